"""Pruning, prompts and decoding together: questions about one pruned video through the paged
cache, against attention in 64 bits over the rows themselves."""
import pytest
import torch

from attention_ref import DH, attend, hidden_mask
from paper_2608_25332_gb300 import provip as P
from paper_2608_25332_gb300.serving import QuestionCache

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__
    __graft_entry__.build()
    P.provip_device_status(clear=True)
    yield
    rc, bits = P.provip_device_status(clear=True)
    assert rc == 0 and bits == 0, f"device status {rc} {bits}"


def near(out, q, k, v, hidden, dtype, what):
    o, _, bound, _ = attend(q, k, v, hidden, DH ** -0.5, dtype, dtype == torch.bfloat16)
    err = (out.double() - o).abs()
    assert torch.isfinite(out).all() and (err <= bound).all(), f"{what}: {float((err / bound).max()):.3g} of its bound"


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_questions_about_one_pruned_video(dtype):
    g = torch.Generator(device=DEV).manual_seed(3)
    rand = lambda *s: torch.randn(*s, generator=g, device=DEV).to(dtype)
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device=DEV)
    H_q, H_kv, nsys, nv, nt, keep, D, layers, B, page = 8, 2, 7, 300, 20, 90, 64, 2, 5, 16
    L = nsys + nv + nt
    # the pruning layer of one sample: its kept rows are the prefix of the layers behind it
    Q, K, V, hidden = rand(1, L, H_q, DH), rand(1, L, H_kv, DH), rand(1, L, H_kv, DH), rand(1, L, D)
    pruned = P.provip_prune(Q, K, V, hidden, None, None, i32([nsys + nv]), i32([nt]), i32([L]), nsys, nv, keep)
    n = nsys + keep
    prefix = [(pruned["K"][0, :n], pruned["V"][0, :n]), (rand(n, H_kv, DH), rand(n, H_kv, DH))]
    cache = QuestionCache(layers, B, H_q, H_kv, page, 60, 120, dtype, DEV)
    cache.set_prefix([p[0] for p in prefix], [p[1] for p in prefix])
    rows = [[None] * B for _ in range(layers)]  # every question's own rows so far

    def check(layer, b, out, q, m):
        k, v = (torch.cat([prefix[layer][i], rows[layer][b][i]]) for i in range(2))
        hid = hidden_mask(m, rows[layer][b][0].shape[0], n, True, DEV)
        for h in range(H_q):
            near(out[:, h], q[:, h], k[:, h * H_kv // H_q], v[:, h * H_kv // H_q], hid, dtype, f"layer {layer} question {b} head {h}")

    def prompts(lens):
        cache.begin(i32(lens))
        T = sum(lens)
        for layer in range(layers):
            q, k, v = rand(T, H_q, DH), rand(T, H_kv, DH), rand(T, H_kv, DH)
            out = cache.prompt(layer, q, k, v)
            at = 0
            for b, m in enumerate(lens):
                if m:
                    rows[layer][b] = [k[at:at + m], v[at:at + m]]
                    check(layer, b, out[at:at + m], q[at:at + m], m)
                at += m

    def decode(new):
        cache.begin(i32(new))
        for layer in range(layers):
            q, k, v = rand(B, H_q, DH), rand(B, H_kv, DH), rand(B, H_kv, DH)
            out = cache.decode(layer, q, k, v)
            for b, m in enumerate(new):
                if m > 0:
                    rows[layer][b] = [torch.cat([r, x[b:b + 1]]) for r, x in zip(rows[layer][b], (k, v))]
                    check(layer, b, out[b:b + 1], q[b:b + 1], 1)
                elif m < 0:
                    rows[layer][b] = None

    prompts([30, 1, 64, 17, 5])
    for _ in range(18):
        decode([1] * B)
    assert cache.kv_len.tolist() == [48, 19, 82, 35, 23]
    decode([1, -1, 1, 1, -1])
    held = sum(-(-x // page) for x in (49, 83, 36)) + -(-n // page)
    assert int(cache.n_free) == 60 - held
    prompts([0, 40, 0, 0, 3])  # two more questions in the slots that came free
    for _ in range(3):
        decode([1] * B)
    assert cache.kv_len.tolist() == [52, 43, 86, 39, 6]
    torch.cuda.synchronize()
