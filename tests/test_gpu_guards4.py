"""Guard bytes around every output, pool and workspace of the rotation and of the 4-bit cache, called at the C entry
points: workspaces of exactly the size reported, rows further apart than they are long (what lies between them is
NaN in inputs, and stays as it was in outputs), and the same values as the binding's calls give."""
import ctypes

import pytest
import torch

import cache4_ref as ref
from paper_2608_25332_gb300 import provip as P
from test_gpu_cache4 import case, decode
from test_gpu_guards import FILL, Guarded, guarded_ws

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = {torch.float32: P.F32, torch.bfloat16: P.BF16}


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__
    __graft_entry__.build()
    P.provip_device_status(clear=True)
    yield
    rc, bits = P.provip_device_status(clear=True)
    assert rc == 0 and bits == 0, f"device status {rc} {bits}"


def stream():
    return torch.cuda.current_stream(DEV).cuda_stream


def apart(x):
    """rows x [T, H, 128] with a head of NaN behind each"""
    wide = torch.full((x.shape[0], x.shape[1] + 1, 128), float("nan"), dtype=x.dtype, device=DEV)
    wide[:, :-1] = x
    return wide


class Rows:
    """Guarded rows [T, H, 128] whose stride is a head longer than they are."""

    def __init__(self, T, H, dtype):
        self.g, self.stride = Guarded((T, H + 1, 128), dtype), (H + 1) * 128
        self.ptr, self.t = self.g.t.data_ptr(), self.g.t[:, :H]

    def check(self, what):
        self.g.check(what)
        between = self.g.t[:, -1].contiguous().view(torch.uint8)
        assert bool((between == FILL).all()), f"{what}: written between rows"


def rotary(T):
    g = torch.Generator(device=DEV).manual_seed(T)
    pos = torch.randint(0, 30000, (3, T), device=DEV, generator=g).to(torch.int32)
    return P.Rotary(sections=(16, 24, 24)), pos


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("T,H_q,H_kv", [(1, 1, 1), (3, 28, 4), (48, 5, 3), (511, 17, 2), (512, 17, 9), (700, 28, 4)])
def test_rotate(T, H_q, H_kv, dtype):
    g = torch.Generator(device=DEV).manual_seed(T + H_q)
    Q, K = torch.randn(T, H_q, 128, device=DEV, generator=g).to(dtype), torch.randn(T, H_kv, 128, device=DEV, generator=g).to(dtype)
    w = (1 + torch.randn(2, 128, device=DEV, generator=g) / 4).to(dtype)
    rot, pos = rotary(T)
    want = P.provip_rotate(Q, K, pos, rot, w[0], w[1])
    q_in, k_in, q, k = apart(Q), apart(K), Rows(T, H_q, dtype), Rows(T, H_kv, dtype)
    rc = P.lib().provip_rotate(q_in.data_ptr(), q.stride, k_in.data_ptr(), k.stride, T, None, H_q, H_kv, 128, pos.data_ptr(), T, *rot.args,
                               w[0].data_ptr(), w[1].data_ptr(), 1e-6, DTYPES[dtype], q.ptr, q.stride, k.ptr, k.stride, stream())
    assert rc == 0
    for rows, x, what in ((q, want[0], "q_out"), (k, want[1], "k_out")):
        rows.check(what)
        assert torch.equal(rows.t, x), what


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("four", [0, 1])
@pytest.mark.parametrize("T,H_q,H_kv,page", [(1, 4, 1, 8), (99, 28, 4, 16), (512, 8, 17, 256), (600, 5, 5, 64)])
def test_rotate_append(T, H_q, H_kv, page, four, dtype):
    g = torch.Generator(device=DEV).manual_seed(T + four)
    Q, K, V = (torch.randn(T, h, 128, device=DEV, generator=g).to(dtype) for h in (H_q, H_kv, H_kv))
    rot, pos = rotary(T)
    n = -(-T // page)
    slot = torch.randperm(n * page, device=DEV, generator=g)[:T].to(torch.int32)  # first and last slot as a rule
    slot[0], shape, kind = n * page - 1, ((n, H_kv, page * 72) if four else (n, page, H_kv, 128)), torch.uint8 if four else dtype
    slot[1:][slot[1:] == n * page - 1] = -1
    pools = [Guarded(shape, kind) for _ in range(2)]
    q, k = Rows(T, H_q, dtype), Rows(T, H_kv, dtype)
    q_in, k_in, v_in = apart(Q), apart(K), apart(V)
    want_pools = [x.t.clone() for x in pools]
    want_q, want_k = P.provip_rotate_append(Q, K, V, pos, rot, slot, *want_pools, want_k=True)
    rc = P.lib().provip_rotate_append(q_in.data_ptr(), q.stride, k_in.data_ptr(), k.stride, v_in.data_ptr(), k.stride, T, None, H_q, H_kv, 128,
                                      pos.data_ptr(), T, *rot.args, None, None, 1e-6, DTYPES[dtype], q.ptr, q.stride, k.ptr, k.stride,
                                      slot.data_ptr(), n, page, four, pools[0].t.data_ptr(), pools[1].t.data_ptr(), stream())
    assert rc == 0
    for x, want, what in ((q, want_q, "q_out"), (k, want_k, "k_out")):
        x.check(what)
        assert torch.equal(x.t, want), what
    for x, want in zip(pools, want_pools):
        x.check("pool")
        assert torch.equal(x.t.view(torch.uint8), want.view(torch.uint8))


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("T,H,page", [(1, 1, 8), (99, 32, 16), (513, 5, 64), (40, 17, 256)])
def test_rows_in_and_out(T, H, page, dtype):
    g = torch.Generator(device=DEV).manual_seed(T + H)
    K, V = (torch.randn(T, H, 128, device=DEV, generator=g).to(dtype) for _ in range(2))
    n = -(-T // page)
    slot = (n * page - 1 - torch.arange(T, device=DEV)).to(torch.int32)
    pools = [Guarded((n, H, page * 72), torch.uint8) for _ in range(2)]
    want_pools = [x.t.clone() for x in pools]
    P.provip_kv_append4(K, V, slot, *want_pools)
    k_in, v_in, k, v = apart(K), apart(V), Rows(T, H, dtype), Rows(T, H, dtype)
    L, at = P.lib(), [x.t.data_ptr() for x in pools]
    assert L.provip_kv_append4(k_in.data_ptr(), k.stride, v_in.data_ptr(), v.stride, T, H, 128, slot.data_ptr(), n, page, DTYPES[dtype], *at,
                               stream()) == 0
    assert L.provip_kv_read4(slot.data_ptr(), T, H, 128, *at, n, page, DTYPES[dtype], k.ptr, k.stride, v.ptr, v.stride, stream()) == 0
    for x, want in zip(pools, want_pools):
        x.check("pool")
        assert torch.equal(x.t, want)
    for x, want in zip((k, v), P.provip_kv_read4(slot, *want_pools, dtype=dtype)):
        x.check("rows out")
        assert torch.equal(x.t, want)


ROWS = [1, 2, 3, 8, 9, 16, 17, 128, 129, 256, 257]  # query rows a key/value head, where one form of the prefix ends
SHAPES = [([(37 * i) % 70 for i in range(n)], 2, 2, 16, 300) for n in ROWS] + \
    [([3000], 28, 4, 64, 0), ([9, 2100, 0], 7, 1, 8, 0), ([0, 0], 16, 1, 16, 5000), ([700] * 20, 28, 4, 64, 2000), ([50] * 300, 32, 32, 16, 0)]


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("lens,H_q,H_kv,page,prefix", SHAPES)
def test_decode(lens, H_q, H_kv, page, prefix, dtype):
    c = case(len(lens) + page, lens, H_q, H_kv, page, prefix, dtype)
    want, B, most, L = decode(c), len(lens), max(lens), P.lib()
    out, lse, q_in = Rows(B, H_q, dtype), Guarded((B, H_q), torch.float32), apart(c["Q"])
    need = L.provip_decode_attention4_workspace_size(B, H_q, H_kv, most, prefix, DTYPES[dtype])
    ws = guarded_ws(need)
    rc = L.provip_decode_attention4(q_in.data_ptr(), out.stride, B, H_q, H_kv, 128, c["k"].data_ptr(), c["v"].data_ptr(), c["k"].shape[0], page,
                                    c["table"].data_ptr(), c["table"].shape[1], c["kv"].data_ptr(), most,
                                    c["prefix_table"].data_ptr() if prefix else None, prefix, ctypes.c_float(128 ** -0.5), DTYPES[dtype], out.ptr,
                                    out.stride, lse.t.data_ptr(), ws.t.data_ptr(), need, stream())
    assert rc == 0
    out.check("out"), lse.check("lse"), ws.check("workspace")
    assert torch.equal(out.t, want["out"]) and torch.equal(lse.t, want["lse"])
    for b in sorted({0, B // 2, B - 1}):  # (and those are right)
        j = torch.arange(lens[b], device=DEV)
        slots = c["table"][b].long()[j // page] * page + j % page if lens[b] else j
        j = torch.arange(prefix, device=DEV)
        slots = torch.cat([c["prefix_table"].long()[j // page] * page + j % page, slots]) if prefix else slots
        K, V = ref.values(c["k"], page, slots), ref.values(c["v"], page, slots)
        for h in range(0, H_q, 5):
            g = h // (H_q // H_kv)
            o, _, bound, _ = ref.attend(c["Q"][b, h], K[:, g], V[:, g], 128 ** -0.5, dtype)
            assert ((out.t[b, h].double() - o).abs() <= bound).all(), (b, h)


def test_two_streams_at_once():
    """rotation into pages and decoding on two streams that nothing orders, each with buffers of its own, as alone"""
    sides = [torch.cuda.Stream(DEV) for _ in range(2)]
    work = []
    for i in range(2):
        g = torch.Generator(device=DEV).manual_seed(50 + i)
        T, H_q, H_kv = 3000 + 7 * i, 28, 4
        Q, K, V = torch.randn(T, H_q + 2 * H_kv, 128, device=DEV, generator=g).to(torch.bfloat16).split([H_q, H_kv, H_kv], 1)
        rot, pos = rotary(T)
        slot = torch.randperm(T + 61, device=DEV, generator=g)[:T].to(torch.int32)
        pools = P.pages4(-(-(T + 61) // 64), 64, H_kv, DEV), P.pages4(-(-(T + 61) // 64), 64, H_kv, DEV)
        out = (torch.zeros(T, H_q, 128, dtype=torch.bfloat16, device=DEV), None)
        c = case(60 + i, [200 + i] * 30, 28, 4, 64, 1500, torch.bfloat16)
        step = P.DecodeAttention4(30, 28, 4, 201, 1500, device=DEV)
        work.append(dict(call=lambda Q=Q, K=K, V=V, pos=pos, rot=rot, slot=slot, pools=pools, out=out, c=c, step=step: (
            P.provip_rotate_append(Q, K, V, pos, rot, slot, *pools, out=out),
            step(c["Q"], c["k"], c["v"], c["table"], c["kv"], c["prefix_table"])), results=[*pools, out[0], step.out, step.lse]))
    want = []
    for w in work:
        w["call"]()
        torch.cuda.synchronize()
        want.append([x.clone() for x in w["results"]])
    for _ in range(10):
        for w in work:
            for x in w["results"]:
                x.zero_()
        torch.cuda.synchronize()
        for _ in range(5):
            for w, side in zip(work, sides):
                with torch.cuda.stream(side):
                    w["call"]()
        torch.cuda.synchronize()
        for w, results in zip(work, want):
            assert all(torch.equal(a, b) for a, b in zip(w["results"], results))
