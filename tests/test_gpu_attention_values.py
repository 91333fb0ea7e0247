"""Attention over values and scores that are NaN, infinite or near the largest number, against
the definition in 64 bits (bounds: attention_ref.py)."""
import math

import pytest
import torch

from attention_ref import DH, attend, check, hidden_mask
from paper_2608_25332_gb300 import provip as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF16, F32 = torch.bfloat16, torch.float32
FORMS = [(F32, P.ALGO_AUTO), (BF16, P.ALGO_SIMT), (BF16, P.ALGO_AUTO)]
IDS = ["f32", "bf16_simt", "bf16"]


@pytest.fixture(scope="module", autouse=True)
def _lib():
    import __graft_entry__
    __graft_entry__.build()
    P.provip_device_status(clear=True)
    yield
    rc, bits = P.provip_device_status(clear=True)
    assert rc == 0 and bits == 0, f"device status {rc} {bits}"


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(g, *shape, dtype=F32):
    return torch.randn(*shape, generator=g, device=DEV).to(dtype)


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def tc(dtype, algo):
    return dtype == BF16 and algo != P.ALGO_SIMT


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
@pytest.mark.parametrize("n,lq,H", [(1500, 1500, 8), (3000, 20, 2)])
def test_a_nan_key_costs_no_more_than_another(n, lq, H, dtype, algo):
    """every row sees the key, so every row is NaN, which its own sum shows: nothing is computed
    again (key by key, that took a thousand times as long). The second size has its keys
    shared out over parts."""
    g = gen(1)
    Q, K, V = randn(g, lq, H, DH, dtype=dtype), randn(g, n, H, DH, dtype=dtype), randn(g, n, H, DH, dtype=dtype)
    step = P.PromptAttention(lq, 1, H, H, lq, n, 0, True, None, dtype, DEV, algo)
    args = i32([0]), i32([lq]), i32([0]), i32([n])

    def best():
        t = []
        for _ in range(5):
            a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
            a.record()
            r = step(Q, K, V, *args)
            b.record()
            b.synchronize()
            t.append(a.elapsed_time(b))
        return min(t[1:]), r

    clean, r = best()
    assert torch.isfinite(r["out"]).all() and torch.isfinite(r["lse"]).all()
    K[5, H - 1, 3] = math.nan
    poisoned, r = best()
    row = torch.arange(lq, device=DEV) + n - lq >= 5
    assert torch.isnan(r["out"][row, H - 1]).all() and torch.isnan(r["lse"][row, H - 1]).all()
    assert torch.isfinite(r["out"][:, :H - 1]).all() and torch.isfinite(r["out"][~row]).all() and torch.isfinite(r["lse"][~row]).all()
    assert poisoned < 4 * clean + 0.05, (clean, poisoned)


def test_rows_computed_again_over_a_long_list():
    """One infinite value that every row of a head sees: its rows are computed again key by key,
    which takes longer than any one wait's limit, and nothing gives up on them."""
    g = gen(2)
    n, lq, H = 160000, 128, 80
    Q = randn(g, lq, H, DH, dtype=BF16)
    K = torch.empty(n, H, DH, dtype=BF16, device=DEV).normal_(generator=g)
    V = torch.empty(n, H, DH, dtype=BF16, device=DEV).normal_(generator=g)
    V[7, 1, 0] = math.inf
    r = P.provip_prompt_attention(Q, K, V, i32([0]), i32([lq]), i32([0]), i32([n]), lq, n)
    torch.cuda.synchronize()
    assert P.provip_device_status() == (0, 0)
    assert (r["out"][:, 1, 0] == math.inf).all()
    V[7, 1, 0] = 0.0
    for h in (1, 79):
        ref = attend(Q[:, h], K[:, h], V[:, h], hidden_mask(lq, n, 0, True, DEV), DH ** -0.5, BF16, True)
        out = r["out"][:, h].clone()
        out[:, 0] = torch.where(out[:, 0] == math.inf, ref[0][:, 0].to(BF16), out[:, 0])
        check(out, r["lse"][:, h], ref, f"head {h}")


def huge(g, *shape, dtype):
    """values of 0.5 to 1 times 3e38, of one sign in the first half of a head's elements: no sum of two
    of those is a finite float, every mean of them is"""
    v = (0.5 + 0.5 * torch.rand(*shape, generator=g, device=DEV)) * 3e38
    v[..., DH // 2:] *= torch.where(torch.rand(*shape[:-1], DH // 2, generator=g, device=DEV) < 0.5, -1.0, 1.0)
    return v.to(dtype)


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
@pytest.mark.parametrize("lq,lk,prefix,H_q,H_kv", [(300, 300, 0, 4, 2), (20, 3000, 0, 2, 2), (40, 40, 2500, 7, 1), (1, 2, 0, 1, 1)])
def test_values_whose_sums_pass_the_largest_float(lq, lk, prefix, H_q, H_kv, dtype, algo):
    """a row is a mean of values: it is finite where they are (the second and third sizes have
    their keys shared out over parts)"""
    g = gen(3)
    Q, K, V = randn(g, lq, H_q, DH, dtype=dtype), randn(g, lk, H_kv, DH, dtype=dtype), huge(g, lk, H_kv, DH, dtype=dtype)
    pre = (randn(g, prefix, H_kv, DH, dtype=dtype), huge(g, prefix, H_kv, DH, dtype=dtype)) if prefix else (None, None)
    r = P.provip_prompt_attention(Q, K, V, i32([0]), i32([lq]), i32([0]), i32([lk]), lq, lk, *pre, algo=algo)
    torch.cuda.synchronize()
    for h in range(H_q):
        kv = h * H_kv // H_q
        k, v = (torch.cat([p[:, kv], x[:, kv]]) if prefix else x[:, kv] for p, x in zip(pre, (K, V)))
        ref = attend(Q[:, h], k, v, hidden_mask(lq, lk, prefix, True, DEV), DH ** -0.5, dtype, tc(dtype, algo))
        check(r["out"][:, h], r["lse"][:, h], ref, f"head {h}")


def decode_case(g, lens, H_q, H_kv, prefix, dtype, values, page=16):
    """the arguments of a decode call, and its keys and values a request"""
    held, pre = [-(-n // page) for n in lens], -(-prefix // page)
    order = torch.randperm(sum(held) + pre + 2, generator=g, device=DEV).to(torch.int32)
    K, V = (torch.full((len(order), page, H_kv, DH), math.nan, dtype=dtype, device=DEV) for _ in range(2))
    table = torch.full((len(lens), max(held) + 1), -1, dtype=torch.int32, device=DEV)
    at = pre
    seqs = []
    for b, n in [(-1, prefix)] + list(enumerate(lens)):
        pages = order[:pre] if b < 0 else order[at:at + held[b]]
        k, v, j = randn(g, n, H_kv, DH, dtype=dtype), values(g, n, H_kv, DH, dtype=dtype), torch.arange(n, device=DEV)
        K[pages.long()[j // page], j % page], V[pages.long()[j // page], j % page] = k, v
        seqs.append((k, v))
        if b >= 0:
            table[b, :held[b]] = pages
            at += held[b]
    Q = randn(g, len(lens), H_q, DH, dtype=dtype)
    kw = dict(prefix_table=order[:pre].clone(), prefix_len=prefix) if prefix else {}
    return (Q, K, V, table, i32(lens), max(lens)), kw, [tuple(torch.cat(x) for x in zip(seqs[0], s)) for s in seqs[1:]]


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
@pytest.mark.parametrize("lens,prefix,H_q,H_kv", [([2, 130, 700], 0, 4, 4), ([3000], 0, 7, 1), ([300] * 40, 0, 8, 4), ([1, 90], 700, 14, 2),
                                                  ([5, 260], 300, 16, 1)])
def test_decoding_values_whose_sums_pass_the_largest_float(lens, prefix, H_q, H_kv, dtype, algo):
    """requests a CTA each, spans that cut them, a prefix, and groups of more than eight heads"""
    args, kw, seqs = decode_case(gen(4), lens, H_q, H_kv, prefix, dtype, huge)
    r = P.provip_decode_attention(*args, algo=algo, **kw)
    torch.cuda.synchronize()
    for b, (k, v) in enumerate(seqs):
        for h in range(H_q):
            kv = h * H_kv // H_q
            ref = attend(args[0][b:b + 1, h], k[:, kv], v[:, kv], torch.zeros(1, len(k), dtype=torch.bool, device=DEV), DH ** -0.5, dtype,
                         tc(dtype, algo))
            check(r["out"][b:b + 1, h], r["lse"][b:b + 1, h], ref, f"request {b} head {h}")


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
@pytest.mark.parametrize("prefix", [0, 300])
def test_decoding_infinite_values_that_are_seen(prefix, dtype, algo):
    """they show in their element, and in no other"""
    def values(g, *shape, dtype):
        v = huge(g, *shape, dtype=dtype)
        if shape[0]:
            v[0, :, 3], v[0, :, 40] = math.inf, math.nan
        return v

    args, kw, seqs = decode_case(gen(5), [2, 130, 700], 14, 2, prefix, dtype, values)
    r = P.provip_decode_attention(*args, algo=algo, **kw)
    torch.cuda.synchronize()
    assert (r["out"][..., 3] == math.inf).all() and torch.isnan(r["out"][..., 40]).all()
    fine = torch.arange(DH, device=DEV)
    fine = fine[(fine != 3) & (fine != 40)]
    for b, (k, v) in enumerate(seqs):
        for h in range(14):
            v2 = v[:, h // 7].clone()
            v2[:, [3, 40]] = 0.0
            o, lse, bound, _ = attend(args[0][b:b + 1, h], k[:, h // 7], v2, torch.zeros(1, len(k), dtype=torch.bool, device=DEV),
                                      DH ** -0.5, dtype, tc(dtype, algo))
            out = r["out"][b:b + 1, h].double()
            assert torch.isfinite(out[:, fine]).all() and ((out - o).abs() <= bound)[:, fine].all(), (b, h)


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
@pytest.mark.parametrize("prefix", [0, 300])
def test_decoding_one_infinite_value_among_huge_ones(prefix, dtype, algo):
    """the others' sum passes the largest float with the other sign: the infinite value shows all
    the same"""
    def values(g, *shape, dtype):
        v = huge(g, *shape, dtype=dtype)
        v[..., 5] = -v[..., 5]
        if shape[0]:
            v[-1, :, 3], v[-1, :, 5] = -math.inf, math.inf
            v[-1, :, 90], v[0, :, 100] = math.inf, -math.inf
        return v

    args, kw, seqs = decode_case(gen(6), [40, 130, 700], 14, 2, prefix, dtype, values)
    r = P.provip_decode_attention(*args, algo=algo, **kw)
    torch.cuda.synchronize()
    for at, want in ((3, -math.inf), (5, math.inf), (90, math.inf), (100, -math.inf)):
        assert (r["out"][..., at] == want).all(), at
    assert torch.isfinite(r["lse"]).all()
