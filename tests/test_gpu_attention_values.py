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
