"""Rows in and out of 4-bit pages, and decoding from them, against their definition."""
import copy
import math
import random

import numpy as np
import pytest
import torch

import cache4_ref as ref
from paper_2608_25332_gb300 import provip as P

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


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


# ---------------------------------------------------------------------------
# rows in and out
# ---------------------------------------------------------------------------
def odd_rows(g, T, H, dtype):
    """Rows with ties, zeros, one-sided groups, and magnitudes from one end of the type to the other."""
    x = torch.randn(T, H, 4, 32, device=DEV, generator=g)
    kind = torch.randint(0, 12, (T, H, 4, 1), device=DEV, generator=g)
    x = torch.where(kind == 0, torch.zeros_like(x), x)
    x = torch.where(kind == 1, x.abs(), x)
    x = torch.where(kind == 2, torch.randint(-8, 9, x.shape, device=DEV, generator=g).float(), x)  # ties in plenty
    x = torch.where(kind == 3, torch.randint(-17, 18, x.shape, device=DEV, generator=g).float() / 2, x)
    x = torch.where(kind == 4, x * 2.0 ** 90, x)
    x = torch.where(kind == 5, x * 2.0 ** -118, x)
    x = torch.where(kind == 6, x * 2.0 ** -126, x)
    x = torch.where(kind == 7, x * 2.0 ** 105, x)
    x = torch.where(kind == 8, x.sign() * 3.0, x)
    return x.view(T, H, 128).to(dtype)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H,page", [(1, 1, 8), (3, 5, 16), (70, 4, 64), (99, 32, 16), (40, 3, 256)])
def test_codes_and_scales(T, H, page, dtype):
    """byte for byte as the definition gives them, operation by operation; other slots as they were"""
    g = gen(T * 7 + H)
    K, V = odd_rows(g, T, H, dtype), odd_rows(g, T, H, dtype)
    n = -(-T // page) + 1
    slot = torch.randperm(n * page, device=DEV, generator=g)[:T].to(torch.int32)
    slot[::5] = -1
    blank = torch.randint(0, 256, (2, n, H, page * 72), device=DEV, generator=g, dtype=torch.uint8)
    got = blank.clone()
    P.provip_kv_append4(K, V, slot, got[0], got[1])
    want, where = blank.cpu(), slot.tolist()
    for x, pool in ((K, want[0]), (V, want[1])):
        codes, bits = ref.pack(x.float().cpu().numpy().reshape(T * H, 128))
        for t, s in enumerate(where):
            for h in range(H if s >= 0 else 0):
                ref.put(pool, page, s, h, codes[t * H + h], bits[t * H + h])
    got = got.cpu()
    # (codes of a group whose scale is NaN may be anything)
    for i, x in enumerate((K, V)):
        for t, s in enumerate(where):
            for h in range(H if s >= 0 else 0):
                c0, b0 = ref.row_bytes(want[i], page, s, h)
                c1, b1 = ref.row_bytes(got[i], page, s, h)
                assert (b0 == b1).all(), (t, h, b0, b1)
                fine = np.repeat(((b0 & 0x7F80) != 0x7F80)[None], 8, 0).reshape(-1).repeat(2)  # byte 2 (4 g + q)
                assert (c0[fine] == c1[fine]).all(), (t, h)
                got[i][s // page, h, s % page * 64:s % page * 64 + 64] = want[i][s // page, h, s % page * 64:s % page * 64 + 64]
    assert torch.equal(want, got)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_values_are_near(dtype):
    """Every value is off by half a scale at most, but where the other sign's end is cut off. There |x| goes to
    7 |d|, and |d| >= most / 8 (1 - 2^-8) (half a step of bf16; exact for bf16 rows), so it is off by at most
    most - 7 most / 8 (1 - 2^-8) = most / 8 (1 + 7 2^-8)."""
    g = gen(5)
    x = (torch.randn(200, 4, 128, device=DEV, generator=g) * torch.exp2(torch.randint(-20, 20, (200, 4, 1), device=DEV, generator=g).float())).to(dtype)
    pools = P.pages4(13, 16, 4, DEV), P.pages4(13, 16, 4, DEV)
    slot = torch.arange(200, dtype=torch.int32, device=DEV)
    P.provip_kv_append4(x, -x, slot, *pools)
    for sign, pool in ((1, pools[0]), (-1, pools[1])):
        v = ref.values(pool, 16, slot) * sign
        grp, gv = x.double().view(200, 4, 4, 32), v.view(200, 4, 4, 32)
        most = grp.abs().amax(-1, keepdim=True)
        d = most / 8
        cut = grp.abs() > 7.5 * d * (1 - 2.0 ** -8)
        worst = (grp - gv).abs() / torch.where(cut, d * (1 + 7 * 2.0 ** -8), d / 2 * (1 + 2.0 ** -8))
        assert float(worst.max()) <= 1


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_read_gives_what_codes_stand_for(dtype):
    g = gen(6)
    for T, H, page in ((1, 1, 8), (37, 5, 16), (300, 32, 64), (13, 4, 256)):
        n = 5 * 256 // page
        pool = ref.random_pool(g, n, page, H, DEV)
        other = ref.random_pool(g, n, page, H, DEV)
        slot = torch.randint(0, n * page, (T,), device=DEV, generator=g).to(torch.int32)  # some twice
        slot[T // 2:T // 2 + 2] = -1
        k, v = P.provip_kv_read4(slot, pool, other, dtype)
        for got, p in ((k, pool), (v, other)):
            want = torch.where((slot >= 0)[:, None, None], ref.values(p, page, slot.clamp(min=0)), 0.0)
            assert torch.equal(got, want.to(torch.float32).to(dtype))
        # into strided rows that hold something
        out = torch.full((T, 2 * H, 128), 7.0, dtype=dtype, device=DEV)
        P.provip_kv_read4(slot, pool, other, out=(out[:, :H], out[:, H:]))
        keep = (slot >= 0)[:, None, None]
        assert torch.equal(out, torch.where(keep, torch.cat([k, v], 1), out.new_tensor(7.0)))


def test_every_scale_fraction():
    """groups whose largest value has each of the 256 fractions of a bf16, at several exponents, with values all
    over the codes' range and next to their borders: codes as the reciprocal rounded to nearest gives them"""
    g = gen(12)
    frac = torch.arange(128, device=DEV).float() / 128 + 1
    rows = []
    for exp in (-100, -20, 0, 7, 60, 90):
        for sign in (1.0, -1.0):
            e = sign * frac * 2.0 ** exp
            d = -e / 8
            x = torch.rand(128, 32, device=DEV, generator=g) * 15.5 - 8
            x[:, 1:16] = torch.round(x[:, 1:16]) + 0.5  # borders, and one step of fp32 off them
            x[:, 4:8] *= 1 + 2.0 ** -23
            x[:, 8:12] *= 1 - 2.0 ** -23
            x = x.clamp(-7.9, 7.9) * d[:, None]
            x[:, 0] = e
            rows.append(x)
    x = torch.cat(rows).view(-1, 1, 128)
    n = x.shape[0]
    pools = P.pages4(-(-n // 64), 64, 1, DEV), P.pages4(-(-n // 64), 64, 1, DEV)
    P.provip_kv_append4(x, x, torch.arange(n, dtype=torch.int32, device=DEV), *pools)
    codes, bits = ref.pack(x.cpu().numpy().reshape(-1, 128))
    want = (codes.reshape(-1, 4, 32) - 8) * ref.bf16_value(bits).astype(np.float64)[..., None]
    got = ref.values(pools[0], 64, torch.arange(n, device=DEV)).cpu().numpy().reshape(-1, 4, 32)
    assert (got == want).all()


def test_not_finite_and_huge_groups_stand_for_nan():
    x = torch.ones(4, 1, 128, device=DEV)
    x[0, 0, 40], x[1, 0, 3], x[2, 0, 100], x[3, 0, 127] = math.nan, math.inf, -math.inf, 2.0 ** 100
    pools = P.pages4(1, 8, 1, DEV), P.pages4(1, 8, 1, DEV)
    P.provip_kv_append4(x, x, torch.arange(4, dtype=torch.int32, device=DEV), *pools)
    k, v = P.provip_kv_read4(torch.arange(4, dtype=torch.int32, device=DEV), *pools, dtype=torch.float32)
    want = torch.ones(4, 4, dtype=torch.bool)
    for t, q in enumerate((1, 0, 3, 3)):
        want[t, q] = False
    for r in (k, v):
        assert torch.equal(torch.isfinite(r.view(4, 4, 32)).all(-1).cpu(), want)
        assert torch.equal(torch.isnan(r.view(4, 4, 32)).all(-1).cpu(), ~want)
        assert (r.view(4, 4, 32)[want.to(DEV)] == 1).all()


def test_bad_slots_are_reported():
    x = torch.randn(3, 2, 128, device=DEV)
    pools = P.pages4(2, 8, 2, DEV), P.pages4(2, 8, 2, DEV)
    P.provip_kv_append4(x, x, i32([16, 3, 2 ** 31 - 1]), *pools)
    assert P.provip_device_status(clear=True)[1] == P.DEVSTAT_BAD_ARG
    out = torch.full((2, 3, 2, 128), 5.0, device=DEV)
    P.provip_kv_read4(i32([16, 3, -2]), *pools, out=(out[0], out[1]))
    assert P.provip_device_status(clear=True)[1] == P.DEVSTAT_BAD_ARG
    assert (out[:, [0, 2]] == 5).all() and (out[:, 1] != 5).any()


# ---------------------------------------------------------------------------
# decoding
# ---------------------------------------------------------------------------
def case(seed, lens, H_q, H_kv, page, prefix=0, dtype=torch.bfloat16, spread=1.0, extra_pages=0, stride=0):
    """requests' pages in a random order; every page that none holds, and rows past each end, have NaN scales"""
    g, rng = gen(seed), random.Random(seed)
    held, pre = [-(-n // page) for n in lens], -(-prefix // page)
    n = sum(held) + pre + 2
    ids = list(range(n))
    rng.shuffle(ids)
    width = max(held + [0]) + extra_pages
    table, at = [], pre
    for h in held:
        table.append(ids[at:at + h] + [-7] * (width - h))
        at += h
    pools = []
    for _ in range(2):
        pool = ref.random_pool(g, n, page, H_kv, DEV, spread)
        scales = pool[..., page * 64:].view(torch.bfloat16).view(n, H_kv, page, 4)
        for pg in ids[at:]:
            scales[pg] = math.nan
        for size, pages in zip(lens + [prefix], table + [ids[:pre]]):
            if size % page:
                scales[pages[size // page], :, size % page:] = math.nan
        pools.append(pool)
    B = len(lens)
    Q = torch.randn(B, H_q + stride, 128, device=DEV, generator=g).to(dtype)[:, :H_q]
    return dict(Q=Q, k=pools[0], v=pools[1], table=i32(table).view(B, width), kv=i32(lens), prefix_table=i32(ids[:pre]) if prefix else None,
                lens=lens, page=page, prefix=prefix, H_kv=H_kv)


def rows_of(c, b):
    page = c["page"]
    j = torch.arange(c["lens"][b], device=DEV)
    slots = c["table"][b].long()[j // page] * page + j % page if len(j) else j
    if c["prefix"]:
        j = torch.arange(c["prefix"], device=DEV)
        slots = torch.cat([c["prefix_table"].long()[j // page] * page + j % page, slots])
    return ref.values(c["k"], page, slots), ref.values(c["v"], page, slots)


def check(c, r, scale=128 ** -0.5, rows=None, what=""):
    H_q = c["Q"].shape[1]
    for b in range(len(c["lens"])) if rows is None else rows:
        K, V = rows_of(c, b)
        for h in range(H_q):
            g = h // (H_q // c["H_kv"])
            o, lse, bo, bl = ref.attend(c["Q"][b, h], K[:, g], V[:, g], scale, c["Q"].dtype)
            got, gl = r["out"][b, h].double(), r["lse"][b, h].double()
            assert torch.isfinite(got).all(), (what, b, h)
            err = (got - o).abs()
            assert (err <= bo).all(), f"{what} request {b} head {h}: off by {float((err / bo).max()):.3g} of its bound"
            if K.shape[0] == 0:
                assert float(gl) == -math.inf
            else:
                assert abs(float(gl - lse)) <= bl, f"{what} request {b} head {h}: lse off by {abs(float(gl - lse)) / bl:.3g}"


def decode(c, kv_max=None, **kw):
    return P.provip_decode_attention4(c["Q"], c["k"], c["v"], c["table"], c["kv"], max(c["lens"]) if kv_max is None else kv_max,
                                      c["prefix_table"], c["prefix"], **kw)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("lens,H_q,H_kv,page,prefix", [
    ([1], 1, 1, 8, 0), ([2, 0, 17], 4, 4, 8, 0), ([31, 32, 33, 127, 128, 129], 4, 2, 16, 0), ([211], 32, 32, 16, 0),
    ([500, 3, 90], 28, 4, 64, 0), ([700, 1291], 8, 1, 32, 0), ([100, 257], 16, 1, 256, 0), ([64, 300], 24, 2, 128, 0),
    ([40, 200], 64, 1, 16, 0), ([65, 10], 37, 1, 8, 0), ([5, 0, 60], 4, 2, 8, 9), ([0], 28, 4, 16, 100), ([0, 0], 3, 3, 16, 0),
    ([1, 512, 77, 300, 5], 28, 4, 64, 2339), ([9, 30], 64, 2, 32, 500), ([3] * 40, 4, 4, 16, 33), ([1, 2, 3], 8, 8, 128, 1)])
def test_decode(lens, H_q, H_kv, page, prefix, dtype):
    c = case(sum(lens) + H_q + page, lens, H_q, H_kv, page, prefix, dtype)
    check(c, decode(c))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_long_rows(dtype):
    """lists of many parts, with one long request among short ones, and a long prefix"""
    c = case(1, [9379, 5, 800], 4, 2, 64, 0, dtype)
    check(c, decode(c))
    c = case(2, [20, 3000], 7, 1, 16, 9251, dtype)
    check(c, decode(c))


@pytest.mark.parametrize("lens,H_q,H_kv,page,prefix", [
    ([3, 0, 9], 28, 4, 16, 100), ([1] * 20, 28, 4, 64, 1000), ([2, 40] * 19, 8, 2, 8, 333), ([7] * 70, 4, 4, 32, 65), ([1] * 64, 28, 4, 64, 9251),
    ([0] * 33, 2, 1, 256, 1), ([5] * 9, 64, 2, 128, 700), ([4] * 300, 1, 1, 16, 2000)])
def test_a_prefix_for_many_rows(lens, H_q, H_kv, page, prefix):
    """blocks of 32, 64 and 128 rows"""
    c = case(len(lens) + page, lens, H_q, H_kv, page, prefix, torch.bfloat16)
    check(c, decode(c), rows=range(0, len(lens), max(len(lens) // 5, 1)))


@pytest.mark.parametrize("spread", [2.0 ** -110, 2.0 ** -40, 2.0 ** 12, 2.0 ** 90])
def test_a_prefix_of_any_size(spread):
    c = case(21, [5] * 12, 28, 4, 16, 300, torch.bfloat16, spread)
    scale = 1.0 / (spread * 11.3)
    check(c, decode(c, scale=scale), scale, rows=(0, 7))


def test_a_prefix_whose_values_grow():
    """keys' scales and values' scales over 2^24 along the list, and groups of a row 2^20 apart: each weight keeps
    its bits next to the largest"""
    c = case(22, [5] * 12, 28, 4, 16, 640, torch.bfloat16)
    j = torch.arange(640, device=DEV)
    slots = c["prefix_table"].long()[j // 16] * 16 + j % 16
    s = c["v"][..., 16 * 64:].view(torch.bfloat16).view(-1, 4, 16, 4)
    grow = torch.exp2((j % 320).float() / 320 * 24 - 12)
    s[slots // 16, :, slots % 16] = (s[slots // 16, :, slots % 16].float() * grow[:, None, None]).to(torch.bfloat16)
    s[..., 2] *= 2.0 ** -20
    s = c["k"][..., 16 * 64:].view(torch.bfloat16).view(-1, 4, 16, 4)
    s[slots // 16, :, slots % 16] = (s[slots // 16, :, slots % 16].float() * (0.05 + j.float()[:, None, None] / 300)).to(torch.bfloat16)
    check(c, decode(c), rows=(0, 11))


def test_a_prefix_with_keys_far_apart():
    """a few keys' values, and a few groups of keys, 2^12 to 2^150 from the others, at the front and later"""
    c = case(25, [5] * 12, 28, 4, 16, 640, torch.bfloat16)
    s = c["v"][..., 16 * 64:].view(torch.bfloat16).view(-1, 4, 16, 4)
    for at, f in ((0, 2.0 ** -70), (1, 2.0 ** -12), (100, 2.0 ** 12), (333, 2.0 ** 80), (500, 2.0 ** -60)):
        s[c["prefix_table"][at // 16].long(), at % 4, at % 16] *= f
    s[c["prefix_table"][5:9].long(), 3] *= 2.0 ** 15
    s = c["k"][..., 16 * 64:].view(torch.bfloat16).view(-1, 4, 16, 4)
    s[c["prefix_table"][3].long(), 1, 7, 2] *= 2.0 ** -14
    s[c["prefix_table"][11:13].long(), :, :, 1] *= 2.0 ** -30
    check(c, decode(c), rows=(0, 5, 11))


def test_a_prefix_that_is_not_finite_shows_where_it_should():
    c = case(23, [5] * 12, 28, 4, 16, 100, torch.bfloat16)
    page = int(c["prefix_table"][3])
    c["v"][..., 16 * 64:].view(torch.bfloat16).view(-1, 4, 16, 4)[page, 2, 5, 1] = math.nan
    bad = ~torch.isfinite(decode(c)["out"]).view(12, 4, 7, 4, 32).all(-1)
    want = torch.zeros(12, 4, 7, 4, dtype=torch.bool, device=DEV)
    want[:, 2, :, 1] = True
    assert torch.equal(bad, want)
    c["k"][..., 16 * 64:].view(torch.bfloat16).view(-1, 4, 16, 4)[page, 0, 5, 1] = math.nan
    r = decode(c)
    want[:, 0] = True
    assert torch.equal(~torch.isfinite(r["out"]).view(12, 4, 7, 4, 32).all(-1), want)
    assert torch.isnan(r["lse"].view(12, 4, 7)[:, 0]).all() and torch.isfinite(r["lse"].view(12, 4, 7)[:, 1:]).all()


def test_a_bad_prefix_page_is_reported():
    c = case(24, [5] * 12, 28, 4, 16, 100, torch.bfloat16)
    for bad in (-1, c["k"].shape[0]):
        c["prefix_table"][2] = bad
        decode(c)
        assert P.provip_device_status(clear=True)[1] == P.DEVSTAT_BAD_ARG


def test_many_requests():
    lens = [(i * 37) % 300 for i in range(300)]
    c = case(3, lens, 8, 2, 16, 0, torch.bfloat16)
    check(c, decode(c), rows=range(0, 300, 23))


def test_a_bound_above_the_lengths():
    """the host's bound sizes the launch only"""
    c = case(4, [30, 200, 0, 129], 4, 2, 16, 0, torch.bfloat16, extra_pages=400)
    a = decode(c)
    check(c, a)
    check(c, decode(c, kv_max=6000))


def test_scales_far_apart_and_strided_queries():
    for spread in (2.0 ** -60, 2.0 ** 12, 2.0 ** 90):
        c = case(5, [150, 33], 8, 4, 16, 20, torch.float32, spread, stride=3)
        scale = 1.0 / (spread * 11.3)
        check(c, decode(c, scale=scale), scale)


def test_groups_that_differ_by_far():
    """one group's values a thousand times another's: each keeps its own scale's precision"""
    c = case(6, [90], 4, 4, 16, 0, torch.bfloat16)
    for pool in (c["k"], c["v"]):
        s = pool[..., 16 * 64:].view(torch.bfloat16).view(-1, 4, 16, 4)
        s[..., 1] *= 2.0 ** -12
        s[..., 2] *= 2.0 ** 10
    c["Q"] *= 2.0 ** -9
    r = decode(c)
    check(c, r)
    K, V = rows_of(c, 0)
    o, _, _, _ = ref.attend(c["Q"][0, 0], K[:, 0], V[:, 0], 128 ** -0.5, torch.bfloat16)
    got = r["out"][0, 0].double()
    for q in range(4):
        x, y = got[32 * q:32 * q + 32], o[32 * q:32 * q + 32]
        assert float((x - y).norm() / y.norm()) < 2.0 ** -7


def test_a_maximum_that_comes_late():
    """scores that grow along the list, so that the running maximum is raised again and again"""
    c = case(7, [640], 2, 1, 16, 0, torch.float32)
    K, _ = rows_of(c, 0)
    j = torch.arange(640, device=DEV)
    slots = c["table"][0].long()[j // 16] * 16 + j % 16
    s = c["k"][..., 16 * 64:].view(torch.bfloat16).view(-1, 1, 16, 4)
    s[slots // 16, 0, slots % 16] = (0.02 * (1 + j.float()))[:, None].to(torch.bfloat16)
    check(c, decode(c))


def test_keys_that_are_not_finite_show_in_their_own_rows_only():
    c = case(8, [70, 70], 4, 2, 16, 0, torch.bfloat16)
    page, row = int(c["table"][1, 2]), 3
    c["v"][..., 16 * 64:].view(torch.bfloat16).view(-1, 2, 16, 4)[page, 1, row, 2] = math.nan
    r = decode(c)
    bad = ~torch.isfinite(r["out"]).view(2, 4, 4, 32).all(-1)
    assert bad.nonzero().tolist() == [[1, 2, 2], [1, 3, 2]]
    c = case(8, [70, 70], 4, 2, 16, 0, torch.bfloat16)
    c["k"][..., 16 * 64:].view(torch.bfloat16).view(-1, 2, 16, 4)[page, 1, row, 2] = math.nan
    r = decode(c)
    assert torch.isnan(r["out"][1, 2:]).all() and torch.isnan(r["lse"][1, 2:]).all()
    r["out"][1, 2:], r["lse"][1, 2:] = 0, 0
    assert torch.isfinite(r["out"]).all() and torch.isfinite(r["lse"]).all()


def test_bad_lengths_and_pages_are_reported():
    c = case(9, [40, 60, 20], 4, 2, 16, 0, torch.bfloat16)
    good = decode(c)
    for bad in (-1, 61, 2 ** 31 - 1):
        c["kv"][0] = bad
        r = decode(c)
        assert P.provip_device_status(clear=True)[1] == P.DEVSTAT_BAD_ARG
        assert not r["out"][0].any() and (r["lse"][0] == -math.inf).all()
        assert torch.equal(r["out"][1:], good["out"][1:])
    c["kv"][0] = 40
    for bad in (-1, c["k"].shape[0], 2 ** 31 - 1):
        c["table"][2, 0] = bad
        r = decode(c)
        assert P.provip_device_status(clear=True)[1] == P.DEVSTAT_BAD_ARG
        assert torch.equal(r["out"][:2], good["out"][:2])


def test_repeated_calls_and_graphs_agree():
    """the same bits from call to call, in a graph, and of two graphs with a workspace each"""
    c = case(10, [700, 30, 257], 28, 4, 16, 300, torch.bfloat16)
    first = decode(c)
    steps = [P.DecodeAttention4(3, 28, 4, 700, 300, device=DEV) for _ in range(2)]
    args = (c["Q"], c["k"], c["v"], c["table"], c["kv"], c["prefix_table"])
    graphs = []
    for step in steps:
        step(*args)
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            step(*args)
        graphs.append(gr)
    streams = [torch.cuda.Stream(DEV) for _ in steps]
    for _ in range(20):
        for step in steps:
            step.out.zero_()
        torch.cuda.synchronize()
        for gr, st in zip(graphs, streams):
            with torch.cuda.stream(st):
                gr.replay()
        torch.cuda.synchronize()
        for step in steps:
            assert torch.equal(step.out, first["out"]) and torch.equal(step.lse, first["lse"])


def test_a_cache_past_32_bits():
    """pages more than 2^32 bytes into the pool"""
    page, H = 256, 8
    n = 2 ** 33 // (page * 72 * H)
    small = case(11, [600, 40], 16, H, page, 0, torch.bfloat16)
    pools = []
    ids = [n - 1 - 3 * i for i in range(small["k"].shape[0])]
    for name in ("k", "v"):
        pool = torch.zeros(n, H, page * 72, dtype=torch.uint8, device=DEV)
        pool[torch.tensor(ids, device=DEV)] = small[name]
        pools.append(pool)
    table = torch.where(small["table"] >= 0, i32(ids)[small["table"].clamp(min=0).long()], small["table"])
    want = decode(small)
    got = P.provip_decode_attention4(small["Q"], *pools, table, small["kv"], 600)
    assert torch.equal(want["out"], got["out"]) and torch.equal(want["lse"], got["lse"])


def test_a_step_copied_or_given_another_output():
    """outputs and workspace are those that the step has at the call"""
    c = case(12, [70, 300], 8, 2, 16, 40, torch.bfloat16)
    want = decode(c)
    step = P.DecodeAttention4(2, 8, 2, 300, 40, device=DEV)
    other = copy.deepcopy(step)
    del step
    r = other(c["Q"], c["k"], c["v"], c["table"], c["kv"], c["prefix_table"])
    assert torch.equal(r["out"], want["out"]) and torch.equal(r["lse"], want["lse"])
    other.out = torch.zeros_like(want["out"])
    assert torch.equal(other(c["Q"], c["k"], c["v"], c["table"], c["kv"], c["prefix_table"])["out"], want["out"])


@pytest.mark.parametrize("B,H_q,H_kv,most", [(15, 32, 32, 900), (33, 16, 16, 300), (130, 4, 4, 40), (512, 1, 1, 17), (513, 1, 1, 17), (129, 37, 1, 9)])
def test_more_units_than_run_at_once(B, H_q, H_kv, most):
    """requests of all lengths in any order, none and the longest among them, and one out of range"""
    rng = random.Random(B)
    lens = [rng.randint(0, most) for _ in range(B)]
    lens[B // 2], lens[B // 3], lens[0], lens[-1] = most, 0, most // 2, most
    c = case(B, lens, H_q, H_kv, 8)
    r = decode(c)
    check(c, r, rows=rng.sample(range(B), min(B, 30)) + [0, B // 3, B // 2, B - 1])
    for bad in (-1, most + 1, 2 ** 31 - 1, -2 ** 31):
        kv = c["kv"].clone()
        kv[3] = bad
        again = P.provip_decode_attention4(c["Q"], c["k"], c["v"], c["table"], kv, most)
        assert P.provip_device_status(clear=True)[1] == P.DEVSTAT_BAD_ARG
        assert not again["out"][3].any() and (again["lse"][3] == -math.inf).all()
        rest = [b for b in range(B) if b != 3]
        assert torch.equal(again["out"][rest], r["out"][rest]) and torch.equal(again["lse"][rest], r["lse"][rest])
