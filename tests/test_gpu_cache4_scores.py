"""Decoding from 4-bit pages where scores leave the range of a float: keys out of sight at a list's front, and
products of queries and keys that pass the largest float before the scale brings them back."""
import pytest
import torch

import cache4_ref as ref
from paper_2608_25332_gb300 import provip as P
from test_gpu_cache4 import _lib, case, check, decode, rows_of  # noqa: F401 (_lib: this module's fixture too)

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
PAGE = 16


def first_value(pool, slots, d):
    """the rows' first group becomes (-8 d, 0, ..., 0)"""
    pg, row = slots // PAGE, slots % PAGE
    codes = pool[..., :PAGE * 64].unflatten(-1, (PAGE, 64))
    for g in range(8):  # values 4 g .. + 3: code 8 stands for 0
        codes[pg, :, row, 8 * g] = 0x88
        codes[pg, :, row, 8 * g + 1] = 0x88
    codes[pg, :, row, 0] = 0x80
    pool[..., PAGE * 64:].view(torch.bfloat16).unflatten(-1, (PAGE, 4))[pg, :, row, 0] = d


def prefix_slots(c):
    j = torch.arange(c["prefix"], device=DEV)
    return c["prefix_table"].long()[j // PAGE] * PAGE + j % PAGE


def own_slots(c):
    out = []
    for b, n in enumerate(c["lens"]):
        j = torch.arange(n, device=DEV)
        out.append(c["table"][b].long()[j // PAGE] * PAGE + j % PAGE)
    return torch.cat(out)


# (fp32 and few rows go one way, more than 16 bf16 rows a key/value head another; many heads make parts long)
@pytest.mark.parametrize("dtype,B,H_q,H_kv", [(torch.bfloat16, 17, 152, 152), (torch.bfloat16, 20, 76, 76), (torch.bfloat16, 40, 14, 2),
                                              (torch.bfloat16, 3, 76, 76), (torch.float32, 17, 76, 76)])
@pytest.mark.parametrize("hidden", [[(0, 128)], [(0, 256), (384, 512)], [(0, 640)], [(130, 600)]])
@pytest.mark.parametrize("level", [0.0, -250.0])
def test_keys_out_of_sight_at_the_front(dtype, B, H_q, H_kv, hidden, level):
    """Scores of -inf in fp32 (-2^99 times a scale of 2^36) beside ordinary ones, which count as ever: also where a
    part begins with a tile or more of the former. `level`: a common addend of all other scores, below which
    a weight against nothing would vanish."""
    c = case(H_q + len(hidden), [5] * B, H_q, H_kv, PAGE, 650, dtype, spread=2.0 ** -40)
    scale = 2.0 ** 40 / 11.3
    c["Q"][:, :, 0] = 1.0
    slots = prefix_slots(c)
    if level:
        first_value(c["k"], torch.cat([slots, own_slots(c)]), -level / 8 / scale)
    out = torch.zeros(650, dtype=torch.bool, device=DEV)
    for lo, hi in hidden:
        out[lo:hi] = True
    first_value(c["k"], slots[out], 2.0 ** 96)
    r = decode(c, scale=scale)
    seen = torch.cat([~out, torch.ones(5, dtype=torch.bool, device=DEV)])
    for b in (0, B - 1):
        K, V = rows_of(c, b)
        for h in range(0, H_q, 13):
            g = h // (H_q // H_kv)
            o, lse, bo, bl = ref.attend(c["Q"][b, h], K[seen, g], V[seen, g], scale, dtype)
            got, gl = r["out"][b, h].double(), r["lse"][b, h].double()
            assert ((got - o).abs() <= bo).all(), (b, h)
            assert abs(float(gl - lse)) <= bl, (b, h)


@pytest.mark.parametrize("dtype,lens", [(torch.bfloat16, [5] * 12), (torch.bfloat16, [40]), (torch.float32, [5] * 12)])
def test_products_past_the_largest_float(dtype, lens):
    """queries around 2^56 and keys around 2^70, whose products' sums pass 2^128, under a scale of 2^-122"""
    c = case(31, lens, 28, 4, PAGE, 300, dtype, spread=2.0 ** 70)
    c["Q"] *= 2.0 ** 56
    scale = 2.0 ** -122
    r = decode(c, scale=scale)
    for b in (0, len(lens) - 1):
        K, V = rows_of(c, b)
        for h in range(28):
            o, lse, bo, bl = ref.attend(c["Q"][b, h], K[:, h // 7], V[:, h // 7], scale, dtype)
            # Scores lie hundreds apart, and a weight below 2^-126 of the largest is no normal float: it may be zero,
            # by the exponential, by the factor of a raised maximum, and by that of the join. Here values are
            # around 2^70, so that is not below the bound's own 1e-30.
            bo = bo + 3 * 2.0 ** -126 * V[:, h // 7].abs().sum(0)
            got, gl = r["out"][b, h].double(), r["lse"][b, h].double()
            assert ((got - o).abs() <= bo).all(), (b, h)
            assert abs(float(gl - lse)) <= bl, (b, h)


def test_a_large_query_beside_small_ones():
    """rows of very different size in one call: each as it is by itself"""
    c = case(32, [5] * 12, 28, 4, PAGE, 300, torch.bfloat16)
    sizes = torch.tensor([1.0, 2.0 ** 18, 2.0 ** 19, 2.0 ** 20, 2.0 ** 21, 2.0 ** 60, 2.0 ** 90, 2.0 ** -90, 0.0, 2.0 ** -20, 1.5, 2.0 ** 33])
    for scale in (2.0 ** -21, 2.0 ** -40):
        for b, s in enumerate(sizes.tolist()):
            alone = dict(c, Q=c["Q"][b:b + 1] * s, table=c["table"][b:b + 1], kv=c["kv"][b:b + 1], lens=c["lens"][:1])
            check(alone, decode(alone, scale=scale), scale)
        all_of = dict(c, Q=(c["Q"].float() * sizes.to(DEV)[:, None, None]).to(torch.bfloat16))
        check(all_of, decode(all_of, scale=scale), scale)


@pytest.mark.parametrize("dtype,lens", [(torch.bfloat16, [5] * 12), (torch.bfloat16, [300]), (torch.float32, [5] * 12), (torch.float32, [300])])
@pytest.mark.parametrize("large", [2.0 ** 12, 2.0 ** 25])
def test_a_query_value_far_above_the_others(dtype, lens, large):
    """one that meets zeros in every key: scores are the others', each taken to 2^-39 of it"""
    c = case(33, lens, 28, 4, PAGE, 200, dtype)
    first_value(c["k"], torch.cat([prefix_slots(c), own_slots(c)]), 0.0)
    c["Q"][:, :, 5] = large
    scale = 1 / 11.3
    r = decode(c, scale=scale)
    for b in (0, len(lens) - 1):
        K, V = rows_of(c, b)
        for h in range(0, 28, 3):
            k, v = K[:, h // 7], V[:, h // 7]
            o, lse, bo, bl = ref.attend(c["Q"][b, h], k, v, scale, dtype)
            # a score is off by that much of each key's magnitudes more; it moves the output by twice as much of the mean of |v|
            e = float(k.abs().sum(1).max()) * scale * large * 2.0 ** -39
            p = torch.softmax(k @ c["Q"][b, h].double() * scale, 0)
            got, gl = r["out"][b, h].double(), r["lse"][b, h].double()
            assert ((got - o).abs() <= bo + 2 * e * (p @ v.abs())).all(), (b, h)
            assert abs(float(gl - lse)) <= bl + e, (b, h)
