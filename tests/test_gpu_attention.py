"""Attention over prompts and over the paged cache against the definition in 64 bits, at the
lengths, masks, layouts and values where it can go wrong (bounds: attention_ref.py)."""
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


def randn(g, *shape, dtype=F32):
    return torch.randn(*shape, generator=g, device=DEV).to(dtype)


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def starts(lens):
    out = [0]
    for x in lens:
        out.append(out[-1] + x)
    return out


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def tc(dtype, algo):
    return dtype == BF16 and algo != P.ALGO_SIMT


def run_prompt(seed, lq, lk, H_q, H_kv, prefix, causal, dtype, algo, scale=None, fused=False, gap=0, sink=True):
    """packed sequences, `gap` rows of NaN between them; checks every row"""
    g = gen(seed)
    B = len(lq)
    qs, ks = [x + gap * i for i, x in enumerate(starts(lq)[:-1])], [x + gap * i for i, x in enumerate(starts(lk)[:-1])]
    Tq, Tk = sum(lq) + gap * B, sum(lk) + gap * B
    Q, K, V = (randn(g, t, h, DH, dtype=dtype) for t, h in ((Tq, H_q), (Tk, H_kv), (Tk, H_kv)))
    if gap:
        for t, st, ln in ((Q, qs, lq), (K, ks, lk), (V, ks, lk)):
            live = torch.zeros(t.shape[0], dtype=torch.bool, device=DEV)
            for s, n in zip(st, ln):
                live[s:s + n] = True
            t[~live] = math.nan
    u = randn(g, H_kv, DH)
    u = u / u.norm(dim=1, keepdim=True)
    if sink:
        for s, n in zip(ks, lk):
            if n:
                K[s] = (8 * math.sqrt(DH) * u).to(dtype)
        Q += u.repeat_interleave(H_q // H_kv, 0).to(dtype)
    if fused:
        assert Tq == Tk
        buf = torch.cat([Q, K, V], 1)
        Q, K, V = buf.split([H_q, H_kv, H_kv], 1)
    Kp = Vp = None
    if prefix:
        Kp, Vp = randn(g, prefix, H_kv, DH, dtype=dtype), randn(g, prefix, H_kv, DH, dtype=dtype)
    step = P.PromptAttention(Tq, B, H_q, H_kv, max(lq), max(lk), prefix, causal, scale, dtype, DEV, algo)
    step.out.fill_(7.0)
    step.lse.fill_(7.0)
    r = step(Q, K, V, i32(qs), i32(lq), i32(ks), i32(lk), Kp, Vp)
    torch.cuda.synchronize()
    covered = torch.zeros(Tq, dtype=torch.bool, device=DEV)
    for b in range(B):
        rows, keys = slice(qs[b], qs[b] + lq[b]), slice(ks[b], ks[b] + lk[b])
        covered[rows] = True
        if lq[b] == 0:
            continue
        hid = hidden_mask(lq[b], lk[b], prefix, causal, DEV)
        for h in range(H_q):
            kv = h // (H_q // H_kv)
            k, v = K[keys, kv], V[keys, kv]
            if prefix:
                k, v = torch.cat([Kp[:, kv], k]), torch.cat([Vp[:, kv], v])
            ref = attend(Q[rows, h], k, v, hid, step.scale, dtype, tc(dtype, algo))
            check(r["out"][rows, h], r["lse"][rows, h], ref, f"sequence {b} head {h}")
    assert (r["out"][~covered] == 7).all() and (r["lse"][~covered] == 7).all(), "rows outside every sequence were written"
    return r


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
@pytest.mark.parametrize("lens", [[1], [2], [63], [64], [65], [127], [128], [129], [255], [256], [257], [511], [700], [3, 0, 200, 1, 64]],
                         ids=lambda v: "_".join(map(str, v)))
def test_whole_prompts(lens, dtype, algo):
    run_prompt(1, lens, lens, 4, 4, 0, True, dtype, algo, fused=True)


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
@pytest.mark.parametrize("H_q,H_kv", [(1, 1), (8, 4), (14, 2), (3, 1), (28, 4), (64, 1), (40, 40)])
def test_head_layouts(H_q, H_kv, dtype, algo):
    run_prompt(2, [150, 37], [150, 37], H_q, H_kv, 0, True, dtype, algo)


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lq,lk", [([1], [1000]), ([1], [1]), ([5, 130], [300, 131]), ([200], [60]), ([7], [0]), ([130, 1, 3], [0, 5, 2]),
                                   ([300], [301]), ([129, 64], [1400, 64])], ids=lambda v: "_".join(map(str, v)))
def test_rows_and_keys_of_other_numbers(lq, lk, causal, dtype, algo):
    """fewer keys than rows leave rows without a key (causal) and one key per sequence at the
    least; without keys every row is empty"""
    run_prompt(3, lq, lk, 6, 2, 0, causal, dtype, algo)


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
@pytest.mark.parametrize("prefix", [1, 64, 127, 128, 129, 1000])
def test_shared_prefix(prefix, dtype, algo):
    run_prompt(4, [40, 1, 0, 129], [40, 1, 0, 129], 14, 2, prefix, True, dtype, algo)


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
def test_prefix_alone(dtype, algo):
    run_prompt(5, [40, 3], [0, 0], 4, 2, 333, True, dtype, algo)


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
@pytest.mark.parametrize("prefix", [0, 70])
def test_padded_layout_with_nan_padding(prefix, dtype, algo):
    run_prompt(6, [100, 33, 128, 1], [100, 33, 200, 129], 7, 1, prefix, True, dtype, algo, gap=29)


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
def test_scale(dtype, algo):
    run_prompt(7, [90], [90], 2, 1, 0, True, dtype, algo, scale=0.5, sink=False)
    run_prompt(7, [90], [90], 2, 1, 0, True, dtype, algo, scale=1e-3, sink=False)


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
def test_long_and_many(dtype, algo):
    run_prompt(8, [2100], [2100], 2, 1, 0, True, dtype, algo)
    run_prompt(9, [40] * 37, [41] * 37, 4, 2, 0, True, dtype, algo)


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
@pytest.mark.parametrize("at", [0, 100, 140, 299])
def test_hidden_keys_may_hold_anything(at, dtype, algo):
    """NaN and infinities in key and value rows from `at` on touch no row before it"""
    g = gen(10)
    n, H = 300, 4
    Q, K, V = (randn(g, n, H, DH, dtype=dtype) for _ in range(3))
    one = lambda k, v: P.provip_prompt_attention(Q, k, v, i32([0]), i32([n]), i32([0]), i32([n]), n, n, algo=algo)
    a = one(K, V)
    K2, V2 = K.clone(), V.clone()
    K2[at:, 0], V2[at:, 0] = math.nan, math.nan
    V2[at:, 1] = math.inf
    K2[at:, 2] = math.inf
    V2[at:, 3, ::2] = -math.inf
    b = one(K2, V2)
    torch.cuda.synchronize()
    fine = b["out"][:at]
    assert torch.isfinite(fine).all() and torch.isfinite(b["lse"][:at]).all()
    for h in range(H):
        ref = attend(Q[:at, h], K[:at, h], V[:at, h], hidden_mask(at, at, 0, True, DEV), DH ** -0.5, dtype, tc(dtype, algo)) if at else None
        if ref:
            check(fine[:, h], b["lse"][:at, h], ref, f"head {h}")
    # the poisoned rows show it
    assert torch.isnan(b["out"][at:, 0]).all() and torch.isnan(b["lse"][at:, 0]).all()
    assert (b["out"][at:, 1] == math.inf).all()
    assert torch.isfinite(b["lse"][at:, 1]).all()
    assert (b["out"][at:, 3, ::2] == -math.inf).all() and torch.isfinite(b["out"][at:, 3, 1::2]).all()
    assert torch.isfinite(a["out"]).all()


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
def test_a_row_whose_scores_are_all_minus_infinity(dtype, algo):
    """0 / 0 of the formula, next to rows that are fine and to rows without a key"""
    n, H = 70, 1
    Q, K, V = torch.ones(n, H, DH, device=DEV), -torch.ones(n, H, DH, device=DEV), torch.ones(n, H, DH, device=DEV)
    Q[5] = math.inf
    Q, K, V = Q.to(dtype), K.to(dtype), V.to(dtype)
    r = P.provip_prompt_attention(Q, K, V, i32([0]), i32([n]), i32([0]), i32([n]), n, n, algo=algo)
    torch.cuda.synchronize()
    assert torch.isnan(r["out"][5]).all() and torch.isnan(r["lse"][5]).all()
    keep = torch.arange(n, device=DEV) != 5
    assert (r["out"][keep] == 1).all()


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
def test_rows_past_2_31_elements(dtype, algo):
    """key rows of one sequence start beyond the 32-bit offsets of the buffer"""
    g = gen(11)
    H, n = 32, 130
    rows = (1 << 31) // (H * DH) + 1000
    K = torch.empty(rows, H, DH, dtype=dtype, device=DEV)
    V = torch.empty(rows, H, DH, dtype=dtype, device=DEV)
    K[-n:], V[-n:] = randn(g, n, H, DH, dtype=dtype), randn(g, n, H, DH, dtype=dtype)
    Q = randn(g, n, H, DH, dtype=dtype)
    r = P.provip_prompt_attention(Q, K, V, i32([0]), i32([n]), i32([rows - n]), i32([n]), n, n, algo=algo)
    torch.cuda.synchronize()
    for h in (0, 31):
        ref = attend(Q[:, h], K[-n:, h], V[-n:, h], hidden_mask(n, n, 0, True, DEV), DH ** -0.5, dtype, tc(dtype, algo))
        check(r["out"][:, h], r["lse"][:, h], ref, f"head {h}")


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
def test_bad_lengths_are_reported_and_skipped(dtype, algo):
    g = gen(12)
    Q, K, V = (randn(g, 100, 2, DH, dtype=dtype) for _ in range(3))
    for qs, ql, ks, kl in ([-1, 40, 0, 40], [0, 51, 0, 40], [60, 41, 0, 40], [0, 40, -3, 40], [0, 40, 70, 40], [0, 40, 0, -1],
                           [0, -2, 0, 40], [0, 40, 0, 51]):
        step = P.PromptAttention(100, 2, 2, 2, 50, 50, dtype=dtype, device=DEV, algo=algo)
        step.out.fill_(7.0)
        r = step(Q, K, V, i32([qs, 90]), i32([ql, 10]), i32([ks, 50]), i32([kl, 50]))
        torch.cuda.synchronize()
        rc, bits = P.provip_device_status(clear=True)
        assert rc == P.ERR_INVALID_ARG and bits == P.DEVSTAT_BAD_ARG, (qs, ql, ks, kl)
        assert (r["out"][:90] == 7).all()
        ref = attend(Q[90:, 0], K[50:, 0], V[50:, 0], hidden_mask(10, 50, 0, True, DEV), DH ** -0.5, dtype, tc(dtype, algo))
        check(r["out"][90:, 0], r["lse"][90:, 0], ref, "the good sequence")


# ---------------------------------------------------------------------------
# paged cache
# ---------------------------------------------------------------------------
def run_decode(seed, lens, H_q, H_kv, prefix, page, dtype, algo, kv_max=None, check_heads=None, spare=3, top=False):
    g = gen(seed)
    B = len(lens)
    held, pre = [-(-n // page) for n in lens], -(-prefix // page)
    pages = sum(held) + pre + spare
    order = torch.randperm(pages, generator=g, device=DEV).to(torch.int32)
    if top:  # the pages in use are the pool's last
        order = torch.arange(pages - 1, -1, -1, device=DEV, dtype=torch.int32)
    pool = torch.full((2, pages, page, H_kv, DH), math.nan, dtype=dtype, device=DEV) if not top else \
        torch.empty((2, pages, page, H_kv, DH), dtype=dtype, device=DEV)
    prefix_table = order[:pre].clone()
    width = max(max(held), -(-(kv_max or 1) // page)) + 2
    table = torch.full((B, width), -1, dtype=torch.int32, device=DEV)
    at = pre
    seqs = []
    u = randn(g, H_kv, DH)
    u = u / u.norm(dim=1, keepdim=True)

    def fill(tab, n, sink):
        kv = randn(g, 2, n, H_kv, DH, dtype=dtype)
        if sink and n:
            kv[0, 0] = (8 * math.sqrt(DH) * u).to(dtype)
        j = torch.arange(n, device=DEV)
        for i in range(2):
            pool[i, tab.long()[j // page], j % page] = kv[i]
        return kv

    pk = fill(prefix_table, prefix, True)
    for b, n in enumerate(lens):
        table[b, :held[b]] = order[at:at + held[b]]
        at += held[b]
        seqs.append(fill(table[b], n, prefix == 0))
    Q = randn(g, B, H_q + 2, DH, dtype=dtype)[:, 1:-1]  # a slice: rows further apart
    Q += u.repeat_interleave(H_q // H_kv, 0).to(dtype)
    step = P.DecodeAttention(B, H_q, H_kv, max(lens) if kv_max is None else kv_max, prefix, None, dtype, DEV, algo)
    r = step(Q, pool[0], pool[1], table, i32(lens), prefix_table if prefix else None)
    torch.cuda.synchronize()
    for b in range(B):
        for h in check_heads or range(H_q):
            kv = h // (H_q // H_kv)
            k, v = (torch.cat([pk[i][:, kv], seqs[b][i][:, kv]]) for i in range(2))
            ref = attend(Q[b:b + 1, h], k, v, torch.zeros(1, len(k), dtype=torch.bool, device=DEV), DH ** -0.5, dtype, tc(dtype, algo))
            check(r["out"][b:b + 1, h], r["lse"][b:b + 1, h], ref, f"request {b} head {h}")
    return step, (Q, pool[0], pool[1], table, i32(lens), prefix_table if prefix else None)


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
@pytest.mark.parametrize("page", [8, 16, 32, 64, 128, 256])
def test_decode_pages(page, dtype, algo):
    lens = [0, 1, page - 1, page, page + 1, 127, 128, 129, 400]
    run_decode(20, lens, 4, 2, 0, page, dtype, algo)
    run_decode(21, lens, 4, 2, page + 3, page, dtype, algo)


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
@pytest.mark.parametrize("prefix", [0, 1, 64, 130, 1000])
@pytest.mark.parametrize("H_q,H_kv", [(1, 1), (32, 32), (28, 4), (6, 3), (10, 2), (16, 1), (64, 1)])
def test_decode_heads_and_prefix(H_q, H_kv, prefix, dtype, algo):
    run_decode(22, [0, 3, 70, 260], H_q, H_kv, prefix, 16, dtype, algo)


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
def test_decode_one_request(dtype, algo):
    run_decode(23, [1], 4, 4, 0, 16, dtype, algo)
    run_decode(24, [3000], 4, 4, 0, 16, dtype, algo)
    run_decode(25, [0], 4, 4, 500, 64, dtype, algo)
    run_decode(26, [0], 4, 4, 0, 64, dtype, algo)


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
def test_decode_many_requests(dtype, algo):
    """more rows of a group than a tile has, lengths far below the host's bound"""
    run_decode(27, [(37 * i) % 90 for i in range(150)], 6, 2, 200, 16, dtype, algo, kv_max=100, check_heads=[0, 5])
    run_decode(28, [(37 * i) % 300 for i in range(70)], 4, 4, 0, 32, dtype, algo, check_heads=[3])


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
def test_decode_past_2_31_elements(dtype, algo):
    H, page = 32, 64
    run_decode(29, [130, 40], H, H, 70, page, dtype, algo, spare=(1 << 31) // (H * DH * page) + 10, top=True, check_heads=[0, 31])


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
def test_decode_reports_bad_lengths_and_pages(dtype, algo):
    step, args = run_decode(30, [100, 33], 4, 2, 0, 16, dtype, algo)
    good = [step(*args)[k].clone() for k in ("out", "lse")]
    Q, k, v, table, kv_len, _ = args
    for bad in (-1, 101):
        r = step(Q, k, v, table, i32([bad, 33]))
        torch.cuda.synchronize()
        rc, bits = P.provip_device_status(clear=True)
        assert rc == P.ERR_INVALID_ARG and bits == P.DEVSTAT_BAD_ARG
        assert torch.equal(r["out"][1], good[0][1]) and (r["out"][0] == 0).all() and (r["lse"][0] == -math.inf).all()
    for page in (-1, 1 << 30, k.shape[0]):
        t = table.clone()
        t[0, 2] = page
        r = step(Q, k, v, t, kv_len)
        torch.cuda.synchronize()
        rc, bits = P.provip_device_status(clear=True)
        assert rc == P.ERR_INVALID_ARG and bits == P.DEVSTAT_BAD_ARG, page
        assert torch.equal(r["out"][1], good[0][1])


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
def test_decode_unseen_slots_may_change(dtype, algo):
    """slots past a length do not reach the result (the pool starts as NaN; here they change)"""
    step, args = run_decode(31, [65, 3], 4, 4, 21, 16, dtype, algo)
    Q, k, v, table, kv_len, pt = args
    a = {x: y.clone() for x, y in step(*args).items()}
    k2, v2 = k.clone(), v.clone()
    k2[torch.isnan(k2)] = math.inf
    v2[torch.isnan(v2)] = -math.inf
    b = step(Q, k2, v2, table, kv_len, pt)
    torch.cuda.synchronize()
    assert torch.equal(a["out"], b["out"]) and torch.equal(a["lse"], b["lse"])


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
def test_streams_and_graphs(dtype, algo):
    """another stream than the default, and a captured call whose inputs change between replays"""
    step, args = run_decode(32, [200, 17, 90], 8, 2, 150, 16, dtype, algo)
    Q, k, v, table, kv_len, pt = args
    want = [{x: y.clone() for x, y in step(q, k, v, table, n, pt).items()} for q, n in ((Q, kv_len), (-Q, kv_len // 2))]
    s = torch.cuda.Stream(DEV)
    q, n = Q.clone(), kv_len.clone()
    torch.cuda.synchronize()
    with torch.cuda.stream(s):
        r = step(q, k, v, table, n, pt)
        assert torch.equal(r["out"], want[0]["out"])
        step.out.zero_()
    s.synchronize()
    gr = torch.cuda.CUDAGraph()
    with torch.cuda.graph(gr):
        r = step(q, k, v, table, n, pt)
    for i, (qq, nn) in enumerate(((Q, kv_len), (-Q, kv_len // 2), (Q, kv_len))):
        q.copy_(qq)
        n.copy_(nn)
        gr.replay()
        torch.cuda.synchronize()
        assert torch.equal(r["out"], want[i % 2]["out"]) and torch.equal(r["lse"], want[i % 2]["lse"])


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
def test_the_same_call_gives_the_same_bits(dtype, algo):
    g = gen(33)
    Q, K, V = (randn(g, 900, 6, DH, dtype=dtype) for _ in range(3))
    a = (i32([0, 500]), i32([500, 400]), i32([0, 500]), i32([500, 400]))
    x, y = (P.provip_prompt_attention(Q, K, V, *a, 500, 500, algo=algo) for _ in range(2))
    assert torch.equal(x["out"], y["out"]) and torch.equal(x["lse"], y["lse"])


@pytest.mark.parametrize("dtype", [F32, BF16])
def test_without_lse(dtype):
    g = gen(34)
    Q, K, V = (randn(g, 64, 2, DH, dtype=dtype) for _ in range(3))
    a = (Q, K, V, i32([0]), i32([64]), i32([0]), i32([64]), 64, 64)
    x, y = P.provip_prompt_attention(*a), P.provip_prompt_attention(*a, want_lse=False)
    assert y["lse"] is None and torch.equal(x["out"], y["out"])


# ---------------------------------------------------------------------------
# sizes at which the work is cut up differently
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
def test_more_sequences_than_the_lanes_hold(dtype, algo):
    """600 sequences (256 at a time are walked through), some without rows"""
    lens = [(7 * i) % 5 + (130 if i in (3, 299, 599) else 0) for i in range(600)]
    run_prompt(40, lens, lens, 2, 1, 0, True, dtype, algo)


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
@pytest.mark.parametrize("rows", [3, 300])
def test_bounds_far_above_the_lengths(rows, dtype, algo):
    """host bounds that promise long keys: most parts of a row are empty"""
    g = gen(41)
    H_q, H_kv, Tk = 4, 2, 200000
    K, V = (torch.full((Tk, H_kv, DH), math.nan, dtype=dtype, device=DEV) for _ in range(2))
    lens, starts_ = [rows, 77 + rows], [5, 100000]
    for s, n in zip(starts_, lens):
        K[s:s + n], V[s:s + n] = randn(g, n, H_kv, DH, dtype=dtype), randn(g, n, H_kv, DH, dtype=dtype)
    Q = randn(g, 2 * rows, H_q, DH, dtype=dtype)
    r = P.provip_prompt_attention(Q, K, V, i32([0, rows]), i32([rows, rows]), i32(starts_), i32(lens), rows, Tk, algo=algo)
    torch.cuda.synchronize()
    for b in range(2):
        for h in range(H_q):
            k, v = (x[starts_[b]:starts_[b] + lens[b], h // 2] for x in (K, V))
            ref = attend(Q[b * rows:(b + 1) * rows, h], k, v, hidden_mask(rows, lens[b], 0, True, DEV), DH ** -0.5, dtype, tc(dtype, algo))
            check(r["out"][b * rows:(b + 1) * rows, h], r["lse"][b * rows:(b + 1) * rows, h], ref, f"sequence {b} head {h}")


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
def test_values_that_grow_along_the_keys(dtype, algo):
    """the running maximum rises many times, by more than any lag: every tile rescales"""
    g = gen(42)
    n = 1500
    Q, K, V = (randn(g, n, 2, DH, dtype=dtype) for _ in range(3))
    q, k = Q.float(), K.float()
    q[..., 0], k[..., 0] = 4.0, torch.arange(n, device=DEV)[:, None] * 0.25  # logits up to 130 above the first
    Q, K = q.to(dtype), k.to(dtype)
    r = P.provip_prompt_attention(Q, K, V, i32([0]), i32([n]), i32([0]), i32([n]), n, n, algo=algo)
    torch.cuda.synchronize()
    for h in range(2):
        ref = attend(Q[:, h], K[:, h], V[:, h], hidden_mask(n, n, 0, True, DEV), DH ** -0.5, dtype, tc(dtype, algo))
        check(r["out"][:, h], r["lse"][:, h], ref, f"head {h}")


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
def test_decode_values_that_grow_along_the_keys(dtype, algo):
    g = gen(43)
    n, page, H = 1100, 16, 2
    pages = -(-n // page)
    K, V = randn(g, pages, page, H, DH, dtype=dtype), randn(g, pages, page, H, DH, dtype=dtype)
    k = K.float().reshape(-1, H, DH)
    k[..., 0] = torch.arange(pages * page, device=DEV)[:, None] * 0.25
    K = k.to(dtype).reshape(pages, page, H, DH)
    Q = randn(g, 1, 4, DH, dtype=dtype)
    Q[..., 0] = 4.0
    table = torch.arange(pages, dtype=torch.int32, device=DEV)[None]
    r = P.provip_decode_attention(Q, K, V, table, i32([n]), n, algo=algo)
    torch.cuda.synchronize()
    for h in range(4):
        kk, vv = (x.reshape(-1, H, DH)[:n, h // 2] for x in (K, V))
        ref = attend(Q[:, h], kk, vv, torch.zeros(1, n, dtype=torch.bool, device=DEV), DH ** -0.5, dtype, tc(dtype, algo))
        check(r["out"][:, h], r["lse"][:, h], ref, f"head {h}")


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
@pytest.mark.parametrize("power", [10, 14, 15, 16, 20, 30, 50])
def test_scores_of_any_size(power, dtype, algo):
    """Scores of 2^(2 power) and more, all exact and far apart, where a rounding of the maximum is
    worth many powers of two: the weight lies on the keys that share the largest. (How evenly is
    not said: parts are joined by log-sum-exps in 32 bits, whose last place is worth more than the
    parts' numbers of such keys.)"""
    g = gen(49)
    n, page, H = 400, 16, 2
    pages = n // page
    c = torch.arange(n, device=DEV) % 7 + 1
    c[::3] = 1 + torch.arange(len(c[::3]), device=DEV) // 60
    K = torch.zeros(pages, page, H, DH, dtype=dtype, device=DEV)
    K.view(n, H, DH)[..., 0] = (c * 2.0 ** power).to(dtype)[:, None]
    V = randn(g, pages, page, H, DH, dtype=dtype)
    Q = torch.zeros(4, 4, DH, dtype=dtype, device=DEV)
    Q[..., 0] = 2.0 ** power
    Q[2:, :, 0] = -(2.0 ** power)  # these rows' largest is that of c = 1
    args = (K.view(n, H, DH), V.view(n, H, DH))
    whole = P.provip_prompt_attention(Q, *args, i32([0]), i32([4]), i32([0]), i32([n]), 4, n, causal=False, algo=algo)
    table = torch.arange(pages, dtype=torch.int32, device=DEV)[None].expand(4, -1).contiguous()
    step = P.provip_decode_attention(Q, K, V, table, i32([n] * 4), n, algo=algo)
    torch.cuda.synchronize()
    for r in (whole, step):
        for t in range(4):
            top = c == (c.max() if t < 2 else c.min())
            x = (1 if t < 2 else -1) * float(c[top][0]) * 2.0 ** (2 * power) * DH ** -0.5
            for h in range(4):
                v = args[1][top, h // 2].double()
                # a mean of them, with bf16 weights and a bf16 output
                o, slack = r["out"][t, h].double(), 2.0 ** -7 * v.abs().amax(0) + 2.0 ** -12
                assert ((o >= v.amin(0) - slack) & (o <= v.amax(0) + slack)).all(), (t, h)
                lse = x + math.log(int(top.sum()))
                assert abs(float(r["lse"][t, h]) - lse) <= abs(lse) * 2.0 ** -21, (t, h)


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
@pytest.mark.parametrize("prefix", [0, 64])
def test_decode_first_scores_minus_infinity(prefix, dtype, algo):
    """the first tiles have no weight, and the scores behind them lie where 2^score underflows"""
    g = gen(48)
    n, page, H = 700, 16, 2
    pages = -(-n // page)
    K, V = randn(g, pages, page, H, DH, dtype=dtype), randn(g, pages, page, H, DH, dtype=dtype)
    k = K.reshape(-1, H, DH)
    k[..., 0] = -2000.0
    k[:prefix + 300, :, 0] = -math.inf
    Q = randn(g, 1, 4, DH, dtype=dtype)
    Q[..., 0] = 4.0
    table = torch.arange(pages, dtype=torch.int32, device=DEV)
    kw = dict(algo=algo, prefix_table=table[:prefix // page], prefix_len=prefix) if prefix else dict(algo=algo)
    r = P.provip_decode_attention(Q, K, V, table[None, prefix // page:].contiguous(), i32([n - prefix]), n - prefix, **kw)
    torch.cuda.synchronize()
    for h in range(4):
        kk, vv = (x.reshape(-1, H, DH)[prefix + 300:n, h // 2] for x in (K, V))  # the keys that have a weight
        ref = attend(Q[:, h], kk, vv, torch.zeros(1, len(kk), dtype=torch.bool, device=DEV), DH ** -0.5, dtype, tc(dtype, algo))
        check(r["out"][:, h], r["lse"][:, h], ref, f"head {h}")


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
def test_decode_more_requests_than_the_lanes_hold(dtype, algo):
    run_decode(44, [(13 * i) % 40 + (700 if i % 211 == 5 else 0) for i in range(700)], 2, 1, 0, 16, dtype, algo, check_heads=[1])
    run_decode(45, [(13 * i) % 40 for i in range(300)], 3, 1, 50, 8, dtype, algo, kv_max=2000, check_heads=[2])


@pytest.mark.parametrize("lens", [[300], [1500, 20, 700], [129] * 40, [1, 2000]], ids=lambda v: "_".join(map(str, v[:4])))
def test_decode_bits_stay(lens):
    """twenty calls in a row, nothing waiting between them: units of several tiles, and units
    that the CTAs' spans cut"""
    step, args = run_decode(46, lens, 4, 4, 0, 16, BF16, P.ALGO_AUTO, check_heads=[0])
    want = {k: v.clone() for k, v in step(*args).items()}
    got = []
    for _ in range(20):
        r = step(*args)
        got.append((r["out"].clone(), r["lse"].clone()))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want["out"]) and torch.equal(l, want["lse"]) for o, l in got)


@pytest.mark.parametrize("dtype,algo", FORMS, ids=IDS)
@pytest.mark.parametrize("pad", [0, 8, 24])
def test_guard_bytes_and_row_strides(pad, dtype, algo):
    """outputs with rows further apart (16-byte, not 32-byte multiples among them) and the
    workspace inside red zones; what lies between and around the rows stays"""
    import ctypes
    g = gen(47)
    L = P.lib()
    dt = P._dtype_of(dtype)
    H_q, H_kv, lens = 6, 2, [130, 0, 7]
    T = sum(lens)
    Q, K, V = (randn(g, T, h, DH, dtype=dtype) for h in (H_q, H_kv, H_kv))
    st, ln = i32(starts(lens)[:-1]), i32(lens)
    want = P.provip_prompt_attention(Q, K, V, st, ln, st, ln, 130, 130, algo=algo)
    stride, zone = H_q * DH + pad, 512
    buf = torch.full((zone + T * stride + zone,), 3.0, dtype=dtype, device=DEV)
    lse = torch.full((zone + T * H_q + zone,), 3.0, device=DEV)
    need = L.provip_prompt_attention_workspace_size(T, 3, H_q, H_kv, 130, 130, 0, dt, algo)
    ws = torch.full((need + 2048,), 0xA5, dtype=torch.uint8, device=DEV)
    at = lambda t, n: ctypes.c_void_p(t.data_ptr() + n * t.element_size())
    rc = L.provip_prompt_attention(Q.data_ptr(), H_q * DH, K.data_ptr(), H_kv * DH, V.data_ptr(), H_kv * DH, T, T, 3, H_q, H_kv, DH,
                                   st.data_ptr(), ln.data_ptr(), st.data_ptr(), ln.data_ptr(), 130, 130, None, 0, None, 0, 0, 1,
                                   DH ** -0.5, dt, algo, at(buf, zone), stride, at(lse, zone), at(ws, 1024), need,
                                   P._stream(torch.device(DEV)))
    torch.cuda.synchronize()
    assert rc == 0
    rows = buf[zone:zone + T * stride].view(T, stride)
    assert torch.equal(rows[:, :H_q * DH].reshape(T, H_q, DH), want["out"]) and (rows[:, H_q * DH:] == 3).all()
    assert (buf[:zone] == 3).all() and (buf[-zone:] == 3).all()
    assert torch.equal(lse[zone:-zone].view(T, H_q), want["lse"]) and (lse[:zone] == 3).all() and (lse[-zone:] == 3).all()
    assert (ws[:1024] == 0xA5).all() and (ws[1024 + need:] == 0xA5).all()
    # decoding
    page, B = 16, 3
    kp, vp = randn(g, 40, page, H_kv, DH, dtype=dtype), randn(g, 40, page, H_kv, DH, dtype=dtype)
    table, kl = torch.arange(30, dtype=torch.int32, device=DEV).view(B, 10), i32([160, 0, 33])
    pt = torch.arange(30, 40, dtype=torch.int32, device=DEV)
    Qd = randn(g, B, H_q, DH, dtype=dtype)
    for prefix in (0, 150):
        want = P.provip_decode_attention(Qd, kp, vp, table, kl, 160, pt if prefix else None, prefix, algo=algo)
        need = L.provip_decode_attention_workspace_size(B, H_q, H_kv, 160, prefix, dt, algo)
        buf.fill_(3.0)
        lse.fill_(3.0)
        ws = torch.full((need + 2048,), 0xA5, dtype=torch.uint8, device=DEV)
        rc = L.provip_decode_attention(Qd.data_ptr(), H_q * DH, B, H_q, H_kv, DH, kp.data_ptr(), vp.data_ptr(), 40, page, table.data_ptr(), 10,
                                       kl.data_ptr(), 160, pt.data_ptr() if prefix else None, prefix, DH ** -0.5, dt, algo, at(buf, zone),
                                       stride, at(lse, zone), at(ws, 1024), need, P._stream(torch.device(DEV)))
        torch.cuda.synchronize()
        assert rc == 0
        rows = buf[zone:zone + B * stride].view(B, stride)
        assert torch.equal(rows[:, :H_q * DH].reshape(B, H_q, DH), want["out"]) and (rows[:, H_q * DH:] == 3).all()
        assert (buf[:zone] == 3).all() and (buf[zone + B * stride:] == 3).all()
        assert torch.equal(lse[zone:zone + B * H_q].view(B, H_q), want["lse"]) and (lse[zone + B * H_q:] == 3).all()
        assert (ws[:1024] == 0xA5).all() and (ws[1024 + need:] == 0xA5).all()
