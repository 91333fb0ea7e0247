"""Norm and position rotation of queries and keys, and keys and values into pages on the way."""
import pytest
import torch

import cache4_ref as ref
from paper_2608_25332_gb300 import provip as P

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
EPS = 1e-6


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


def inputs(seed, T, H_q, H_kv, dtype, axes=1, far=4096, norm=True, fused=True):
    g = gen(seed)
    x = torch.randn(T, H_q + 2 * H_kv, 128, device=DEV, generator=g).to(dtype)
    Q, K, V = x.split([H_q, H_kv, H_kv], 1)
    if not fused:
        Q, K, V = Q.contiguous(), K.contiguous(), V.contiguous()
    pos = torch.randint(-far, far + 1, (axes, T), device=DEV, generator=g).to(torch.int32)
    w = (1 + 0.3 * torch.randn(2, 128, device=DEV, generator=g)).to(dtype)
    return Q, K, V, pos, (w[0] if norm else None, w[1] if norm else None)


def rotary(axes=1, base=10000.0, factor=1.0):
    return P.Rotary(sections=(16, 24, 24) if axes == 3 else None, base=base, factor=factor)


def near(got, x, pos, rot, w, what):
    want, size = ref.turn(x, pos, list(rot.inv_freq), list(rot.axis), w, EPS, rot.factor)
    bound = size + torch.finfo(got.dtype).eps / 2 * (want.abs() + size) + 1e-38
    err = (got.double() - want).abs()
    assert (err <= bound).all(), f"{what}: off by {float((err / bound).max()):.3g} of its bound"


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H_q,H_kv,axes,norm,fused", [
    (1, 1, 1, 1, True, True), (3, 28, 4, 3, True, True), (48, 32, 32, 1, False, True), (17, 5, 3, 3, False, False),
    (257, 40, 40, 1, True, True), (1000, 28, 4, 3, True, False), (2, 64, 1, 3, True, True), (1291, 17, 17, 1, True, True)])
def test_rotate(T, H_q, H_kv, axes, norm, fused, dtype):
    Q, K, _, pos, w = inputs(T + H_q, T, H_q, H_kv, dtype, axes, norm=norm, fused=fused)
    rot = rotary(axes)
    q, k = P.provip_rotate(Q, K, pos, rot, *w, EPS)
    near(q, Q, pos, rot, w[0], "Q")
    near(k, K, pos, rot, w[1], "K")


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_far_positions_and_odd_plans(dtype):
    """positions up to the type's ends, frequencies past a turn a position and negative ones, a factor"""
    Q, K, _, pos, w = inputs(3, 9, 4, 2, dtype, 2)
    pos[0] = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31, 10 ** 6, -10 ** 6 - 1, 123456789, 2 ** 30], dtype=torch.int32)
    freq = [(-1) ** i * 2.0 ** (-i / 2) for i in range(60)] + [0.0, 7.25, -12.5, 1e6]
    # (a double holds 2^31 f to 2^-22 of a radian: only frequencies it can hold times a position exactly)
    freq = [round(f * 2 ** 20) / 2 ** 20 for f in freq]
    rot = P.Rotary(freq, axis=[i % 2 for i in range(64)], factor=1.25)
    q, k = P.provip_rotate(Q, K, pos, rot, w[0], None, EPS)
    near(q, Q, pos, rot, w[0], "Q")
    near(k, K, pos, rot, None, "K")


def test_in_place_and_rows_behind_the_last():
    """outputs in the fused buffer itself; rows past the count stay as they were"""
    for n in (0, 1, 5, 12):
        Q, K, V, pos, w = inputs(n, 12, 6, 2, torch.bfloat16, 3)
        rot = rotary(3)
        want_q, want_k = P.provip_rotate(Q, K, pos, rot, *w, EPS)
        q0, k0, v0 = Q.clone(), K.clone(), V.clone()
        P.provip_rotate(Q, K, pos, rot, *w, EPS, out=(Q, K), n_rows=torch.tensor([n], dtype=torch.int32, device=DEV))
        assert torch.equal(Q, torch.cat([want_q[:n], q0[n:]])) and torch.equal(K, torch.cat([want_k[:n], k0[n:]]))
        assert torch.equal(V, v0)


def test_a_bad_count_is_reported():
    Q, K, _, pos, w = inputs(4, 6, 2, 2, torch.float32)
    for n, rows in ((-1, 0), (7, 6)):
        out = torch.zeros(2, 6, 2, 128, device=DEV)
        P.provip_rotate(Q, K, pos, rotary(), out=(out[0], out[1]), n_rows=torch.tensor([n], dtype=torch.int32, device=DEV))
        assert P.provip_device_status(clear=True)[1] == P.DEVSTAT_BAD_ARG
        assert bool((out[:, :rows] != 0).any(-1).all()) and not out[:, rows:].any()


def test_a_compactions_padded_positions():
    """[P, B, L] position ids with T = B L, as a compaction leaves them"""
    Q, K, _, pos, w = inputs(5, 3 * 7, 4, 2, torch.bfloat16, 3)
    rot = rotary(3)
    q, k = P.provip_rotate(Q, K, pos, rot, *w, EPS)
    q3, k3 = P.provip_rotate(Q, K, pos.view(3, 3, 7), rot, *w, EPS)
    assert torch.equal(q, q3) and torch.equal(k, k3)


def test_one_axis_of_many():
    """a model with one axis takes the first of three"""
    Q, K, _, pos, _ = inputs(6, 10, 4, 4, torch.float32, 3)
    a = P.provip_rotate(Q, K, pos, rotary(1))
    b = P.provip_rotate(Q, K, pos[:1].contiguous(), rotary(1))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_one_row_of_ids_for_every_axis():
    """text behind a video: the same position on all three axes, as a view without a copy"""
    Q, K, _, pos, w = inputs(14, 33, 6, 2, torch.bfloat16)
    a = P.provip_rotate(Q, K, pos.expand(3, 33), rotary(3), *w, EPS)
    b = P.provip_rotate(Q, K, pos.repeat(3, 1), rotary(3), *w, EPS)
    c = P.provip_rotate(Q, K, pos, rotary(1), *w, EPS)  # (and with the same frequencies)
    assert all(torch.equal(x, y) and torch.equal(x, z) for x, y, z in zip(a, b, c))


def test_values_that_are_not_finite_stay_in_their_head():
    Q, K, _, pos, w = inputs(7, 4, 6, 2, torch.bfloat16, fused=False)
    Q[1, 2, 5], Q[2, 3, 70], K[3, 1, 0] = float("nan"), float("inf"), -float("inf")
    rot = rotary()
    for norms in ((None, None), w):
        q, k = P.provip_rotate(Q, K, pos, rot, *norms, EPS)
        bad_q, bad_k = ~torch.isfinite(q).all(-1), ~torch.isfinite(k).all(-1)
        assert bad_q.nonzero().tolist() == [[1, 2], [2, 3]] and bad_k.nonzero().tolist() == [[3, 1]]


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H_q,H_kv,axes,page", [(1, 4, 4, 1, 8), (5, 28, 4, 3, 16), (256, 28, 4, 3, 16), (300, 32, 32, 1, 64),
                                                  (33, 10, 5, 1, 256)])
def test_append_on_the_way(T, H_q, H_kv, axes, page, dtype):
    """pages hold what rotating first and appending then gives, bit for bit; other slots stay"""
    Q, K, V, pos, w = inputs(T, T, H_q, H_kv, dtype, axes)
    rot, g = rotary(axes), gen(T)
    n = -(-T // page) + 1
    slot = torch.randperm(n * page, device=DEV, generator=g)[:T].to(torch.int32)
    slot[torch.rand(T, device=DEV, generator=g) < 0.2] = -1
    q, k = P.provip_rotate(Q, K, pos, rot, *w, EPS)
    blank = torch.randn(2, n, page, H_kv, 128, device=DEV, generator=g).to(dtype)
    want, got = blank.clone(), blank.clone()
    P.provip_kv_append(k, V, slot, want[0], want[1])
    for want_k in (False, True):
        got.copy_(blank)
        q2, k2 = P.provip_rotate_append(Q, K, V, pos, rot, slot, got[0], got[1], *w, EPS, want_k=want_k)
        assert torch.equal(q, q2) and torch.equal(want, got)
        assert torch.equal(k, k2) if want_k else k2 is None
    # and into 4 bits
    blank4 = torch.randint(0, 256, (2, n, H_kv, page * 72), device=DEV, generator=g, dtype=torch.uint8)
    want4, got4 = blank4.clone(), blank4.clone()
    P.provip_kv_append4(k, V, slot, want4[0], want4[1])
    q2, k2 = P.provip_rotate_append(Q, K, V, pos, rot, slot, got4[0], got4[1], *w, EPS, want_k=True)
    assert torch.equal(q, q2) and torch.equal(k, k2) and torch.equal(want4, got4)


def test_append_reports_slots_past_the_pool():
    Q, K, V, pos, w = inputs(8, 4, 4, 2, torch.bfloat16)
    pages = torch.zeros(2, 2, 8, 2, 128, dtype=torch.bfloat16, device=DEV)
    pages4 = torch.zeros(2, 2, 2, 8 * 72, dtype=torch.uint8, device=DEV)
    for pool in (pages, pages4):
        slot = torch.tensor([15, 16, -5, 2 ** 31 - 1], dtype=torch.int32, device=DEV)
        q, k = P.provip_rotate_append(Q, K, V, pos, rotary(), slot, pool[0], pool[1], want_k=True)
        assert P.provip_device_status(clear=True)[1] == P.DEVSTAT_BAD_ARG
        want = P.provip_rotate(Q, K, pos, rotary())
        assert torch.equal(q, want[0]) and torch.equal(k, want[1])
    assert torch.equal(pages[0, 1, 7], want[1][0]) and torch.equal(pages[1, 1, 7], V[0])
    assert int((pages != 0).any(-1).sum()) == 4


def test_rows_behind_the_last_stay_out_of_the_cache():
    Q, K, V, pos, _ = inputs(9, 6, 4, 2, torch.bfloat16)
    pages = torch.zeros(2, 1, 8, 2, 128, dtype=torch.bfloat16, device=DEV)
    slot = torch.arange(6, dtype=torch.int32, device=DEV)
    P.provip_rotate_append(Q, K, V, pos, rotary(), slot, pages[0], pages[1], n_rows=torch.tensor([2], dtype=torch.int32, device=DEV))
    assert pages[:, 0, :2].any(-1).all() and not pages[:, 0, 2:].any()


def test_captured_and_on_a_side_stream():
    """a graph of the call replays on new inputs; two streams work side by side"""
    Q, K, V, pos, w = inputs(10, 20, 8, 4, torch.bfloat16, 3)
    rot = rotary(3)
    pages = P.pages4(4, 8, 4, DEV), P.pages4(4, 8, 4, DEV)
    slot = torch.arange(20, dtype=torch.int32, device=DEV)
    out = (torch.empty(20, 8, 128, dtype=torch.bfloat16, device=DEV), None)
    side = torch.cuda.Stream(DEV)
    side.wait_stream(torch.cuda.current_stream(DEV))
    with torch.cuda.stream(side):
        P.provip_rotate_append(Q, K, V, pos, rot, slot, *pages, *w, EPS, out=out)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        P.provip_rotate_append(Q, K, V, pos, rot, slot, *pages, *w, EPS, out=out)
    for seed in (11, 12):
        Q2, K2, V2, pos2, _ = inputs(seed, 20, 8, 4, torch.bfloat16, 3)
        Q.copy_(Q2), K.copy_(K2), V.copy_(V2), pos.copy_(pos2)
        graph.replay()
        torch.cuda.synchronize()
        other = P.pages4(4, 8, 4, DEV), P.pages4(4, 8, 4, DEV)
        q, _ = P.provip_rotate_append(Q2, K2, V2, pos2, rot, slot, *other, *w, EPS)
        assert torch.equal(q, out[0]) and all(torch.equal(a, b) for a, b in zip(pages, other))


def test_offsets_past_32_bits():
    """rows and slots that lie more than 2^32 bytes into their tensors"""
    T, H = 3, 2
    big = torch.zeros(3, 2 ** 30 + 2 ** 27, dtype=torch.bfloat16, device=DEV)  # rows 2.25 GiB apart
    Q, K, V, pos, _ = inputs(13, T, H, H, torch.bfloat16, fused=False)
    rows = big.as_strided((T, H, 128), (big.stride(0), 128, 1))
    rows.copy_(Q)
    rot = rotary()
    want_q, want_k = P.provip_rotate(Q, K, pos, rot)
    q, k = P.provip_rotate(rows, K, pos, rot, out=(rows, torch.empty_like(K)))
    assert torch.equal(rows, want_q) and torch.equal(k, want_k)
    del big, rows, q
    page = 256
    n = 2 ** 33 // (page * 72 * 8)  # of 8 heads: 8 GiB
    pools = [torch.zeros(n, 8, page * 72, dtype=torch.uint8, device=DEV) for _ in range(2)]
    Q, K, V, pos, _ = inputs(14, T, 8, 8, torch.bfloat16)
    slot = torch.tensor([n * page - 1, 0, n * page // 2 + 77], dtype=torch.int32, device=DEV)
    P.provip_rotate_append(Q, K, V, pos, rot, slot, *pools)
    small = [torch.zeros(1, 8, page * 72, dtype=torch.uint8, device=DEV) for _ in range(2)]
    P.provip_rotate_append(Q, K, V, pos, rot, torch.arange(3, dtype=torch.int32, device=DEV), *small)
    a = P.provip_kv_read4(slot, *pools)
    b = P.provip_kv_read4(torch.arange(3, dtype=torch.int32, device=DEV), *small)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1]) and a[0].any() and a[1].any()
