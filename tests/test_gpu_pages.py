"""Block tables, slot maps and rows of the paged cache against plain Python."""
import random

import pytest
import torch

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


def i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def plain(kv, new, page, stack, table, T_max):
    """one step, request by request"""
    stack, table, kv_out = list(stack), [list(r) for r in table], []
    for b, n in enumerate(new):
        if n < 0:
            stack += table[b][:-(-kv[b] // page)]
    row, slots, shut = [0], [], False
    for b, n in enumerate(new):
        if n < 0:
            kv_out.append(0)
            row.append(row[-1])
            continue
        held, want = -(-kv[b] // page), -(-(kv[b] + n) // page)
        if want > held and (shut or want - held > len(stack)):
            shut = True
            kv_out.append(kv[b])
            slots += [-1] * n
        else:
            for i in range(held, want):
                table[b][i] = stack.pop()
            slots += [table[b][p // page] * page + p % page for p in range(kv[b], kv[b] + n)]
            kv_out.append(kv[b] + n)
        row.append(row[-1] + n)
    return kv_out, row, slots + [-1] * (T_max - len(slots)), stack, table


def one_step(rng, B, page, kv_hi, new_hi, ended, free, extra=0, inplace=False):
    kv = [rng.randint(0, kv_hi) for _ in range(B)]
    new = [-1 if ended and rng.randrange(ended) == 0 else rng.randint(0, new_hi) for _ in range(B)]
    held = [-(-k // page) for k in kv]
    width = max(-(-(k + max(n, 0)) // page) for k, n in zip(kv, new)) + 1
    ids = list(range(sum(held) + free))
    rng.shuffle(ids)
    table, at = [], 0
    for h in held:
        table.append(ids[at:at + h] + [-7] * (width - h))
        at += h
    T_max = sum(max(n, 0) for n in new) + extra
    want = plain(kv, new, page, ids[at:], table, T_max)
    stack = i32(ids[at:] + [-9] * (len(ids) - free + 1))
    d_kv, d_table, d_free = i32(kv), i32(table), i32([free])
    step = P.PageTables(B, page, T_max, DEV)
    r = step(d_kv, i32(new), stack, d_free, d_table, inplace=inplace)
    torch.cuda.synchronize()
    assert r["kv_len"].tolist() == want[0]
    assert r["row_start"].tolist() == want[1]
    assert r["slot_map"].tolist() == want[2]
    n = int(r["free_count"])
    assert n == len(want[3]) and stack[:n].tolist() == want[3]
    assert d_table.tolist() == want[4]
    if inplace:
        assert d_kv.tolist() == want[0] and int(d_free) == n
    else:
        assert d_kv.tolist() == kv and int(d_free) == free


@pytest.mark.parametrize("inplace", [False, True])
@pytest.mark.parametrize("B,page,kv_hi,new_hi,ended,free", [
    (1, 16, 0, 0, 0, 0), (1, 16, 0, 1, 0, 1), (1, 8, 100, 1, 0, 3), (1, 16, 50, 700, 0, 100), (5, 256, 1000, 1, 2, 4), (33, 16, 300, 1, 4, 40),
    (256, 16, 500, 1, 16, 300), (64, 64, 0, 1100, 0, 2000), (64, 64, 0, 1100, 0, 300), (64, 32, 200, 90, 3, 5), (64, 32, 200, 90, 0, 0),
    (1000, 16, 40, 3, 5, 100), (1024, 16, 40, 3, 5, 1000), (1025, 16, 40, 3, 5, 100), (2600, 8, 30, 20, 4, 3000), (2600, 8, 30, 20, 4, 2000),
    (7, 128, 3, 5000, 0, 500)])
def test_one_step(B, page, kv_hi, new_hi, ended, free, inplace):
    rng = random.Random(B * 1000 + page + kv_hi + new_hi + free)
    for extra in (0, 5):
        one_step(rng, B, page, kv_hi, new_hi, ended, free, extra, inplace)


def test_a_run_of_steps_conserves_the_pages():
    """60 steps in place: every page is held once or free, lengths and tables as planned"""
    rng = random.Random(7)
    B, page, pages, width = 40, 16, 120, 20
    ids = list(range(pages))
    rng.shuffle(ids)
    stack, free, table, kv = i32(ids), i32([pages]), torch.full((B, width), -1, dtype=torch.int32, device=DEV), i32([0] * B)
    h_stack, h_table, h_kv = list(ids), [[-1] * width for _ in range(B)], [0] * B
    step = P.PageTables(B, page, B * 30, DEV)
    for _ in range(60):
        new = [-1 if rng.random() < 0.08 else rng.choice([0, 1, 1, 1, 30]) for _ in range(B)]
        new = [min(n, width * page - k) for n, k in zip(new, h_kv)]
        h_kv, row, slots, h_stack, h_table = plain(h_kv, new, page, h_stack, h_table, B * 30)
        r = step(kv, i32(new), stack, free, table, inplace=True)
        torch.cuda.synchronize()
        assert r["slot_map"].tolist() == slots and r["row_start"].tolist() == row
        assert kv.tolist() == h_kv and int(free) == len(h_stack) and stack[:len(h_stack)].tolist() == h_stack
        held = [table[b, :-(-h_kv[b] // page)].tolist() for b in range(B)]
        assert sorted(sum(held, []) + h_stack) == list(range(pages))


def test_bad_requests_are_reported_and_left():
    page, width = 16, 4
    table = i32([[0, 1, -1, -1], [2, -1, -1, -1], [3, -1, -1, -1]])
    for kv, new in (([-5, 3, 3], [2, 2, 2]), ([30, 3, 3], [60, 2, 2]), ([100, 3, 3], [1, 2, 2]), ([100, 3, 3], [-1, 2, 2])):
        t = table.clone()
        step = P.PageTables(3, page, 70, DEV)
        r = step(i32(kv), i32(new), i32(list(range(4, 20))), i32([10]), t)
        torch.cuda.synchronize()
        rc, bits = P.provip_device_status(clear=True)
        assert rc == P.ERR_INVALID_ARG and bits == P.DEVSTAT_BAD_ARG, (kv, new)
        assert r["kv_len"].tolist()[1:] == [5, 5] and torch.equal(t, table)
        assert int(r["free_count"]) == 10
        n = max(new[0], 0)
        assert r["slot_map"].tolist() == [-1] * n + [35, 36, 51, 52] + [-1] * (66 - n)
    # more rows than T_max: the last request is left
    step = P.PageTables(3, page, 5, DEV)
    r = step(i32([3, 3, 3]), i32([2, 2, 2]), i32(list(range(4, 20))), i32([10]), table.clone())
    torch.cuda.synchronize()
    assert P.provip_device_status(clear=True) == (P.ERR_INVALID_ARG, P.DEVSTAT_BAD_ARG)
    assert r["kv_len"].tolist() == [5, 5, 3] and r["slot_map"].tolist() == [3, 4, 35, 36, -1]
    # a stack without room for what comes back
    step = P.PageTables(3, page, 5, DEV)
    r = step(i32([3, 3, 3]), i32([-1, -1, 0]), i32([9]), i32([0]), table.clone())
    torch.cuda.synchronize()
    assert P.provip_device_status(clear=True) == (P.ERR_INVALID_ARG, P.DEVSTAT_BAD_ARG)
    assert int(r["free_count"]) == 1


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("T,H,d,page", [(1, 1, 8, 16), (3, 4, 128, 16), (256, 4, 128, 16), (257, 32, 128, 64), (1000, 40, 128, 8), (77, 3, 64, 3), (5, 512, 128, 16)])
def test_append(T, H, d, page, dtype):
    g = torch.Generator(device=DEV).manual_seed(T)
    pages = -(-T // page) + 2
    buf = torch.randn(T, 2 * H + 4 * (8 // d if d < 8 else 1), d, generator=g, device=DEV).to(dtype)
    K, V = buf[:, :H], buf[:, H:2 * H]
    slot = torch.randperm(pages * page, generator=g, device=DEV)[:T].to(torch.int32)
    slot[::5] = -1
    kp, vp = (torch.full((pages, page, H, d), x, dtype=dtype, device=DEV) for x in (3.0, 4.0))
    wk, wv = kp.clone(), vp.clone()
    keep = slot >= 0
    wk.flatten(0, 1)[slot[keep].long()] = K[keep]
    wv.flatten(0, 1)[slot[keep].long()] = V[keep]
    P.provip_kv_append(K, V, slot, kp, vp)
    torch.cuda.synchronize()
    assert torch.equal(kp, wk) and torch.equal(vp, wv)
    # slots past the pool are reported and skipped
    slot[1::5] = pages * page + 3
    P.provip_kv_append(-K, -V, slot, kp, vp)
    torch.cuda.synchronize()
    if T > 1:
        assert P.provip_device_status(clear=True) == (P.ERR_INVALID_ARG, P.DEVSTAT_BAD_ARG)
    keep = (slot >= 0) & (slot < pages * page)
    wk.flatten(0, 1)[slot[keep].long()] = -K[keep]
    wv.flatten(0, 1)[slot[keep].long()] = -V[keep]
    assert torch.equal(kp, wk) and torch.equal(vp, wv)


def test_append_bits_and_nothing():
    """bytes are kept as they are (NaN payloads, -0), and no rows are no work"""
    bits = torch.randint(-2 ** 31, 2 ** 31 - 1, (50, 2, 128), dtype=torch.int32, device=DEV)
    K = bits.view(torch.float32)
    kp = torch.zeros(4, 16, 2, 128, device=DEV)
    vp = torch.zeros_like(kp)
    P.provip_kv_append(K, K, torch.arange(50, dtype=torch.int32, device=DEV), kp, vp)
    torch.cuda.synchronize()
    assert torch.equal(kp.view(torch.int32).flatten(0, 1)[:50], bits) and torch.equal(vp.view(torch.int32).flatten(0, 1)[:50], bits)
    P.provip_kv_append(K[:0], K[:0], torch.empty(0, dtype=torch.int32, device=DEV), kp, vp)


def test_append_past_2_31_elements():
    H, page = 32, 64
    pages = (1 << 31) // (H * 128 * page) + 4
    kp = torch.empty(pages, page, H, 128, dtype=torch.bfloat16, device=DEV)
    vp = torch.empty_like(kp)
    K = torch.randn(3, H, 128, device=DEV).to(torch.bfloat16)
    n = pages * page
    P.provip_kv_append(K, -K, i32([n - 1, 5, n - 70]), kp, vp)
    torch.cuda.synchronize()
    for i, s in enumerate((n - 1, 5, n - 70)):
        assert torch.equal(kp[s // page, s % page], K[i]) and torch.equal(vp[s // page, s % page], -K[i])
