"""Calls of the rotation and of the 4-bit cache as a serving program makes them: keys and values into pages from a fused
buffer that is rotated in place, a captured call whose count of rows changes, many ways of sharing pages."""
import pytest
import torch

import cache4_ref as ref
from paper_2608_25332_gb300 import provip as P
from test_gpu_cache4 import case, check, decode
from test_gpu_rotate import EPS, inputs, rotary

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


def pools(bits, n, page, H, dtype):
    if bits == 4:
        return P.pages4(n, page, H, DEV), P.pages4(n, page, H, DEV)
    return tuple(torch.zeros(n, page, H, 128, dtype=dtype, device=DEV) for _ in range(2))


@pytest.mark.parametrize("bits", [4, 16])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("T,H_q,H_kv,count", [(7, 4, 2, 5), (600, 28, 4, 600), (700, 9, 17, 1), (700, 9, 17, 0)])
def test_in_place_into_pages(T, H_q, H_kv, count, dtype, bits):
    """queries and keys rotated where they lie, beside the values that go with them; rows past the count stay, in the
    buffer and out of the pages"""
    Q, K, V, pos, w = inputs(T + bits, T, H_q, H_kv, dtype, 3)
    rot, page = rotary(3), 16
    n = -(-T // page)
    slot = torch.randperm(n * page, device=DEV, generator=torch.Generator(device=DEV).manual_seed(1))[:T].to(torch.int32)
    want_pools = pools(bits, n, page, H_kv, dtype)
    want_q, want_k = P.provip_rotate_append(Q[:count], K[:count], V[:count], pos[:, :count], rot, slot[:count], *want_pools, *w, EPS,
                                            want_k=True)
    q0, k0, v0, got = Q.clone(), K.clone(), V.clone(), pools(bits, n, page, H_kv, dtype)
    P.provip_rotate_append(Q, K, V, pos, rot, slot, *got, *w, EPS, out=(Q, K), n_rows=torch.tensor([count], dtype=torch.int32, device=DEV))
    assert torch.equal(Q, torch.cat([want_q, q0[count:]])) and torch.equal(K, torch.cat([want_k, k0[count:]])) and torch.equal(V, v0)
    assert all(torch.equal(a, b) for a, b in zip(got, want_pools))


def test_a_captured_call_takes_the_count_of_each_replay():
    T = 40
    Q, K, V, pos, w = inputs(2, T, 8, 4, torch.bfloat16, 3)
    rot, count = rotary(3), torch.tensor([3], dtype=torch.int32, device=DEV)
    slot = torch.arange(T, dtype=torch.int32, device=DEV)
    got, out = pools(4, 5, 8, 4, None), (torch.zeros(T, 8, 128, dtype=torch.bfloat16, device=DEV), None)
    call = lambda: P.provip_rotate_append(Q, K, V, pos, rot, slot, *got, *w, EPS, out=out, n_rows=count)
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    for n in (40, 0, 17):
        want_pools = pools(4, 5, 8, 4, None)
        want, _ = P.provip_rotate_append(Q[:n], K[:n], V[:n], pos[:, :n], rot, slot[:n], *want_pools, *w, EPS)
        count.fill_(n), out[0].zero_(), got[0].zero_(), got[1].zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out[0][:n], want) and not out[0][n:].any() and all(torch.equal(a, b) for a, b in zip(got, want_pools))


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_requests_that_share_pages(dtype):
    """several requests' tables name the same pages, and the prefix's among them"""
    c = case(3, [64, 40, 64, 17, 1], 8, 2, 16, 100, dtype)
    c["table"][1, :3], c["table"][3, :2], c["table"][2, 1] = c["table"][0, :3], c["table"][0, 1:3], c["prefix_table"][2]
    check(c, decode(c))


def test_no_rows():
    """calls without a row do nothing, and are no error"""
    Q, K, V, pos, w = inputs(4, 3, 4, 2, torch.bfloat16)
    none, got = torch.zeros(0, dtype=torch.int32, device=DEV), pools(4, 2, 8, 2, None)
    q, k = P.provip_rotate(Q[:0], K[:0], pos[:, :0], rotary(), *w, EPS)
    assert q.shape == (0, 4, 128) and k.shape == (0, 2, 128)
    P.provip_rotate_append(Q[:0], K[:0], V[:0], pos[:, :0], rotary(), none, *got, *w, EPS)
    P.provip_kv_append4(K[:0], V[:0], none, *got)
    k, v = P.provip_kv_read4(none, *got)
    assert k.shape == (0, 2, 128) and not got[0].any() and not got[1].any()
    assert torch.equal(ref.values(got[0], 8, torch.arange(16, device=DEV)), torch.zeros(16, 2, 128, dtype=torch.float64, device=DEV))
