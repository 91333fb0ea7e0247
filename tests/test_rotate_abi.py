"""Refusals of the rotation's and the 4-bit cache's calls (CPU: all of them come before any CUDA call)."""
import copy
import ctypes
import math
import pickle

import pytest
import torch

from paper_2608_25332_gb300 import build as pbuild

FAKE = 0x10000  # never dereferenced
OFF = 0x10008


@pytest.fixture(scope="module")
def L():
    pbuild.build()
    from paper_2608_25332_gb300 import provip
    return provip.lib()


def freq(at=None, value=0.0):
    return (ctypes.c_double * 64)(*[value if i == at else 1.0 for i in range(64)])


def axis(value):
    return (ctypes.c_int * 64)(*[value] * 64)


def rotate(L, **kw):
    a = dict(Q=FAKE, qs=1024, K=FAKE * 2, ks=512, T=5, n=None, H_q=8, H_kv=4, d_h=128, pos=FAKE, ps=5, axes=3, freq=freq(), axis=None,
             factor=1.0, wq=None, wk=None, eps=1e-6, dtype=1, qo=FAKE * 3, qos=1024, ko=FAKE * 4, kos=512)
    a.update(kw)
    return L.provip_rotate(*a.values(), None)


COMMON_BAD = [dict(Q=None), dict(K=None), dict(qo=None), dict(pos=None), dict(freq=None), dict(T=-1), dict(H_q=0), dict(H_kv=0), dict(qs=1000),
              dict(ks=500), dict(qos=8), dict(axes=0), dict(axes=300), dict(ps=4), dict(ps=-1, axes=1), dict(freq=freq(7, math.nan)),
              dict(freq=freq(63, math.inf)), dict(freq=freq(0, -1.1e6)), dict(axis=axis(3)), dict(axis=axis(-1)), dict(factor=math.nan),
              dict(factor=math.inf), dict(wq=FAKE, eps=-1.0), dict(wk=FAKE, eps=math.nan), dict(qo=FAKE, qos=1032)]
COMMON_UNSUPPORTED = [dict(d_h=64), dict(dtype=2), dict(Q=OFF), dict(K=OFF), dict(qo=OFF), dict(ko=OFF), dict(qs=1028), dict(kos=516), dict(wq=OFF),
                      dict(wk=OFF), dict(T=2 ** 31 - 1, ps=2 ** 31 - 1)]


def test_rotate_refusals(L):
    for bad in COMMON_BAD + [dict(ko=None), dict(kos=100), dict(ko=FAKE * 2, kos=520)]:
        assert rotate(L, **bad) == -1, bad
        assert b"rotate" in L.provip_last_error()
    for bad in COMMON_UNSUPPORTED:
        assert rotate(L, **bad) == -2, bad
    assert rotate(L, T=0) == 0


def append(L, **kw):
    a = dict(Q=FAKE, qs=1024, K=FAKE * 2, ks=512, V=FAKE, vs=512, T=5, n=None, H_q=8, H_kv=4, d_h=128, pos=FAKE, ps=5, axes=3, freq=freq(),
             axis=None, factor=1.0, wq=None, wk=None, eps=1e-6, dtype=1, qo=FAKE * 3, qos=1024, ko=None, kos=512, slot=FAKE, n_pages=4, page=16,
             four=0, kp=FAKE, vp=FAKE)
    a.update(kw)
    return L.provip_rotate_append(*a.values(), None)


def test_append_refusals(L):
    for four in (0, 1):
        for bad in COMMON_BAD + [dict(V=None), dict(vs=8), dict(slot=None), dict(kp=None), dict(vp=None), dict(n_pages=0), dict(four=2),
                                 dict(ko=FAKE * 2, kos=520)]:
            assert append(L, **{"four": four, **bad}) == -1, bad
        for bad in COMMON_UNSUPPORTED[:-1] + [dict(V=OFF), dict(vs=516), dict(page=12), dict(page=4), dict(page=512), dict(kp=OFF), dict(vp=OFF),
                                              dict(n_pages=2 ** 30)]:
            if bad != dict(kos=516):
                assert append(L, **{"four": four, **bad}) == -2, bad
        assert append(L, T=0, four=four) == 0


def test_rows_refusals(L):
    ap = lambda **kw: L.provip_kv_append4(*dict(dict(K=FAKE, ks=512, V=FAKE, vs=512, T=3, H=4, d=128, slot=FAKE, n=4, page=16, dtype=1, kp=FAKE,
                                                     vp=FAKE), **kw).values(), None)
    rd = lambda **kw: L.provip_kv_read4(*dict(dict(slot=FAKE, T=3, H=4, d=128, kp=FAKE, vp=FAKE, n=4, page=16, dtype=1, K=FAKE, ks=512, V=FAKE,
                                                   vs=512), **kw).values(), None)
    for f in (ap, rd):
        for bad in (dict(K=None), dict(V=None), dict(slot=None), dict(kp=None), dict(vp=None), dict(T=-1), dict(H=0), dict(n=0), dict(ks=8),
                    dict(vs=511)):
            assert f(**bad) == -1, bad
        for bad in (dict(dtype=5), dict(d=64), dict(K=OFF), dict(V=OFF), dict(vp=OFF), dict(ks=516), dict(page=24), dict(page=512),
                    dict(n=2 ** 28)):
            assert f(**bad) == -2, bad
        assert f(T=0) == 0


def decode(L, **kw):
    a = dict(Q=FAKE, qs=1024, B=2, H_q=8, H_kv=4, d_h=128, kp=FAKE, vp=FAKE, n=10, page=16, bt=FAKE, mp=4, kl=FAKE, km=64, pt=None, P=0, scale=0.1,
             dtype=1, out=FAKE, os=1024, lse=None, ws=None, wsb=0)
    a.update(kw)
    return L.provip_decode_attention4(*a.values(), None)


def test_decode_refusals(L):
    for bad in (dict(Q=None), dict(kp=None), dict(vp=None), dict(out=None), dict(bt=None), dict(kl=None), dict(B=0), dict(n=0), dict(mp=-1),
                dict(km=65), dict(km=-1), dict(P=-1), dict(P=5), dict(H_kv=3), dict(scale=0.0), dict(scale=math.inf), dict(qs=100), dict(os=100)):
        assert decode(L, **bad) == -1, bad
    for bad in (dict(d_h=64), dict(page=12), dict(page=4), dict(page=512), dict(dtype=7), dict(Q=OFF), dict(kp=OFF), dict(qs=1025), dict(B=70000),
                dict(mp=2 ** 27, km=2 ** 31 - 100), dict(n=2 ** 28), dict(H_q=8 * 65, H_kv=8, qs=8 * 65 * 128, os=8 * 65 * 128)):
        assert decode(L, **bad) == -2, bad
    need = L.provip_decode_attention4_workspace_size(2, 8, 4, 6400, 0, 1)
    assert need > 0 and decode(L, mp=400, km=6400, ws=FAKE, wsb=need - 1) == -3


def test_workspace_sizes(L):
    d = L.provip_decode_attention4_workspace_size
    assert d(0, 8, 4, 10, 0, 1) == 0 and d(2, 8, 3, 10, 0, 1) == 0 and d(2, 8, 4, -1, 0, 1) == 0
    assert d(2, 8, 4, 4000, 5000, 1) > d(2, 8, 4, 4000, 0, 1) > 0
    assert d(100, 32, 32, 100, 0, 1) == 0  # one part a row


def test_binding_refusals():
    """what the Python binding rejects before it calls the library"""
    from paper_2608_25332_gb300 import provip as P
    for kw in (dict(inv_freq=[1.0] * 63), dict(axis=[0] * 63), dict(axis=[-1] + [0] * 63), dict(sections=(16, 24, 23)),
               dict(axis=[0] * 64, sections=(64,))):
        with pytest.raises(P.ProvipError):
            P.Rotary(**kw)
    r = P.Rotary(sections=(16, 24, 24), base=1e6)
    assert r.n_axes == 3 and list(r.axis) == [0] * 16 + [1] * 24 + [2] * 24 and r.inv_freq[0] == 1.0 and r.inv_freq[32] == 1e6 ** -0.5
    for c in (copy.copy(r), copy.deepcopy(r), pickle.loads(pickle.dumps(r))):  # of their own: the first may be gone
        assert c.args[1] is c.inv_freq is not r.inv_freq and c.args[2] is c.axis and (c.n_axes, c.factor) == (r.n_axes, r.factor)
        assert list(c.inv_freq) == list(r.inv_freq) and list(c.axis) == list(r.axis)
    assert P.pages4(3, 16, 2, "cpu").shape == (3, 2, 16 * 72)
    t, i = torch.zeros(4, 2, 128), torch.zeros(1, 4, dtype=torch.int32)
    pool = P.pages4(3, 16, 2, "cpu")
    for call in (lambda: P.provip_rotate(t, t, i, r), lambda: P.provip_kv_append4(t, t, i[0], pool, pool),
                 lambda: P.provip_kv_read4(i[0], pool, pool), lambda: P.provip_rotate_append(t, t, t, i, r, i[0], pool, pool)):
        with pytest.raises(P.ProvipError):
            call()  # not on the GPU
    with pytest.raises(P.ProvipError):
        P._positions(i, 4, 1, 0)
