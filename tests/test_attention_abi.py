"""Refusals of the attention and cache calls (CPU: all of them come before any CUDA call)."""
import ctypes
import math

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


def prompt(L, **kw):
    a = dict(Q=FAKE, qs=1024, K=FAKE, ks=512, V=FAKE, vs=512, T_q=50, T_k=60, B=2, H_q=8, H_kv=4, d_h=128, st=FAKE, ql=FAKE,
             kst=FAKE, kl=FAKE, qm=50, km=60, Kp=None, kps=0, Vp=None, vps=0, P=0, causal=1, scale=0.1, dtype=1, algo=1, out=FAKE,
             os=1024, lse=None, ws=None, wsb=0)
    a.update(kw)
    return L.provip_prompt_attention(*a.values(), None)


def test_prompt_refusals(L):
    for bad in (dict(Q=None), dict(K=None), dict(out=None), dict(st=None), dict(kl=None), dict(B=0), dict(T_q=-1), dict(qm=51),
                dict(km=61), dict(P=-1), dict(H_kv=3), dict(H_q=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=math.nan),
                dict(scale=math.inf), dict(algo=3), dict(qs=1000), dict(ks=500), dict(os=8), dict(P=5), dict(P=5, Kp=FAKE),
                dict(P=5, Kp=FAKE, Vp=FAKE, kps=512, vps=100)):
        assert prompt(L, **bad) == -1, bad
    for bad in (dict(d_h=64), dict(dtype=2), dict(dtype=0, algo=2), dict(Q=OFF), dict(V=OFF), dict(qs=1028), dict(vs=516),
                dict(P=5, Kp=OFF, Vp=FAKE, kps=512, vps=512), dict(H_q=8 * 65, H_kv=8, qs=8 * 65 * 128, ks=1024, vs=1024, os=8 * 65 * 128),
                dict(B=70000)):
        assert prompt(L, **bad) == -2, bad
    assert prompt(L, T_q=0, qm=0) == 0  # no row, no work
    need = L.provip_prompt_attention_workspace_size(50, 2, 8, 4, 50, 600, 5000, 1, 1)
    assert need > 0
    assert prompt(L, T_k=600, km=600, P=5000, Kp=FAKE, Vp=FAKE, kps=512, vps=512, ws=FAKE, wsb=need - 1) == -3
    assert b"workspace" in L.provip_last_error()


def decode(L, **kw):
    a = dict(Q=FAKE, qs=1024, B=2, H_q=8, H_kv=4, d_h=128, kp=FAKE, vp=FAKE, n=10, page=16, bt=FAKE, mp=4, kl=FAKE, km=64, pt=None,
             P=0, scale=0.1, dtype=1, algo=1, out=FAKE, os=1024, lse=None, ws=None, wsb=0)
    a.update(kw)
    return L.provip_decode_attention(*a.values(), None)


def test_decode_refusals(L):
    for bad in (dict(Q=None), dict(kp=None), dict(vp=None), dict(out=None), dict(bt=None), dict(kl=None), dict(B=0), dict(n=0), dict(mp=-1),
                dict(km=65), dict(km=-1), dict(P=-1), dict(P=5), dict(H_kv=3), dict(scale=0.0), dict(algo=4), dict(qs=100), dict(os=100)):
        assert decode(L, **bad) == -1, bad
    for bad in (dict(d_h=64), dict(page=12), dict(page=4), dict(page=512), dict(dtype=7), dict(dtype=0, algo=2), dict(Q=OFF), dict(kp=OFF),
                dict(qs=1025), dict(B=70000)):
        assert decode(L, **bad) == -2, bad
    assert decode(L, mp=400, km=6400) == -3


def test_tables_and_append_refusals(L):
    t = lambda **kw: L.provip_page_tables(*dict(dict(kv=FAKE, new=FAKE, B=2, page=16, fp=FAKE, nf=5, fc=FAKE, bt=FAKE, mp=3, T=9, o1=FAKE, o2=FAKE,
                                                     o3=FAKE, o4=FAKE), **kw).values(), None)
    for bad in (dict(kv=None), dict(new=None), dict(fp=None), dict(fc=None), dict(bt=None), dict(o1=None), dict(o2=None), dict(o3=None),
                dict(o4=None), dict(B=0), dict(nf=-1), dict(mp=-1), dict(T=-1)):
        assert t(**bad) == -1, bad
    assert t(page=24) == -2 and t(page=0) == -2
    ap = lambda **kw: L.provip_kv_append(*dict(dict(K=FAKE, ks=512, V=FAKE, vs=512, T=3, H=4, d=128, slot=FAKE, n=4, page=16, dtype=1, kp=FAKE,
                                                    vp=FAKE), **kw).values(), None)
    for bad in (dict(K=None), dict(slot=None), dict(kp=None), dict(T=-1), dict(H=0), dict(n=0), dict(page=0), dict(ks=8), dict(vs=8)):
        assert ap(**bad) == -1, bad
    for bad in (dict(dtype=5), dict(K=OFF), dict(vp=OFF), dict(ks=516), dict(H=1, d=4, ks=8, vs=8)):
        assert ap(**bad) == -2, bad
    assert ap(T=0) == 0


def test_workspace_sizes(L):
    f = L.provip_prompt_attention_workspace_size
    assert f(0, 0, 8, 4, 0, 0, 0, 1, 0) == 0 and f(100, 2, 8, 3, 50, 50, 0, 1, 0) == 0
    d = L.provip_decode_attention_workspace_size
    assert d(0, 8, 4, 10, 0, 1, 0) == 0 and d(2, 8, 4, 4000, 0, 1, 0) > 0
    assert d(2, 8, 4, 4000, 5000, 1, 0) > d(2, 8, 4, 4000, 0, 1, 0)


def test_binding_refusals():
    """what the Python binding rejects before it calls the library"""
    from paper_2608_25332_gb300 import provip as P
    t = torch.zeros(4, 2, 128)
    with pytest.raises(P.ProvipError):
        P._rows(t, 2, torch.float32, "Q")  # not on the GPU
    with pytest.raises(P.ProvipError):
        P._ints(torch.zeros(3, dtype=torch.int64), 3, "k_len")
    with pytest.raises(P.ProvipError):
        P._dtype_of(torch.float16)
    with pytest.raises(P.ProvipError):
        P.provip_kv_append(t, t[:, :1], torch.zeros(4, dtype=torch.int32), torch.zeros(1, 16, 2, 128), torch.zeros(1, 16, 2, 128))
