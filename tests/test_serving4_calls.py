"""QuestionCache with a rotary and with pages of 4 bits, against attention over the rows themselves (CPU: the
binding's calls are the model's, cache4_model.py)."""
import pytest
import torch

import cache4_ref as ref
from cache4_model import Model4, held
from cache_model import DH, Model
from paper_2608_25332_gb300 import provip as P
from paper_2608_25332_gb300.serving import QuestionCache

H_Q, H_KV, PAGE, LAYERS = 4, 2, 8, 2
EPS = 1e-5


class Run:
    """A cache and what its questions hold: own rows as prompts see them, and as pages do."""

    def __init__(self, monkeypatch, bits, rotary, normed=False, B=6, n_pages=60, max_len=40, prefix=11, **kw):
        self.model, self.g, self.B, self.bits = Model4(monkeypatch), torch.Generator().manual_seed(1), B, bits
        self.rotary = P.Rotary(sections=(16, 24, 24)) if rotary else None
        self.norms = [(1 + self.rand(DH) / 4, 1 + self.rand(DH) / 4) for _ in range(LAYERS)] if normed else None
        self.cache = QuestionCache(LAYERS, B, H_Q, H_KV, PAGE, n_pages, max_len, torch.float32, "cpu", bits=bits, rotary=self.rotary,
                                   norms=self.norms, eps=EPS, **kw)
        self.rows = [[[torch.zeros(0, H_KV, DH)] * 2 for _ in range(B)] for _ in range(LAYERS)]
        self.prefix = [[torch.zeros(0, H_KV, DH)] * 2 for _ in range(LAYERS)]
        if prefix:
            self.set_prefix(prefix)

    def rand(self, *shape):
        return torch.randn(*shape, generator=self.g)

    def kept(self, x):
        return held(x) if self.bits == 4 else x

    def set_prefix(self, n):
        given = [[self.rand(n, H_KV, DH) for _ in range(LAYERS)] for _ in range(2)]
        self.prefix = [[self.kept(given[i][layer].clone()) for i in range(2)] for layer in range(LAYERS)]
        self.cache.set_prefix(*given)
        for x in (*given[0], *given[1]):
            x.fill_(7.0)  # (copied by then)

    def begin(self, new):
        self.new = new
        self.cache.begin(torch.tensor(new, dtype=torch.int32))
        self.rows = [[[x[:0] for x in r] if n < 0 else r for n, r in zip(new, layer)] for layer in self.rows]

    def turned(self, layer, q, k, pos):
        if self.rotary is None:
            return q, k
        w = self.norms[layer] if self.norms else (None, None)
        f, a = list(self.rotary.inv_freq), list(self.rotary.axis)
        return tuple(ref.turn(x, pos, f, a, y, EPS, 1.0)[0].float() for x, y in ((q, w[0]), (k, w[1])))

    def inputs(self, n):
        pos = torch.randint(0, 5000, (3, n), generator=self.g).to(torch.int32) if self.rotary else None
        return self.rand(n, H_Q, DH), self.rand(n, H_KV, DH), self.rand(n, H_KV, DH), pos

    def prompt(self, pad=0, **kw):
        T = sum(max(n, 0) for n in self.new)
        for layer in range(LAYERS):
            q, k, v, pos = self.inputs(T + pad)
            out, at = self.cache.prompt(layer, q, k, v, pos=pos, **kw), 0
            tq, tk = self.turned(layer, q, k, pos)
            for b, n in enumerate(self.new):
                n = max(n, 0)
                for i in range(at, at + n):  # (own rows unrounded)
                    kk, vv = (torch.cat([p.float(), x[at:i + 1]]) for p, x in zip(self.prefix[layer], (tk, v)))
                    assert torch.allclose(out[i], Model.attend(tq[i], kk, vv, DH ** -0.5), atol=1e-5), (layer, b, i)
                if n:
                    self.rows[layer][b] = [torch.cat([r.double(), self.kept(x[at:at + n]).double()]) for r, x in
                                           zip(self.rows[layer][b], (tk, v))]
                at += n
        assert not self.model.reports

    def decode(self):
        for layer in range(LAYERS):
            q, k, v, pos = self.inputs(self.B)
            out = self.cache.decode(layer, q, k, v, pos=pos)
            tq, tk = self.turned(layer, q, k, pos)
            for b, n in enumerate(self.new):
                if n > 0:
                    self.rows[layer][b] = [torch.cat([r.double(), self.kept(x[b:b + 1]).double()]) for r, x in
                                           zip(self.rows[layer][b], (tk, v))]
                kk, vv = (torch.cat([p.double(), r.double()]) for p, r in zip(self.prefix[layer], self.rows[layer][b]))
                assert torch.allclose(out[b], Model.attend(tq[b], kk, vv, DH ** -0.5), atol=1e-5), (layer, b)
        assert not self.model.reports


@pytest.mark.parametrize("bits,rotary,normed", [(4, False, False), (4, True, True), (16, True, False), (16, True, True)])
def test_prompts_and_decoding(monkeypatch, bits, rotary, normed):
    r = Run(monkeypatch, bits, rotary, normed)
    r.begin([3, 0, 9, 1, 0, 2])
    r.prompt(pad=4)
    for _ in range(2):
        r.begin([1, 0, 1, 1, 0, 1])
        r.decode()
    r.begin([1, 0, -1, 1, 0, -1])
    r.decode()
    r.begin([0, 5, 2, 0, 0, 0])  # new questions, also in a slot that came free
    r.prompt()
    r.begin([-1, -1, -1, -1, -1, -1])
    r.set_prefix(19)
    r.begin([2, 2, 0, 0, 0, 1])
    r.prompt()
    r.begin([1, 1, 0, 0, 0, 1])
    r.decode()


@pytest.mark.parametrize("bits", [4, 16])
def test_more_rows_than_slots(monkeypatch, bits):
    """rows behind the last question, past what the tables hand out"""
    r = Run(monkeypatch, bits, True, max_new=7)
    r.begin([3, 0, 2, 0, 1, 0])
    r.prompt(pad=9)


def test_a_prefix_without_pages_is_reported(monkeypatch):
    r = Run(monkeypatch, 4, False, n_pages=6, prefix=0)
    r.begin([30, 0, 0, 0, 0, 0])
    r.prompt()
    r.cache.set_prefix(*[[r.rand(20, H_KV, DH) for _ in range(LAYERS)] for _ in range(2)])
    r.begin([0, 3, 0, 0, 0, 0])
    q, k, v, _ = r.inputs(3)
    r.cache.prompt(0, q, k, v)
    assert "slot" in r.model.reports


def test_four_bits_take_the_room(monkeypatch):
    r = Run(monkeypatch, 4, False)
    assert all(x.dtype is torch.uint8 and x.shape == (60, H_KV, PAGE * 72) for pool in r.cache.pools for x in pool)
    assert not r.cache.prefix  # held in the pages alone


def test_refusals(monkeypatch):
    Model4(monkeypatch)
    rot = P.Rotary()
    make = lambda **kw: QuestionCache(LAYERS, 2, H_Q, H_KV, PAGE, 20, 16, torch.float32, "cpu", **kw)
    w = torch.ones(DH)
    for kw in (dict(bits=8), dict(norms=[(w, w)] * LAYERS), dict(rotary=rot, norms=[(w, w)])):
        with pytest.raises(P.ProvipError):
            make(**kw)
    q, k = torch.zeros(2, H_Q, DH), torch.zeros(2, H_KV, DH)
    pos = torch.zeros(1, 2, dtype=torch.int32)
    for cache, bad in ((make(), pos), (make(rotary=rot), None), (make(rotary=rot), pos[:, :1]), (make(rotary=rot), pos[0])):
        cache.begin(torch.ones(2, dtype=torch.int32))
        for call in (cache.prompt, cache.decode):
            with pytest.raises(P.ProvipError):
                call(0, q, k, k, pos=bad)
