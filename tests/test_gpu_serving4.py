"""QuestionCache with a rotary and pages of 4 bits on the GPU: questions about one pruned video from the
compaction to the answers, against attention over the rows themselves in 64 bits."""
import pytest
import torch

import cache4_ref as ref
from attention_ref import attend as attend_rows
from cache4_model import held
from paper_2608_25332_gb300 import provip as P
from paper_2608_25332_gb300.serving import QuestionCache

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DH, LAYERS, EPS = 128, 2, 1e-6


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


class Run:
    def __init__(self, bits, dtype=torch.bfloat16, B=5, H_q=8, H_kv=2, page=16, n_pages=60, max_len=80, normed=True):
        self.g = torch.Generator(device=DEV).manual_seed(3)
        self.B, self.H_q, self.H_kv, self.dtype, self.bits, self.page = B, H_q, H_kv, dtype, bits, page
        self.rotary = P.Rotary(sections=(16, 24, 24), base=1e6)
        self.norms = [tuple((1 + torch.randn(DH, generator=self.g, device=DEV) / 4).to(dtype) for _ in range(2))
                      for _ in range(LAYERS)] if normed else None
        self.cache = QuestionCache(LAYERS, B, H_q, H_kv, page, n_pages, max_len, dtype, DEV, bits=bits, rotary=self.rotary,
                                   norms=self.norms, eps=EPS)
        self.rows = [[[self.rand(0, H_kv)] * 2 for _ in range(B)] for _ in range(LAYERS)]

    def rand(self, n, h):
        return torch.randn(n, h, DH, generator=self.g, device=DEV).to(self.dtype)

    def kept(self, x):
        """as the pages stand for it"""
        return held(x) if self.bits == 4 else x.double()

    def set_prefix(self, K, V):
        self.prefix = [[self.kept(x) for x in kv] for kv in zip(K, V)]
        self.cache.set_prefix(K, V)

    def begin(self, new):
        self.new = new
        self.cache.begin(i32(new))
        self.rows = [[[x[:0] for x in r] if n < 0 else r for n, r in zip(new, layer)] for layer in self.rows]

    def inputs(self, n):
        pos = torch.randint(0, 30000, (3, n), generator=self.g, device=DEV).to(torch.int32)
        fused = self.rand(n, self.H_q + 2 * self.H_kv)
        return (*fused.split([self.H_q, self.H_kv, self.H_kv], 1), pos)

    def turned(self, layer, q, k, pos):
        w = self.norms[layer] if self.norms else (None, None)
        return P.provip_rotate(q, k, pos, self.rotary, *w, EPS)

    def near(self, layer, out, q, kk, vv, what):
        for h in range(self.H_q):
            g = h * self.H_kv // self.H_q
            o, _, bound, _ = ref.attend(q[h], kk[:, g], vv[:, g], DH ** -0.5, self.dtype)
            assert ((out[h].double() - o).abs() <= bound).all(), what

    def near_prompt(self, layer, out, q, kk, vv, what):
        """the prompts' attention takes the prefix's rows rounded to its type"""
        for h in range(self.H_q):
            g = h * self.H_kv // self.H_q
            o, _, bound, _ = attend_rows(q[None, h], kk[:, g], vv[:, g], torch.zeros(1, len(kk), dtype=torch.bool, device=DEV), DH ** -0.5,
                                         self.dtype, self.dtype == torch.bfloat16)
            assert ((out[None, h].double() - o).abs() <= bound).all(), what

    def prompt(self, pad=0):
        T = sum(max(n, 0) for n in self.new)
        for layer in range(LAYERS):
            q, k, v, pos = self.inputs(T + pad)
            out, at = self.cache.prompt(layer, q, k, v, pos=pos).clone(), 0
            tq, tk = self.turned(layer, q, k, pos)
            for b, n in enumerate(self.new):
                n = max(n, 0)
                pre = [p.to(self.dtype) for p in self.prefix[layer]]
                for i in range(at, at + n, max(n // 3, 1)):
                    kk, vv = (torch.cat([p, x[at:i + 1]]) for p, x in zip(pre, (tk, v)))
                    self.near_prompt(layer, out[i], tq[i], kk, vv, ("prompt", layer, b, i))
                if n:
                    self.rows[layer][b] = [torch.cat([r.double(), self.kept(x[at:at + n])]) for r, x in zip(self.rows[layer][b], (tk, v))]
                at += n

    def took(self, layer, k, v):
        for b, n in enumerate(self.new):
            if n > 0:
                self.rows[layer][b] = [torch.cat([r.double(), self.kept(x[b:b + 1])]) for r, x in zip(self.rows[layer][b], (k, v))]

    def check(self, layer, out, q):
        for b in range(self.B):
            kk, vv = (torch.cat([p, r.double()]) for p, r in zip(self.prefix[layer], self.rows[layer][b]))
            self.near(layer, out[b], q[b], kk, vv, ("decode", layer, b))

    def decode(self):
        for layer in range(LAYERS):
            q, k, v, pos = self.inputs(self.B)
            out = self.cache.decode(layer, q, k, v, pos=pos)
            tq, tk = self.turned(layer, q, k, pos)
            self.took(layer, tk, v)
            self.check(layer, out, tq)


def compacted(run, B=1, N_v=300, keep=40, vis_start=5, text=20):
    """a layer's rows after a compaction: the first vis_start + keep are the shared prefix"""
    L = vis_start + N_v + text
    scores = torch.rand(B, N_v, generator=run.g, device=DEV)
    K, V = (run.rand(B * L, run.H_kv).view(B, L, run.H_kv, DH) for _ in range(2))
    hidden = torch.zeros(B, L, 64, dtype=run.dtype, device=DEV)
    r = P.provip_topk_compact(scores, keep, hidden, K, V, None, i32([L] * B), vis_start)
    return r["K"][0, :vis_start + keep], r["V"][0, :vis_start + keep]


@pytest.mark.parametrize("bits,dtype,normed", [(4, torch.bfloat16, True), (16, torch.bfloat16, False), (4, torch.float32, True),
                                               (16, torch.float32, True)])
def test_questions_about_a_pruned_video(bits, dtype, normed):
    r = Run(bits, dtype, normed=normed)
    layers = [compacted(r) for _ in range(LAYERS)]
    r.set_prefix([k for k, _ in layers], [v for _, v in layers])
    r.begin([30, 1, 0, 17, 5])
    r.prompt(pad=3)
    for _ in range(3):
        r.begin([1, 1, 0, 1, 1])
        r.decode()
    r.begin([1, -1, 0, 1, -1])
    r.decode()
    r.begin([0, 33, 2, 0, 0])
    r.prompt()
    r.begin([1, 1, 1, 1, 0])
    r.decode()
    r.begin([-1] * 5)
    r.set_prefix([r.rand(63, 2) for _ in range(LAYERS)], [r.rand(63, 2) for _ in range(LAYERS)])
    r.begin([2, 0, 0, 0, 9])
    r.prompt()
    r.begin([1, 0, 0, 0, 1])
    r.decode()
    assert r.cache.kv_len.tolist() == [3, 0, 0, 0, 10]


@pytest.mark.parametrize("bits", [4, 16])
def test_a_captured_decode_step(bits):
    """a decode step in a graph follows the steps begun later, on another stream too"""
    r = Run(bits, H_q=28, H_kv=4)
    r.set_prefix([r.rand(37, 4) for _ in range(LAYERS)], [r.rand(37, 4) for _ in range(LAYERS)])
    r.begin([20, 3, 0, 9, 40])
    r.prompt()
    q, k, v, pos = r.inputs(r.B)
    held_in = [t.clone() for t in (q, k, v, pos)]
    r.begin([1, 1, 0, 1, 1])
    outs = [r.cache.decode(layer, *held_in[:3], pos=held_in[3]) for layer in range(LAYERS)]
    for layer in range(LAYERS):
        tq, tk = r.turned(layer, *held_in[:2], held_in[3])
        r.took(layer, tk, held_in[2])
    r.check(LAYERS - 1, outs[-1], tq)
    torch.cuda.synchronize()
    graph, out = torch.cuda.CUDAGraph(), []
    r.begin([1, 1, 0, 1, 1])
    with torch.cuda.graph(graph):
        for layer in range(LAYERS):
            out.append(r.cache.decode(layer, *held_in[:3], pos=held_in[3]).clone())
    side = torch.cuda.Stream(DEV)
    for step, new in enumerate(([1, 1, 0, 1, 1], [1, -1, 1, 1, 0], [1, 1, 1, 1, 1])):
        if step:
            # a prompt of another size in between, and whatever takes memory that came free
            r.begin([0, 0, 7 + step, 0, 0] if step == 1 else [0, 3, 0, 0, 0])
            r.prompt()
            _ = [torch.full((5, 28, DH), 9.0, dtype=r.dtype, device=DEV) for _ in range(8)]
            r.begin(new)
        for to, x in zip(held_in, r.inputs(r.B)):
            to.copy_(x)
        side.wait_stream(torch.cuda.current_stream(DEV))
        with torch.cuda.stream(side):
            graph.replay()
        torch.cuda.current_stream(DEV).wait_stream(side)
        for layer in range(LAYERS):
            tq, tk = r.turned(layer, *held_in[:2], held_in[3])
            r.took(layer, tk, held_in[2])
            r.check(layer, out[layer], tq)
