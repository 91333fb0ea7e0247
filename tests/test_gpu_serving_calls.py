"""QuestionCache's calls on the GPU, at the steps and sizes where they could go wrong, against
attention over the rows themselves in 64 bits (bounds: attention_ref.py)."""
import pytest
import torch

from attention_ref import DH, attend
from paper_2608_25332_gb300 import provip as P
from paper_2608_25332_gb300.serving import QuestionCache

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
DTYPES = [torch.float32, torch.bfloat16]
H_Q, H_KV, PAGE = 8, 2, 16


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
    """A cache of one layer and what its questions hold."""

    def __init__(self, dtype, B=8, n_pages=60, max_len=70, prefix=37, **kw):
        self.g, self.dtype, self.B = torch.Generator(device=DEV).manual_seed(5), dtype, B
        self.cache = QuestionCache(1, B, H_Q, H_KV, PAGE, n_pages, max_len, dtype, DEV, **kw)
        self.rows = [[self.rand(0, H_KV)] * 2 for _ in range(B)]
        self.set_prefix(prefix)

    def rand(self, n, h):
        return torch.randn(n, h, DH, generator=self.g, device=DEV).to(self.dtype)

    def set_prefix(self, n):
        self.prefix = [self.rand(n, H_KV) for _ in range(2)]
        given = [x.clone() for x in self.prefix]
        self.cache.set_prefix([given[0]], [given[1]])
        return given

    def begin(self, new):
        self.new = new
        self.cache.begin(i32(new))
        self.rows = [[x[:0] for x in r] if n < 0 else r for n, r in zip(new, self.rows)]

    def near(self, out, b, q):
        k, v = (torch.cat([p, r]) for p, r in zip(self.prefix, self.rows[b]))
        for h in range(H_Q):
            kv = h * H_KV // H_Q
            o, _, bound, _ = attend(q[None, h], k[:, kv], v[:, kv], torch.zeros(1, len(k), dtype=torch.bool, device=DEV), DH ** -0.5,
                                    self.dtype, self.dtype == torch.bfloat16)
            assert ((out[None, h].double() - o).abs() <= bound).all(), (b, h)

    def prompt(self, pad=0):
        T, at = sum(max(n, 0) for n in self.new), 0
        q, k, v = self.rand(T + pad, H_Q), self.rand(T + pad, H_KV), self.rand(T + pad, H_KV)
        out = self.cache.prompt(0, q, k, v)
        for b, n in enumerate(self.new):
            for i in range(at, at + max(n, 0)):
                self.rows[b] = [torch.cat([r, x[i:i + 1]]) for r, x in zip(self.rows[b], (k, v))]
                self.near(out[i], b, q[i])
            at += max(n, 0)

    def decode(self):
        q, k, v = self.rand(self.B, H_Q), self.rand(self.B, H_KV), self.rand(self.B, H_KV)
        out = self.cache.decode(0, q, k, v)
        for b, n in enumerate(self.new):
            if n > 0:
                self.rows[b] = [torch.cat([r, x[b:b + 1]]) for r, x in zip(self.rows[b], (k, v))]
            self.near(out[b], b, q[b])
        torch.cuda.synchronize()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("new", [[1, 1, 1, 1, 0, 0, 0, 0], [1, -1, 1, 0, 0, 1, -1, 0], [0] * 8])
def test_decode_with_fewer_slots_than_questions(new, dtype):
    """a step's slots are fewer than the questions, and idle or ended ones follow its last row"""
    r = Run(dtype, max_new=4)
    r.begin([1, 0, 2, 0, 1, 0, 0, 0])
    r.prompt()
    r.begin(new)
    r.decode()


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_prompt_behind_tokens_of_its_question_is_reported(dtype):
    """prompt() sees the step's own rows and the prefix, none of the pages: a second turn is
    reported, the other questions' rows are as ever"""
    r = Run(dtype, B=3)
    r.begin([5, 40, 0])
    r.prompt()
    r.begin([4, 0, 30])
    q, k, v = r.rand(34, H_Q), r.rand(34, H_KV), r.rand(34, H_KV)
    out = r.cache.prompt(0, q, k, v)
    torch.cuda.synchronize()
    rc, bits = P.provip_device_status(clear=True)
    assert rc == P.ERR_INVALID_ARG and bits == P.DEVSTAT_BAD_ARG
    for i in range(4, 34):
        r.rows[2] = [torch.cat([x, y[i:i + 1]]) for x, y in zip(r.rows[2], (k, v))]
        r.near(out[i], 2, q[i])
    r.rows[0] = [torch.cat([x, y[:4]]) for x, y in zip(r.rows[0], (k, v))]
    r.begin([1, 1, 1])  # the rows are in the cache all the same
    r.decode()
    r.begin([-1, 1, 0])  # an ended question's slot takes a prompt again
    r.decode()
    r.begin([21, 0, 0])
    r.prompt()


@pytest.mark.parametrize("dtype", DTYPES)
def test_prompts_and_decoding_see_the_same_prefix(dtype):
    """the rows given to set_prefix may be the outputs of a pruning step, which its next call
    overwrites"""
    r = Run(dtype, B=3)
    r.begin([-1, -1, -1])
    for x in r.set_prefix(53):
        x.fill_(7.0)
    r.begin([3, 0, 20])
    r.prompt()
    r.begin([1, 0, 1])
    r.decode()


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_prefix_that_the_pool_cannot_hold(dtype):
    """refused where no pool state could hold it; where others hold the pages, reported by every
    decoding instead of attending over a page of someone else's"""
    r = Run(dtype, B=2, n_pages=6, prefix=3)
    with pytest.raises(P.ProvipError, match="pages"):
        r.set_prefix(6 * PAGE + 1)
    r = Run(dtype, B=2, n_pages=7, prefix=3)
    r.begin([40, 0])
    r.set_prefix(5 * PAGE)
    r.begin([1, 0])
    r.cache.decode(0, r.rand(2, H_Q), r.rand(2, H_KV), r.rand(2, H_KV))
    torch.cuda.synchronize()
    rc, bits = P.provip_device_status(clear=True)
    assert rc == P.ERR_INVALID_ARG and bits == P.DEVSTAT_BAD_ARG


@pytest.mark.parametrize("dtype", DTYPES)
def test_another_prefix_returns_the_first_ones_pages(dtype):
    r = Run(dtype, B=3, n_pages=12, prefix=30)
    for n in (100, 5, 12 * PAGE, 1, 0, 33):  # (12 pages: all, those of the prefix before among them)
        r.set_prefix(n)
        held = -(-n // PAGE)
        assert int(r.cache.n_free) == 12 - held
        assert sorted(r.cache.free[:12 - held].tolist() + r.cache.prefix_table[:held].tolist()) == list(range(12))
    r.begin([3, 0, 19])
    r.prompt()
    r.begin([1, 0, 1])
    r.decode()


@pytest.mark.parametrize("dtype", DTYPES)
def test_prompts_of_many_sizes_keep_one_set_of_buffers(dtype):
    r = Run(dtype, B=2, n_pages=200, max_len=1200)
    for n in (700, 1100, 1200):
        r.begin([n, 0])
        q, k, v = r.rand(n, H_Q), r.rand(n, H_KV), r.rand(n, H_KV)
        r.cache.prompt(0, q, k, v)
        r.begin([-1, 0])
    torch.cuda.synchronize()
    held = torch.cuda.memory_allocated()
    for n in range(1000, 1100):
        r.begin([n, 0])
        r.cache.prompt(0, q[:n], k[:n], v[:n])
        r.begin([-1, 0])
    torch.cuda.synchronize()
    assert torch.cuda.memory_allocated() <= held


@pytest.mark.parametrize("dtype", DTYPES)
def test_buffers_that_are_dropped_wait_for_their_stream(dtype):
    """The prefix was copied on another stream than the one that reads it last: once another takes
    its place, the first stream gets its memory only behind that use."""
    n = 5000
    r = Run(dtype, B=1, n_pages=1000, max_len=64, prefix=n)
    r.begin([4])
    q, k, v = r.rand(4, H_Q), r.rand(4, H_KV), r.rand(4, H_KV)
    want = r.cache.prompt(0, q, k, v).clone()
    new, other = [i32([x]) for x in (-1, 4)], [r.rand(n, H_KV) for _ in range(2)]
    side = torch.cuda.Stream(DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        r.cache.begin(new[0])
        r.cache.begin(new[1])
        torch.cuda._sleep(200_000_000)  # about a tenth of a second
        got = r.cache.prompt(0, q, k, v)
        r.cache.set_prefix([other[0]], [other[1]])
    junk = [torch.full_like(other[0], 7.0) for _ in range(6)]  # (of the size that was dropped)
    torch.cuda.synchronize()
    assert torch.equal(got, want) and len(junk)


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_table_that_is_dropped_waits_for_its_stream(dtype):
    """the same for the prefix's table, which decoding reads"""
    n = 5000
    r = Run(dtype, B=1, n_pages=1000, max_len=64, prefix=n)
    new, other = [i32([x]) for x in (1, -1, 1)], [r.rand(n, H_KV) for _ in range(2)]
    q, k, v = r.rand(1, H_Q), r.rand(1, H_KV), r.rand(1, H_KV)
    r.cache.begin(new[0])
    want = r.cache.decode(0, q, k, v).clone()
    width = r.cache.prefix_table.numel()
    side = torch.cuda.Stream(DEV)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        r.cache.begin(new[1])
        r.cache.begin(new[2])
        torch.cuda._sleep(200_000_000)
        got = r.cache.decode(0, q, k, v)
        r.cache.set_prefix([other[0]], [other[1]])
    junk = [torch.zeros(2, width, dtype=torch.int32, device=DEV) for _ in range(200)]
    torch.cuda.synchronize()
    assert torch.equal(got, want) and len(junk)


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_question_may_fill_its_last_page(dtype):
    """the tables hand out whole pages: with max_len 20 and pages of 16 a question holds 32 tokens"""
    r = Run(dtype, B=2, max_len=20)
    r.begin([30, 0])
    r.prompt()
    for _ in range(2):
        r.begin([1, 0])
        r.decode()
    assert r.cache.kv_len.tolist() == [32, 0]


@pytest.mark.parametrize("dtype", DTYPES)
def test_a_captured_layer_sees_the_steps_begun_after_it(dtype):
    r = Run(dtype, B=4)
    r.begin([3, 0, 20, 1])
    r.prompt()
    q, k, v = r.rand(4, H_Q), r.rand(4, H_KV), r.rand(4, H_KV)
    r.begin([1, 0, 1, 1])
    r.cache.decode(0, q, k, v)  # (its buffers)
    r.rows = [[torch.cat([x, y[b:b + 1]]) for x, y in zip(rows, (k, v))] if r.new[b] > 0 else rows for b, rows in enumerate(r.rows)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = r.cache.decode(0, q, k, v)
    for new in ([1, 0, 1, 1], [0, 0, -1, 1], [1, -1, 0, 1]):
        r.begin(new)
        for x, h in ((q, H_Q), (k, H_KV), (v, H_KV)):
            x.copy_(r.rand(4, h))
        graph.replay()
        torch.cuda.synchronize()
        for b, n in enumerate(new):
            if n > 0:
                r.rows[b] = [torch.cat([x, y[b:b + 1]]) for x, y in zip(r.rows[b], (k, v))]
            r.near(out[b], b, q[b])
