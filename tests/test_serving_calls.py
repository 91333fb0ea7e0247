"""QuestionCache's calls against attention over the rows themselves (CPU: the binding's calls
are the model's, cache_model.py)."""
import pytest
import torch

from cache_model import DH, Model
from paper_2608_25332_gb300 import provip as P
from paper_2608_25332_gb300.serving import QuestionCache

H_Q, H_KV, PAGE, LAYERS = 4, 2, 8, 2


class Run:
    """A cache and what its questions hold."""

    def __init__(self, monkeypatch, B=8, n_pages=60, max_len=40, prefix=11, **kw):
        self.model, self.g, self.B = Model(monkeypatch), torch.Generator().manual_seed(1), B
        self.cache = QuestionCache(LAYERS, B, H_Q, H_KV, PAGE, n_pages, max_len, torch.float32, "cpu", **kw)
        self.rows = [[[torch.zeros(0, H_KV, DH)] * 2 for _ in range(B)] for _ in range(LAYERS)]
        self.prefix = [[torch.zeros(0, H_KV, DH)] * 2 for _ in range(LAYERS)]
        if prefix:
            self.set_prefix(prefix)

    def rand(self, n, h):
        return torch.randn(n, h, DH, generator=self.g)

    def set_prefix(self, n):
        self.prefix = [[self.rand(n, H_KV) for _ in range(2)] for _ in range(LAYERS)]
        given = [[p[i].clone() for p in self.prefix] for i in range(2)]
        self.cache.set_prefix(*given)
        return given

    def begin(self, new):
        self.new = new
        self.cache.begin(torch.tensor(new, dtype=torch.int32))
        self.rows = [[[x[:0] for x in r] if n < 0 else r for n, r in zip(new, layer)] for layer in self.rows]

    def want(self, layer, b, q):
        k, v = (torch.cat([p, r]) for p, r in zip(self.prefix[layer], self.rows[layer][b]))
        return Model.attend(q, k, v, DH ** -0.5)

    def prompt(self, pad=0, **kw):
        T = sum(max(n, 0) for n in self.new)
        for layer in range(LAYERS):
            q, k, v = self.rand(T + pad, H_Q), self.rand(T + pad, H_KV), self.rand(T + pad, H_KV)
            out, at = self.cache.prompt(layer, q, k, v, **kw), 0
            for b, n in enumerate(self.new):
                for i in range(at, at + max(n, 0)):
                    self.rows[layer][b] = [torch.cat([r, x[i:i + 1]]) for r, x in zip(self.rows[layer][b], (k, v))]
                    assert torch.allclose(out[i], self.want(layer, b, q[i])), (layer, b, i)
                at += max(n, 0)
        assert not self.model.reports

    def decode(self):
        for layer in range(LAYERS):
            q, k, v = self.rand(self.B, H_Q), self.rand(self.B, H_KV), self.rand(self.B, H_KV)
            out = self.cache.decode(layer, q, k, v)
            for b, n in enumerate(self.new):
                if n > 0:
                    self.rows[layer][b] = [torch.cat([r, x[b:b + 1]]) for r, x in zip(self.rows[layer][b], (k, v))]
                assert torch.allclose(out[b], self.want(layer, b, q[b])), (layer, b)
        assert not self.model.reports


def test_prompts_and_decoding(monkeypatch):
    r = Run(monkeypatch)
    r.begin([3, 0, 9, 1, 0, 17, 2, 0])
    r.prompt()
    for _ in range(3):
        r.begin([1, 0, 1, 1, 0, 1, 1, 0])
        r.decode()
    r.begin([1, 0, -1, 1, 0, -1, 1, 0])
    r.decode()


@pytest.mark.parametrize("max_new", [4, 5, 8])
@pytest.mark.parametrize("new", [[1, 1, 1, 1, 0, 0, 0, 0], [1, -1, 1, 0, 0, 1, -1, 0], [0] * 8, [0, 0, 0, 0, 1, 1, 1, 1]])
def test_decode_with_fewer_slots_than_questions(monkeypatch, max_new, new):
    """a step's slots are fewer than the questions, and idle or ended ones follow its last row"""
    r = Run(monkeypatch, max_new=max_new)
    r.begin([1, 0, 2, 0, 1, 0, 0, 0])
    r.prompt()
    r.begin(new)
    r.decode()


def test_decode_without_slots(monkeypatch):
    r = Run(monkeypatch, max_new=0)
    r.begin([0] * 8)
    r.decode()


def test_a_prompt_behind_tokens_of_its_question_is_reported(monkeypatch):
    """prompt() sees the step's own rows and the prefix, none of the pages: a second turn is
    reported and its rows are left untouched, the other questions' are as ever"""
    r = Run(monkeypatch, B=3)
    r.begin([5, 9, 0])
    r.prompt()
    r.begin([4, 0, 3])
    q, k, v = r.rand(7, H_Q), r.rand(7, H_KV), r.rand(7, H_KV)
    for layer in range(LAYERS):
        out = r.cache.prompt(layer, q, k, v)
        assert r.model.reports == ["sequence"]
        r.model.reports.clear()
        if layer == 0:
            assert torch.isnan(out[:4]).all()
        for i in range(4, 7):
            r.rows[layer][2] = [torch.cat([x, y[i:i + 1]]) for x, y in zip(r.rows[layer][2], (k, v))]
            assert torch.allclose(out[i], r.want(layer, 2, q[i]))
        r.rows[layer][0] = [torch.cat([x, y[:4]]) for x, y in zip(r.rows[layer][0], (k, v))]
    r.begin([1, 1, 1])  # the rows are in the cache all the same
    r.decode()
    r.begin([-1, 1, 0])  # an ended question's slot takes a prompt again
    r.decode()
    r.begin([6, 0, 0])
    r.prompt()


def test_prompts_and_decoding_see_the_same_prefix(monkeypatch):
    """the rows given to set_prefix may be the outputs of a pruning step, which its next call
    overwrites"""
    r = Run(monkeypatch, prefix=0)
    given = r.set_prefix(13)
    for i in range(2):
        for x in given[i]:
            x.fill_(7.0)
    r.begin([3, 0, 9, 1, 0, 17, 2, 0])
    r.prompt()
    r.begin([1, 0, 1, 1, 0, 1, 1, 0])
    r.decode()


def test_a_prefix_that_the_pool_cannot_hold(monkeypatch):
    """refused where no pool state could hold it; where others hold the pages, reported by every
    decoding instead of attending over a page of someone else's"""
    r = Run(monkeypatch, n_pages=6, prefix=0)
    with pytest.raises(P.ProvipError, match="pages"):
        r.set_prefix(6 * PAGE + 1)
    assert r.cache.prefix_len == 0 and int(r.cache.n_free) == 6
    r.prefix = [[torch.zeros(0, H_KV, DH)] * 2 for _ in range(LAYERS)]
    r.begin([20, 0, 0, 0, 0, 0, 0, 0])  # three of the six pages
    r.prompt()
    r.set_prefix(4 * PAGE)
    r.begin([1, 0, 0, 0, 0, 0, 0, 0])
    r.cache.decode(0, r.rand(8, H_Q), r.rand(8, H_KV), r.rand(8, H_KV))
    assert "page" in r.model.reports
    assert int(r.cache.n_free) == 3


def test_another_prefix_returns_the_first_ones_pages(monkeypatch):
    r = Run(monkeypatch, n_pages=12, prefix=30)
    assert int(r.cache.n_free) == 8
    for n in (70, 5, 96, 1, 0, 33, 33):  # (96: every page of the pool, those of the prefix before among them)
        r.set_prefix(n)
        assert int(r.cache.n_free) == 12 - -(-n // PAGE)
        assert sorted(r.cache.free[:int(r.cache.n_free)].tolist() + r.cache.prefix_table[:-(-n // PAGE)].tolist()) == list(range(12))
    r.begin([3, 0, 9, 1, 0, 10, 2, 0])  # the seven pages that are left
    r.prompt()
    r.begin([1, 0, 1, 1, 0, 1, 1, 0])
    r.decode()
    r.begin([-1, 0, -1, -1, 0, -1, -1, 0])
    r.set_prefix(90)
    r.begin([0, 2, 0, 0, 0, 0, 0, 0])  # the pool is all the prefix's
    assert r.cache.kv_len.tolist() == [0] * 8 and int(r.cache.n_free) == 0
    r.model.reports.clear()
    # a prefix that got no pages has none to return
    r.set_prefix(0)
    r.begin([40, 0, 0, 0, 0, 0, 0, 0])
    r.set_prefix(60)
    assert int(r.cache.n_free) == 7 and r.cache.prefix_table.tolist()[:8] == [-1] * 8
    r.set_prefix(56)
    assert int(r.cache.n_free) == 0 and -1 not in r.cache.prefix_table.tolist()[:7]


def test_prompts_of_many_sizes_keep_one_set_of_buffers(monkeypatch):
    r = Run(monkeypatch, B=2)
    for n in list(range(1, 12)) + [3, 3, 20]:
        r.begin([n, 0])
        r.prompt()
        assert r.model.kept("PromptAttention") == 1
        r.begin([-1, 0])
        r.decode()
    assert r.model.kept("DecodeAttention") == 1


def test_the_lengths_of_a_step_may_change_after_begin(monkeypatch):
    """a caller may write the next step's lengths into the same tensor before this one's layers"""
    r = Run(monkeypatch, B=3)
    lens = torch.tensor([2, 0, 5], dtype=torch.int32)
    r.new = lens.tolist()
    r.cache.begin(lens)
    lens.fill_(-1)
    r.prompt()
    lens.copy_(torch.tensor([1, 0, 1]))
    r.new = lens.tolist()
    r.cache.begin(lens)
    lens.fill_(0)
    r.decode()
    r.begin([1, 0, 1])
    r.decode()


def test_a_question_may_fill_its_last_page(monkeypatch):
    """the tables hand out whole pages: with max_len 20 and pages of 8 a question holds 24 tokens"""
    r = Run(monkeypatch, B=2, max_len=20)
    r.begin([22, 0])
    r.prompt()
    for _ in range(2):
        r.begin([1, 0])
        r.decode()
    assert r.cache.kv_len.tolist() == [24, 0]
    r.begin([1, 0])  # its table is full
    assert r.cache.kv_len.tolist() == [24, 0] and r.model.reports


@pytest.mark.parametrize("pad", [0, 1, 9])
def test_prompts_with_rows_behind_the_last_question(monkeypatch, pad):
    """padding rows, more in all than the step's slots"""
    r = Run(monkeypatch, B=3, max_new=12)
    r.begin([4, 0, 8])
    r.prompt(pad=pad)
    r.begin([1, 1, 1])
    r.decode()


def test_a_prefix_is_given_for_every_layer(monkeypatch):
    r = Run(monkeypatch, B=2)
    one, two = r.rand(5, H_KV), r.rand(6, H_KV)
    for k, v in (([one], [one]), ([one] * 2, [one]), ([one] * 3, [one] * 3), ([one, two], [one, one]), ([one, one], [one, two]), ([], [])):
        with pytest.raises(P.ProvipError):
            r.cache.set_prefix(k, v)
    r.begin([3, 2])  # nothing has changed
    r.prompt()
    r.begin([1, 1])
    r.decode()


def test_decoding_more_than_one_token_of_a_question_is_reported(monkeypatch):
    """its other new tokens have slots, but no rows: what lies there is not attended to"""
    r = Run(monkeypatch, B=3)
    r.begin([2, 3, 1])
    r.prompt()
    r.begin([1, 2, 1])
    q, k, v = r.rand(3, H_Q), r.rand(3, H_KV), r.rand(3, H_KV)
    for layer in range(LAYERS):
        out = r.cache.decode(layer, q, k, v)
        assert r.model.reports == ["kv_len"]
        r.model.reports.clear()
        for b in (0, 2):
            r.rows[layer][b] = [torch.cat([x, y[b:b + 1]]) for x, y in zip(r.rows[layer][b], (k, v))]
            assert torch.allclose(out[b], r.want(layer, b, q[b]))


def test_the_lengths_of_a_step_are_checked(monkeypatch):
    """int32, one for every question: a shorter tensor is not spread over them"""
    r = Run(monkeypatch, B=3)
    for bad in (torch.tensor([1]), torch.tensor([1], dtype=torch.int32), torch.tensor([1, 1, 1]), torch.ones(2, dtype=torch.int32),
                torch.ones(6, dtype=torch.int32)[::2], torch.tensor(1, dtype=torch.int32)):
        with pytest.raises(P.ProvipError):
            r.cache.begin(bad)
    r.new = [2, 0, 1]
    r.cache.begin(torch.tensor([2, 0, 1, 7], dtype=torch.int32))  # (more may follow)
    r.prompt()


def test_a_steps_rows_are_checked(monkeypatch):
    """with fewer rows of K or V than of Q some tokens would not be stored"""
    r = Run(monkeypatch, B=3)
    r.begin([2, 0, 1])
    q, k, v = r.rand(3, H_Q), r.rand(3, H_KV), r.rand(3, H_KV)
    for kk, vv in ((k[:2], v[:2]), (k[:2], v), (k, v[:2])):
        with pytest.raises(P.ProvipError):
            r.cache.prompt(0, q, kk, vv)
    r.prompt()
    r.begin([1, 1, 1])
    for qq, kk, vv in ((q, k[:2], v[:2]), (q, k, v[:2]), (q[:2], k, v), (q[:2], k[:2], v[:2])):
        with pytest.raises(P.ProvipError):
            r.cache.decode(0, qq, kk, vv)
    r.decode()


def test_a_refused_prefix_leaves_the_one_before(monkeypatch):
    """types and shapes are checked before any page changes hands"""
    r = Run(monkeypatch, B=2, n_pages=12, prefix=30)
    for bad in (r.rand(9, H_KV).double(), r.rand(9, H_KV + 1), r.rand(9, H_KV)[..., :64]):
        fine = r.rand(9, H_KV)
        for k, v in (([fine, bad], [fine, fine]), ([fine, fine], [bad, fine])):
            with pytest.raises(P.ProvipError):
                r.cache.set_prefix(k, v)
    assert int(r.cache.n_free) == 8 and r.cache.prefix_len == 30
    r.begin([3, 2])
    r.prompt()
    r.begin([1, 1])
    r.decode()
