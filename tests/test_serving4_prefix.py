"""A shared prefix whose rows lie in any way, and one that is refused (CPU: the binding's calls are the model's, which
here refuses layouts as the binding does)."""
import pytest
import torch

from cache4_model import Model4, held
from cache_model import DH, Model
from paper_2608_25332_gb300 import provip as P
from paper_2608_25332_gb300.serving import QuestionCache

LAYERS, H_Q, H_KV, PAGE = 2, 4, 2, 8


class Strict(Model4):
    def kv_append4(self, K, V, slot_map, k_pages, v_pages):
        for x in (K, V):
            T, H, _ = x.shape
            s0, s1, s2 = x.stride()
            if T and (s2 != 1 or (s1 != DH and H > 1)):
                raise P.ProvipError(P.ERR_INVALID_ARG, "heads")
            if (T > 1 and (s0 < H * DH or s0 * x.element_size() % 16)) or x.data_ptr() % 16:
                raise P.ProvipError(P.ERR_UNSUPPORTED, "stride or alignment")
        super().kv_append4(K, V, slot_map, k_pages, v_pages)


def laid_out(kind, x):
    """the rows x [n, H, 128] in another layout"""
    n, H, d = x.shape
    if kind == "transposed":
        return x.transpose(0, 1).contiguous().transpose(0, 1)
    if kind == "off":  # 4 bytes behind a boundary
        return torch.cat([x.new_zeros(1), x.flatten()])[1:].view(n, H, d)
    if kind == "odd stride":
        return torch.cat([x.flatten(1), x.new_zeros(n, 1)], 1)[:, :H * d].unflatten(1, (H, d))
    if kind == "columns":
        return x.permute(2, 0, 1).contiguous().permute(1, 2, 0)
    if kind == "slice":
        return torch.cat([x, x], 1)[:, :H]
    return x


def cache(bits=4, n_pages=12):
    return QuestionCache(LAYERS, 2, H_Q, H_KV, PAGE, n_pages, 16, torch.float32, "cpu", bits=bits)


def decode(c, g, prefix):
    """a token of each question behind the prefix"""
    c.begin(torch.ones(2, dtype=torch.int32))
    for layer in range(LAYERS):
        q, k, v = torch.randn(2, H_Q, DH, generator=g), torch.randn(2, H_KV, DH, generator=g), torch.randn(2, H_KV, DH, generator=g)
        out = c.decode(layer, q, k, v)
        for b in range(2):
            kk, vv = (torch.cat([p[layer], held(x[b:b + 1])]) for p, x in zip(prefix, (k, v)))
            assert torch.allclose(out[b], Model.attend(q[b], kk, vv, DH ** -0.5), atol=1e-5)
    c.begin(torch.full((2,), -1, dtype=torch.int32))


@pytest.mark.parametrize("kind", ["transposed", "off", "odd stride", "columns", "slice", "as it is", "expanded"])
def test_rows_in_any_layout(monkeypatch, kind):
    model, g = Strict(monkeypatch), torch.Generator().manual_seed(3)
    c = cache()
    for n in (11, 1, 30):
        rows = [[torch.randn(n, H_KV, DH, generator=g) for _ in range(LAYERS)] for _ in range(2)]
        if kind == "expanded":
            rows = [[x[:1].expand(n, H_KV, DH) for x in y] for y in rows]
        prefix = [[held(x.contiguous()) for x in y] for y in rows]
        c.set_prefix(*[[laid_out(kind, x) for x in y] for y in rows])
        decode(c, g, prefix)
    assert not model.reports


def test_a_refused_prefix_leaves_the_one_before(monkeypatch):
    """shapes, types and sizes that are refused: pages, lengths and the table stay, and the prefix is still decoded from"""
    Strict(monkeypatch)
    g = torch.Generator().manual_seed(4)
    c = cache()
    rows = [[torch.randn(11, H_KV, DH, generator=g) for _ in range(LAYERS)] for _ in range(2)]
    prefix = [[held(x) for x in y] for y in rows]
    c.set_prefix(*rows)
    state = lambda: [x.clone() for x in (c.n_free, c.free, c._prefix_held, c.prefix_table, *(y for pool in c.pools for y in pool))]
    before = state()
    new = lambda n=30, h=H_KV, **kw: [torch.zeros(n, h, DH, **kw) for _ in range(LAYERS)]
    for k, v in ((new(), new(29)), (new(h=3), new(h=3)), (new(dtype=torch.bfloat16), new(dtype=torch.bfloat16)), (new(), new()[:1]),
                 (new(97), new(97)), ([x[0] for x in new()], [x[0] for x in new()])):
        with pytest.raises(P.ProvipError):
            c.set_prefix(k, v)
        assert all(torch.equal(a, b) for a, b in zip(before, state())) and c.prefix_len == 11
    decode(c, g, prefix)


@pytest.mark.parametrize("bits", [4, 16])
def test_a_type_that_no_page_takes(monkeypatch, bits):
    Strict(monkeypatch)
    with pytest.raises(P.ProvipError):
        QuestionCache(LAYERS, 2, H_Q, H_KV, PAGE, 12, 16, torch.float16, "cpu", bits=bits)
