"""A shared prefix in 4 bits whose rows lie in any way."""
import pytest
import torch

from paper_2608_25332_gb300 import provip as P
from paper_2608_25332_gb300.serving import QuestionCache
from test_serving4_prefix import laid_out

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


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("kind", ["transposed", "off", "odd stride", "columns", "slice", "expanded"])
def test_rows_in_any_layout(kind, dtype):
    """pages, prompts and decoding as for contiguous rows, bit for bit"""
    g = torch.Generator(device=DEV).manual_seed(5)
    rand = lambda *s: torch.randn(*s, device=DEV, generator=g).to(dtype)
    rows = [[rand(1 if kind == "expanded" else 37, 4, 128).expand(37, 4, 128) for _ in range(2)] for _ in range(2)]
    q, k, v = rand(5, 8, 128), rand(5, 4, 128), rand(5, 4, 128)
    q1, k1, v1 = rand(2, 8, 128), rand(2, 4, 128), rand(2, 4, 128)
    got = []
    for plain in (True, False):
        c = QuestionCache(2, 2, 8, 4, 16, 20, 32, dtype, DEV, bits=4)
        c.set_prefix(*[[x.contiguous() if plain else laid_out(kind, x) for x in y] for y in rows])
        c.begin(torch.tensor([3, 2], dtype=torch.int32, device=DEV))
        r = [c.prompt(layer, q, k, v).clone() for layer in range(2)]
        c.begin(torch.tensor([1, 1], dtype=torch.int32, device=DEV))
        r += [c.decode(layer, q1, k1, v1).clone() for layer in range(2)]
        got.append(r + [x for pool in c.pools for x in pool])
    assert all(torch.equal(a, b) for a, b in zip(*got)) and all(torch.isfinite(x.float()).all() for x in got[0][:4])
