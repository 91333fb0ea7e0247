"""Position rotation by negative frequencies: the other way round, and as far."""
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


@pytest.mark.parametrize("base", [1e4, 1e6, 1e12])
def test_a_negative_frequency_is_a_negative_position(base):
    """-f at p turns by the angle of f at -p, which is the same integer: the same bits, at any position"""
    g = torch.Generator(device=DEV).manual_seed(int(base) % 1000)
    T = 40
    Q, K = torch.randn(2, T, 3, 128, device=DEV, generator=g)
    pos = torch.randint(-2 ** 31 + 1, 2 ** 31, (1, T), device=DEV, generator=g).to(torch.int32)
    pos[0, :5] = torch.tensor([0, 1, -1, 2 ** 31 - 1, -2 ** 31 + 1], dtype=torch.int32)
    freq = [base ** (-i / 64) for i in range(64)]
    a = P.provip_rotate(Q, K, pos, P.Rotary([-f for f in freq]))
    b = P.provip_rotate(Q, K, -pos, P.Rotary(freq))
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])
