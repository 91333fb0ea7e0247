"""Tensors of too few or too many dimensions, and of the wrong sizes, to the binding of the rotation and of the 4-bit cache (CPU:
refused before the library is called)."""
import pytest
import torch

from paper_2608_25332_gb300 import build as pbuild
from paper_2608_25332_gb300 import provip as P

ROWS, POOL, POOL16 = torch.zeros(4, 2, 128), P.pages4(3, 16, 2, "cpu"), torch.zeros(3, 16, 2, 128)
IDS, SLOT, ROT = torch.zeros(1, 4, dtype=torch.int32), torch.zeros(4, dtype=torch.int32), P.Rotary()


@pytest.fixture(scope="module", autouse=True)
def _lib():
    pbuild.build()


def flat(t):
    """the tensor with fewer dimensions, down to none, and with one more"""
    out = [t[None]]
    while t.dim():
        t = t[0]
        out.append(t)
    return out


CALLS = {
    "Q": lambda t: [lambda: P.provip_rotate(t, ROWS, IDS, ROT), lambda: P.provip_rotate_append(t, ROWS, ROWS, IDS, ROT, SLOT, POOL, POOL),
                    lambda: P.provip_decode_attention4(t, POOL, POOL, IDS.view(4, 1), SLOT, 8)],
    "K": lambda t: [lambda: P.provip_rotate(ROWS, t, IDS, ROT), lambda: P.provip_rotate_append(ROWS, t, ROWS, IDS, ROT, SLOT, POOL, POOL),
                    lambda: P.provip_kv_append4(t, ROWS, SLOT, POOL, POOL)],
    "V": lambda t: [lambda: P.provip_rotate_append(ROWS, ROWS, t, IDS, ROT, SLOT, POOL, POOL),
                    lambda: P.provip_kv_append4(ROWS, t, SLOT, POOL, POOL)],
    "out": lambda t: [lambda: P.provip_rotate(ROWS, ROWS, IDS, ROT, out=(t, ROWS)), lambda: P.provip_rotate(ROWS, ROWS, IDS, ROT, out=(ROWS, t)),
                      lambda: P.provip_kv_read4(SLOT, POOL, POOL, out=(t, ROWS)), lambda: P.provip_kv_read4(SLOT, POOL, POOL, out=(ROWS, t))],
}


@pytest.mark.parametrize("name", list(CALLS))
def test_rows(name):
    for t in flat(ROWS) + [ROWS[:3], ROWS[:, :1], ROWS[..., :64]]:
        for call in CALLS[name](t):
            with pytest.raises(P.ProvipError):
                call()


def test_pages():
    for t in flat(POOL) + flat(POOL16):
        for call in (lambda: P.provip_kv_append4(ROWS, ROWS, SLOT, t, POOL), lambda: P.provip_kv_append4(ROWS, ROWS, SLOT, POOL, t),
                     lambda: P.provip_kv_read4(SLOT, t, POOL), lambda: P.provip_kv_read4(SLOT, POOL, t),
                     lambda: P.provip_rotate_append(ROWS, ROWS, ROWS, IDS, ROT, SLOT, t, POOL),
                     lambda: P.provip_rotate_append(ROWS, ROWS, ROWS, IDS, ROT, SLOT, POOL, t),
                     lambda: P.provip_rotate_append(ROWS, ROWS, ROWS, IDS, ROT, SLOT, t, POOL16),
                     lambda: P.provip_rotate_append(ROWS, ROWS, ROWS, IDS, ROT, SLOT, POOL16, t),
                     lambda: P.provip_decode_attention4(ROWS, t, POOL, IDS.view(4, 1), SLOT, 8)):
            with pytest.raises(P.ProvipError):
                call()


def test_position_ids():
    for t in flat(IDS)[1:] + [IDS.float(), IDS[:, :3], IDS.long(), IDS[:0], IDS[None, None]]:
        with pytest.raises(P.ProvipError):
            P._positions(t, 4, 1, -1)  # (the device's number of a CPU tensor)
    assert P._positions(IDS[None], 4, 1, -1)[0] == IDS.data_ptr()


def test_a_plan_stays_as_it_is_made():
    """an attribute set afterwards would change nothing of the calls: it is refused"""
    r = P.Rotary(factor=0.5)
    for name, value in (("factor", 2.0), ("n_axes", 3), ("inv_freq", [1.0] * 64), ("axis", [0] * 64), ("args", ()), ("scale", 1.0)):
        with pytest.raises(P.ProvipError):
            setattr(r, name, value)
    assert r.factor == 0.5 and r.args == (1, r.inv_freq, r.axis, 0.5)
