"""The rotation's table against its definition, written out: position p turns pair i by the angle p theta^(-2 i / dim)."""
import math

import pytest
import torch

from paper_2605_13473_amd import binding as ob


@pytest.mark.parametrize("rows,dim,theta", [(1, 16, 10000.0), (300, 64, 10000.0), (50, 128, 500000.0), (7, 48, 500.0)])
def test_cosines_then_sines(rows, dim, theta):
    t = ob.rotary_table(rows, dim, theta, device="cpu")
    assert t.dtype == torch.float32 and t.shape == (rows, dim) and t.is_contiguous()
    for p in range(rows):
        for i in range(dim // 2):
            angle = p / theta ** (2 * i / dim)
            assert abs(float(t[p, i]) - math.cos(angle)) < 2.0 ** -24 and abs(float(t[p, dim // 2 + i]) - math.sin(angle)) < 2.0 ** -24


def test_known_angles():
    t = ob.rotary_table(100001, 32, 10000.0, device="cpu")
    assert bool((t[0, :16] == 1).all()) and bool((t[0, 16:] == 0).all())
    # pair 8 of 16 turns by a hundredth of the position (10000^(-1/2)); the defaults are theta = 10000 and pair 0 by the position itself
    for p in (1, 1571, 100000):
        assert abs(float(t[p, 8]) - math.cos(p / 100)) < 2.0 ** -24 and abs(float(t[p, 24]) - math.sin(p / 100)) < 2.0 ** -24
        assert abs(float(t[p, 0]) - math.cos(p)) < 2.0 ** -24 and abs(float(t[p, 16]) - math.sin(p)) < 2.0 ** -24
    assert torch.equal(t[:50], ob.rotary_table(50, 32, device="cpu"))
