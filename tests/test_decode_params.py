"""Numbers past the fields of the parameter block of attention are not taken for other numbers."""
import pytest

from paper_2605_13473_amd import binding as ob


def test_numbers_past_their_field():
    p = ob.make_decode_params(2, 8, 4, 64, True, 100, window=2 ** 32 + 5)
    assert p.window == 2 ** 31 - 1 and ob.osdn_paged_decode_workspace_bytes(p) == ob.osdn_paged_decode_workspace_bytes(ob.make_decode_params(2, 8, 4, 64, True, 100))
    for kw in (dict(max_length=2 ** 32 + 100), dict(max_length=-2 ** 32), dict(window=-2 ** 32), dict(shares=2 ** 32 + 1), dict(shares=-2 ** 32)):
        p = ob.make_decode_params(2, 8, 4, 64, True, **{"max_length": 100000, **kw})
        field, = (n for n in kw)
        assert getattr(p, field) == (2 ** 31 - 1 if kw[field] > 0 else -2 ** 31)
        assert ob.osdn_paged_decode_workspace_bytes(p) == 0             # (refused)


@pytest.mark.parametrize("window", [0, None, 1, 2 ** 31 - 1])
def test_numbers_in_their_field(window):
    p = ob.make_decode_params(2, 8, 4, 64, False, 100, 0.5, window, -1)
    assert (p.window, p.max_length, p.shares, p.scale, p.io_dtype) == (window or 0, 100, -1, 0.5, ob.OSDN_F32)
