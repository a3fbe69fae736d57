"""Attention over a paged cache where a row is empty, or a length is none."""
import pytest
import torch

from tests.test_gpu_paged import call, make_decode

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("shares", [0, -1, 5])
@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_a_slot_that_nobody_uses(io, shares):
    """Without a token there is nothing to look up: zero and minus infinity, whatever stands for the sequence."""
    x = make_decode([600, 600, 600, 600, 600], 4, 2, 128, 16, io=io, shares=shares, window=100)
    want, wlse = call(x)
    x["lengths"].copy_(torch.tensor([0, 600, -1, 600, -2 ** 31], dtype=torch.int32))
    seq = torch.tensor([-1, 1, 5, 3, 2 ** 31 - 1], dtype=torch.int32, device="cuda")
    o, lse = call(x, seq=seq)
    assert bool((o[::2] == 0).all()) and bool((lse[::2] == -float("inf")).all())
    close = dict(rtol=2.0 ** -7, atol=2.0 ** -7) if io == "bf16" else dict(rtol=1e-4, atol=1e-5)         # (other cuts of the used rows)
    assert torch.allclose(o[1::2], want[1::2], **close) and torch.allclose(lse[1::2], wlse[1::2], rtol=1e-5, atol=1e-5)


@pytest.mark.parametrize("K,io,order", [(64, "bf16", "head"), (128, "bf16", "token"), (256, "bf16", "head"), (128, "f32", "head")])
def test_lengths_that_are_no_lengths(K, io, order):
    """The largest numbers for a length, with windows that begin next to them: NaN, and the rows beside them as they are."""
    x = make_decode([700, 33, 700, 1], 4, 2, K, 16, io=io, order=order)
    for window in (0, 1, 40, 1000):
        for shares in (0, -1, 6):
            x["lengths"].copy_(torch.tensor([700, 33, 700, 1], dtype=torch.int32))
            y = dict(x, window=window, shares=shares)
            want, wlse = call(y)
            x["lengths"].copy_(torch.tensor([2 ** 31 - 1, 33, 2 ** 31 - 40, 1], dtype=torch.int32))
            o, lse = call(y)
            assert bool(o[::2].isnan().all()) and bool(lse[::2].isnan().all())
            close = dict(rtol=2.0 ** -7, atol=2.0 ** -7) if io == "bf16" else dict(rtol=1e-4, atol=1e-5)     # (other cuts)
            assert torch.allclose(o[1::2], want[1::2], **close) and torch.allclose(lse[1::2], wlse[1::2], rtol=1e-5, atol=1e-5)
