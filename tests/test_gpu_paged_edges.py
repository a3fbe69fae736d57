"""Attention over a paged cache where a row is empty, cut or not whole: slots that nobody uses, lengths that are none, a page that is missing in one
part of a row, results off 16 bytes."""
import pytest
import torch

from paper_2605_13473_amd import binding as ob
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


# a row of 6000 tokens in several parts, joined by a wavefront each, or (more than 16 shares for a group of rows) by a workgroup each
PARTS = [dict(Hq=4, Hk=1, K=128, shares=7), dict(Hq=4, Hk=1, K=128, shares=200), dict(Hq=8, Hk=4, K=128, order="token", shares=9),
         dict(Hq=8, Hk=4, K=64, order="token", shares=150), dict(Hq=4, Hk=2, K=256, shares=40), dict(Hq=4, Hk=1, K=64, io="f32", shares=7),
         dict(Hq=2, Hk=1, K=256, io="f32", shares=100)]


@pytest.mark.parametrize("case", PARTS, ids=lambda c: "-".join(str(v) for v in c.values()))
def test_a_page_missing_in_one_part_of_a_row(case):
    x = make_decode([6000, 5000, 70], page=64, **case)
    want, wlse = call(x)
    assert bool(want.isfinite().all())
    for at, entry in ((40, -1), (0, 10 ** 6), (5999 // 64, 2 ** 31 - 1)):
        table = x["table"].clone()
        table[0, at] = entry
        o, lse = call(dict(x, table=table))
        assert bool(o[0].isnan().all()) and bool(lse[0].isnan().all()), at
        assert torch.equal(o[1:], want[1:]) and torch.equal(lse[1:], wlse[1:]), at
    # outside the window it is not looked at
    x["window"] = 1000
    want, wlse = call(x)
    table = x["table"].clone()
    table[0, 40] = -1
    o, lse = call(dict(x, table=table))
    assert torch.equal(o, want) and torch.equal(lse, wlse) and bool(o.isfinite().all())


@pytest.mark.parametrize("case", PARTS, ids=lambda c: "-".join(str(v) for v in c.values()))
def test_results_of_parts_off_16_bytes(case):
    x = make_decode([6000, 5000, 70], page=64, **case)
    want, wlse = call(x)
    B, Hq, K = x["q"].shape
    wide = torch.full((B, Hq, K + 5), 7.0, device="cuda", dtype=x["q"].dtype)
    o, lse = wide[..., 3:3 + K], torch.empty(B, Hq, device="cuda")
    p = ob.make_decode_params(B, Hq, x["kc"].shape[2], K, x["q"].dtype == torch.bfloat16, 6000, None, 0, x["shares"])
    ws = torch.empty(ob.osdn_paged_decode_workspace_bytes(p), dtype=torch.uint8, device="cuda")
    ob.osdn_paged_decode(p, x["q"], x["kc"], x["vc"], x["table"], x["lengths"], None, o, lse, ws)
    assert torch.equal(o, want) and torch.equal(lse, wlse)
    assert bool((wide[..., :3] == 7.0).all()) and bool((wide[..., 3 + K:] == 7.0).all())


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
