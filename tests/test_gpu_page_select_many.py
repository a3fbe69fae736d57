"""Selection for more queries than a launch takes, and of all pages."""
import pytest
import torch

from paper_2605_13473_amd import binding as ob
from tests import heads_reference as ref
from tests import pages_reference as pages
from tests.test_gpu_page_select import bounds_of, make, rnd

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("B,max_length", [(70000, 91), (300, 1 << 25)])
def test_more_queries_than_a_launch_takes(B, max_length):
    """By their number, and by the scores that they may have (300 x 2 heads x 2^22 pages of 8 tokens)."""
    g = torch.Generator(device="cuda").manual_seed(5)
    x = make([90, 41], 4, 2, 64, 8)
    b = bounds_of(x)
    seq = torch.randint(0, 2, (B,), dtype=torch.int32, device="cuda", generator=g)
    lengths = torch.minimum(torch.randint(0, 91, (B,), dtype=torch.int32, device="cuda", generator=g), x["lengths"][seq.long()])
    q = rnd(g, B, 4, 64).bfloat16()
    chosen, tokens = ob.page_select(q, b, x["table"], lengths, 8, 4, seq=seq, max_length=max_length)
    assert chosen.shape == (B, 2, 4) and tokens.shape == (B, 2)
    for at in (0, B // 2 - 20, B - 40):
        s = slice(at, at + 40)
        want = pages.select(ref.f64(q[s]), ref.f64(b), x["table"].cpu(), lengths[s].cpu(), seq[s].cpu(), 8, 4, 1, 1, max_length)
        assert torch.equal(chosen[s].cpu(), want[0]) and torch.equal(tokens[s].cpu(), want[1])
    for bad in (lengths[:5], lengths.long()):
        with pytest.raises((TypeError, ValueError)):
            ob.page_select(q, b, x["table"], bad, 8, 4, seq=seq, max_length=max_length)


@pytest.mark.parametrize("form", [dict(io="bf16"), dict(io="f32"), dict(io="bf16", mx=True), dict(io="f32", mx=True)], ids=str)
def test_all_pages_cut_alike_are_the_bits_of_the_whole_sequence(form):
    """As many pages as there are, a row to a workgroup on both sides: the same sums in the same order."""
    x = make([300, 47, 0, 16], 8, 2, 128, 16, **form)
    chosen, tokens = ob.page_select(x["q"], bounds_of(x), x["table"], x["lengths"], 16, 25)
    p = ob.make_decode_params(4, 8, 2, 128, x["dt"] == torch.bfloat16, 400, shares=-1)
    out = [(torch.empty_like(x["q"]), torch.empty(4, 8, device="cuda")) for _ in range(2)]
    if x["mx"]:
        ob.osdn_paged_decode_pages_mx(p, x["q"], x["cache"], chosen, tokens, *out[0])
        ob.osdn_paged_decode_mx(p, x["q"], x["cache"], x["table"], x["lengths"], None, *out[1])
    else:
        ob.osdn_paged_decode_pages(p, x["q"], *x["cache"], chosen, tokens, *out[0])
        ob.osdn_paged_decode(p, x["q"], *x["cache"], x["table"], x["lengths"], None, *out[1])
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1])
