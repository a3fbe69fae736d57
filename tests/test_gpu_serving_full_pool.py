"""The example stack where its pool runs out of pages: the sequences that find none wait, the others' tokens stay with them."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kw", [dict(), dict(mx=True), dict(pages=2), dict(mx=True, pages=2)], ids=str)
def test_a_token_that_finds_no_page_waits(kw):
    from examples.hybrid_stack import Config, Serving, make_weights
    c = Config(longest=64)
    w = make_weights(c)
    g = torch.Generator(device="cuda").manual_seed(2)
    text = [torch.randn(n, c.width, device="cuda", generator=g).bfloat16() for n in (2 * c.page, 20, c.page + 5)]
    tokens = torch.randn(4, 3, c.width, device="cuda", generator=g).bfloat16()
    full, wide = Serving(c, w, 3, held=6, **kw), Serving(c, w, 3, **kw)         # 2 + 2 + 2 pages: none for the first one's next token
    for i, t in enumerate(text):
        assert torch.equal(full.prompt(i, t), wide.prompt(i, t))
    state = full.S[0].clone(), full.d[0].clone(), full.table[0].clone(), full.lengths.clone()
    for x in tokens[:2]:
        got, want = full.token(x, 64), wide.token(x, 64)
        assert bool(torch.isnan(got[0]).all()) and bool(want.isfinite().all())
        assert torch.equal(got[1:], want[1:])
    assert torch.equal(full.S[0], state[0]) and torch.equal(full.d[0], state[1]) and torch.equal(full.table[0], state[2]) and torch.equal(full.S[1:], wide.S[1:])
    assert full.lengths.tolist() == [2 * c.page, 22, c.page + 7]
    with pytest.raises(MemoryError):
        full.prompt(0, text[0])
    assert torch.equal(full.S[0], state[0]) and full.lengths.tolist() == [2 * c.page, 22, c.page + 7]
    full.finish([2])
    again = Serving(c, w, 3, **kw)
    again.prompt(0, text[0])
    assert torch.equal(full.token(tokens[2], 64)[0], again.token(tokens[2], 64)[0])


def test_the_first_tokens_of_a_plan_are_not_those_of_the_rows():
    """What the rows are kept apart for: the plan leaves the served sequences' tokens side by side."""
    from examples.hybrid_stack import Config, Serving, make_weights
    c = Config(longest=64)
    s = Serving(c, make_weights(c), 2, held=3)
    x = torch.randn(2 * c.page, c.width, device="cuda").bfloat16()
    s.prompt(0, x)
    s.prompt(1, x[:3])
    _, seq, _ = s.places(torch.ones_like(s.lengths), 2)
    assert seq.tolist() == [[1, -1]]
