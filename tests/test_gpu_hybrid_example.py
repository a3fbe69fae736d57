"""The example stack of recurrence and attention: prompts and tokens one by one against whole texts, and the training step of its mixer
against differences of its loss."""
import pytest
import torch

pytestmark = pytest.mark.gpu


def test_tokens_one_by_one_are_the_text_at_once():
    """Every output is a sum of three terms of order one, from bf16 operands in another order (the chunked and the recurrent form of the
    recurrence differ by up to 2e-2 of a chain's magnitude by this library's own bound): 2^-4 of the largest, 2^-6 in norm."""
    from examples.hybrid_stack import run
    pairs, _ = run(sequences=3, prompt=130, new=20)
    for got, want in pairs:
        got, want = got.float(), want.float()
        assert got.shape == want.shape and bool(want.isfinite().all())
        assert (got - want).abs().max() <= 2.0 ** -4 * want.abs().max()
        assert (got - want).norm() <= 2.0 ** -6 * want.norm()


def test_training_step_of_the_mixer_against_differences():
    """fp32: the gradient along a direction against central differences of the loss (h = 1e-2 of a unit direction: the third derivative
    leaves 1e-4 relative, fp32 sums of the loss 2^-22 sqrt(terms) |loss terms| / h)."""
    from examples.hybrid_stack import mixer_step
    from paper_2605_13473_amd import binding as ob
    g = torch.Generator(device="cuda").manual_seed(3)
    B, T, H, K = 1, 100, 2, 64
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)
    x = dict(q=rnd(B, T, H, K), k=rnd(B, T, H, K), v=rnd(B, T, H, K), beta=torch.sigmoid(rnd(B, T, H)), log_alpha=-torch.nn.functional.softplus(rnd(B, T, H)))
    dO = rnd(B, T, H, K)
    _, grads = mixer_step(**x, dO=dO)
    loss = lambda **kw: float((mixer_step(**dict(x, **kw), dO=dO)[0].double() * dO.double()).sum())
    for n in ("q", "k"):
        u = rnd(B, T, H, K)
        u = u / u.norm() * x[n].norm() * 1e-2
        diff = (loss(**{n: x[n] + u}) - loss(**{n: x[n] - u})) / 2
        got = float((grads["d" + n].double() * u.double()).sum())
        size = float((grads["d" + n].double() * u.double()).norm() * 1.0)
        assert abs(got - diff) <= 2e-2 * (abs(got) + size)
