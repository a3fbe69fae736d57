"""The training step of the example's mixer (norm in front of the recurrence, forward and backward) against the loss in 64 bits: the oracle's
recurrence on rows normed in 64 bits, by central differences."""
import numpy as np
import pytest
import torch

import oracle
from examples.hybrid_stack import UNIT, mixer_step
from paper_2605_13473_amd import binding as ob
from tests import heads_reference as ref
from tests.gpu_util import F32_REL

pytestmark = pytest.mark.gpu
B, T, H, K = 1, 100, 2, 64


def _inputs(seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)
    x = dict(q=rnd(B, T, H, K), k=rnd(B, T, H, K), v=rnd(B, T, H, K), beta=torch.sigmoid(rnd(B, T, H)), log_alpha=-torch.nn.functional.softplus(rnd(B, T, H)))
    return x, rnd(B, T, H, K)


def _unit(rows):
    return rows / torch.sqrt((rows * rows).sum(-1, keepdim=True) + UNIT.eps)


def _loss(x, dO):
    a = {n: np.ascontiguousarray(t.numpy()) for n, t in x.items()}
    a["q"], a["k"] = (np.ascontiguousarray(_unit(x[n]).numpy()) for n in "qk")
    o = oracle.fwd(a["q"], a["k"], a["v"], a["beta"], a["log_alpha"], None, None, None, oracle.Hyper())[0]
    return float((o * dO.numpy()).sum())


@pytest.mark.parametrize("n", ["q", "k"])
def test_along_the_gradient(n):
    """u: the gradient itself, so that <dx, u> is as large as it can be.  The recurrence's gradients are within F32_REL of their largest magnitude (this
    library's bound in fp32), which the norm's derivative J carries to F32_REL max |g| sum |J u|; the norm itself adds 2^-19 of the magnitudes that
    meet in an element (tests/test_gpu_qk_norm.py), at most 1.5 r (max |g| + |x r| sum |x r| max |g|).  The differences: a step of 1e-5 of x leaves h^2
    = 1e-10 of the third derivative, and 1e-16 / 1e-5 of the loss's terms: 1e-6 of the value together."""
    x, dO = _inputs(3)
    _, grads = mixer_step(**x, dO=dO)
    qn, kn = ob.qk_norm(x["q"], x["k"], hp=UNIT)
    _, _, _, ctx = ob.forward(qn, kn, x["v"], x["beta"], x["log_alpha"], for_backward=True)
    g = ref.f64(ob.backward(ctx, dO)["d" + n])
    x64, dx = {m: ref.f64(t) for m, t in x.items()}, ref.f64(grads["d" + n])
    rows = x64[n]
    r = 1 / torch.sqrt((rows * rows).sum(-1, keepdim=True) + UNIT.eps)
    u = dx / dx.norm() * rows.norm()
    h = 1e-5
    diff = (_loss({**x64, n: rows + h * u}, ref.f64(dO)) - _loss({**x64, n: rows - h * u}, ref.f64(dO))) / (2 * h)
    xr = rows * r
    Ju = r * (u - xr * (xr * u).sum(-1, keepdim=True))
    gmax = g.abs().amax(-1, keepdim=True)
    own = 1.5 * r * (gmax + xr.abs() * (xr.abs() * gmax).sum(-1, keepdim=True))
    got = float((dx * u).sum())
    tol = F32_REL * float(g.abs().max()) * float(Ju.abs().sum()) + 2.0 ** -19 * float((own * u.abs()).sum()) + 1e-6 * abs(got)
    assert tol <= 2e-3 * abs(got)                       # (it says something)
    assert abs(got - diff) <= tol, (got, diff, tol)


@pytest.mark.parametrize("n", ["q", "k"])
def test_along_the_rows(n):
    """A row's length is normed away: <dx, x> = r <g, x> (1 - r^2 |x|^2) = r^3 eps <g, x>, where each of the two terms is r <g, x>.  What is
    left besides is the rounding of dx: 2^-19 of the magnitudes that meet in each of its elements, times the row's."""
    x, dO = _inputs(4)
    _, grads = mixer_step(**x, dO=dO)
    qn, kn = ob.qk_norm(x["q"], x["k"], hp=UNIT)
    _, _, _, ctx = ob.forward(qn, kn, x["v"], x["beta"], x["log_alpha"], for_backward=True)
    g, rows, dx = ref.f64(ob.backward(ctx, dO)["d" + n]), ref.f64(x[n]), ref.f64(grads["d" + n])
    r = 1 / torch.sqrt((rows * rows).sum(-1, keepdim=True) + UNIT.eps)
    gx = (g * rows).sum(-1)
    gmax = g.abs().amax(-1, keepdim=True)
    size = 1.5 * r * (gmax + (rows * r).abs() * ((rows * r).abs() * gmax).sum(-1, keepdim=True))
    left = (dx * rows).sum(-1) - r[..., 0] ** 3 * UNIT.eps * gx
    bound = 2.0 ** -19 * (size * rows.abs()).sum(-1)
    assert (left.abs() <= bound).all(), float((left.abs() / bound).max())
    assert float((bound / (r[..., 0] * gx).abs()).median()) < 1e-2       # (without the second term it would be the first)
