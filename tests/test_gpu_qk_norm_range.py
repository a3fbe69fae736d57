"""Norm and rotation at the ends of the range of fp32: rows whose sum of squares passes it, products with weights that do, rows that are not looked at."""
import math

import pytest
import torch

from paper_2605_13473_amd import binding as ob
from tests import heads_reference as ref
from tests.test_gpu_qk_norm import check, make

pytestmark = pytest.mark.gpu

KINDS = [dict(rotary=0, weighted=False), dict(rotary=0), dict(rotary=64, weighted=False), dict(rotary=64), dict(rotary=32, interleaved=True)]


def _with_large_rows(kind, io, norm):
    """Inputs with rows of 1e30, of 3e38 and with one element of 1e20 among the others, and the same with zeros in their place."""
    x = make(B=2, T=5, Hq=3, Hk=2, K=64, io=io, norm=norm, seed=4, **kind)
    g = torch.Generator(device="cuda").manual_seed(8)
    y = dict(x, **{n: x[n].clone() for n in ("q", "k", "dq", "dk")})
    for n in "qk":
        t = x[n]
        t[0, 1] = 1e30 * torch.randn(t.shape[2:], device="cuda", generator=g)
        t[1, 3] = 3e38 * torch.sign(torch.randn(t.shape[2:], device="cuda", generator=g))
        t[1, 0, 1, 7] = 1e20
        for m in (n, "d" + n):
            y[m][0, 1] = y[m][1, 3] = y[m][1, 0, 1] = 0
    return x, y


@pytest.mark.parametrize("norm", ["l2", "rms"])
@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS, ids=str)
def test_rows_whose_squares_pass_fp32(kind, io, norm):
    """They become zeros, and an append writes zeros."""
    x, y = _with_large_rows(kind, io, norm)
    z, want = (ob.qk_norm(i["q"], i["k"], i["wq"], i["wk"], i["table"], None, i["hp"]) for i in (x, y))
    assert torch.equal(z[0], want[0]) and torch.equal(z[1], want[1])
    kc, vc = (torch.full((2, 8, 2, 64), 5.0, device="cuda", dtype=x["q"].dtype) for _ in range(2))
    pos = torch.arange(5, dtype=torch.int32, device="cuda").expand(2, -1).contiguous()
    q = ob.paged_append(x["k"], x["k"], kc, vc, torch.tensor([[1], [0]], dtype=torch.int32, device="cuda"), pos, None, x["q"], x["wq"], x["wk"], x["table"], x["hp"])
    assert torch.equal(q, want[0]) and torch.equal(kc[[1, 0], :5], want[1])


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS, ids=str)
def test_large_weights_on_large_rows(kind, io):
    """Products of a row and its weights that pass fp32 where the normed row does not: the bound of the forward pass (2^-19 of the row's
    largest magnitude before the rotation)."""
    x = make(B=2, T=5, Hq=3, Hk=2, K=64, io=io, norm="rms", seed=5, **kind)
    if x["wq"] is None:
        x["wq"], x["wk"] = (torch.ones(64, device="cuda") for _ in range(2))
    for n in "qk":
        x[n].mul_(1e15)
        x["w" + n].mul_(1e25)
    z = ob.qk_norm(x["q"], x["k"], x["wq"], x["wk"], x["table"], None, x["hp"])
    pos, table, hp = torch.arange(5).expand(2, -1), ref.f64(x["table"]), x["hp"]
    for n, got in zip("qk", z):
        rows, w = ref.f64(x[n]), ref.f64(x["w" + n])
        want, y = (ref.norm_rows(rows, w, t, pos, hp.norm, hp.eps, hp.interleaved) for t in (table, None))
        check(got, want, y.abs().amax(-1, keepdim=True), io == "bf16", n)


@pytest.mark.parametrize("norm", ["l2", "rms"])
@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS, ids=str)
def test_gradients_of_rows_whose_squares_pass_fp32(kind, io, norm):
    """They are zero, and the gradients of the weights are what they are without those rows."""
    x, y = _with_large_rows(kind, io, norm)
    g, want = (ob.qk_norm_backward(i["q"], i["k"], i["dq"], i["dk"], i["wq"], i["wk"], i["table"], None, i["hp"]) for i in (x, y))
    for n in g:
        assert (g[n] is None and want[n] is None) or torch.equal(g[n], want[n]), n


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS, ids=str)
def test_without_a_norm_gradients_of_rows_do_not_see_them(kind, io):
    """dx = w . R(-p) dz: what a row holds has no part in it, infinite or not a number."""
    x = make(B=2, T=5, Hq=3, Hk=2, K=64, io=io, norm="none", seed=6, **kind)
    args = (x["wq"], x["wk"], x["table"], None, x["hp"])
    want = ob.qk_norm_backward(x["q"], x["k"], x["dq"], x["dk"], *args)
    for n in "qk":
        x[n][0, 2, 1, 7], x[n][1, 1, 0, 3], x[n][1, 4, 1] = math.inf, math.nan, -math.inf
    got = ob.qk_norm_backward(x["q"], x["k"], x["dq"], x["dk"], *args)
    assert torch.equal(got["dq"], want["dq"]) and torch.equal(got["dk"], want["dk"]) and bool(got["dq"].isfinite().all())
