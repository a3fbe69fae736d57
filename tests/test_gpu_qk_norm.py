"""Norm of queries and keys with the position rotation, forward and backward, against the definition in 64 bits.

Tolerances.  Forward: a row's factor r comes from a sum of squares whose depth is at most 16 fused steps, and an element sees at most
six more roundings, each of 2^-24 of the row's largest magnitude before the rotation: e = 2^-19 of it.  A bf16 result is that, rounded once: it
lies between the roundings of the exact value less e and plus e.
Backward: the same with the magnitudes that are subtracted from one another.  dweight: every term 2^-19 of its magnitude, the
sums over rows at most 64 deep: 2^-18 of the sum of magnitudes."""
import pytest
import torch

from paper_2605_13473_amd import binding as ob
from tests import heads_reference as ref

pytestmark = pytest.mark.gpu
EPS32 = 2.0 ** -19


def rnd(g, *s):
    return torch.randn(*s, device="cuda", generator=g)


def make(B, T, Hq, Hk, K, io="bf16", norm="rms", weighted=True, rotary=0, interleaved=False, positions=None, layout="plain", seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.bfloat16 if io == "bf16" else torch.float32

    def rows(H):
        x = rnd(g, B, T, H, K) * torch.exp(rnd(g, B, T, H, 1))
        if layout == "fused":           # slices of one projection
            return x
        if layout == "heads_first":     # [B,H,T,K] seen as [B,T,H,K]
            return x.to(dt).transpose(1, 2).contiguous().transpose(1, 2)
        if layout == "odd":             # rows that start off 16 bytes, a step that is no multiple of them
            y = torch.empty(B, T, H, K + 5, device="cuda", dtype=dt)[..., 3:3 + K]
            return y.copy_(x)
        if layout == "longer":          # a part of a longer axis: batch is not T x token
            y = torch.empty(B, T + 3, H, K, device="cuda", dtype=dt)[:, 1:1 + T]
            return y.copy_(x)
        return x.to(dt)

    q, k = rows(Hq), rows(Hk)
    if layout == "fused":
        f = torch.cat([q.flatten(2), k.flatten(2), rnd(g, B, T, Hk * K)], dim=2).to(dt)
        q, k, _ = (y.unflatten(2, (-1, K)) for y in f.split([Hq * K, Hk * K, Hk * K], dim=2))
    dq, dk = rows(Hq).to(dt), rows(Hk).to(dt)
    table = ob.rotary_table(max(T, 50), rotary, 10000.0) if rotary else None
    pos = None
    if positions == "given":
        pos = torch.randint(0, 50, (B, T), device="cuda", generator=g, dtype=torch.int32)
        pos.view(-1)[:: 5] = -1
    w = [0.5 + torch.rand(K, device="cuda", generator=g) if weighted else None for _ in range(2)]
    return dict(q=q, k=k, wq=w[0], wk=w[1], table=table, pos=pos, dq=dq, dk=dk, hp=ob.NormHyper(norm=norm, interleaved=interleaved), B=B, T=T)


CASES = [
    dict(B=1, T=1, Hq=1, Hk=1, K=64, norm="l2", weighted=False),
    dict(B=2, T=7, Hq=5, Hk=3, K=128, norm="l2", weighted=False),
    dict(B=2, T=7, Hq=5, Hk=3, K=128, io="f32", norm="l2", rotary=64),
    dict(B=3, T=33, Hq=16, Hk=2, K=128, rotary=128),
    dict(B=3, T=33, Hq=16, Hk=2, K=128, rotary=128, positions="given", layout="fused"),
    dict(B=1, T=70, Hq=7, Hk=1, K=256, rotary=256, interleaved=True),
    dict(B=1, T=70, Hq=9, Hk=9, K=256, rotary=96, layout="heads_first"),
    dict(B=2, T=19, Hq=3, Hk=3, K=256, io="f32", rotary=256, layout="fused"),
    dict(B=2, T=19, Hq=6, Hk=6, K=64, io="f32", rotary=16, interleaved=True, positions="given"),
    dict(B=2, T=19, Hq=9, Hk=2, K=64, rotary=64, norm="none", layout="odd"),
    dict(B=2, T=19, Hq=9, Hk=2, K=64, rotary=48, norm="none", weighted=False, interleaved=True, layout="longer"),
    dict(B=2, T=11, Hq=4, Hk=2, K=128, io="f32", rotary=128, layout="odd"),
    dict(B=2, T=11, Hq=4, Hk=2, K=128, rotary=112, layout="odd", positions="given"),
    dict(B=5, T=410, Hq=12, Hk=4, K=64, rotary=32, layout="longer"),
    dict(B=4, T=1031, Hq=16, Hk=16, K=128, norm="l2", weighted=False),
    dict(B=1, T=2049, Hq=8, Hk=2, K=128, rotary=128, positions="given"),
]


def check(got, want, scale, bf16, name):
    got = got.double().cpu()
    lo, hi = want - EPS32 * scale, want + EPS32 * scale
    if bf16:                # (rounding keeps the order; through fp32, whose own rounding is far below e)
        lo, hi = (x.float().bfloat16().double() for x in (lo, hi))
    bad = ~((got >= lo) & (got <= hi))
    assert not bad.any(), f"{name}: {int(bad.sum())} of {bad.numel()} off, the worst by {float((got - want).abs()[bad].max()):.3g}"


def reference(x):
    pos = torch.arange(x["T"]).expand(x["B"], -1) if x["pos"] is None else x["pos"].cpu().long()
    table, hp = ref.f64(x["table"]), x["hp"]
    out = {}
    for n in "qk":
        rows, w = ref.f64(x[n]).contiguous().requires_grad_(), None if x["w" + n] is None else ref.f64(x["w" + n]).requires_grad_()
        z = ref.norm_rows(rows, w, table, pos, hp.norm, hp.eps, hp.interleaved)
        out[n] = (rows, w, z)
    return out, pos, table


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(v) for v in c.values()))
def test_forward_and_backward(case):
    x = make(**case)
    bf16 = x["q"].dtype == torch.bfloat16
    out, pos, table = reference(x)
    z = ob.qk_norm(x["q"], x["k"], x["wq"], x["wk"], x["table"], x["pos"], x["hp"])
    g = ob.qk_norm_backward(x["q"], x["k"], x["dq"], x["dk"], x["wq"], x["wk"], x["table"], x["pos"], x["hp"])
    for n, got in zip("qk", z):
        rows, w, want = out[n]
        y = ref.norm_rows(rows.detach(), None if w is None else w.detach(), None, pos, x["hp"].norm, x["hp"].eps, False)
        check(got, want.detach(), y.abs().amax(-1, keepdim=True), bf16, n)
        dz = ref.f64(x["d" + n])
        grads = torch.autograd.grad(want, [rows] + ([w] if w is not None else []), dz)
        # the magnitudes that meet in an element of dx
        m = {"l2": 1.0, "rms": 1.0 / rows.shape[-1], "none": 0.0}[x["hp"].norm]
        xr = rows.detach()
        r = (m * (xr * xr).sum(-1, keepdim=True) + x["hp"].eps) ** -0.5 if m else torch.ones_like(xr[..., :1])
        dy = ref.turn(dz, table, pos.clamp(min=0), x["hp"].interleaved, -1.0)
        gmax = 1.5 * dz.abs().amax(-1, keepdim=True) * (1.0 if w is None else w.detach().abs().max())
        scale = r * (gmax + xr.abs() * r * r * m * (gmax * xr.abs()).sum(-1, keepdim=True))
        check(g["d" + n], grads[0], scale, bf16, "d" + n)
        if w is not None:
            alive = (pos >= 0)[..., None, None]
            size = (torch.where(alive, 1.5 * dz.abs().amax(-1, keepdim=True) * xr.abs() * r, torch.zeros_like(xr))).sum((0, 1, 2))
            assert ((g["dweight_" + n].double().cpu() - grads[1]).abs() <= 2.0 ** -18 * size).all()
        else:
            assert g["dweight_" + n] is None


@pytest.mark.parametrize("norm", ["l2", "rms"])
def test_gradient_against_differences(norm):
    """The kernel's gradients (fp32) along a direction, against central differences of the definition in 64 bits: the third
    derivative leaves h^2 = 1e-8 relative, the kernel 2^-18."""
    x = make(B=2, T=9, Hq=4, Hk=2, K=64, io="f32", norm=norm, rotary=32, positions="given", seed=3)
    out, pos, table = reference(x)
    g = ob.qk_norm_backward(x["q"], x["k"], x["dq"], x["dk"], x["wq"], x["wk"], x["table"], x["pos"], x["hp"])
    gen = torch.Generator().manual_seed(0)
    for n in "qk":
        rows, w, _ = out[n]
        rows, w, dz = rows.detach(), w.detach(), ref.f64(x["d" + n])
        loss = lambda a, b: (ref.norm_rows(a, b, table, pos, norm, x["hp"].eps, False) * dz).sum()
        u, uw = torch.randn(rows.shape, generator=gen, dtype=torch.float64) * rows.abs().mean(-1, keepdim=True), torch.randn(w.shape, generator=gen, dtype=torch.float64)
        for ua, ub, grad, along in ((u, 0 * uw, g["d" + n], u), (0 * u, uw, g["dweight_" + n], uw)):
            h = 1e-4
            diff = (loss(rows + h * ua, w + h * ub) - loss(rows - h * ua, w - h * ub)) / (2 * h)
            got = (ref.f64(grad) * along).sum()
            size = (ref.f64(grad).abs() * along.abs()).sum()
            assert abs(got - diff) <= (2.0 ** -18 + 1e-6) * size


def test_in_place_and_into_slices():
    """Outputs may be the inputs themselves, and slices of a wider tensor whose rest is left alone."""
    x = make(B=2, T=21, Hq=6, Hk=2, K=128, rotary=64, layout="fused")
    p = ob.make_norm_params(2, 21, 6, 2, 128, True, x["hp"], x["table"])
    want = ob.qk_norm(x["q"], x["k"], x["wq"], x["wk"], x["table"], None, x["hp"])
    g = ob.qk_norm_backward(x["q"], x["k"], x["dq"], x["dk"], x["wq"], x["wk"], x["table"], None, x["hp"])
    wide = torch.full((2, 21, 10 * 128), 7.0, device="cuda", dtype=torch.bfloat16)
    dq, dk, rest = (y.unflatten(2, (-1, 128)) for y in wide.split([6 * 128, 2 * 128, 2 * 128], dim=2))
    ob.osdn_qk_norm_bwd(p, x["q"], x["k"], x["wq"], x["wk"], x["table"], None, x["dq"], x["dk"], dq, dk, None, None)
    assert torch.equal(dq, g["dq"]) and torch.equal(dk, g["dk"]) and bool((rest == 7.0).all())
    for a, b in ((x["dq"], x["dk"]), (x["q"].clone(), x["k"].clone())):
        q, k = (x["q"], x["k"]) if a is x["dq"] else (a, b)
        da, db = (a, b) if a is x["dq"] else (x["dq0"], x["dk0"])
        if a is x["dq"]:
            x["dq0"], x["dk0"] = a.clone(), b.clone()
        ob.osdn_qk_norm_bwd(p, q, k, x["wq"], x["wk"], x["table"], None, da, db, a, b, None, None)
        assert torch.equal(a, g["dq"]) and torch.equal(b, g["dk"])
    ob.osdn_qk_norm_fwd(p, x["q"], x["k"], x["wq"], x["wk"], x["table"], None, x["q"], x["k"])
    assert torch.equal(x["q"], want[0]) and torch.equal(x["k"], want[1])


def test_one_of_the_two_and_repeatable():
    x = make(B=2, T=130, Hq=5, Hk=3, K=128, rotary=128)
    q, k = ob.qk_norm(x["q"], x["k"], x["wq"], x["wk"], x["table"], None, x["hp"])
    a, none = ob.qk_norm(x["q"], None, x["wq"], None, x["table"], None, x["hp"])
    none2, b = ob.qk_norm(None, x["k"], None, x["wk"], x["table"], None, x["hp"])
    assert none is None and none2 is None and torch.equal(a, q) and torch.equal(b, k)
    first = ob.qk_norm_backward(x["q"], x["k"], x["dq"], x["dk"], x["wq"], x["wk"], x["table"], None, x["hp"])
    for _ in range(3):
        again = ob.qk_norm_backward(x["q"], x["k"], x["dq"], x["dk"], x["wq"], x["wk"], x["table"], None, x["hp"])
        assert all(torch.equal(first[n], again[n]) for n in first)
    only = ob.qk_norm_backward(None, x["k"], None, x["dk"], None, x["wk"], x["table"], None, x["hp"])
    assert only["dq"] is None and torch.equal(only["dk"], first["dk"])
    # (a call without queries is cut otherwise: the weights' sums in another order, each within the bound of the exact ones)
    size = (1.5 * x["dk"].float().abs().amax(-1, keepdim=True) * ob.qk_norm(None, x["k"], hp=x["hp"])[1].float().abs()).sum((0, 1, 2))
    assert ((only["dweight_k"] - first["dweight_k"]).abs() <= 2 * 2.0 ** -18 * size).all()


def test_rows_of_zeros_and_positions_off_the_table():
    x = make(B=1, T=4, Hq=2, Hk=1, K=64, rotary=64, positions="given")
    x["q"][0, 1] = 0
    x["pos"].copy_(torch.tensor([[3, 7, 50, -1]], dtype=torch.int32))          # the table has 50 rows
    q, k = ob.qk_norm(x["q"], x["k"], x["wq"], x["wk"], x["table"], x["pos"], x["hp"])
    assert bool((q[0, 1] == 0).all()) and bool(q[0, 2].isnan().all()) and bool((q[0, 3] == 0).all()) and bool(k[0, 2].isnan().all())
    assert bool(q[0, :2].isfinite().all()) and bool(k[0, :2].isfinite().all())
    g = ob.qk_norm_backward(x["q"], x["k"], x["dq"], x["dk"], x["wq"], x["wk"], x["table"], x["pos"], x["hp"])
    assert bool(g["dq"][0, 2].isnan().all()) and bool((g["dq"][0, 3] == 0).all()) and bool(g["dq"][0, :2].isfinite().all())


def test_on_another_stream():
    x = make(B=2, T=300, Hq=8, Hk=4, K=128, rotary=128)
    want = ob.qk_norm(x["q"], x["k"], x["wq"], x["wk"], x["table"], None, x["hp"])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        got = ob.qk_norm(x["q"], x["k"], x["wq"], x["wk"], x["table"], None, x["hp"])
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
