"""The paged cache in 4 bits: the codes that an append leaves, what is read back, and attention of one token over it against the definition in 64 bits.

Codes.  A key's elements in 64 bits are off by less than 2^-48 of themselves, and the inputs here have none that lies as near to the border of two codes (the
test looks): codes and scales have to be those of the definition, to the bit.

Tolerances of attention, over the values that the codes stand for.  They, queries and (fp32: their three parts) weights are exact in bf16, so a product is exact and a score, a
sum of K products, at most K + 8 additions deep, of magnitudes that sum to A = scale sum |q_i k_i|, is off by ds <= (K + 8) 2^-24 A.  The weights e^(s - m) are
off by a factor of 1 +- (2 ds + 2^-21), and their sums are fp32, at most 2^-18 deep in all.  o is a mean of values with those weights: off by
twice that of the largest value.  With bf16 I/O a weight is the sum of two bf16 numbers, 2^-16 off, and the result is rounded: 2^-16 of the largest value and 2^-9
of that and of the result.  lse: ds, and 2^-20 of itself or one."""
import math

import pytest
import torch

from paper_2605_13473_amd import binding as ob
from tests import heads_reference as ref
from tests import pages_reference as pages

pytestmark = pytest.mark.gpu


def rnd(g, *s):
    return torch.randn(*s, device="cuda", generator=g)


def make_cache(g, n_pages, page, H, K, order="head"):
    """Codes and scales of random rows; order: which of page, head, slot follows which in memory; `apart`: rows farther apart than they are wide."""
    out = []
    for n in (K // 2, K // 2, K // 32, K // 32):
        if order == "head":
            t = torch.empty(n_pages, H, page, n, dtype=torch.uint8, device="cuda").transpose(1, 2)
        elif order == "token":
            t = torch.empty(n_pages, page, H, n, dtype=torch.uint8, device="cuda")
        elif order == "page_inside":
            t = torch.empty(H, page, n_pages, n, dtype=torch.uint8, device="cuda").permute(2, 1, 0, 3)
        else:
            t = torch.empty(n_pages, page, H, n + 16, dtype=torch.uint8, device="cuda")[..., :n]
        if n == K // 2:
            t.copy_(torch.randint(0, 256, t.shape, dtype=torch.uint8, device="cuda", generator=g))
        else:
            t.copy_(torch.randint(125, 128, t.shape, dtype=torch.uint8, device="cuda", generator=g))
        out.append(t)
    return tuple(out)


def make_table(lengths, page, extra, seed):
    gen = torch.Generator().manual_seed(seed)
    need = [max(0, -(-max(n, 0) // page)) for n in lengths]
    n_pages = sum(need) + 3
    perm = torch.randperm(n_pages, generator=gen).int()
    table = torch.full((len(lengths), max(need + [1]) + extra), -7, dtype=torch.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = perm[at:at + n]
        at += n
    return table, n_pages


# ------------------------------------------------------------------------------- append ----
APPEND = [
    dict(B=1, T=1, Hq=1, Hk=1, K=64, page=16),
    dict(B=2, T=5, Hq=6, Hk=2, K=128, page=8, norm="rms", rotary=128, order="token"),
    dict(B=3, T=7, Hq=5, Hk=5, K=256, page=4, norm="l2", rotary=64, interleaved=True, order="apart"),
    dict(B=2, T=9, Hq=3, Hk=3, K=64, page=32, io="f32", norm="rms", rotary=32),
    dict(B=1, T=33, Hq=0, Hk=7, K=128, page=16, io="f32", norm="l2", rotary=128, interleaved=True),
    dict(B=2, T=4, Hq=8, Hk=2, K=256, page=1, io="f32", rotary=256, order="page_inside"),
    dict(B=4, T=3, Hq=4, Hk=1, K=128, page=64, slices=True, norm="rms", rotary=64),
    dict(B=2, T=3, Hq=4, Hk=1, K=64, page=64, slices="odd", norm="l2", rotary=64),
    dict(B=1, T=600, Hq=2, Hk=9, K=64, page=128, norm="rms"),
]


def make_append(B, T, Hq, Hk, K, page, io="bf16", norm="none", rotary=0, interleaved=False, order="head", slices=False, seed=4):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    if slices:
        pad = 1 if slices == "odd" else 0                                             # rows off 16 bytes
        x = (3 * rnd(g, B, T, (Hq + 2 * Hk) * K + pad)).to(dt)[..., pad:]
        q, k, v = (y.unflatten(2, (-1, K)) for y in x.split([Hq * K, Hk * K, Hk * K], dim=2))
    else:
        q, k, v = ((3 * rnd(g, B, T, H, K)).to(dt) if H else None for H in (Hq, Hk, Hk))
    at = [5 + 11 * b for b in range(B)]
    table, n_pages = make_table([n + T for n in at], page, 1, seed)
    pos = torch.arange(T, dtype=torch.int32)[None] + torch.tensor(at, dtype=torch.int32)[:, None]
    return dict(q=q, k=k, v=v, wq=1 + rnd(g, K) / 8 if norm == "rms" else None, wk=1 + rnd(g, K) / 8 if norm == "rms" else None,
                rotary=ob.rotary_table(700, rotary) if rotary else None, cache=make_cache(g, n_pages, page, Hk, K, order), table=table.cuda(), pos=pos.cuda(),
                hp=ob.NormHyper(norm=norm, interleaved=interleaved))


def far_from_borders(x, codes_of):
    """No element is so near the border of two codes that 64 bits do not tell them: a step of 2^-44 either way leaves all codes."""
    a, b, c = (codes_of(x * f) for f in (1.0 - 2.0 ** -44, 1.0, 1.0 + 2.0 ** -44))
    return all(torch.equal(p, q) and torch.equal(q, r) for p, q, r in zip(a, b, c))


def exact_rows(x, which):
    w = x["w" + which]
    return ref.norm_rows(ref.f64(x[which]), ref.f64(w), ref.f64(x["rotary"]), x["pos"].cpu().long(), x["hp"].norm, x["hp"].eps, x["hp"].interleaved)


def look(x, cache, before, k, v):
    """The cache holds these rows where the tokens are and what it held elsewhere."""
    page, table, pos = cache[0].shape[1], x["table"].cpu(), x["pos"].cpu()
    for part, rows in ((0, k), (1, v)):
        codes, scales = pages.pack(rows)
        want_c, want_s = before[part].clone(), before[part + 2].clone()
        for b in range(pos.shape[0]):
            for t in range(pos.shape[1]):
                p = int(pos[b, t])
                if p < 0 or p // page >= table.shape[1] or not 0 <= int(table[b, p // page]) < want_c.shape[0]:
                    continue
                want_c[int(table[b, p // page]), p % page] = codes[b, t]
                want_s[int(table[b, p // page]), p % page] = scales[b, t]
        assert torch.equal(cache[part + 2].cpu(), want_s)
        assert torch.equal(cache[part].cpu(), want_c)


@pytest.mark.parametrize("case", APPEND, ids=lambda c: "-".join(str(v) for v in c.values()))
def test_append(case):
    x = make_append(**case)
    before = [t.cpu().clone() for t in x["cache"]]
    q = ob.paged_append_mx(x["k"], x["v"], x["cache"], x["table"], x["pos"], q=x["q"], weight_q=x["wq"], weight_k=x["wk"], rotary=x["rotary"], hp=x["hp"])
    k = exact_rows(x, "k")
    if x["hp"].norm != "none":
        assert far_from_borders(k, pages.pack)
    look(x, x["cache"], before, k, ref.f64(x["v"]))
    if x["q"] is None:
        assert q is None
    else:                                       # the queries of the append to a cache of whole bytes
        kc, vc = ob.alloc_paged_cache(x["cache"][0].shape[0], x["cache"][0].shape[1], x["k"].shape[2], x["k"].shape[3], x["k"].dtype)
        want = ob.paged_append(x["k"], x["v"], kc, vc, x["table"], x["pos"], q=x["q"], weight_q=x["wq"], weight_k=x["wk"], rotary=x["rotary"], hp=x["hp"])
        assert torch.equal(q, want)
    # what it reads back
    for dt in (torch.bfloat16, torch.float32):
        kr, vr = ob.paged_read_mx(x["cache"], x["table"], x["pos"], dtype=dt)
        for got, rows in ((kr, k), (vr, ref.f64(x["v"]))):
            assert got.dtype == dt and torch.equal(got.double().cpu(), pages.values(*pages.pack(rows)))


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_values_at_the_ends(io):
    """Zeros, ties, what lies between 6 and 7 scales, the largest and the smallest numbers, infinities and NaN: block by block."""
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    big = torch.finfo(dt).max
    rows = torch.zeros(1, 12, 1, 64)
    rows[0, 1, 0, :32] = torch.arange(32) / 4.0 - 1.0                  # ties of every border, and 6.75
    rows[0, 1, 0, 32:] = -torch.arange(32) / 4.0 + 0.75
    rows[0, 2, 0, 0], rows[0, 2, 0, 33] = 7.0, 7.03125                 # the border of two scales
    rows[0, 3, 0, :32], rows[0, 3, 0, 32:] = big, -big
    rows[0, 4, 0, :32], rows[0, 4, 0, 40] = 2.0 ** -120, 2.0 ** -126   # the least scale
    rows[0, 5, 0, 3] = math.inf
    rows[0, 6, 0, 60] = math.nan
    rows[0, 7, 0, 9], rows[0, 7, 0, 10] = -math.inf, 1.0
    rows[0, 8, 0] = 2.0 ** torch.arange(64).float() * 2.0 ** -40
    rows[0, 9, 0, ::2] = -0.0
    rows[0, 10, 0] = 1e-40 if io == "f32" else 1e-38
    rows[0, 11, 0] = 3.0 * 2.0 ** -122
    k = rows.to(dt).cuda()
    g = torch.Generator(device="cuda").manual_seed(1)
    table, n_pages = make_table([12], 16, 0, 2)
    x = dict(table=table.cuda(), pos=torch.arange(12, dtype=torch.int32)[None].cuda())
    cache = make_cache(g, n_pages, 16, 1, 64)
    before = [t.cpu().clone() for t in cache]
    ob.paged_append_mx(k, k.flip(1), cache, x["table"], x["pos"], hp=ob.NormHyper(norm="none"))
    look(x, cache, before, ref.f64(k), ref.f64(k.flip(1)))
    kr, _ = ob.paged_read_mx(cache, x["table"], x["pos"], dtype=torch.float32)
    nan = torch.isnan(kr[0, :, 0]).cpu()
    want = torch.zeros(12, 64, dtype=torch.bool)
    want[5, :32] = want[6, 32:] = want[7, :32] = True
    assert torch.equal(nan, want) and bool(torch.isfinite(kr[0, :, 0].cpu()[~want]).all())


@pytest.mark.parametrize("T,Hq,Hk,K", [(1, 1, 1, 64), (37, 7, 3, 128), (300, 5, 2, 256)])
def test_queries_in_place(T, Hq, Hk, K):
    """q_out may be q: the same rows as into an array of their own."""
    x = make_append(2, T, Hq, Hk, K, 16, norm="rms", rotary=K)
    q = x["q"].clone()
    want = ob.paged_append_mx(x["k"], x["v"], x["cache"], x["table"], x["pos"], q=q, rotary=x["rotary"], hp=ob.NormHyper("rms"))
    p = ob._params_of(q, x["k"], ob.NormHyper("rms"), x["rotary"])
    ob.osdn_paged_append_mx(p, q, x["k"], x["v"], x["cache"], x["table"], None, None, x["rotary"], x["pos"], None, q)
    assert torch.equal(q, want) and not torch.equal(q, x["q"])


def test_rows_past_what_fp32_squares():
    """Keys whose squares leave the range of fp32: in 64 bits they have a norm; a row with an infinity is NaN in its blocks that hold one and zero in the others."""
    k = torch.full((1, 3, 1, 128), 1e30, device="cuda")
    k[0, 1, 0, 5] = math.inf
    k[0, 2] *= 1e-36
    table = torch.zeros(1, 1, dtype=torch.int32, device="cuda")
    pos = torch.arange(3, dtype=torch.int32, device="cuda")[None]
    cache = ob.alloc_paged_cache_mx(1, 4, 1, 128)
    ob.paged_append_mx(k, torch.zeros_like(k), cache, table, pos, hp=ob.NormHyper(norm="rms"))
    kr, vr = ob.paged_read_mx(cache, table, pos, dtype=torch.float32)
    assert bool((kr[0, 0] == 1.0).all()) and bool((vr == 0).all())
    assert bool(torch.isnan(kr[0, 1, 0, :32]).all()) and bool((kr[0, 1, 0, 32:] == 0).all())
    assert bool(torch.isfinite(kr[0, 2]).all())


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_every_scale_and_code(io):
    """All sixteen codes under all scales, those that no append leaves among them, as read and as the bounds of a page.  (4 * 2^126 and more, under the scales 253 and 254, is
    more than the type holds: infinite, as rounded to it.)"""
    codes = torch.tensor([(2 * i % 16) | ((2 * i + 1) % 16) << 4 for i in range(32)], dtype=torch.uint8).expand(256, 1, 1, 32)
    scales = torch.stack([torch.arange(256), 255 - torch.arange(256)], dim=-1).to(torch.uint8)[:, None, None]
    cache = tuple(t.contiguous().cuda() for t in (codes, codes.flip(-1), scales, scales))
    table, pos = torch.arange(256, dtype=torch.int32, device="cuda")[None], torch.arange(256, dtype=torch.int32, device="cuda")[None]
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    got = ob.paged_read_mx(cache, table, pos, dtype=dt)
    for x, i in zip(got, range(2)):
        want = pages.values(cache[i].cpu(), cache[i + 2].cpu())[:, 0].to(dt).double()
        assert torch.equal(x[0].double().cpu().nan_to_num(1e300), want.nan_to_num(1e300))
    bounds = ob.alloc_page_bounds(256, 1, 64, dt).zero_()
    ob.page_bounds((cache[0], cache[2]), table, torch.zeros(1, dtype=torch.int32, device="cuda"), torch.tensor([256], dtype=torch.int32, device="cuda"), bounds)
    want = pages.values(cache[0].cpu(), cache[2].cpu())[:, 0, 0].to(dt).double()
    for side in range(2):
        assert torch.equal(bounds[:, 0, side].double().cpu().nan_to_num(1e300), want.nan_to_num(1e300))


def test_tokens_without_a_place():
    """No token, a sequence or a page that is not there, a position past the table: not appended, nothing else touched; read as zeros and NaN."""
    x = make_append(2, 6, 4, 2, 128, 8, norm="rms", rotary=128)
    x["pos"][0, 1] = -1
    x["pos"][0, 4] = -2 ** 31
    x["pos"][1, 3] = 8 * x["table"].shape[1]
    x["table"][1, 2] = -1
    x["table"][0, 1] = x["cache"][0].shape[0]
    before = [t.cpu().clone() for t in x["cache"]]
    seq = torch.tensor([[0] * 6, [1] * 5 + [7]], dtype=torch.int32, device="cuda")
    q = ob.paged_append_mx(x["k"], x["v"], x["cache"], x["table"], x["pos"], seq, q=x["q"], weight_q=x["wq"], weight_k=x["wk"], rotary=x["rotary"], hp=x["hp"])
    k = exact_rows(x, "k") if int(x["pos"].max()) < 700 else None
    assert bool((q[0, 1] == 0).all()) and bool((q[0, 4] == 0).all())
    x["pos"][1, 5] = -1                          # (for the reference: a sequence that is not there)
    look(x, x["cache"], before, k, ref.f64(x["v"]))
    x["pos"][1, 5] = 5
    kr, vr = ob.paged_read_mx(x["cache"], x["table"], x["pos"], seq)
    for r in (kr, vr):
        assert bool((r[0, 1] == 0).all()) and bool((r[0, 4] == 0).all()) and bool(torch.isnan(r[1, 3]).all()) and bool(torch.isnan(r[1, 5]).all())


# ------------------------------------------------------------------------------- decode ----
DECODE = [
    dict(lengths=[1], Hq=1, Hk=1, K=64, page=16),
    dict(lengths=[1], Hq=4, Hk=4, K=64, page=1, io="f32"),
    dict(lengths=[0, 1, 2, 31, 32, 33], Hq=8, Hk=2, K=128, page=16),
    dict(lengths=[0, -3, 127, 128, 129, 255], Hq=6, Hk=2, K=128, page=32, io="f32"),
    dict(lengths=[1531], Hq=16, Hk=4, K=128, page=16, order="token"),
    dict(lengths=[700, 0, 3, 1025], Hq=5, Hk=1, K=256, page=8),
    dict(lengths=[700, 0, 3, 1025], Hq=5, Hk=5, K=256, page=64, io="f32", order="apart"),
    dict(lengths=[300, 77], Hq=40, Hk=2, K=64, page=128, order="page_inside"),
    dict(lengths=[300, 77], Hq=33, Hk=1, K=128, page=4, io="f32"),
    dict(lengths=[300, 77, 5, 0], Hq=8, Hk=2, K=128, page=16, window=1),
    dict(lengths=[300, 77, 5, 0], Hq=8, Hk=2, K=128, page=16, window=50),
    dict(lengths=[2000, 1999, 40], Hq=7, Hk=1, K=64, page=2, window=1000, io="f32"),
    dict(lengths=[2000, 1999, 40], Hq=16, Hk=1, K=256, page=1024, window=33),
    dict(lengths=[5000, 4096, 4097, 1], Hq=4, Hk=1, K=64, page=256, shares=33),
    dict(lengths=[5000, 4096, 4097, 1], Hq=4, Hk=1, K=128, page=64, shares=7),
    dict(lengths=[130] * 70, Hq=2, Hk=2, K=64, page=32),
    dict(lengths=[20000], Hq=2, Hk=1, K=128, page=64),
    dict(lengths=[(37 * i) % 200 - 3 for i in range(600)], Hq=2, Hk=1, K=64, page=16, shares=50),
    dict(lengths=[(91 * i) % 400 for i in range(300)], Hq=3, Hk=1, K=256, page=32, io="f32", window=150),
    dict(lengths=[900, 33, 512, 1], Hq=16, Hk=8, K=128, page=16, order="token"),
]


def make_decode(lengths, Hq, Hk, K, page, io="bf16", order="head", window=0, shares=0, seed=2):
    g = torch.Generator(device="cuda").manual_seed(seed)
    table, n_pages = make_table(lengths, page, extra=2, seed=seed)
    return dict(q=rnd(g, len(lengths), Hq, K).to(torch.bfloat16 if io == "bf16" else torch.float32), cache=make_cache(g, n_pages, page, Hk, K, order), table=table.cuda(),
                lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"), window=window, shares=shares, longest=max(max(lengths), 0))


def call(x, seq=None, max_length=None, scale=None):
    B, Hq, K = x["q"].shape
    p = ob.make_decode_params(B, Hq, x["cache"][0].shape[2], K, x["q"].dtype == torch.bfloat16, x["longest"] if max_length is None else max_length, scale,
                              x["window"], x["shares"])
    n = ob.osdn_paged_decode_mx_workspace_bytes(p)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda") if n else None            # (fp32 NaN: nothing in it is read before it is written)
    o, lse = torch.empty_like(x["q"]), torch.empty(B, Hq, device="cuda")
    ob.osdn_paged_decode_mx(p, x["q"], x["cache"], x["table"], x["lengths"], seq, o, lse, ws)
    return o, lse


def hold(o, lse, want, wlse, size, vmax, K, bf16):
    ds = (K + 8) * 2.0 ** -24 * size
    tol = 2 * (2 * ds + 2.0 ** -21 + 2.0 ** -18 + (2.0 ** -16 if bf16 else 0.0))[..., None] * vmax + (2.0 ** -9 * (vmax + want.abs()) if bf16 else 0.0)
    err = (o.double().cpu() - want).abs()
    assert (err <= tol).all(), f"o: worst {float((err / tol).nan_to_num(9e9).max()):.3g} of the tolerance"
    empty = torch.isinf(wlse)
    assert torch.equal(torch.isinf(lse.cpu()) & (lse.cpu() < 0), empty) and bool((o.cpu()[empty] == 0).all())
    lt = ds + 2.0 ** -20 * wlse.abs().clamp(min=1.0)
    assert ((lse.double().cpu() - wlse).abs()[~empty] <= lt[~empty]).all()


def compare(x, o, lse, seq=None, scale=None):
    B, Hq, K = x["q"].shape
    k, v = (pages.values(x["cache"][i].cpu(), x["cache"][i + 2].cpu()) for i in range(2))
    want, wlse, size = ref.decode(ref.f64(x["q"]), k, v, x["table"].cpu(), x["lengths"].cpu(), torch.arange(B) if seq is None else seq.cpu(), K ** -0.5 if scale is None else scale,
                                  x["window"])
    hold(o, lse, want, wlse, size, float(v.nan_to_num(0.0).abs().max()), K, x["q"].dtype == torch.bfloat16)


@pytest.mark.parametrize("case", DECODE, ids=lambda c: "-".join(str(v) for v in c.values())[:80])
def test_decode(case):
    x = make_decode(**case)
    o, lse = call(x)
    compare(x, o, lse)
    # what no length shows: not looked at, whatever stands there
    shown = torch.zeros(x["cache"][0].shape[:2], dtype=torch.bool)
    page = x["cache"][0].shape[1]
    for b, n in enumerate(case["lengths"]):
        j = torch.arange(max(0, n - case.get("window", 0)) if case.get("window") else 0, max(n, 0))
        shown[x["table"].cpu()[b][j // page].long(), j % page] = True
    for poison in (255, 254, 0):
        for c in x["cache"]:
            c.masked_fill_(~shown.cuda()[..., None, None], poison)
        o2, lse2 = call(x)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
    # a launch sized for more than is there, and other cuts: the same answer
    for shares in (-1, 1, 3, 1000):
        compare(x, *call(dict(x, shares=shares)))
    compare(x, *call(x, max_length=x["longest"] + 777 if x["longest"] + 777 <= x["table"].shape[1] * page else x["longest"]))


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("group", [1, 4, 20])
def test_rows_that_may_be_many(io, group):
    """A bound of the lengths beyond 64 MB of rows: their codes are loaded past the caches, in shares and a row each; the lengths themselves stay small."""
    for B, lengths in ((3, [1531, 0, 77]), (130, [1 + 37 * b % 530 for b in range(130)])):
        for K in (64, 128):
            x = make_decode(lengths, 4 * group, 4, K, 16, io)
            compare(x, *call(x, max_length=1 << 17 if B == 3 else 2000 * 128 // K))


@pytest.mark.parametrize("Hq,Hk,K", [(6, 3, 64), (8, 4, 128), (18, 1, 64), (4, 4, 256), (40, 2, 128)])
def test_heads_side_by_side(Hq, Hk, K):
    """More sequences than XCDs, and some over: the workgroups of a sequence on one of them."""
    x = make_decode([(97 * b) % 260 for b in range(19)], Hq, Hk, K, 8, order="token")
    compare(x, *call(x))
    x = make_decode([(97 * b) % 260 for b in range(16)], Hq, Hk, K, 8, order="token", shares=-1)
    compare(x, *call(x))


def test_decode_slices_several_queries_and_scale():
    x = make_decode([200, 33], 8, 2, 128, 16)
    wide = torch.randn(2, 12, 128, device="cuda").bfloat16()
    wide[:, 2:10] = x["q"]
    a, lse = ob.paged_decode_mx(wide[:, 2:10], x["cache"], x["table"], x["lengths"], want_lse=True)
    compare(x, a, lse)
    b = ob.paged_decode_mx(x["q"], x["cache"], x["table"], x["lengths"], max_length=200)
    compare(x, b, lse)
    odd = torch.empty(2, 8, 131, device="cuda", dtype=torch.bfloat16)[..., 3:]          # rows off 16 bytes, written too
    odd.copy_(x["q"])
    p = ob.make_decode_params(2, 8, 2, 128, True, 200)
    n = ob.osdn_paged_decode_mx_workspace_bytes(p)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
    ob.osdn_paged_decode_mx(p, odd, x["cache"], x["table"], x["lengths"], None, odd, None, ws)
    assert torch.equal(odd, b)
    seq = torch.tensor([1, 0, 0, 1, 0], dtype=torch.int32, device="cuda")
    y = dict(x, q=torch.randn(5, 8, 128, device="cuda").bfloat16(), lengths=torch.tensor([33, 199, 200, 1, 0], dtype=torch.int32, device="cuda"))
    o, lse = ob.paged_decode_mx(y["q"], y["cache"], y["table"], y["lengths"], seq, scale=0.3, want_lse=True)
    compare(y, o, lse, seq, 0.3)


def test_blocks_that_are_nan_and_what_is_not_there():
    x = make_decode([40, 40, 40, 40, 40, 200], 4, 2, 128, 16)
    o, lse = call(x)
    t = x["table"]
    x["cache"][2][int(t[0, 1]), 3, 1, 2] = 255          # a key of head 1
    x["cache"][3][int(t[1, 0]), 5, 0, 0] = 255          # a value of head 0: its first 32 elements
    t[2, 1] = -1
    x["lengths"][3] = 10 ** 6                           # more than was promised
    seq = torch.tensor([0, 1, 2, 3, 77, 5], dtype=torch.int32, device="cuda")
    o2, l2 = call(x, seq=seq)
    nan = torch.isnan(o2).cpu()
    want = torch.zeros_like(nan)
    want[0, 2:] = True
    want[1, :2, :32] = True
    want[2:5] = True
    assert torch.equal(nan, want)
    assert torch.equal(torch.isnan(l2).cpu(), want.all(-1))
    same = ~want
    assert torch.equal(o2.cpu()[5], o.cpu()[5]) and torch.equal(o2.cpu()[same], o.cpu()[same])


def test_more_queries_than_a_launch_takes():
    g = torch.Generator(device="cuda").manual_seed(8)
    x = make_decode([60, 3], 2, 1, 64, 16)
    B = 70000
    seq = torch.randint(0, 2, (B,), dtype=torch.int32, device="cuda", generator=g)
    lengths = torch.minimum(torch.randint(0, 61, (B,), dtype=torch.int32, device="cuda", generator=g), torch.tensor([60, 3], dtype=torch.int32, device="cuda")[seq.long()])
    q = rnd(g, B, 2, 64).bfloat16()
    o, lse = ob.paged_decode_mx(q, x["cache"], x["table"], lengths, seq, max_length=60, want_lse=True)
    for at in (0, 34999, 35000, 69990):
        s = slice(at, at + 10)
        compare(dict(x, q=q[s], lengths=lengths[s]), o[s], lse[s], seq[s])


def test_fp32_holds_more_than_bf16():
    """fp32 queries and weights are not rounded on their way: far closer than one rounding to bf16 would leave them."""
    x = make_decode([777, 64], 8, 2, 128, 16, io="f32")
    o, lse = call(x)
    k, v = (pages.values(x["cache"][i].cpu(), x["cache"][i + 2].cpu()) for i in range(2))
    want, wlse, _ = ref.decode(ref.f64(x["q"]), k, v, x["table"].cpu(), x["lengths"].cpu(), torch.arange(2), 128 ** -0.5, 0)
    assert float((o.double().cpu() - want).norm() / want.norm()) < 2.0 ** -18


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_append_read_and_attend_in_a_graph(io):
    """Tokens one by one through append, read and attention, captured once: every replay against the eager calls."""
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(6)
    B, Hq, Hk, K, page = 3, 4, 2, 128, 4
    rot = ob.rotary_table(64, K)
    table = torch.randperm(B * 10, generator=torch.Generator().manual_seed(1)).int().view(B, 10).cuda()
    text = [rnd(g, 12, B, 1, H, K).to(dt) for H in (Hq, Hk, Hk)]
    hp = ob.NormHyper(norm="rms")

    def step(q, k, v, cache, pos, lengths):
        qr = ob.paged_append_mx(k, v, cache, table, pos, q=q, rotary=rot, hp=hp)
        back = ob.paged_read_mx(cache, table, pos, dtype=dt)
        return (*ob.paged_decode_mx(qr[:, 0], cache, table, lengths, max_length=12, want_lse=True), *back)

    eager, graphed = (tuple(t.zero_() for t in ob.alloc_paged_cache_mx(B * 10, page, Hk, K)) for _ in range(2))
    pos = torch.zeros(B, 1, dtype=torch.int32, device="cuda")
    lengths = torch.ones(B, dtype=torch.int32, device="cuda")
    held = [t[0].clone() for t in text]
    graph = torch.cuda.CUDAGraph()
    step(*held, graphed, pos, lengths)
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = step(*held, graphed, pos, lengths)
    for i in range(12):
        pos.fill_(i)
        lengths.fill_(i + 1)
        for h, t in zip(held, text):
            h.copy_(t[i])
        graph.replay()
        want = step(*held, eager, pos, lengths)
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(out, want))
        assert all(torch.equal(a, b) for a, b in zip(eager, graphed))


@pytest.mark.parametrize("step", [3 << 30, 5 << 30])
def test_offsets_past_32_bits(step):
    """Pages 3 (one rule finds a row's place in all four arrays) and 5 GiB apart: what is appended, read and attended to is that of a small cache, to the bit."""
    g = torch.Generator(device="cuda").manual_seed(8)
    far = [torch.zeros(2 * s + 2048, dtype=torch.uint8, device="cuda").as_strided((3, 8, 2, n), (s, 2 * n, n, 1)) for n, s in ((64, step), (64, step), (4, step // 16), (4, step // 16))]
    near = [t.clone() for t in make_cache(g, 3, 8, 2, 128, "token")]
    for a, b in zip(far, near):
        a.copy_(b)
    table = torch.tensor([[2, 0, 1]], dtype=torch.int32, device="cuda")
    k, v, q = rnd(g, 1, 21, 2, 128).bfloat16(), rnd(g, 1, 21, 2, 128).bfloat16(), rnd(g, 1, 4, 128).bfloat16()
    pos, n = torch.arange(2, 23, dtype=torch.int32, device="cuda")[None], torch.tensor([23], dtype=torch.int32, device="cuda")
    got = []
    for cache in (tuple(near), tuple(far)):
        ob.paged_append_mx(k, v, cache, table, pos, hp=ob.NormHyper("rms"))
        bounds = ob.alloc_page_bounds(3, 2, 128).zero_()
        ob.page_bounds((cache[0], cache[2]), table, torch.zeros_like(n), n, bounds)
        chosen, tokens = ob.page_select(q, bounds, table, n, 8, 2)
        got.append([*ob.paged_read_mx(cache, table, pos), ob.paged_decode_mx(q, cache, table, n), bounds, chosen, ob.paged_decode_pages_mx(q, cache, chosen, tokens)])
    for a, b in zip(*got):
        assert torch.equal(a, b)
