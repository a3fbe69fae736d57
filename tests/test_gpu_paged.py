"""The paged cache: what an append writes and leaves, and attention of one token over the cache against the definition in 64 bits.

Tolerances of attention.  A score is a sum of K products, at most K / 4 + 8 additions deep, of magnitudes that sum to A = scale sum |q_i k_i|:
it is off by ds <= (K / 4 + 8) 2^-24 A.  The weights e^(s - m) are then off by a factor of 1 +- (2 ds + 2^-21) (the maximum's own error
included), and their sums are fp32, at most 2^-18 deep in all.  o is a mean of values with those weights: off by twice that of the largest value.
With bf16 I/O every weight is rounded once more and so is the result: 2^-9 of the largest value and of the result (the result's own rounding
is 2^-8 of it at most, which is below that; the weights' roundings fall either way).  lse: ds, and 2^-20 of itself or one."""
import math

import pytest
import torch

from paper_2605_13473_amd import binding as ob
from tests import heads_reference as ref

pytestmark = pytest.mark.gpu


def rnd(g, *s):
    return torch.randn(*s, device="cuda", generator=g)


def make_cache(g, n_pages, page, H, K, dt, order):
    """order: which of page, head, slot follows which in memory; `apart`: rows farther apart than they are wide."""
    if order == "head":
        return rnd(g, n_pages, H, page, K).to(dt).transpose(1, 2)
    if order == "token":
        return rnd(g, n_pages, page, H, K).to(dt)
    if order == "page_inside":
        return rnd(g, H, page, n_pages, K).to(dt).permute(2, 1, 0, 3)
    return rnd(g, n_pages, page, H, K + 8).to(dt)[..., :K]


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
]


def make_decode(lengths, Hq, Hk, K, page, io="bf16", order="head", window=0, shares=0, seed=2, spread=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    table, n_pages = make_table(lengths, page, extra=2, seed=seed)
    kc, vc = (make_cache(g, n_pages, page, Hk, K, dt, order) for _ in range(2))
    return dict(q=(spread * rnd(g, len(lengths), Hq, K)).to(dt), kc=kc, vc=vc, table=table.cuda(), lengths=torch.tensor(lengths, dtype=torch.int32, device="cuda"),
                window=window, shares=shares, longest=max(max(lengths), 0))


def call(x, seq=None, max_length=None, scale=None, **kw):
    B, Hq, K = x["q"].shape
    p = ob.make_decode_params(B, Hq, x["kc"].shape[2], K, x["q"].dtype == torch.bfloat16, x["longest"] if max_length is None else max_length, scale,
                              x["window"], x["shares"])
    n = ob.osdn_paged_decode_workspace_bytes(p)
    ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda") if n else None            # (fp32 NaN: nothing in it is read before it is written)
    o, lse = torch.empty_like(x["q"]), torch.empty(B, Hq, device="cuda")
    ob.osdn_paged_decode(p, x["q"], x["kc"], x["vc"], x["table"], x["lengths"], seq, o, lse, ws)
    return o, lse


def compare(x, o, lse, seq=None, scale=None):
    B, Hq, K = x["q"].shape
    scale = K ** -0.5 if scale is None else scale
    want, wlse, size = ref.decode(ref.f64(x["q"]), ref.f64(x["kc"]), ref.f64(x["vc"]), x["table"].cpu(), x["lengths"].cpu(),
                                  torch.arange(B) if seq is None else seq.cpu(), scale, x["window"])
    bf16 = x["q"].dtype == torch.bfloat16
    ds = (K / 4 + 8) * 2.0 ** -24 * size
    vmax = float(ref.f64(x["vc"]).nan_to_num(0.0, 0.0, 0.0).abs().max())
    tol = 2 * (2 * ds + 2.0 ** -21 + 2.0 ** -18)[..., None] * vmax + (2.0 ** -9 * (vmax + want.abs()) if bf16 else 0.0)
    err = (o.double().cpu() - want).abs()
    assert (err <= tol).all(), f"o: worst {float((err / tol).nan_to_num(9e9).max()):.3g} of the tolerance"
    empty = torch.isinf(wlse)
    assert torch.equal(torch.isinf(lse.cpu()) & (lse.cpu() < 0), empty) and bool((o.cpu()[empty] == 0).all())
    lt = ds + 2.0 ** -20 * wlse.abs().clamp(min=1.0)
    assert ((lse.double().cpu() - wlse).abs()[~empty] <= lt[~empty]).all()


@pytest.mark.parametrize("case", DECODE, ids=lambda c: "-".join(str(v) for v in c.values())[:80])
def test_decode(case):
    x = make_decode(**case)
    o, lse = call(x)
    compare(x, o, lse)
    # what no length shows: not looked at, whatever stands there
    shown = torch.zeros(x["kc"].shape[:2], dtype=torch.bool)
    page = x["kc"].shape[1]
    for b, n in enumerate(case["lengths"]):
        j = torch.arange(max(0, n - case.get("window", 0)) if case.get("window") else 0, max(n, 0))
        shown[x["table"].cpu()[b][j // page].long(), j % page] = True
    for poison in (math.nan, math.inf, -math.inf):
        for c in (x["kc"], x["vc"]):
            c.masked_fill_(~shown.cuda()[..., None, None], poison)
        o2, lse2 = call(x)
        assert torch.equal(o, o2) and torch.equal(lse, lse2)
    # a launch sized for more than is there, and other cuts: the same answer
    for shares in (-1, 1, 3, 1000):
        compare(x, *call(dict(x, shares=shares)))
    compare(x, *call(x, max_length=x["longest"] + 777 if x["longest"] + 777 <= x["table"].shape[1] * page else x["longest"]))


def test_decode_conveniences_slices_and_strides():
    x = make_decode([200, 33], 8, 2, 128, 16)
    wide = torch.randn(2, 12, 128, device="cuda").bfloat16()
    wide[:, 2:10] = x["q"]
    a = ob.paged_decode(wide[:, 2:10], x["kc"], x["vc"], x["table"], x["lengths"])
    b, lse = ob.paged_decode(x["q"], x["kc"], x["vc"], x["table"], x["lengths"], max_length=200, want_lse=True)
    compare(x, a, lse)
    compare(x, b, lse)
    odd = torch.empty(2, 8, 131, device="cuda", dtype=torch.bfloat16)[..., 3:]          # rows off 16 bytes, written too
    odd.copy_(x["q"])
    p = ob.make_decode_params(2, 8, 2, 128, True, 200)
    n = ob.osdn_paged_decode_workspace_bytes(p)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda") if n else None
    ob.osdn_paged_decode(p, odd, x["kc"], x["vc"], x["table"], x["lengths"], None, odd, None, ws)
    assert torch.equal(odd, b)


def test_several_queries_of_one_sequence():
    """Drafted tokens, or a prompt token by token: queries that share a row of the table, each with its own length."""
    x = make_decode([90, 41], 4, 2, 64, 16, io="f32")
    g = torch.Generator(device="cuda").manual_seed(9)
    seq = torch.tensor([0] * 90 + [1] * 41, dtype=torch.int32, device="cuda")
    x["lengths"] = torch.cat([torch.arange(1, 91), torch.arange(1, 42)]).int().cuda()
    x["q"] = rnd(g, 131, 4, 64)
    compare(x, *call(x, seq=seq), seq=seq)


@pytest.mark.parametrize("spread,scale", [(300.0, 0.5), (1e-3, 0.125), (2.0, -0.2), (2.0, 0.0)])
def test_scores_far_apart_and_equal(spread, scale):
    x = make_decode([600, 45], 4, 1, 64, 32, io="f32", spread=spread, shares=33)
    o, lse = call(x, scale=scale)
    compare(x, o, lse, scale=scale)


def test_scores_of_minus_infinity_weigh_nothing():
    """A key whose product with the query is minus infinity has no part; where every key is such a one the row is empty."""
    x = make_decode([40, 20], 2, 1, 64, 16)
    x["q"].fill_(1.0)
    table = x["table"].cpu()
    x["kc"][table[0, 0].long(), :4, 0, 0] = -math.inf
    x["kc"][table[1, 0].long(), :, 0, 5] = -math.inf
    x["kc"][table[1, 1].long(), :4, 0, 5] = -math.inf
    o, lse = call(x)
    kept = torch.arange(4, 40)
    k, v = (ref.f64(c)[table[0][kept // 16].long(), kept % 16, 0] for c in (x["kc"], x["vc"]))
    s = k.sum(-1) / 8
    assert torch.allclose(lse[0].double().cpu(), torch.logsumexp(s, 0).expand(2), rtol=1e-5, atol=1e-5)
    assert ((o[0].double().cpu() - torch.softmax(s, 0) @ v).abs() <= 2.0 ** -7 * float(v.abs().max())).all()
    assert bool((o[1] == 0).all()) and bool((lse[1] == -math.inf).all())


def test_decode_says_so_when_promises_are_not_kept():
    x = make_decode([40, 40, 40, 40], 4, 2, 128, 16)
    x["lengths"][1] = 41                        # above max_length
    x["table"][2, 1] = -1                       # a page that is not there
    x["table"][3, 2] = 10 ** 6
    x["longest"] = 40
    o, lse = call(x)
    assert bool(o[0].isfinite().all()) and bool(o[1:].isnan().all()) and bool(lse[1:].isnan().all())
    seq = torch.tensor([0, 4, -1, 0], dtype=torch.int32, device="cuda")
    x["lengths"].fill_(40)
    o, lse = call(x, seq=seq)
    assert bool(o[1:3].isnan().all()) and torch.equal(o[3].isfinite(), torch.ones_like(o[3], dtype=torch.bool))
    x = make_decode([40], 4, 2, 128, 16)
    x["table"] = x["table"][:, :2].contiguous()         # a table of two pages for forty tokens
    for shares in (0, -1, 5):
        o, lse = call(dict(x, shares=shares), max_length=400)
        assert bool(o.isnan().all()) and bool(lse.isnan().all())


def test_offsets_beyond_32_bits():
    """A cache whose far pages stand more than 2^32 elements behind its start."""
    g = torch.Generator(device="cuda").manual_seed(4)
    n_pages, page, H, K = 270000, 64, 2, 128                           # 4.4e9 elements, 8.8 GB each
    kc, vc = (torch.empty(n_pages, H, page, K, dtype=torch.bfloat16, device="cuda").transpose(1, 2) for _ in range(2))
    far = torch.tensor([[269999, 3, 269990]], dtype=torch.int32, device="cuda")
    k, v, q = (rnd(g, 1, 150, h, K).bfloat16() for h in (H, H, 4))
    pos = torch.arange(150, dtype=torch.int32, device="cuda")[None]
    ob.paged_append(k, v, kc, vc, far, pos, hp=ob.NormHyper(norm="none"))
    o = ob.paged_decode(q[:, 0], kc, vc, far, torch.tensor([150], dtype=torch.int32, device="cuda"))
    near_k, near_v = kc[far[0].long()].clone(), vc[far[0].long()].clone()
    want = ob.paged_decode(q[:, 0], near_k, near_v, torch.arange(3, dtype=torch.int32, device="cuda")[None], torch.tensor([150], dtype=torch.int32, device="cuda"))
    assert torch.equal(o, want) and torch.equal(near_k.transpose(1, 2)[0].transpose(0, 1), k[0, :64])


# ------------------------------------------------------------------------------------ append ----
APPEND = [
    dict(B=1, T=1, Hq=1, Hk=1, K=64, page=16),
    dict(B=3, T=1, Hq=16, Hk=4, K=128, page=16, rotary=128),
    dict(B=3, T=37, Hq=5, Hk=3, K=128, page=8, rotary=64, order="token", layout="fused"),
    dict(B=2, T=20, Hq=0, Hk=2, K=256, page=64, rotary=256, norm="none", weighted=False),
    dict(B=2, T=20, Hq=3, Hk=1, K=64, page=1, io="f32", norm="l2", rotary=32, interleaved=True, order="apart"),
    dict(B=2, T=20, Hq=6, Hk=2, K=256, page=4, io="f32", rotary=96, layout="odd", order="page_inside"),
    dict(B=1, T=700, Hq=9, Hk=9, K=64, page=32, rotary=64, packed=True),
    dict(B=1, T=9000, Hq=2, Hk=2, K=128, page=32, rotary=0, norm="none", weighted=False, packed=True),
]


@pytest.mark.parametrize("case", APPEND, ids=lambda c: "-".join(str(v) for v in c.values()))
def test_append(case):
    c = dict(dict(io="bf16", norm="rms", weighted=True, rotary=0, interleaved=False, order="head", layout="plain", packed=False), **case)
    B, T, Hq, Hk, K, page = c["B"], c["T"], c["Hq"], c["Hk"], c["K"], c["page"]
    g = torch.Generator(device="cuda").manual_seed(5)
    dt = torch.bfloat16 if c["io"] == "bf16" else torch.float32
    if c["packed"]:                             # sequences of any length on one axis, and tokens that do not exist
        lens = [1, 130, 0, T // 2, T - 131 - T // 2 - 5]
        seq = torch.cat([torch.full((n,), i) for i, n in enumerate(lens)] + [torch.zeros(5)]).int()
        pos = torch.cat([torch.arange(n) for n in lens] + [torch.full((5,), -1)]).int()
        total = lens
    else:                                       # behind what is there already
        before = [3 + 11 * b for b in range(B)]
        seq = torch.arange(B).repeat_interleave(T).int()
        pos = torch.cat([torch.arange(n, n + T) for n in before]).int()
        total = [n + T for n in before]
    table, n_pages = make_table(total, page, extra=1, seed=6)
    kc, vc = (make_cache(g, n_pages, page, Hk, K, dt, c["order"]) for _ in range(2))
    kc0, vc0 = kc.clone(), vc.clone()
    if c["layout"] == "fused":
        x = rnd(g, B, T, (Hq + 2 * Hk) * K).to(dt)
        q, k, v = (y.unflatten(2, (-1, K)) for y in x.split([Hq * K, Hk * K, Hk * K], dim=2))
    elif c["layout"] == "odd":
        q, k, v = (torch.empty(B, T, h, K + 3, device="cuda", dtype=dt)[..., 1:K + 1].copy_(rnd(g, B, T, h, K)) for h in (Hq, Hk, Hk))
    else:
        q, k, v = (rnd(g, B, T, h, K).to(dt) for h in (Hq, Hk, Hk))
    w = [0.5 + torch.rand(K, device="cuda", generator=g) if c["weighted"] else None for _ in range(2)]
    rot = ob.rotary_table(max(total), c["rotary"], 500.0) if c["rotary"] else None
    hp = ob.NormHyper(norm=c["norm"], interleaved=c["interleaved"])
    pos, seq = pos.view(B, T).cuda(), seq.view(B, T).cuda()
    got = ob.paged_append(k, v, kc, vc, table.cuda(), pos, seq if c["packed"] else None, q if Hq else None, w[0] if Hq else None, w[1], rot, hp)
    # the rows are those of the norm by itself, the places those of the table, and nothing else has changed
    wq, wk = ob.qk_norm(q if Hq else None, k, w[0] if Hq else None, w[1], rot, pos, hp)
    assert (got is None) if not Hq else torch.equal(got, wq)
    p, s = pos.cpu().view(-1).long(), seq.cpu().view(-1).long()
    alive = p >= 0
    at = table[s[alive], p[alive] // page].long().cuda(), (p[alive] % page).cuda()
    kc0[at], vc0[at] = wk.reshape(-1, Hk, K)[alive.cuda()], v.reshape(-1, Hk, K)[alive.cuda()]
    assert torch.equal(kc, kc0) and torch.equal(vc, vc0)


def test_append_leaves_out_what_has_no_place():
    g = torch.Generator(device="cuda").manual_seed(7)
    kc, vc = (make_cache(g, 4, 16, 2, 64, torch.bfloat16, "head") for _ in range(2))
    k0, v0 = kc.clone(), vc.clone()
    table = torch.tensor([[0, -1], [99, 2]], dtype=torch.int32, device="cuda")
    k, v = (rnd(g, 1, 6, 2, 64).bfloat16() for _ in range(2))
    pos = torch.tensor([[-1, 17, 3, 40, 5, 2 ** 31 - 1]], dtype=torch.int32, device="cuda")        # none, no page, no page, off the table, no sequence (twice)
    seq = torch.tensor([[0, 0, 1, 0, 2, -1]], dtype=torch.int32, device="cuda")
    ob.paged_append(k, v, kc, vc, table, pos, seq, hp=ob.NormHyper(norm="none"))
    assert torch.equal(kc, k0) and torch.equal(vc, v0)


def test_serving_loop_in_a_graph():
    """One captured step (append, then attention) replayed over tokens with the lengths advanced on the device, against eager
    calls on a second cache."""
    B, Hq, Hk, K, page, steps = 3, 8, 2, 128, 16, 9
    g = torch.Generator(device="cuda").manual_seed(8)
    lens0 = [5, 14, 40]
    table, n_pages = make_table([n + steps for n in lens0], page, 0, 3)
    table = table.cuda()
    caches = [tuple(make_cache(torch.Generator(device="cuda").manual_seed(i), n_pages, page, Hk, K, torch.bfloat16, "head") for i in (1, 2)) for _ in range(2)]
    x = [torch.randn(B, 1, (Hq + 2 * Hk) * K, device="cuda", generator=g).bfloat16() for _ in range(steps)]
    rot, w = ob.rotary_table(64, K), 0.5 + torch.rand(K, device="cuda", generator=g)
    hp = ob.NormHyper(norm="rms")

    def step(inp, pos, length, cache):
        q, k, v = (y.unflatten(2, (-1, K)) for y in inp.split([Hq * K, Hk * K, Hk * K], dim=2))
        q = ob.paged_append(k, v, *cache, table, pos, q=q, weight_q=w, weight_k=w, rotary=rot, hp=hp)
        return ob.paged_decode(q[:, 0], *cache, table, length, max_length=40 + steps)

    inp, pos = torch.empty_like(x[0]), torch.tensor(lens0, dtype=torch.int32, device="cuda")[:, None]
    length = pos[:, 0] + 1
    warm = torch.cuda.Stream()
    warm.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(warm):
        inp.copy_(x[0])
        step(inp, pos, length, caches[0])
    torch.cuda.current_stream().wait_stream(warm)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(inp, pos, length, caches[0])
    for i in range(steps):
        inp.copy_(x[i])
        graph.replay()
        p = torch.tensor(lens0, dtype=torch.int32, device="cuda")[:, None] + i
        want = step(x[i], p, p[:, 0] + 1, caches[1])
        assert torch.equal(out, want), i
        pos += 1
        length += 1
        torch.cuda.synchronize()


@pytest.mark.parametrize("K", [64, 128, 256])
def test_fp32_scores_are_summed_in_parts(K):
    """fp32, scores of a spread of 4.  Rounding a sum of n products of variance s^2 one by one is off by less than 2^-24 s sqrt(n (n + 1) / 2) in the mean
    square; in sums of at most 32 products, K / 32 of them (four at least), and those two by two, K = 256 comes to 2^-24 s sqrt(8 x 528 + 3 x 256) = 71
    2^-24 s, as one sum to 181 2^-24 s; s = 4 and the scale 1 / 16 make 1.05e-6 and 2.7e-6 of a score, a weight, and so of o in norm.  The score's
    scaling and the maximum's subtraction, each off by 2^-25 of about 4 sqrt(log2 e), and e^x with its 2^-23, add 0.4e-6: 1.15e-6 in all."""
    x = make_decode([861, 1500], 8, 4, K, 16, io="f32", seed=11, spread=4.0)
    o, _ = call(x)
    want, _, _ = ref.decode(ref.f64(x["q"]), ref.f64(x["kc"]), ref.f64(x["vc"]), x["table"].cpu(), x["lengths"].cpu(), torch.arange(2), K ** -0.5, 0)
    assert float((o.double().cpu() - want).norm() / want.norm()) < 1.15e-6


# More rows than the chip holds workgroups: four (two) short ones together, a wavefront each; and rows whose heads stand side by side
MANY = [
    dict(lengths=[(7 * i) % 34 - 2 for i in range(400)], Hq=8, Hk=4, K=64, page=16),
    dict(lengths=[(7 * i) % 125 for i in range(300)], Hq=4, Hk=4, K=128, page=8, order="token"),
    dict(lengths=[(5 * i) % 17 for i in range(400)], Hq=6, Hk=2, K=256, page=16, window=9),
    dict(lengths=[(11 * i) % 65 - 1 for i in range(200)], Hq=4, Hk=4, K=256, page=32, io="f32"),
    dict(lengths=[(3 * i) % 60 for i in range(450)], Hq=8, Hk=4, K=64, page=2, io="f32", order="page_inside"),
    dict(lengths=[(13 * i) % 50 for i in range(500)], Hq=40, Hk=1, K=64, page=64),
    dict(lengths=[(131 * i) % 700 for i in range(90)], Hq=8, Hk=4, K=128, page=16, order="token"),
    dict(lengths=[(131 * i) % 700 for i in range(90)], Hq=6, Hk=6, K=64, page=16, order="token", io="f32"),
]


@pytest.mark.parametrize("case", MANY, ids=lambda c: "-".join(str(v) for k, v in c.items() if k != "lengths"))
def test_decode_many_rows(case):
    test_decode(case)


APPEND_MANY = [
    dict(B=1, T=23000, Hq=2, Hk=2, K=128, page=32, rotary=128, packed=True),
    dict(B=1, T=13000, Hq=9, Hk=9, K=64, page=64, rotary=32, packed=True, order="token"),
    dict(B=2, T=1100, Hq=15, Hk=9, K=256, page=16, io="f32", norm="l2", rotary=64, interleaved=True, order="page_inside"),
]


@pytest.mark.parametrize("case", APPEND_MANY, ids=lambda c: "-".join(str(v) for v in c.values()))
def test_append_many_tokens(case):
    test_append(case)
