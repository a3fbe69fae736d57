"""Bounds of the keys of a page, the pages that a query reads, and attention over them.  Bounds and choices are exact: every number against tokens and pages taken
one by one.  Tolerances of attention: as in test_gpu_paged_mx, over the cache's values (a cache of fp32 sums K products too)."""
import math

import pytest
import torch

from paper_2605_13473_amd import binding as ob
from tests import heads_reference as ref
from tests import pages_reference as pages
from tests.test_gpu_paged import make_cache as make_rows
from tests.test_gpu_paged_mx import hold, make_cache, make_table, rnd

pytestmark = pytest.mark.gpu

i32 = lambda x: torch.as_tensor(x, dtype=torch.int32)


def make(lengths, Hq, Hk, K, page, io="bf16", order="head", mx=False, seed=3):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    table, n_pages = make_table(lengths, page, 2, seed)
    if mx:
        cache = make_cache(g, n_pages, page, Hk, K, order)
        values = [pages.values(cache[i].cpu(), cache[i + 2].cpu()) for i in range(2)]
        keys = (cache[0], cache[2])
    else:
        cache = tuple(make_rows(g, n_pages, page, Hk, K, dt, order) for _ in range(2))
        values = [ref.f64(c) for c in cache]
        keys = cache[0]
    return dict(q=rnd(g, len(lengths), Hq, K).to(dt), cache=cache, keys=keys, values=values, table=table.cuda(), lengths=i32(lengths).cuda(), page=page, mx=mx, dt=dt,
                n_pages=n_pages, longest=max(max(lengths), 1))


FORMS = [dict(io="bf16"), dict(io="f32"), dict(io="bf16", mx=True), dict(io="f32", mx=True)]


@pytest.mark.parametrize("form", FORMS, ids=str)
@pytest.mark.parametrize("case", [
    dict(lengths=[1], Hk=1, K=64, page=16), dict(lengths=[37, 0, 16, 5], Hk=2, K=128, page=16, order="token"), dict(lengths=[9, 300, 64], Hk=3, K=256, page=8, order="apart"),
    dict(lengths=[200, 1], Hk=5, K=64, page=1), dict(lengths=[700], Hk=9, K=128, page=256, order="page_inside")], ids=lambda c: "-".join(str(v) for v in c.values()))
def test_bounds(case, form):
    """Tokens come in several parts, of a page's length and not; the bounds are those of all that came, and the other pages' stay."""
    x = make(Hq=case["Hk"], **case, **form)
    B, K, Hk = len(case["lengths"]), case["K"], case["Hk"]
    bounds = ob.alloc_page_bounds(x["n_pages"], Hk, K, x["dt"]).copy_(torch.randn(x["n_pages"], Hk, 2, K))
    want = ref.f64(bounds)
    at = torch.zeros(B, dtype=torch.int32)
    for part in (3, 1, 40, 7, 10 ** 4):
        to = torch.minimum(at + part, x["lengths"].cpu())
        ob.page_bounds(x["keys"], x["table"], at.cuda(), to.cuda(), bounds, max_new=part if part < 100 else None)
        want = pages.bounds(x["values"][0], x["table"].cpu(), at, to, torch.arange(B), want)
        assert torch.equal(ref.f64(bounds), want)
        at = to
    assert torch.equal(at, x["lengths"].cpu())


def test_bounds_of_what_is_not_there_and_not_a_number():
    x = make([40, 30, 20, 64, 50], 2, 2, 128, 8)
    B = 5
    seq = i32([0, 1, 9, 3, -1])
    cached, lengths = i32([-5, 0, 0, 70, 0]), i32([40, 30, 20, 64, 50])
    x["table"][0, 2] = -1
    x["table"][1, 1] = x["n_pages"]
    lengths[3] = 10 ** 6                                # (from 70 on its row holds some more pages, none of them there)
    g = int(x["table"][0, 1])
    x["cache"][0][g, 3, 1, 5] = math.nan
    x["cache"][0][g, 4, 0, 7] = math.inf
    bounds = ob.alloc_page_bounds(x["n_pages"], 2, 128).zero_()
    ob.page_bounds(x["keys"], x["table"], cached.cuda(), lengths.cuda(), bounds, seq=seq.cuda(), max_new=100)
    keys = ref.f64(x["cache"][0])
    want = pages.bounds(keys, x["table"].cpu(), cached, lengths, seq, torch.zeros(x["n_pages"], 2, 2, 128, dtype=torch.float64))
    got = ref.f64(bounds)
    nan = torch.isnan(want)
    assert int(nan.sum()) == 2 and torch.equal(torch.isnan(got), nan) and torch.equal(got[~nan], want[~nan])
    # no more than max_new tokens of a sequence
    bounds.zero_()
    ob.page_bounds(x["keys"], x["table"], torch.zeros(1, dtype=torch.int32, device="cuda"), i32([30]).cuda(), bounds, seq=i32([1]).cuda(), max_new=3)
    want = pages.bounds(keys, x["table"].cpu(), i32([0]), i32([3]), i32([1]), torch.zeros(x["n_pages"], 2, 2, 128, dtype=torch.float64))
    assert torch.equal(ref.f64(bounds), want)


def bounds_of(x):
    b = ob.alloc_page_bounds(x["n_pages"], x["cache"][0].shape[2], x["q"].shape[2], x["dt"]).fill_(math.nan)
    ob.page_bounds(x["keys"], x["table"], torch.zeros_like(x["lengths"]), x["lengths"], b)
    return b


def check_choice(x, bounds, n, first=1, last=1, seq=None, lengths=None, max_length=None):
    lengths = x["lengths"] if lengths is None else lengths
    longest = x["longest"] if max_length is None else max_length
    got = ob.page_select(x["q"], bounds, x["table"], lengths, x["page"], n, seq=None if seq is None else seq.cuda(), first=first, last=last, max_length=longest)
    want = pages.select(ref.f64(x["q"]), ref.f64(bounds), x["table"].cpu(), lengths.cpu(), torch.arange(len(lengths)) if seq is None else seq, x["page"], n, first, last, longest)
    assert torch.equal(got[1].cpu(), want[1]) and torch.equal(got[0].cpu(), want[0])
    return got


def check_attention(x, chosen, tokens, scale=None, shares=None, max_length=None):
    B, Hq, K = x["q"].shape
    Hk = chosen.shape[1]
    G = Hq // Hk
    s = K ** -0.5 if scale is None else scale
    if shares is None:
        call = ob.paged_decode_pages_mx if x["mx"] else ob.paged_decode_pages
        o, lse = call(x["q"], *((x["cache"],) if x["mx"] else x["cache"]), chosen, tokens, scale=scale, max_length=max_length, want_lse=True)
    else:
        p = ob.make_decode_params(B, Hq, Hk, K, x["dt"] == torch.bfloat16, chosen.shape[2] * x["page"], scale, 0, shares)
        n = (ob.osdn_paged_decode_pages_mx_workspace_bytes if x["mx"] else ob.osdn_paged_decode_pages_workspace_bytes)(p)
        ws = torch.full((n,), 255, dtype=torch.uint8, device="cuda") if n else None
        o, lse = torch.empty_like(x["q"]), torch.empty(B, Hq, device="cuda")
        call = ob.osdn_paged_decode_pages_mx if x["mx"] else ob.osdn_paged_decode_pages
        call(p, x["q"], *((x["cache"],) if x["mx"] else x["cache"]), chosen, tokens, o, lse, ws)
    q = ref.f64(x["q"])
    want, wlse, size = torch.zeros(B, Hq, K, dtype=torch.float64), torch.zeros(B, Hq, dtype=torch.float64), torch.zeros(B, Hq, dtype=torch.float64)
    for h in range(Hk):
        of = slice(h * G, (h + 1) * G)
        want[:, of], wlse[:, of], size[:, of] = ref.decode(q[:, of], x["values"][0][:, :, h:h + 1], x["values"][1][:, :, h:h + 1], chosen.cpu()[:, h], tokens.cpu()[:, h],
                                                           torch.arange(B), s, 0)
    hold(o, lse, want, wlse, size, float(x["values"][1].abs().max()), K, x["dt"] == torch.bfloat16)
    return o, lse


SELECT = [
    dict(lengths=[1], Hq=1, Hk=1, K=64, page=16, n=2),
    dict(lengths=[300, 0, 17, 129], Hq=8, Hk=2, K=128, page=8, n=4),
    dict(lengths=[300, 0, 17, 129], Hq=8, Hk=2, K=128, page=8, n=7, order="token", first=2, last=3),
    dict(lengths=[300, 64, 63, 65], Hq=5, Hk=5, K=256, page=4, n=9, first=0),
    dict(lengths=[300, 64, 63, 65], Hq=40, Hk=2, K=64, page=2, n=21, order="apart"),
    dict(lengths=[3000], Hq=7, Hk=1, K=128, page=1, n=100, first=0, last=1),
    dict(lengths=[9000, 40], Hq=6, Hk=3, K=64, page=2, n=33, order="page_inside"),
    dict(lengths=[700, 701], Hq=9, Hk=9, K=64, page=16, n=5, first=2, last=3),
    dict(lengths=[50, 20], Hq=4, Hk=2, K=128, page=16, n=60),
    dict(lengths=[(97 * b) % 260 for b in range(19)], Hq=6, Hk=3, K=64, page=8, n=9, order="token"),
]


@pytest.mark.parametrize("form", FORMS, ids=str)
@pytest.mark.parametrize("case", SELECT, ids=lambda c: "-".join(str(v) for v in c.values()))
def test_select_and_attend(case, form):
    case = dict(case)
    n, first, last = case.pop("n"), case.pop("first", 1), case.pop("last", 1)
    x = make(**case, **form)
    bounds = bounds_of(x)
    chosen, tokens = check_choice(x, bounds, n, first, last)
    check_attention(x, chosen, tokens)
    for shares in (-1, 1, 3, 1000):
        check_attention(x, chosen, tokens, shares=shares)
    check_choice(x, bounds, n, first, last, max_length=x["longest"] + 555 if -(-(x["longest"] + 555) // x["page"]) <= x["table"].shape[1] else None)


@pytest.mark.parametrize("io", ["bf16", "f32"])
def test_chosen_rows_that_may_be_many(io):
    """A bound of the tokens that makes them 2^19 rows of 128 elements in 4 bits: their codes are loaded past the caches."""
    x = make([700, 41, 0, 260], 6, 3, 128, 8, io, "token", mx=True)
    chosen, tokens = check_choice(x, bounds_of(x), 20)
    check_attention(x, chosen, tokens, max_length=1 << 17)
    for K in (64, 128):
        x = make([700, 41, 0, 260], 6, 3, K, 8, io, mx=True)
        chosen, tokens = check_choice(x, bounds_of(x), 20)
        check_attention(x, chosen, tokens, max_length=1 << 17)


def test_equal_scores_go_to_the_earlier_page():
    x = make([640, 640], 4, 2, 64, 8)
    b = bounds_of(x)
    b[:] = b[int(x["table"][0, 0])][None]                       # all alike
    chosen, _ = check_choice(x, b, 9, 1, 2)
    assert torch.equal(chosen[0, 0].cpu(), x["table"].cpu()[0, [0, 1, 2, 3, 4, 5, 6, 78, 79]])
    x["q"][0] = 0.0                                             # and all zero, of either sign
    check_choice(x, bounds_of(x), 9, 1, 2)
    b[int(x["table"][1, 40])] *= 2.0                            # one stands out, either way
    check_choice(x, b, 3, 1, 1)
    b[::2] += 1.0
    check_choice(x, b, 31, 1, 1)


def test_scores_that_are_not_numbers_and_pages_that_are_not_there():
    x = make([160, 160, 160, 160, 40], 4, 2, 64, 8)
    b = bounds_of(x)
    t = x["table"]
    b[int(t[0, 7]), 0, 1, 3] = math.nan
    b[int(t[0, 9]), 0, 0, 3] = -math.inf
    x["q"][0, 0, 3], x["q"][0, 1, 3] = -1.0, -2.0               # (that one's score is infinite)
    b[int(t[1, 12]), 1, 1] = math.inf                           # infinities and zeros of Q+ or both signs: NaN or infinity
    t[2, 5] = -1
    t[3, 19] = x["n_pages"]                                     # the last page, which is always taken
    lengths = x["lengths"].clone()
    lengths[4] = 10 ** 6
    chosen, tokens = check_choice(x, b, 4, 1, 1, lengths=lengths)
    assert int(t[0, 7]) in chosen[0, 0].tolist() and int(t[0, 9]) in chosen[0, 0].tolist()
    o, lse = ob.paged_decode_pages(x["q"], *x["cache"], chosen, tokens, want_lse=True)
    nan = torch.isnan(o).all(-1).cpu()
    assert torch.equal(nan, torch.isnan(lse).cpu()) and nan.tolist() == [[False] * 4] * 2 + [[True] * 4] * 3
    seq = i32([0, 99, -1, 1, 4])
    chosen, tokens = check_choice(x, b, 4, 1, 1, seq=seq)
    o, _ = ob.paged_decode_pages(x["q"], *x["cache"], chosen, tokens, want_lse=True)
    assert bool(torch.isnan(o[1]).all()) and bool(torch.isnan(o[2]).all()) and not bool(torch.isnan(o[4]).any())


def test_infinite_bounds_come_first_or_last():
    """Bounds that infinite keys leave: an infinite score, of either sign, and one whose Q is zero, which is read before the finite ones."""
    x = make([160, 160, 160], 4, 2, 64, 8)
    b, t = bounds_of(x), x["table"]
    x["q"][:, :, 3] = torch.tensor([2.0, 1.0, 3.0, 0.5], device="cuda")
    for at, (lo, hi) in enumerate(((-math.inf, 1.0), (-math.inf, -math.inf), (1.0, math.inf))):
        b[int(t[at, 11]), :, 0, 3], b[int(t[at, 11]), :, 1, 3] = lo, hi
    for n in (3, 19):
        chosen, _ = ob.page_select(x["q"], b, t, x["lengths"], 8, n)
        for at in range(3):
            assert all((int(t[at, 11]) in row) for row in chosen[at].tolist())
    b[int(t[1, 11]), :, 0, 3] = -3e38                           # (Q- is zero there: with a finite bound the largest is minus infinity, and the score too)
    chosen, _ = ob.page_select(x["q"], b, t, x["lengths"], 8, 19)
    assert all((int(t[1, 11]) not in row) for row in chosen[1].tolist())


def test_all_pages_are_the_whole_sequence():
    """As many pages as there are: the bits of attention over all of it, over either kind of cache."""
    for form in FORMS:
        x = make([300, 47, 0, 16], 8, 2, 128, 16, **form)
        chosen, tokens = ob.page_select(x["q"], bounds_of(x), x["table"], x["lengths"], 16, 25)
        if x["mx"]:
            a, b = ob.paged_decode_pages_mx(x["q"], x["cache"], chosen, tokens, want_lse=True), ob.paged_decode_mx(x["q"], x["cache"], x["table"], x["lengths"], want_lse=True)
        else:
            a, b = ob.paged_decode_pages(x["q"], *x["cache"], chosen, tokens, want_lse=True), ob.paged_decode(x["q"], *x["cache"], x["table"], x["lengths"], want_lse=True)
        assert torch.allclose(a[0].float(), b[0].float(), atol=2.0 ** -7, rtol=2.0 ** -7) and torch.allclose(a[1], b[1], atol=2.0 ** -18, rtol=2.0 ** -18)


def test_scale_strides_and_unaligned_queries():
    x = make([300, 64, 7], 8, 2, 64, 8)
    b = bounds_of(x)
    wide = torch.randn(3, 12, 67, device="cuda").bfloat16()
    wide[:, 2:10, 3:] = x["q"]
    y = dict(x, q=wide[:, 2:10, 3:])
    chosen, tokens = check_choice(y, b, 5)
    o, lse = check_attention(y, chosen, tokens, scale=0.4)
    o2, lse2 = check_attention(x, chosen, tokens, scale=0.4)
    assert torch.equal(o, o2) and torch.equal(lse, lse2)
    check_attention(x, chosen, tokens, max_length=40)


def test_several_queries_of_a_sequence_and_more_than_a_launch_takes():
    g = torch.Generator(device="cuda").manual_seed(5)
    x = make([90, 41], 4, 2, 64, 8)
    b = bounds_of(x)
    seq = torch.randint(0, 2, (40000,), dtype=torch.int32, device="cuda", generator=g)
    lengths = torch.minimum(torch.randint(0, 91, (40000,), dtype=torch.int32, device="cuda", generator=g), x["lengths"][seq.long()])
    q = rnd(g, 40000, 4, 64).bfloat16()
    chosen, tokens = ob.page_select(q, b, x["table"], lengths, 8, 4, seq=seq)
    o, lse = ob.paged_decode_pages(q, *x["cache"], chosen, tokens, want_lse=True)
    for at in (0, 32760, 39990):
        s = slice(at, at + 10)
        y = dict(x, q=q[s], lengths=lengths[s])
        c, t = check_choice(y, b, 4, seq=seq[s].cpu())
        assert torch.equal(c, chosen[s]) and torch.equal(t, tokens[s])
        y_o, y_lse = check_attention(y, c, t)
        assert torch.allclose(o[s].float(), y_o.float(), atol=2.0 ** -7, rtol=2.0 ** -7)


def test_lengths_near_31_bits():
    """Pages of 2^22 tokens, and of so many that the length and a page are more than 31 bits hold: the choice of the definition, and nothing beside it is written."""
    g = torch.Generator(device="cuda").manual_seed(9)
    for page, last in ((2 ** 22, 2 ** 31 - 257), (2 ** 22, 2 ** 31 - 2 ** 22), (2 ** 22, 2 ** 31 - 2 ** 22 + 1), (2 ** 30, 2 ** 30 + 1), (2 ** 30, 2 ** 31 - 300)):
        n, have = i32([last]), -(-last // page)
        q, bounds, table = rnd(g, 1, 4, 64).bfloat16(), rnd(g, 600, 2, 2, 64).bfloat16().sort(2).values, torch.randperm(600, device="cuda", generator=g).int()[None, :have + 1]
        pages_taken = 9 if page < 2 ** 30 else 1
        p = ob.make_select_params(1, 4, 2, 64, True, 2 ** 31 - 256, pages=pages_taken, first=0)
        held = torch.full((3, 1, 2, pages_taken), -5, dtype=torch.int32, device="cuda")
        tokens = torch.empty(1, 2, dtype=torch.int32, device="cuda")
        size = ob.osdn_page_select_workspace_bytes(p, page)
        ob.osdn_page_select(p, ob._pages(table, page, 600), q, bounds, n.cuda(), None, held[1], tokens, torch.empty(size, dtype=torch.uint8, device="cuda") if size else None)
        want = pages.select(ref.f64(q), ref.f64(bounds), table.cpu(), n, torch.arange(1), page, pages_taken, 0, 1, 2 ** 31 - 256)
        assert torch.equal(held[1].cpu(), want[0]) and torch.equal(tokens.cpu(), want[1])
        assert bool((held[0] == -5).all()) and bool((held[2] == -5).all())


def test_bounds_past_32_bits():
    """2^21 + 64 pages, whose bounds are 4.3 GB: those of the last ones, selected as from a small array."""
    g = torch.Generator(device="cuda").manual_seed(3)
    far, Hk, K = 1 << 21, 4, 128
    keys = torch.zeros(far + 64, 1, Hk, K, dtype=torch.bfloat16, device="cuda")
    keys[far:] = rnd(g, 64, 1, Hk, K).bfloat16()
    table = torch.randperm(64, device="cuda", generator=g).int()[None]
    q, n, none = rnd(g, 1, 8, K).bfloat16(), i32([60]).cuda(), i32([0]).cuda()
    small, large = ob.alloc_page_bounds(64, Hk, K).zero_(), torch.zeros(far + 64, Hk, 2, K, dtype=torch.bfloat16, device="cuda")
    ob.page_bounds(keys[far:], table, none, n, small)
    ob.page_bounds(keys, table + far, none, n, large)
    assert torch.equal(large[far:], small) and not bool(large[:1000].any())
    a, b = ob.page_select(q, small, table, n, 1, 7), ob.page_select(q, large, table + far, n, 1, 7)
    assert torch.equal(a[0] + far, b[0]) and torch.equal(a[1], b[1])
    got, want = ob.paged_decode_pages(q, keys, keys, *b), ob.paged_decode_pages(q, keys[far:], keys[far:], *a)
    assert torch.equal(got, want)
