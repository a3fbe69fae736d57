"""The pages of a cache from plan to release as a program uses them: the example stack over a cache in 4 bits, over selected pages, over pages that others gave back; and a step of
all of them together, captured once and replayed as sequences grow."""
import pytest
import torch

from paper_2605_13473_amd import binding as ob
from tests import pages_reference as pages

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kw", [dict(mx=True), dict(pages=64), dict(mx=True, pages=64)], ids=str)
def test_tokens_one_by_one_are_the_text_at_once(kw):
    """As without: the keys and values are the same 4-bit rows either way, and 64 pages of 16 are more than these sequences have.  The bound of the example's own test."""
    from examples.hybrid_stack import run
    pairs, _ = run(sequences=3, prompt=130, new=20, **kw)
    for got, want in pairs:
        got, want = got.float(), want.float()
        assert got.shape == want.shape and bool(want.isfinite().all())
        assert (got - want).abs().max() <= 2.0 ** -4 * want.abs().max()
        assert (got - want).norm() <= 2.0 ** -6 * want.norm()


@pytest.mark.parametrize("mx", [False, True])
def test_few_pages_run(mx):
    from examples.hybrid_stack import run
    pairs, _ = run(sequences=3, prompt=300, new=9, mx=mx, pages=4)
    assert all(bool(got.isfinite().all()) and got.shape == want.shape for got, want in pairs)


def test_pages_that_others_gave_back():
    """A pool that holds two sequences at a time serves four, one after the other, with the outputs of a pool of their own; a prompt that finds no pages leaves everything as it was."""
    from examples.hybrid_stack import Config, Serving, make_weights
    c = Config(longest=64)
    w = make_weights(c)
    g = torch.Generator(device="cuda").manual_seed(2)
    text = [torch.randn(n, c.width, device="cuda", generator=g).bfloat16() for n in (40, 33, 48, 17)]
    s, want = Serving(c, w, 3, held=6), []
    for t in text:
        own = Serving(c, w, 1)
        want.append(own.prompt(0, t))
    assert torch.equal(s.prompt(0, text[0]), want[0]) and torch.equal(s.prompt(2, text[1]), want[1])
    assert int(s.n_free) == 0
    before = s.table.clone(), s.lengths.clone()
    positions, seq, _ = s.places(torch.full((1,), 48, dtype=torch.int32, device="cuda"), 48, 1)
    assert bool((positions == -1).all()) and bool((seq == -1).all()) and torch.equal(s.table, before[0]) and torch.equal(s.lengths, before[1])
    s.finish([0, 2])
    assert int(s.n_free) == 6 and bool((s.table == -1).all())
    assert torch.equal(s.prompt(1, text[2]), want[2]) and torch.equal(s.prompt(0, text[3]), want[3])
    assert int(s.n_free) == 1


@pytest.mark.parametrize("io", ["bf16", "f32"])
@pytest.mark.parametrize("mx", [False, True])
def test_a_step_of_all_of_them_in_a_graph(io, mx):
    """plan, append, bounds, selection and attention captured once, and replayed as the sequences grow over page after page: every replay against the eager calls on a pool of
    their own, with the program's own work between the replays, and in the end the table and the bounds against the plain ones."""
    dt = torch.bfloat16 if io == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(6)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)
    B, Hq, Hk, K, page, N, most = 3, 4, 2, 64, 4, 60, 80
    i32 = dict(dtype=torch.int32, device="cuda")
    free0 = torch.randperm(N, generator=torch.Generator().manual_seed(1)).int().cuda()
    rot, hp = ob.rotary_table(most, K), ob.NormHyper(norm="rms")

    def pool():
        cache = tuple(t.zero_() for t in (ob.alloc_paged_cache_mx(N, page, Hk, K) if mx else ob.alloc_paged_cache(N, page, Hk, K, dt)))
        return dict(cache=cache, table=torch.full((B, most // page), -1, **i32), free=free0.clone(), n_free=torch.full((1,), N, **i32), lengths=torch.zeros(B, **i32),
                    bounds=ob.alloc_page_bounds(N, Hk, K, dt).zero_())

    def step(s, q, k, v, fresh):
        p = ob.paged_plan(s["table"], s["lengths"], fresh, s["free"], s["n_free"], page, B, n_pages=N)
        s["n_free"].copy_(p["n_free"])
        args = (s["table"], p["positions"], p["seq"])
        q = ob.paged_append_mx(k, v, s["cache"], *args, q=q, rotary=rot, hp=hp) if mx else ob.paged_append(k, v, *s["cache"], *args, q=q, rotary=rot, hp=hp)
        keys = (s["cache"][0], s["cache"][2]) if mx else s["cache"][0]
        ob.page_bounds(keys, s["table"], s["lengths"], p["lengths"], s["bounds"], max_new=1)
        s["lengths"].copy_(p["lengths"])
        chosen, tokens = ob.page_select(q[0], s["bounds"], s["table"], (p["positions"] + 1).view(-1), page, 3, seq=p["seq"].view(-1), max_length=most)
        o, lse = (ob.paged_decode_pages_mx(q[0], s["cache"], chosen, tokens, want_lse=True) if mx else ob.paged_decode_pages(q[0], *s["cache"], chosen, tokens, want_lse=True))
        return o, lse, chosen, tokens, p["positions"], p["seq"]

    text = [rnd(30, 1, B, H, K).to(dt) for H in (Hq, Hk, Hk)]
    held, fresh = [t[0].clone() for t in text], torch.zeros(B, **i32)
    eager, graphed, other = pool(), pool(), pool()
    step(other, *held, fresh)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(graphed, *held, fresh)
    for i in range(30):
        fresh.copy_(torch.tensor([1, i % 2, int(i >= 5)], dtype=torch.int32))
        for h, t in zip(held, text):
            h.copy_(t[i])
        graph.replay()
        want = step(eager, *held, fresh)
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert torch.equal(a, b)
        for n in ("table", "lengths", "n_free", "bounds"):
            assert torch.equal(eager[n], graphed[n]), n
        assert all(torch.equal(a, b) for a, b in zip(eager["cache"], graphed["cache"]))
    assert eager["lengths"].tolist() == [30, 15, 25]
    keys = pages.values(eager["cache"][0].cpu(), eager["cache"][2].cpu()) if mx else eager["cache"][0].double().cpu()
    plain = pages.bounds(keys, eager["table"].cpu(), torch.zeros(B, dtype=torch.int32), eager["lengths"].cpu(), torch.arange(B), torch.zeros(N, Hk, 2, K, dtype=torch.float64))
    assert torch.equal(eager["bounds"].double().cpu(), plain)


def test_calls_side_by_side_on_two_streams():
    """Two pools, each on a stream of its own, the calls of one between those of the other: the results of each alone."""
    def work(seed):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)
        k, v, q = rnd(1, 500, 2, 128).bfloat16(), rnd(1, 500, 2, 128).bfloat16(), rnd(1, 8, 128).bfloat16()
        i32 = dict(dtype=torch.int32, device="cuda")
        cache = tuple(t.zero_() for t in ob.alloc_paged_cache_mx(40, 16, 2, 128))
        table, free, bounds = torch.full((1, 40), -1, **i32), torch.randperm(40, device="cuda", generator=g).int(), ob.alloc_page_bounds(40, 2, 128).zero_()
        p = ob.paged_plan(table, torch.zeros(1, **i32), torch.full((1,), 500, **i32), free, torch.full((1,), 40, **i32), 16, 500, want_slots=True)
        yield
        ob.paged_append_mx(k, v, cache, table, p["positions"], p["seq"], hp=ob.NormHyper("none"))
        yield
        ob.page_bounds((cache[0], cache[2]), table, torch.zeros(1, **i32), p["lengths"], bounds)
        yield
        chosen, tokens = ob.page_select(q, bounds, table, p["lengths"], 16, 6)
        yield
        o = ob.paged_decode_pages_mx(q, cache, chosen, tokens)
        yield
        full = ob.paged_decode_mx(q, cache, table, p["lengths"])
        yield
        return [o, full, chosen, tokens, bounds, table, p["slots"], *ob.paged_read_mx(cache, table, p["positions"], p["seq"])]

    def drive(work, stream):
        with torch.cuda.stream(stream):
            try:
                next(work)
            except StopIteration as e:
                return e.value

    alone = []
    for seed in (1, 2):
        w, r = work(seed), None
        while r is None:
            r = drive(w, torch.cuda.current_stream())
        torch.cuda.synchronize()
        alone.append(r)
    streams, works, results = [torch.cuda.Stream(), torch.cuda.Stream()], [work(1), work(2)], [None, None]
    torch.cuda.synchronize()
    while None in results:
        for i in range(2):
            if results[i] is None:
                results[i] = drive(works[i], streams[i])
    torch.cuda.synchronize()
    for got, want in zip(results, alone):
        assert all(torch.equal(a, b) for a, b in zip(got, want))
