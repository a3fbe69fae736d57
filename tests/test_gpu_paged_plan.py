"""The page table and the places of new tokens from the lengths of requests, and pages given back: every number against requests taken one by one."""
import pytest
import torch

from paper_2605_13473_amd import binding as ob
from tests import pages_reference as ref

pytestmark = pytest.mark.gpu

i32 = lambda x: torch.as_tensor(x, dtype=torch.int32)


def make(cached, fresh, page, rows=None, spare=1000, order="own", max_pages=None, seed=1):
    """A pool in use: the sequences hold what they have cached, the rest is on the list."""
    g = torch.Generator().manual_seed(seed)
    B = len(cached)
    rows = B if rows is None else rows
    seq = torch.arange(B) if order == "own" else torch.randperm(rows, generator=g)[:B]
    held = [-(-max(c, 0) // page) for c in cached]
    width = max_pages or max([-(-(max(c, 0) + max(f, 0)) // page) for c, f in zip(cached, fresh)] + [1]) + 1
    n_pages = sum(held) + spare
    perm = torch.randperm(n_pages, generator=g).int()
    table = torch.full((rows, width), -1, dtype=torch.int32)
    at = 0
    for b, n in enumerate(held):
        n = min(n, width)
        table[seq[b], :n] = perm[at:at + n]
        at += n
    free = torch.full((n_pages,), -9, dtype=torch.int32)
    free[:spare] = perm[n_pages - spare:]
    return dict(table=table, cached=i32(cached), fresh=i32(fresh), seq=seq.int(), free=free, n_free=i32([spare]), page=page, n_pages=n_pages)


def check_plan(x, tokens, use_seq=True):
    dev = {n: t.cuda() if isinstance(t, torch.Tensor) else t for n, t in x.items()}
    table = x["table"].clone()
    want = ref.plan(table, x["cached"], x["fresh"], x["seq"], x["free"], x["n_free"][0], x["page"], tokens, x["n_pages"])
    got = ob.paged_plan(dev["table"], dev["cached"], dev["fresh"], dev["free"], dev["n_free"], x["page"], tokens, seq=dev["seq"] if use_seq else None,
                        n_pages=x["n_pages"], want_slots=True)
    for name, w in zip(("lengths", "starts", "positions", "seq", "slots", "n_free"), want):
        assert got[name].flatten().tolist() == (w if isinstance(w, list) else [w]), name
    assert torch.equal(dev["table"].cpu(), table)
    assert torch.equal(dev["free"].cpu(), x["free"]) and torch.equal(dev["n_free"].cpu(), x["n_free"])
    return got


CASES = [
    dict(cached=[0], fresh=[1], page=16),
    dict(cached=[15], fresh=[1], page=16),
    dict(cached=[16], fresh=[1], page=16),
    dict(cached=[0, 5, 16, 17], fresh=[0, 0, 0, 0], page=16),
    dict(cached=[0, 5, 16, 17, 0], fresh=[100, 3, 1, 0, 1], page=1),
    dict(cached=[3, 0, 64, 1], fresh=[300, 64, 65, 2], page=64, rows=9, order="any"),
    dict(cached=[7 * i for i in range(300)], fresh=[1] * 300, page=8, rows=400, order="any"),
    dict(cached=[(13 * i) % 200 for i in range(70)], fresh=[(37 * i) % 90 for i in range(70)], page=32),
    dict(cached=[(13 * i) % 50 for i in range(2500)], fresh=[i % 3 for i in range(2500)], page=4, rows=2600, order="any", spare=3000),
    dict(cached=[0] * 3, fresh=[5000, 1, 4000], page=128),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: f"{len(c['cached'])}-{sum(c['fresh'])}-{c['page']}")
@pytest.mark.parametrize("extra", [0, 77, 5000])
def test_plan(case, extra):
    x = make(**case)
    check_plan(x, max(1, sum(case["fresh"]) + extra), use_seq=case.get("order") == "any")


def test_lengths_that_31_bits_do_not_hold():
    """A row of the table that holds more than 2^31 tokens: the request that would pass them is not served, one that ends at them is."""
    top = 2 ** 31 - 1
    for fresh in ([5, 1, 0], [4, 1, 3]):
        x = make([0, 0, 0], fresh, 2 ** 16, spare=9, max_pages=2 ** 15 + 4)
        x["cached"] = i32([top - 4, 7, top])
        check_plan(x, 40)
        check_plan(x, 4000)


@pytest.mark.parametrize("spare", [0, 1, 2, 5, 11])
def test_pages_that_do_not_do_for_all(spare):
    x = make([3, 0, 8, 15, 16, 1], [1, 30, 8, 1, 40, 2], 8, spare=spare)
    got = check_plan(x, 200)
    assert got["starts"][0] == 0 and int(got["n_free"]) >= 0
    check_plan(make([(5 * i) % 40 for i in range(1500)], [(i * 7) % 5 for i in range(1500)], 4, spare=900 + spare), 4000)


@pytest.mark.parametrize("tokens", [1, 2, 30, 31, 71])
def test_a_token_axis_that_is_too_short(tokens):
    check_plan(make([3, 0, 8, 15, 16, 1], [1, 30, 8, 1, 40, 2], 8), tokens)


def test_requests_that_are_not_served():
    """Rows that are not there, negative numbers, more tokens than a row holds, two requests for one row: no page goes to them, and the rest is served."""
    x = make([4, 9, 0, 2, 3, 7, 20, 30, 0, 5], [3, 1, 2, 9, 4, 1, 50, 6, 3, 2], 8, rows=12, order="any", max_pages=8)
    x["seq"][1] = -1
    x["seq"][2] = 12
    x["cached"][3] = -5
    x["fresh"][4] = -2
    x["seq"][8] = x["seq"][5]                       # both bring tokens
    check_plan(x, 64)
    x["fresh"][8] = 0                               # one brings none: the other is served
    check_plan(x, 64)
    x["fresh"][0] = 2 ** 31 - 1
    check_plan(x, 64)
    x["cached"][0] = 2 ** 31 - 1
    check_plan(x, 64)


def test_lists_and_pages_that_are_not_right():
    x = make([3, 0], [20, 9], 8)
    x["n_free"] = i32([10 ** 6])                    # more than there is room for: as many as there is
    check_plan(x, 40)
    x["n_free"] = i32([-4])
    check_plan(x, 40)
    x = make([3, 0], [20, 9], 8)
    x["table"][0, 0] = x["n_pages"]                 # a page that is not there has no slots
    x["free"][998] = -3
    check_plan(x, 40)


def check_release(x, lengths, use_seq=True):
    table, free = x["table"].clone(), x["free"].clone()
    want = ref.release(table, lengths, x["seq"], free, x["n_free"][0], x["page"], x["n_pages"])
    dev = {n: t.cuda() if isinstance(t, torch.Tensor) else t for n, t in x.items()}
    got = ob.paged_release(dev["table"], lengths.cuda(), dev["free"], dev["n_free"], x["page"], seq=dev["seq"] if use_seq else None, n_pages=x["n_pages"])
    assert int(got) == want
    assert torch.equal(dev["table"].cpu(), table) and torch.equal(dev["free"].cpu(), free)
    return dev, got


@pytest.mark.parametrize("case", [
    dict(cached=[1], fresh=[0], page=16, spare=0), dict(cached=[0, 0], fresh=[0, 0], page=16), dict(cached=[5, 0, 64, 65, 700], fresh=[0] * 5, page=4, rows=8, order="any"),
    dict(cached=[(29 * i) % 300 for i in range(1100)], fresh=[0] * 1100, page=8, rows=1200, order="any"),
    dict(cached=[2, 9000, 3], fresh=[0] * 3, page=2)], ids=lambda c: f"{len(c['cached'])}-{c['page']}")
def test_release(case):
    x = make(**case)
    check_release(x, x["cached"], use_seq=case.get("order") == "any")


def test_release_of_what_is_not_there():
    x = make([20, 30, 40, 9, 12, 50], [0] * 6, 8, rows=9, order="any", max_pages=6)
    x["table"][x["seq"][0], 1] = -1                 # holes
    x["table"][x["seq"][0], 2] = x["n_pages"]
    x["seq"][3] = 99
    lengths = x["cached"].clone()
    lengths[1] = -3
    lengths[5] = 10 ** 9                            # more than a row holds: the row
    check_release(x, lengths)
    x["seq"][4] = x["seq"][2]                       # named twice: kept
    check_release(x, lengths)
    x["n_free"] = i32([x["n_pages"] - 1])           # no room
    check_release(x, lengths)


def test_given_back_and_taken_again():
    """The pages come back in the order that they had, so that the same prompts get the same table."""
    x = make([20, 33, 1, 64], [5, 0, 30, 64], 8, rows=7, order="any")
    dev, n = check_release(x, x["cached"])
    p = ob.paged_plan(dev["table"], torch.zeros(4, dtype=torch.int32, device="cuda"), dev["cached"], dev["free"], n, 8, 200, seq=dev["seq"])
    assert torch.equal(dev["table"].cpu(), x["table"]) and int(p["n_free"]) == int(x["n_free"])
    assert p["slots"] is None


def test_places_in_place_and_in_a_graph():
    """Lengths and the count of free pages over themselves, captured once and replayed as the sequences grow."""
    page, B = 4, 5
    table = torch.full((B, 40), -1, dtype=torch.int32, device="cuda")
    free = torch.randperm(200, generator=torch.Generator().manual_seed(3)).int().cuda()
    n_free, lengths, fresh = i32([200]).cuda(), i32([0, 3, 4, 0, 7]).cuda(), i32([1, 1, 0, 2, 1]).cuda()
    starts, pos, rows = (torch.empty(n, dtype=torch.int32, device="cuda") for n in (B + 1, 8, 8))
    slots = torch.empty(8, dtype=torch.int64, device="cuda")
    g = ob._pages(table, page, 200, free)
    x = dict(table=table.cpu(), lengths=lengths.cpu(), n_free=200)
    for b in range(B):                              # what they have already
        table[b, :2] = torch.tensor([150 + 2 * b, 151 + 2 * b], dtype=torch.int32)
    free[150:160] = -5
    n_free.fill_(150)
    x = dict(table=table.cpu(), lengths=lengths.cpu(), free=free.cpu(), n_free=150)
    call = lambda: ob.osdn_paged_plan(g, B, 8, lengths, fresh, None, n_free, n_free, lengths, starts, pos, rows, slots)
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        call()
    torch.cuda.synchronize()
    for step in range(9):
        if step % 3 == 2:
            call()                                  # the program's own work between the replays
        else:
            graph.replay()
        torch.cuda.synchronize()
        w = ref.plan(x["table"], x["lengths"], fresh.cpu(), torch.arange(B), x["free"], x["n_free"], page, 8, 200)
        x["lengths"], x["n_free"] = i32(w[0]), w[5]
        for got, want in zip((lengths, starts, pos, rows, slots, n_free), w):
            assert got.tolist() == (want if isinstance(want, list) else [want])
        assert torch.equal(table.cpu(), x["table"])


@pytest.mark.parametrize("tokens", [40, 3500, 9000])
def test_outputs_over_the_inputs(tokens):
    """The same numbers where lengths and the count of free pages stand in the place of what they come from, for few tokens and for many."""
    x = make([3, 0, 70, 15, 16, 1], [1, 30, 0, 1, 3, 2] if tokens == 40 else [1, 3000, 0, 2000, 3, 2500], 8, rows=9, order="any")
    table = x["table"].clone()
    want = ref.plan(table, x["cached"], x["fresh"], x["seq"], x["free"], x["n_free"][0], 8, tokens, x["n_pages"])
    d = {n: t.cuda() if isinstance(t, torch.Tensor) else t for n, t in x.items()}
    starts, pos, rows = (torch.empty(n, dtype=torch.int32, device="cuda") for n in (7, tokens, tokens))
    slots = torch.empty(tokens, dtype=torch.int64, device="cuda")
    ob.osdn_paged_plan(ob._pages(d["table"], 8, x["n_pages"], d["free"]), 6, tokens, d["cached"], d["fresh"], d["seq"], d["n_free"], d["n_free"], d["cached"], starts, pos, rows, slots)
    for got, w in zip((d["cached"], starts, pos, rows, slots, d["n_free"]), want):
        assert got.tolist() == (w if isinstance(w, list) else [w])
    assert torch.equal(d["table"].cpu(), table)
    ob.osdn_paged_plan(ob._pages(d["table"], 8, x["n_pages"], d["free"]), 6, tokens, torch.zeros(6, dtype=torch.int32, device="cuda"), d["fresh"], d["seq"], d["n_free"], d["n_free"], d["fresh"],
                       starts, pos, rows)
    # (from nothing, with what the list still holds: lengths are what is new of those that are served)
    again = ref.plan(table, torch.zeros(6, dtype=torch.int32), x["fresh"], x["seq"], x["free"], want[5], 8, tokens, x["n_pages"])
    assert d["fresh"].tolist() == again[0] and int(d["n_free"]) == again[5] and torch.equal(d["table"].cpu(), table)


@pytest.mark.parametrize("rows", [1, 1025, 3000])
def test_release_of_many_entries(rows):
    """More entries than a workgroup takes at a time, and more sequences than a round; some of them with holes."""
    x = make([(53 * i) % 97 * 11 for i in range(rows)] if rows > 1 else [40000], [0] * rows, 2 if rows == 1 else 16, rows=rows + 5, order="any", spare=50)
    x["table"][x["seq"][::7].long(), 0] = -1
    check_release(x, x["cached"])
