"""What the entry points for pages, for the cache in 4 bits and for selected pages refuse, on the CPU: argument errors come before any pointer is used (none here is ever
dereferenced), sizes of workspaces, and the errors of the binding."""
import ctypes

import pytest
import torch

from paper_2605_13473_amd import binding as ob
from tests.test_heads_abi import BAD_CACHE, BAD_DECODE, BAD_NORM, DTYPE, FAKE, NULL, PARAM, SHAPE, WORKSPACE, cache, norm_params, rows

by, none = ctypes.byref, ctypes.POINTER(ob.OsdnRows)()


def of(x, **kw):
    for n, v in kw.items():
        setattr(x, n, v)
    return x


def pages(**kw):
    return of(ob.OsdnPages(FAKE, 8, FAKE, 40, 40, 16, 4, 8), **kw)


def cache_mx(K=64, **kw):
    t, h, ts, hs = 4 * K // 2, K // 2, 4 * K // 32, K // 32
    return of(ob.OsdnCacheMx(FAKE, FAKE, FAKE, FAKE, 16 * t, t, h, 16 * t, t, h, 16 * ts, ts, hs, 16 * ts, ts, hs, FAKE, 8, 10, 16, 4, 8), **kw)


def choice(**kw):
    return of(ob.OsdnSelectParams(2, 8, 4, 64, 1, 100, 5, 4, 1, 1), **kw)


def plan(g, B=3, tokens=20, missing=None):
    a = dict(cached=FAKE, fresh=FAKE, seq=None, n_free=FAKE, n_free_out=FAKE, lengths=FAKE, starts=FAKE, positions=FAKE, rows=FAKE)
    if missing:
        a[missing] = None
    return ob.lib().osdn_paged_plan(g and by(g), B, tokens, *a.values(), None, None)


def release(g, B=3, missing=None):
    a = [None if missing == n else FAKE for n in ("lengths", "n_free", "n_free_out")]
    return ob.lib().osdn_paged_release(g and by(g), B, a[0], None, a[1], a[2], None)


BAD_TABLE = [(dict(table=None), NULL), (dict(n_pages=0), SHAPE), (dict(page_size=0), SHAPE), (dict(page_size=24), SHAPE), (dict(page_size=-16), SHAPE), (dict(n_seqs=0), SHAPE),
             (dict(max_pages=0), SHAPE), (dict(table_stride=7), SHAPE), (dict(table_stride=-8), SHAPE), (dict(table=FAKE + 2), SHAPE)]


@pytest.mark.parametrize("kw,status", BAD_TABLE + [(dict(free_list=None), NULL), (dict(free_capacity=0), SHAPE), (dict(free_list=FAKE + 2), SHAPE), (dict(table_stride=0), SHAPE)], ids=str)
def test_pages(kw, status):
    g = pages(**kw)
    assert plan(g) == status and release(g) == status
    if "free_list" not in kw and "free_capacity" not in kw and kw != dict(table_stride=0):
        assert select(choice(), g) == status


def test_requests():
    for B in (0, -1, 65536):
        assert plan(pages(), B=B) == SHAPE and release(pages(), B=B) == SHAPE
    for tokens in (0, -5, 2 ** 30 + 1, 2 ** 31 - 1):
        assert plan(pages(), tokens=tokens) == SHAPE
    for n in ("cached", "fresh", "n_free", "n_free_out", "lengths", "starts", "positions", "rows"):
        assert plan(pages(), missing=n) == NULL
    for n in ("lengths", "n_free", "n_free_out"):
        assert release(pages(), missing=n) == NULL
    assert plan(None) == NULL and release(None) == NULL
    assert release(pages(max_pages=2 ** 20 + 1, table_stride=2 ** 20 + 1), B=1024) == SHAPE
    L, g = ob.lib(), pages(n_seqs=131073)                                           # rows that are named: of so many
    assert L.osdn_paged_plan(by(g), 3, 20, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None, None) == SHAPE
    assert L.osdn_paged_release(by(g), 3, FAKE, FAKE, FAKE, FAKE, None) == SHAPE


BAD_MX = [(dict(kw), s) for kw, s in BAD_CACHE if set(kw) & {"table", "n_pages", "page_size", "n_seqs", "max_pages", "table_stride"} or None in kw.values()] + [
    (dict(k_scale=None), NULL), (dict(v_scale=None), NULL), (dict(k=FAKE + 8), SHAPE), (dict(v=FAKE + 1), SHAPE), (dict(k_token=136), SHAPE), (dict(v_head=-32), SHAPE), (dict(k_head=16), SHAPE),
    (dict(v_scale_head=1), SHAPE), (dict(k_scale_token=-8), SHAPE), (dict(k_scale_page=1), SHAPE)]


@pytest.mark.parametrize("kw,status", BAD_MX, ids=str)
def test_cache(kw, status):
    L, r, c, p = ob.lib(), by(rows()), cache_mx(**kw), ob.make_decode_params(2, 8, 4, 64, True, 100)
    assert L.osdn_paged_append_mx(by(norm_params()), by(c), r, r, r, None, None, None, FAKE, None, r, None) == status
    assert L.osdn_paged_read_mx(by(norm_params()), by(c), FAKE, None, r, r, None) == status
    assert L.osdn_paged_decode_mx(by(p), by(c), r, FAKE, None, r, None, None, 0, None) == status
    if not set(kw) & {"table", "n_seqs", "max_pages", "table_stride"}:             # (which come with the pages that are chosen)
        assert L.osdn_paged_decode_pages_mx(by(p), by(c), r, FAKE, 4, FAKE, r, None, None, 0, None) == status
    if not any(n.startswith("v") for n in kw):
        assert bounds(choice(), c) == status


def test_scales_of_256_lie_on_two_bytes():
    L, r, p = ob.lib(), by(rows(K=256)), norm_params(K=256)
    for kw in (dict(k_scale=FAKE + 1), dict(v_scale=FAKE + 3), dict(k_scale_token=33), dict(v_scale_page=16 * 32 + 1), dict(k_scale_head=9)):
        assert L.osdn_paged_append_mx(by(p), by(cache_mx(256, **kw)), r, r, r, None, None, None, FAKE, None, r, None) == SHAPE


@pytest.mark.parametrize("kw", [dict(k_page=0), dict(k_token=0), dict(k_head=0), dict(v_token=0), dict(v_scale_page=0), dict(k_scale_token=0), dict(k_scale_head=0), dict(k_token=32), dict(v_page=128),
                                dict(k_scale_token=2), dict(v_scale_page=8)], ids=str)
def test_rows_that_are_written_lie_apart(kw):
    r = by(rows())
    assert ob.lib().osdn_paged_append_mx(by(norm_params()), by(cache_mx(**kw)), r, r, r, None, None, None, FAKE, None, r, None) == SHAPE


@pytest.mark.parametrize("kw,status", [x for x in BAD_NORM if x[1] != NULL], ids=str)
def test_norm_parameters(kw, status):
    r = by(rows())
    assert ob.lib().osdn_paged_append_mx(by(norm_params(**kw)), by(cache_mx()), r, r, r, None, None, None, FAKE, None, r, None) == status
    if not set(kw) & {"Hq", "norm", "eps", "interleaved", "rotary_dim"}:           # (not looked at)
        assert ob.lib().osdn_paged_read_mx(by(norm_params(**kw)), by(cache_mx()), FAKE, None, r, r, None) == status


def test_append_and_read_need_their_rows():
    L, r, c, p = ob.lib(), by(rows()), by(cache_mx()), by(norm_params())
    call = lambda q, k, v, pos, qo, p=p: L.osdn_paged_append_mx(p, c, q, k, v, None, None, None, pos, None, qo, None)
    assert call(r, none, none, FAKE, r, by(norm_params(Hk=0))) == SHAPE
    assert call(r, r, r, None, r) == NULL
    for i in range(4):
        a = [r, r, r, FAKE, r]
        a[i + (i == 3)] = none
        assert call(*a) == NULL
    read = lambda p, c, pos, k, v: L.osdn_paged_read_mx(p, c, pos, None, k, v, None)
    assert [read(*(None if i == j else x for j, x in enumerate((p, c, FAKE, r, r)))) for i in range(5)] == [NULL] * 5
    assert read(by(norm_params(Hk=0)), c, FAKE, r, r) == SHAPE
    for kw in (dict(batch=0), dict(token=63), dict(head=-63), dict(at=FAKE + 1)):
        assert read(p, c, FAKE, by(rows(**kw)), r) == SHAPE and read(p, c, FAKE, r, by(rows(**kw))) == SHAPE


def decode_pages(p, c=None, mx=False, q=None, chosen=FAKE, n=8, tokens=FAKE, o=None, ws=FAKE, size=1 << 40):
    r = by(rows())
    L = ob.lib()
    return (L.osdn_paged_decode_pages_mx if mx else L.osdn_paged_decode_pages)(by(p), c or by((cache_mx if mx else cache)()), r if q is None else q, chosen, n, tokens, r if o is None else o, None, ws, size, None)


@pytest.mark.parametrize("kw,status", BAD_DECODE, ids=str)
def test_decode_parameters(kw, status):
    p = of(ob.make_decode_params(2, 8, 4, 64, True, 100), **kw)
    r = by(rows())
    assert ob.lib().osdn_paged_decode_mx(by(p), by(cache_mx()), r, FAKE, None, r, None, FAKE, 1 << 40, None) == status
    assert decode_pages(p) == status and decode_pages(p, mx=True) == status
    assert ob.osdn_paged_decode_mx_workspace_bytes(p) == ob.osdn_paged_decode_pages_workspace_bytes(p) == ob.osdn_paged_decode_pages_mx_workspace_bytes(p) == 0


@pytest.mark.parametrize("mx", [False, True])
def test_decode_of_chosen_pages(mx):
    p = ob.make_decode_params(2, 8, 4, 64, True, 100000)
    n = ob._pages_bytes(p, mx)
    assert n > 0
    assert decode_pages(p, mx=mx, q=none) == NULL and decode_pages(p, mx=mx, o=none) == NULL
    for kw, status in ((dict(chosen=None), NULL), (dict(tokens=None), NULL), (dict(n=0), SHAPE), (dict(n=-3), SHAPE), (dict(chosen=FAKE + 2), SHAPE), (dict(ws=None, size=0), NULL),
                       (dict(size=n - 1), WORKSPACE), (dict(ws=FAKE + 4), WORKSPACE), (dict(o=by(rows(batch=0))), SHAPE)):
        assert decode_pages(p, mx=mx, **kw) == status, kw
    L, r = ob.lib(), by(rows())
    assert (L.osdn_paged_decode_pages_mx if mx else L.osdn_paged_decode_pages)(by(p), None, r, FAKE, 8, FAKE, r, None, FAKE, n, None) == NULL
    assert decode_pages(of(ob.make_decode_params(2, 8, 4, 64, True, 100), window=5), mx=mx) == PARAM
    assert decode_pages(ob.make_decode_params(16384, 8, 4, 64, True, 100), mx=mx) == SHAPE               # 65536 entries
    assert ob._pages_bytes(ob.make_decode_params(2, 8, 4, 64, True, 128), mx) == 0


def test_decode_mx_workspace():
    L, r, c, p = ob.lib(), by(rows()), by(cache_mx()), ob.make_decode_params(2, 8, 4, 64, True, 100000)
    n = ob.osdn_paged_decode_mx_workspace_bytes(p)
    assert n > 0
    call = lambda q, lens, o, ws, size, c=c: L.osdn_paged_decode_mx(by(p), c, q, lens, None, o, None, ws, size, None)
    assert call(none, FAKE, r, FAKE, n) == call(r, None, r, FAKE, n) == call(r, FAKE, none, FAKE, n) == call(r, FAKE, r, None, n) == call(r, FAKE, r, FAKE, n, None) == NULL
    assert call(r, FAKE, r, FAKE, n - 1) == WORKSPACE and call(r, FAKE, r, FAKE + 4, n) == WORKSPACE
    assert call(r, FAKE, by(rows(batch=0)), FAKE, n) == SHAPE
    assert ob.osdn_paged_decode_mx_workspace_bytes(ob.make_decode_params(2, 8, 4, 64, True, 128)) == 0


def bounds(p, c, cached=FAKE, lengths=FAKE, to=FAKE):
    L = ob.lib()
    f = L.osdn_page_bounds_mx if isinstance(c, ob.OsdnCacheMx) else L.osdn_page_bounds
    return f(p and by(p), c and by(c), cached, lengths, None, to, None)


def select(p, g, q=None, at=FAKE, lengths=FAKE, chosen=FAKE, tokens=FAKE, ws=FAKE, size=1 << 40):
    return ob.lib().osdn_page_select(p and by(p), g and by(g), by(rows()) if q is None else q, at, lengths, None, chosen, tokens, ws, size, None)


BAD_BOTH = [(dict(io_dtype=2), DTYPE), (dict(io_dtype=-1), DTYPE), (dict(B=0), SHAPE), (dict(B=65536), SHAPE), (dict(Hk=0), SHAPE), (dict(Hk=70000), SHAPE), (dict(B=65535, Hk=64), SHAPE), (dict(K=96), SHAPE),
            (dict(K=512), SHAPE)]
BAD_CHOICE = [(dict(Hq=2), SHAPE), (dict(Hq=10), SHAPE), (dict(Hq=70000), SHAPE), (dict(max_length=-1), SHAPE), (dict(max_length=2 ** 31 - 1), SHAPE), (dict(pages=0), PARAM), (dict(first=-1), PARAM),
              (dict(last=0), PARAM), (dict(first=2, last=3), PARAM), (dict(first=2 ** 31 - 1, last=2 ** 31 - 1), PARAM), (dict(pages=2 ** 27), PARAM), (dict(B=65535, Hq=32, Hk=32, max_length=2 ** 25), SHAPE),
              (dict(B=60000, Hq=32, Hk=32, pages=2000, max_length=16), SHAPE)]


@pytest.mark.parametrize("kw,status", BAD_BOTH, ids=str)
def test_choice_and_bounds(kw, status):
    assert bounds(choice(**kw), cache()) == status and bounds(choice(**kw), cache_mx()) == status
    assert select(choice(**kw), pages()) == status
    assert ob.osdn_page_select_workspace_bytes(choice(**kw), 16) == 0


@pytest.mark.parametrize("kw,status", BAD_CHOICE, ids=str)
def test_choice(kw, status):
    assert select(choice(**kw), pages()) == status
    assert ob.osdn_page_select_workspace_bytes(choice(**kw), 16) == 0


def test_pointers_of_bounds_and_choice():
    for c in (cache(), cache_mx()):
        assert bounds(None, c) == NULL
        assert bounds(choice(max_new=0), c) == SHAPE and bounds(choice(max_new=-1), c) == SHAPE
        for kw in (dict(cached=None), dict(lengths=None), dict(to=None)):
            assert bounds(choice(), c, **kw) == NULL
        assert bounds(choice(), c, to=FAKE + 8) == SHAPE
    L = ob.lib()
    assert L.osdn_page_bounds(by(choice()), None, FAKE, FAKE, None, FAKE, None) == L.osdn_page_bounds_mx(by(choice()), None, FAKE, FAKE, None, FAKE, None) == NULL
    for kw, status in [x for x in BAD_CACHE if not any(n.startswith("v") for n in x[0])]:
        if kw not in (dict(k_head=0), dict(k_token=0)):                             # (which may be read so)
            assert bounds(choice(), cache(**kw)) == status, kw
    assert select(None, pages()) == NULL and select(choice(), None) == NULL and select(choice(), pages(), q=none) == NULL
    for kw in (dict(at=None), dict(lengths=None), dict(chosen=None), dict(tokens=None)):
        assert select(choice(), pages(), **kw) == NULL
    assert select(choice(), pages(), at=FAKE + 8) == SHAPE and select(choice(), pages(), q=by(rows(at=FAKE + 1))) == SHAPE
    p = choice(max_length=10 ** 6)
    n = ob.osdn_page_select_workspace_bytes(p, 16)
    assert n == 2 * 4 * 62500 * 8
    assert select(p, pages(), ws=None, size=n) == NULL and select(p, pages(), size=n - 1) == WORKSPACE and select(p, pages(), ws=FAKE + 8) == WORKSPACE
    assert ob.osdn_page_select_workspace_bytes(choice(max_length=64), 16) == 0      # no more pages than are taken


def test_the_binding_says_what_is_wrong():
    i32 = torch.int32
    table, ints, x = torch.zeros(2, 4, dtype=i32), torch.zeros(2, dtype=i32), torch.zeros(2, 4, 64)
    one, mx = torch.zeros(1, dtype=i32), ob.alloc_paged_cache_mx(4, 16, 2, 64, device="cpu")
    assert [tuple(t.shape) for t in mx] == [(4, 16, 2, 32)] * 2 + [(4, 16, 2, 2)] * 2 and mx[0].stride() == (1024, 32, 512, 1) and mx[2].stride() == (64, 2, 32, 1)
    kc, b = torch.zeros(4, 16, 2, 64), ob.alloc_page_bounds(4, 2, 64, torch.float32, device="cpu")
    assert b.shape == (4, 2, 2, 64)
    for call in (lambda: ob.paged_plan(table, ints, ints, ints, one, 16, 5), lambda: ob.paged_release(table, ints, ints, one, 16), lambda: ob.page_select(x, b, table, ints, 16, 2),
                 lambda: ob.page_bounds(kc, table, ints, ints, b), lambda: ob.page_bounds((mx[0], mx[2]), table, ints, ints, b), lambda: ob.page_bounds(mx, table, ints, ints, b),
                 lambda: ob.paged_append_mx(x[None, :, :2], x[None, :, :2], mx, table, table[:1, :2], table[:1, :2]), lambda: ob.paged_decode_mx(x, mx, table, ints), lambda: ob.paged_decode_mx(x, mx[:2], table, ints),
                 lambda: ob.paged_decode_mx(x[0], mx, table, ints), lambda: ob.paged_read_mx(mx, table, table), lambda: ob.paged_read_mx(mx, table, ints), lambda: ob.paged_read_mx(mx, table, table, dtype=torch.float16),
                 lambda: ob.paged_decode_pages(x, kc, kc, table[:, None], table), lambda: ob.paged_decode_pages(x, kc, kc, table, table), lambda: ob.paged_decode_pages_mx(x, mx, table[:, None], table),
                 lambda: ob.paged_decode_pages_mx(x, kc, table[:, None], table), lambda: ob.paged_plan(table, None, ints, ints, one, 16, 5), lambda: ob.paged_plan(None, ints, ints, ints, one, 16, 5)):
        with pytest.raises(TypeError):
            call()
