"""What the entry points around the recurrence refuse, on the CPU: argument errors come before any pointer is used (none here is ever
dereferenced), sizes of workspaces, and the errors of the binding."""
import ctypes

import pytest
import torch

from paper_2605_13473_amd import binding as ob

FAKE = 0x10000
NULL, SHAPE, DTYPE, WORKSPACE, PARAM = -1, -2, -3, -4, -5


def rows(B=2, T=3, H=4, K=64, at=FAKE, **kw):
    r = dict(batch=T * H * K, token=H * K, head=K)
    r.update(kw)
    return ob.OsdnRows(at, r["batch"], r["token"], r["head"])


def norm_params(**kw):
    p = ob.OsdnNormParams(2, 3, 4, 4, 64, 1, 1, 0, 0, 0, 1e-6)
    for n, v in kw.items():
        setattr(p, n, v)
    return p


def cache(**kw):
    c = ob.OsdnCache(FAKE, FAKE, 16 * 4 * 64, 4 * 64, 64, 16 * 4 * 64, 4 * 64, 64, FAKE, 8, 10, 16, 2, 8)
    for n, v in kw.items():
        setattr(c, n, v)
    return c


def norm_fwd(p, q=None, k=None, qo=None, ko=None, rotary=None):
    r = [ctypes.byref(x if x is not None else rows()) for x in (q, k, qo, ko)]
    return ob.lib().osdn_qk_norm_fwd(ctypes.byref(p), r[0], r[1], None, None, rotary, None, r[2], r[3], None)


BAD_NORM = [
    (dict(io_dtype=2), DTYPE), (dict(B=0), SHAPE), (dict(T=0), SHAPE), (dict(T=-1), SHAPE), (dict(K=96), SHAPE), (dict(K=512), SHAPE), (dict(Hq=-1), SHAPE),
    (dict(Hq=0, Hk=0), SHAPE), (dict(Hq=70000), SHAPE), (dict(B=1 << 20, T=1 << 10, Hq=1), SHAPE), (dict(B=1 << 16, T=1 << 16), SHAPE), (dict(norm=3), PARAM), (dict(norm=-1), PARAM),
    (dict(eps=0.0), PARAM), (dict(eps=float("inf")), PARAM), (dict(eps=float("nan")), PARAM), (dict(norm=2, eps=-1.0), PARAM), (dict(interleaved=2), PARAM),
    (dict(rotary_dim=8, rotary_rows=4), SHAPE), (dict(rotary_dim=-16), SHAPE), (dict(rotary_dim=128, rotary_rows=4), SHAPE), (dict(rotary_dim=64), SHAPE),
    (dict(rotary_dim=64, rotary_rows=4), NULL),
]


@pytest.mark.parametrize("kw,status", BAD_NORM, ids=str)
def test_norm_parameters(kw, status):
    p = norm_params(**kw)
    assert norm_fwd(p) == status
    r = ctypes.byref(rows())
    assert ob.lib().osdn_qk_norm_bwd(ctypes.byref(p), r, r, None, None, None, None, r, r, r, r, None, None, None, 0, None) == status
    assert ob.lib().osdn_paged_append(ctypes.byref(p), ctypes.byref(cache()), r, r, r, None, None, None, FAKE, None, r, None) == status
    if status != NULL:
        assert ob.osdn_qk_norm_bwd_workspace_bytes(p) == 0


def test_rows():
    p = norm_params()
    L = ob.lib()
    none = ctypes.POINTER(ob.OsdnRows)()
    r = ctypes.byref(rows())
    for at in range(4):
        a = [r] * 4
        a[at] = none
        assert L.osdn_qk_norm_fwd(ctypes.byref(p), a[0], a[1], None, None, None, None, a[2], a[3], None) == NULL
        a[at] = ctypes.byref(rows(at=0))
        assert L.osdn_qk_norm_fwd(ctypes.byref(p), a[0], a[1], None, None, None, None, a[2], a[3], None) == NULL
    assert norm_fwd(p, q=rows(at=FAKE + 1)) == SHAPE                     # not on an element
    for axis in ("batch", "token", "head"):
        for step in (0, 63, -63):
            assert norm_fwd(p, qo=rows(**{axis: step})) == SHAPE         # rows written over one another
    assert L.osdn_qk_norm_fwd(None, r, r, None, None, None, None, r, r, None) == NULL


def test_gradients_of_weights_need_a_workspace():
    p, L, r = norm_params(), ob.lib(), ctypes.byref(rows())
    n = ob.osdn_qk_norm_bwd_workspace_bytes(p)
    assert n >= 2 * 64 * 4
    call = lambda dwq, dwk, ws, size: L.osdn_qk_norm_bwd(ctypes.byref(p), r, r, None, None, None, None, r, r, r, r, dwq, dwk, ws, size, None)
    for dw in ((FAKE, None), (None, FAKE)):
        assert call(*dw, None, n) == NULL
        assert call(*dw, FAKE + 16, n) == WORKSPACE
        assert call(*dw, FAKE, n - 1) == WORKSPACE


BAD_CACHE = [
    (dict(k=None), NULL), (dict(v=None), NULL), (dict(table=None), NULL), (dict(n_pages=0), SHAPE), (dict(page_size=0), SHAPE), (dict(page_size=24), SHAPE),
    (dict(n_seqs=0), SHAPE), (dict(max_pages=0), SHAPE), (dict(table_stride=7), SHAPE), (dict(table_stride=-8), SHAPE), (dict(k=FAKE + 8), SHAPE),
    (dict(v=FAKE + 2), SHAPE), (dict(table=FAKE + 2), SHAPE), (dict(k_token=257), SHAPE), (dict(v_head=-64), SHAPE), (dict(k_head=0), SHAPE), (dict(v_page=0), SHAPE), (dict(k_token=0), SHAPE), (dict(k_head=56), SHAPE),
    (dict(v_token=56), SHAPE),
]


@pytest.mark.parametrize("kw,status", BAD_CACHE, ids=str)
def test_cache(kw, status):
    L, r, c = ob.lib(), ctypes.byref(rows()), cache(**kw)
    assert L.osdn_paged_append(ctypes.byref(norm_params()), ctypes.byref(c), r, r, r, None, None, None, FAKE, None, r, None) == status
    p = ob.make_decode_params(2, 8, 4, 64, True, 100)
    assert L.osdn_paged_decode(ctypes.byref(p), ctypes.byref(c), r, FAKE, None, r, None, None, 0, None) == status


def test_append_needs_keys_values_and_positions():
    L, r, c = ob.lib(), ctypes.byref(rows()), ctypes.byref(cache())
    none = ctypes.POINTER(ob.OsdnRows)()
    call = lambda p, q, k, v, pos, qo: L.osdn_paged_append(ctypes.byref(p), c, q, k, v, None, None, None, pos, None, qo, None)
    assert call(norm_params(Hk=0), r, none, none, FAKE, r) == SHAPE
    assert call(norm_params(), r, r, r, None, r) == NULL
    assert call(norm_params(), none, r, r, FAKE, r) == NULL
    assert call(norm_params(), r, none, r, FAKE, r) == NULL
    assert call(norm_params(), r, r, none, FAKE, r) == NULL
    assert call(norm_params(), r, r, r, FAKE, none) == NULL


BAD_DECODE = [
    (dict(io_dtype=7), DTYPE), (dict(B=0), SHAPE), (dict(B=65536), SHAPE), (dict(Hk=0), SHAPE), (dict(Hq=2), SHAPE), (dict(Hq=10), SHAPE), (dict(K=96), SHAPE), (dict(max_length=-1), SHAPE), (dict(B=65535, Hq=64), SHAPE),
    (dict(max_length=2 ** 31 - 1), SHAPE), (dict(B=100, Hk=8, max_length=2 ** 30), SHAPE),
    (dict(window=-1), PARAM), (dict(shares=-2), PARAM), (dict(shares=65536), PARAM), (dict(scale=float("nan")), PARAM), (dict(scale=float("inf")), PARAM),
]


@pytest.mark.parametrize("kw,status", BAD_DECODE, ids=str)
def test_decode_parameters(kw, status):
    p = ob.make_decode_params(2, 8, 4, 64, True, 100)
    for n, v in kw.items():
        setattr(p, n, v)
    r = ctypes.byref(rows())
    assert ob.lib().osdn_paged_decode(ctypes.byref(p), ctypes.byref(cache()), r, FAKE, None, r, None, FAKE, 1 << 40, None) == status
    assert ob.osdn_paged_decode_workspace_bytes(p) == 0


def test_decode_pointers_and_workspace():
    L, r, c = ob.lib(), ctypes.byref(rows()), ctypes.byref(cache())
    none = ctypes.POINTER(ob.OsdnRows)()
    p = ob.make_decode_params(2, 8, 4, 64, True, 100000)
    n = ob.osdn_paged_decode_workspace_bytes(p)
    assert n > 0
    call = lambda q, lens, o, ws, size: L.osdn_paged_decode(ctypes.byref(p), c, q, lens, None, o, None, ws, size, None)
    assert call(none, FAKE, r, FAKE, n) == NULL
    assert call(r, None, r, FAKE, n) == NULL
    assert call(r, FAKE, none, FAKE, n) == NULL
    assert call(r, FAKE, r, None, n) == NULL
    assert call(r, FAKE, r, FAKE, n - 1) == WORKSPACE
    assert call(r, FAKE, r, FAKE + 4, n) == WORKSPACE
    assert call(r, FAKE, ctypes.byref(rows(batch=0)), FAKE, n) == SHAPE
    assert ob.osdn_paged_decode_workspace_bytes(ob.make_decode_params(2, 8, 4, 64, True, 128)) == 0          # no second kernel
    assert ob.osdn_paged_decode_workspace_bytes(ob.make_decode_params(2, 8, 4, 64, True, 0)) == 0


def test_the_binding_says_what_is_wrong():
    x = torch.zeros(1, 2, 3, 64)
    with pytest.raises(TypeError, match="q: expected a CUDA"):
        ob.qk_norm(x, x)
    with pytest.raises(TypeError, match="rows"):
        ob.qk_norm(x[0], x)
    with pytest.raises(TypeError, match="rows"):
        ob.qk_norm(None, None)
    with pytest.raises(ValueError, match="norm"):
        ob.qk_norm(x, x, hp=ob.NormHyper(norm="layer"))
    with pytest.raises(TypeError, match="expected q"):
        ob.paged_decode(x, x, x, x, x)
    kc = torch.zeros(4, 16, 3, 64)
    with pytest.raises(TypeError):
        ob.paged_decode(x[0], kc, kc, torch.zeros(2, 2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32))
    with pytest.raises(TypeError):
        ob.paged_append(x, x, kc, kc, torch.zeros(1, 2, dtype=torch.int32), torch.zeros(1, 2, dtype=torch.int32))
