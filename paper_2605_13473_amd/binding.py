"""Thin Python binding of libosdn (argument marshalling only).

``osdn_precond_update``, ``osdn_fwd``, ``osdn_bwd``, ``osdn_workspace_bytes`` and
``osdn_strerror`` mirror the C entry points of ``include/osdn.h`` one to one: they take
torch tensors that already live on the GPU (PyTorch is used for device memory and
streams only), check dtype / contiguity / device, and pass raw pointers.  Every step of
the computation runs in the HIP library; there is no fallback of any kind: if the shared
object is missing this module raises.

``forward`` / ``backward`` are conveniences that allocate the outputs and the workspace; ``qk_norm``, ``paged_append``, ``paged_decode`` and the operators on
a cache's pages (``paged_plan`` .. ``paged_decode_pages_mx``) are, too.
"""
from __future__ import annotations

import ctypes
import os
import struct
import warnings
from dataclasses import dataclass

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libosdn.so")
_lib = None
_step_native = None        # _native.step, once the library is loaded (None: no module that fits it)
_rows_native = None        # _native, for the operators around the recurrence

OSDN_F32, OSDN_BF16 = 0, 1
OSDN_ERR_SHAPE = -2


class OsdnParams(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("T", ctypes.c_int32), ("H", ctypes.c_int32),
        ("K", ctypes.c_int32), ("V", ctypes.c_int32), ("chunk", ctypes.c_int32),
        ("io_dtype", ctypes.c_int32),
        ("scale", ctypes.c_float), ("eta", ctypes.c_float),
        ("d_min", ctypes.c_float), ("d_max", ctypes.c_float), ("eps", ctypes.c_float),
        ("beta_aware", ctypes.c_int32), ("retention_per_channel", ctypes.c_int32),
        ("gate_per_channel", ctypes.c_int32),
        ("segments", ctypes.c_int32), ("p1_pieces", ctypes.c_int32), ("p1_piece_sweeps", ctypes.c_int32),
        ("p1_solved", ctypes.c_int32),
    ]


class OsdnRows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("batch", ctypes.c_int64), ("token", ctypes.c_int64), ("head", ctypes.c_int64)]


class OsdnNormParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "T", "Hq", "Hk", "K", "io_dtype", "norm", "rotary_dim", "rotary_rows",
                                              "interleaved")] + [("eps", ctypes.c_float)]


class OsdnCache(ctypes.Structure):
    _fields_ = ([("k", ctypes.c_void_p), ("v", ctypes.c_void_p)]
                + [(n, ctypes.c_int64) for n in ("k_page", "k_token", "k_head", "v_page", "v_token", "v_head")]
                + [("table", ctypes.c_void_p), ("table_stride", ctypes.c_int64)]
                + [(n, ctypes.c_int32) for n in ("n_pages", "page_size", "n_seqs", "max_pages")])


class OsdnDecodeParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "Hq", "Hk", "K", "io_dtype", "window", "max_length", "shares")] + [
        ("scale", ctypes.c_float)]


class OsdnPages(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("table_stride", ctypes.c_int64), ("free_list", ctypes.c_void_p)] + [
        (n, ctypes.c_int32) for n in ("free_capacity", "n_pages", "page_size", "n_seqs", "max_pages")]


class OsdnCacheMx(ctypes.Structure):
    _fields_ = ([(n, ctypes.c_void_p) for n in ("k", "v", "k_scale", "v_scale")]
                + [(f"{t}_{n}", ctypes.c_int64) for t in ("k", "v", "k_scale", "v_scale") for n in ("page", "token", "head")]
                + [("table", ctypes.c_void_p), ("table_stride", ctypes.c_int64)]
                + [(n, ctypes.c_int32) for n in ("n_pages", "page_size", "n_seqs", "max_pages")])


class OsdnSelectParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("B", "Hq", "Hk", "K", "io_dtype", "max_length", "max_new", "pages", "first", "last")]


class OsdnError(RuntimeError):
    def __init__(self, status: int):
        self.status = status
        super().__init__(f"libosdn error {status}: {osdn_strerror(status)}")


def lib():
    """Load libosdn.so (built in-tree by ``build.py``); raises if it is not there."""
    global _lib, _step_native, _rows_native
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} is missing: build it with `python -m paper_2605_13473_amd.build` "
                "(there is no CPU or PyTorch fallback)")
        L = ctypes.CDLL(LIB_PATH)
        vp, fp = ctypes.c_void_p, ctypes.c_void_p
        pp = ctypes.POINTER(OsdnParams)
        L.osdn_workspace_bytes.restype = ctypes.c_size_t
        L.osdn_workspace_bytes.argtypes = [pp, ctypes.c_int]
        L.osdn_debug_mask_offset.restype = ctypes.c_size_t
        L.osdn_debug_mask_offset.argtypes = [pp]
        L.osdn_strerror.restype = ctypes.c_char_p
        L.osdn_strerror.argtypes = [ctypes.c_int]
        L.osdn_precond_update.restype = ctypes.c_int
        L.osdn_precond_update.argtypes = [pp, vp, fp, fp, fp, vp, fp, fp, vp]
        L.osdn_fwd.restype = ctypes.c_int
        L.osdn_fwd.argtypes = [pp, vp, vp, vp, fp, fp, fp, fp, fp, vp, fp, fp, vp, ctypes.c_size_t, vp]
        L.osdn_fwd_noalloc.restype = ctypes.c_int
        L.osdn_fwd_noalloc.argtypes = [pp, vp, vp, vp, fp, fp, fp, fp, fp, vp, fp, fp, vp]
        L.osdn_bwd.restype = ctypes.c_int
        L.osdn_bwd.argtypes = [pp] + [vp] * 19 + [vp, ctypes.c_size_t, vp]
        ip = ctypes.POINTER(ctypes.c_int32)
        L.osdn_workspace_bytes_packed.restype = ctypes.c_size_t
        L.osdn_workspace_bytes_packed.argtypes = [pp, ip, ctypes.c_int32, ctypes.c_int]
        L.osdn_fwd_packed.restype = ctypes.c_int
        L.osdn_fwd_packed.argtypes = [pp, vp, vp, vp, fp, fp, fp, fp, fp, vp, fp, fp, ip, ctypes.c_int32, vp,
                                      ctypes.c_size_t, vp]
        L.osdn_bwd_packed.restype = ctypes.c_int
        L.osdn_bwd_packed.argtypes = [pp] + [vp] * 19 + [ip, ctypes.c_int32, vp, ctypes.c_size_t, vp]
        L.osdn_step.restype = ctypes.c_int
        L.osdn_step.argtypes = [pp, vp, vp, vp, fp, fp, fp, fp, fp, vp, fp, fp, vp]
        np_, dp = ctypes.POINTER(OsdnNormParams), ctypes.POINTER(OsdnDecodeParams)
        rp, cp = ctypes.POINTER(OsdnRows), ctypes.POINTER(OsdnCache)
        L.osdn_qk_norm_fwd.restype = ctypes.c_int
        L.osdn_qk_norm_fwd.argtypes = [np_, rp, rp, fp, fp, fp, vp, rp, rp, vp]
        L.osdn_qk_norm_bwd_workspace_bytes.restype = ctypes.c_size_t
        L.osdn_qk_norm_bwd_workspace_bytes.argtypes = [np_]
        L.osdn_qk_norm_bwd.restype = ctypes.c_int
        L.osdn_qk_norm_bwd.argtypes = [np_, rp, rp, fp, fp, fp, vp, rp, rp, rp, rp, fp, fp, vp, ctypes.c_size_t, vp]
        L.osdn_paged_append.restype = ctypes.c_int
        L.osdn_paged_append.argtypes = [np_, cp, rp, rp, rp, fp, fp, fp, vp, vp, rp, vp]
        L.osdn_paged_decode_workspace_bytes.restype = ctypes.c_size_t
        L.osdn_paged_decode_workspace_bytes.argtypes = [dp]
        L.osdn_paged_decode.restype = ctypes.c_int
        L.osdn_paged_decode.argtypes = [dp, cp, rp, vp, vp, rp, fp, vp, ctypes.c_size_t, vp]
        mp, gp, sp = ctypes.POINTER(OsdnCacheMx), ctypes.POINTER(OsdnPages), ctypes.POINTER(OsdnSelectParams)
        i32, size = ctypes.c_int32, ctypes.c_size_t
        for name, of in (("osdn_paged_plan", [gp, i32, i32] + [vp] * 11), ("osdn_paged_release", [gp, i32] + [vp] * 5),
                         ("osdn_paged_append_mx", [np_, mp, rp, rp, rp, fp, fp, fp, vp, vp, rp, vp]), ("osdn_paged_read_mx", [np_, mp, vp, vp, rp, rp, vp]),
                         ("osdn_paged_decode_mx", [dp, mp, rp, vp, vp, rp, fp, vp, size, vp]),
                         ("osdn_paged_decode_pages", [dp, cp, rp, vp, i32, vp, rp, fp, vp, size, vp]),
                         ("osdn_paged_decode_pages_mx", [dp, mp, rp, vp, i32, vp, rp, fp, vp, size, vp]),
                         ("osdn_page_bounds", [sp, cp, vp, vp, vp, vp, vp]), ("osdn_page_bounds_mx", [sp, mp, vp, vp, vp, vp, vp]),
                         ("osdn_page_select", [sp, gp, rp, vp, vp, vp, vp, vp, vp, size, vp])):
            getattr(L, name).restype = ctypes.c_int
            getattr(L, name).argtypes = of
        for name, of in (("osdn_paged_decode_mx_workspace_bytes", [dp]), ("osdn_paged_decode_pages_workspace_bytes", [dp]),
                         ("osdn_paged_decode_pages_mx_workspace_bytes", [dp]), ("osdn_page_select_workspace_bytes", [sp, i32])):
            getattr(L, name).restype = size
            getattr(L, name).argtypes = of
        L.osdn_profile_enable.restype = None
        L.osdn_profile_enable.argtypes = [ctypes.c_int]
        L.osdn_profile_kernel_count.restype = ctypes.c_int
        L.osdn_profile_kernel_name.restype = ctypes.c_char_p
        L.osdn_profile_kernel_name.argtypes = [ctypes.c_int]
        L.osdn_profile_read.restype = ctypes.c_int
        L.osdn_profile_read.argtypes = [ctypes.POINTER(ctypes.c_double), ctypes.POINTER(ctypes.c_int), ctypes.c_int]
        _lib = L
        try:
            from . import _native
            _native.bind(ctypes.cast(L.osdn_step, vp).value, ctypes.sizeof(OsdnParams), torch.__version__)
            _native.bind_rows(*(ctypes.cast(f, vp).value for f in (
                L.osdn_qk_norm_fwd, L.osdn_qk_norm_bwd, L.osdn_qk_norm_bwd_workspace_bytes, L.osdn_paged_append, L.osdn_paged_decode,
                L.osdn_paged_decode_workspace_bytes)), *(ctypes.sizeof(c) for c in (OsdnRows, OsdnNormParams, OsdnCache, OsdnDecodeParams)))
            _native.bind_pages(tuple(ctypes.cast(getattr(L, "osdn_" + f), vp).value for f in (
                "paged_plan", "paged_release", "paged_append_mx", "paged_read_mx", "paged_decode_mx", "paged_decode_mx_workspace_bytes", "page_bounds",
                "page_bounds_mx", "page_select", "page_select_workspace_bytes", "paged_decode_pages", "paged_decode_pages_workspace_bytes",
                "paged_decode_pages_mx", "paged_decode_pages_mx_workspace_bytes")), *(ctypes.sizeof(c) for c in (OsdnPages, OsdnCacheMx, OsdnSelectParams)))
            _step_native, _rows_native = _native.step, _native
        except (ImportError, TypeError, AttributeError) as e:       # (TypeError, AttributeError: one of an earlier interface)
            warnings.warn(f"no extension module ({e}): step goes through Python, at twice the time of a small call; "
                          "run python -m paper_2605_13473_amd.build", RuntimeWarning, stacklevel=2)
    return _lib


def osdn_profile_enable(on: bool) -> None:
    lib().osdn_profile_enable(int(bool(on)))


def osdn_profile_read() -> dict:
    """{kernel name: (summed milliseconds, launches)} since the previous read."""
    L = lib()
    n = L.osdn_profile_kernel_count()
    ms = (ctypes.c_double * n)()
    cnt = (ctypes.c_int * n)()
    _check(L.osdn_profile_read(ms, cnt, n))
    return {L.osdn_profile_kernel_name(i).decode(): (ms[i], cnt[i]) for i in range(n)}


def osdn_strerror(status: int) -> str:
    return lib().osdn_strerror(int(status)).decode()


def osdn_workspace_bytes(params: OsdnParams, for_backward: bool) -> int:
    return int(lib().osdn_workspace_bytes(ctypes.byref(params), int(bool(for_backward))))


def osdn_debug_mask_offset(params: OsdnParams) -> int:
    return int(lib().osdn_debug_mask_offset(ctypes.byref(params)))


def _io_torch_dtype(params: OsdnParams):
    return torch.bfloat16 if params.io_dtype == OSDN_BF16 else torch.float32


def _ptr(t, dtype, shape=None, name="tensor"):
    if t is None:
        return None
    # what every good call takes, as one expression; the checks one by one below say what is wrong with a bad one
    if isinstance(t, torch.Tensor) and t.is_cuda and t.dtype == dtype and t.is_contiguous() and (
            shape is None or t.shape == shape):
        return t.data_ptr()
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name}: expected a CUDA/HIP torch tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected dtype {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name}: must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    return t.data_ptr()


def _stream_ptr(stream):
    if stream is None:      # the handle of torch.cuda.current_stream(), without the Stream object
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return stream.cuda_stream


def _check(rc):
    if rc != 0:
        raise OsdnError(rc)


def osdn_precond_update(params, k, beta, retention, d_in, k_tilde, d_out, d_ckpt=None, stream=None):
    p = params
    io, f32 = _io_torch_dtype(p), torch.float32
    _check(lib().osdn_precond_update(
        ctypes.byref(p),
        _ptr(k, io, (p.B, p.T, p.H, p.K), "k"), _ptr(beta, f32, (p.B, p.T, p.H), "beta"),
        _ptr(retention, f32, _ret_shape(p), "retention"), _ptr(d_in, f32, (p.B, p.H, p.K), "d_in"),
        _ptr(k_tilde, io, (p.B, p.T, p.H, p.K), "k_tilde"), _ptr(d_out, f32, (p.B, p.H, p.K), "d_out"),
        _ptr(d_ckpt, f32, None, "d_ckpt"), _stream_ptr(stream)))


def osdn_step(params, q, k, v, beta, log_alpha, retention, d_in, S_in, o, S_out, d_out, stream=None):
    # (`step` comes here with what the extension module leaves to it.)
    p = params
    B, T, H, K, V = p.B, p.T, p.H, p.K, p.V
    io, f32 = _io_torch_dtype(p), torch.float32
    bth, bthk, bthv, bhk, bhvk = (B, T, H), (B, T, H, K), (B, T, H, V), (B, H, K), (B, H, V, K)
    _check(lib().osdn_step(
        ctypes.byref(p), _ptr(q, io, bthk, "q"), _ptr(k, io, bthk, "k"), _ptr(v, io, bthv, "v"),
        _ptr(beta, f32, bth, "beta"), _ptr(log_alpha, f32, bthk if p.gate_per_channel else bth, "log_alpha"),
        _ptr(retention, f32, bthk if p.retention_per_channel else bth, "retention"), _ptr(d_in, f32, bhk, "d_in"),
        _ptr(S_in, f32, bhvk, "S_in"), _ptr(o, io, bthv, "o"), _ptr(S_out, f32, bhvk, "S_out"),
        _ptr(d_out, f32, bhk, "d_out"), _stream_ptr(stream)))


def osdn_fwd(params, q, k, v, beta, log_alpha, retention, d_in, S_in, o, S_out, d_out, workspace,
             stream=None):
    p = params
    io, f32 = _io_torch_dtype(p), torch.float32
    bth, bthk, bthv = (p.B, p.T, p.H), (p.B, p.T, p.H, p.K), (p.B, p.T, p.H, p.V)
    _check(lib().osdn_fwd(
        ctypes.byref(p), _ptr(q, io, bthk, "q"), _ptr(k, io, bthk, "k"), _ptr(v, io, bthv, "v"),
        _ptr(beta, f32, bth, "beta"), _ptr(log_alpha, f32, _gate_shape(p), "log_alpha"),
        _ptr(retention, f32, _ret_shape(p), "retention"), _ptr(d_in, f32, (p.B, p.H, p.K), "d_in"),
        _ptr(S_in, f32, (p.B, p.H, p.V, p.K), "S_in"), _ptr(o, io, bthv, "o"),
        _ptr(S_out, f32, (p.B, p.H, p.V, p.K), "S_out"), _ptr(d_out, f32, (p.B, p.H, p.K), "d_out"),
        _ptr(workspace, torch.uint8, None, "workspace"), ctypes.c_size_t(workspace.numel()),
        _stream_ptr(stream)))


def osdn_fwd_noalloc(params, q, k, v, beta, log_alpha, retention, d_in, S_in, o, S_out, d_out, stream=None):
    p = params
    io, f32 = _io_torch_dtype(p), torch.float32
    bth, bthk, bthv = (p.B, p.T, p.H), (p.B, p.T, p.H, p.K), (p.B, p.T, p.H, p.V)
    _check(lib().osdn_fwd_noalloc(
        ctypes.byref(p), _ptr(q, io, bthk, "q"), _ptr(k, io, bthk, "k"), _ptr(v, io, bthv, "v"),
        _ptr(beta, f32, bth, "beta"), _ptr(log_alpha, f32, _gate_shape(p), "log_alpha"),
        _ptr(retention, f32, _ret_shape(p), "retention"), _ptr(d_in, f32, (p.B, p.H, p.K), "d_in"),
        _ptr(S_in, f32, (p.B, p.H, p.V, p.K), "S_in"), _ptr(o, io, bthv, "o"),
        _ptr(S_out, f32, (p.B, p.H, p.V, p.K), "S_out"), _ptr(d_out, f32, (p.B, p.H, p.K), "d_out"),
        _stream_ptr(stream)))


def osdn_bwd(params, q, k, v, beta, log_alpha, retention, d_in, S_in, dO, dS_out, dd_out,
             dq, dk, dv, dbeta, dlog_alpha, dretention, dd_in, dS_in, workspace, stream=None):
    p = params
    io, f32 = _io_torch_dtype(p), torch.float32
    bth, bthk, bthv = (p.B, p.T, p.H), (p.B, p.T, p.H, p.K), (p.B, p.T, p.H, p.V)
    bhk, bhvk = (p.B, p.H, p.K), (p.B, p.H, p.V, p.K)
    _check(lib().osdn_bwd(
        ctypes.byref(p), _ptr(q, io, bthk, "q"), _ptr(k, io, bthk, "k"), _ptr(v, io, bthv, "v"),
        _ptr(beta, f32, bth, "beta"), _ptr(log_alpha, f32, _gate_shape(p), "log_alpha"),
        _ptr(retention, f32, _ret_shape(p), "retention"), _ptr(d_in, f32, bhk, "d_in"),
        _ptr(S_in, f32, bhvk, "S_in"), _ptr(dO, io, bthv, "dO"), _ptr(dS_out, f32, bhvk, "dS_out"),
        _ptr(dd_out, f32, bhk, "dd_out"), _ptr(dq, io, bthk, "dq"), _ptr(dk, io, bthk, "dk"),
        _ptr(dv, io, bthv, "dv"), _ptr(dbeta, f32, bth, "dbeta"),
        _ptr(dlog_alpha, f32, _gate_shape(p), "dlog_alpha"), _ptr(dretention, f32, _ret_shape(p), "dretention"),
        _ptr(dd_in, f32, bhk, "dd_in"), _ptr(dS_in, f32, bhvk, "dS_in"),
        _ptr(workspace, torch.uint8, None, "workspace"), ctypes.c_size_t(workspace.numel()),
        _stream_ptr(stream)))


def _cu(cu_seqlens):
    """Host int32 array of n_seqs + 1 offsets from a sequence of ints."""
    vals = [int(x) for x in cu_seqlens]
    return (ctypes.c_int32 * len(vals))(*vals), len(vals) - 1


def osdn_workspace_bytes_packed(params: OsdnParams, cu_seqlens, for_backward: bool) -> int:
    cu, n = _cu(cu_seqlens)
    return int(lib().osdn_workspace_bytes_packed(ctypes.byref(params), cu, n, int(bool(for_backward))))


def osdn_fwd_packed(params, q, k, v, beta, log_alpha, retention, d_in, S_in, o, S_out, d_out, cu_seqlens,
                    workspace, stream=None):
    p = params
    cu, n = _cu(cu_seqlens)
    io, f32 = _io_torch_dtype(p), torch.float32
    bth, bthk, bthv = (p.B, p.T, p.H), (p.B, p.T, p.H, p.K), (p.B, p.T, p.H, p.V)
    _check(lib().osdn_fwd_packed(
        ctypes.byref(p), _ptr(q, io, bthk, "q"), _ptr(k, io, bthk, "k"), _ptr(v, io, bthv, "v"),
        _ptr(beta, f32, bth, "beta"), _ptr(log_alpha, f32, _gate_shape(p), "log_alpha"),
        _ptr(retention, f32, _ret_shape(p), "retention"), _ptr(d_in, f32, (n, p.H, p.K), "d_in"),
        _ptr(S_in, f32, (n, p.H, p.V, p.K), "S_in"), _ptr(o, io, bthv, "o"),
        _ptr(S_out, f32, (n, p.H, p.V, p.K), "S_out"), _ptr(d_out, f32, (n, p.H, p.K), "d_out"),
        cu, n, _ptr(workspace, torch.uint8, None, "workspace"), ctypes.c_size_t(workspace.numel()),
        _stream_ptr(stream)))


def osdn_bwd_packed(params, q, k, v, beta, log_alpha, retention, d_in, S_in, dO, dS_out, dd_out,
                    dq, dk, dv, dbeta, dlog_alpha, dretention, dd_in, dS_in, cu_seqlens, workspace, stream=None):
    p = params
    cu, n = _cu(cu_seqlens)
    io, f32 = _io_torch_dtype(p), torch.float32
    bth, bthk, bthv = (p.B, p.T, p.H), (p.B, p.T, p.H, p.K), (p.B, p.T, p.H, p.V)
    bhk, bhvk = (n, p.H, p.K), (n, p.H, p.V, p.K)
    _check(lib().osdn_bwd_packed(
        ctypes.byref(p), _ptr(q, io, bthk, "q"), _ptr(k, io, bthk, "k"), _ptr(v, io, bthv, "v"),
        _ptr(beta, f32, bth, "beta"), _ptr(log_alpha, f32, _gate_shape(p), "log_alpha"),
        _ptr(retention, f32, _ret_shape(p), "retention"), _ptr(d_in, f32, bhk, "d_in"),
        _ptr(S_in, f32, bhvk, "S_in"), _ptr(dO, io, bthv, "dO"), _ptr(dS_out, f32, bhvk, "dS_out"),
        _ptr(dd_out, f32, bhk, "dd_out"), _ptr(dq, io, bthk, "dq"), _ptr(dk, io, bthk, "dk"),
        _ptr(dv, io, bthv, "dv"), _ptr(dbeta, f32, bth, "dbeta"),
        _ptr(dlog_alpha, f32, _gate_shape(p), "dlog_alpha"), _ptr(dretention, f32, _ret_shape(p), "dretention"),
        _ptr(dd_in, f32, bhk, "dd_in"), _ptr(dS_in, f32, bhvk, "dS_in"),
        cu, n, _ptr(workspace, torch.uint8, None, "workspace"), ctypes.c_size_t(workspace.numel()),
        _stream_ptr(stream)))


# ------------------------------------------------------------- conveniences ----
@dataclass
class Hyper:
    scale: float | None = None   # None => K ** -0.5
    eta: float = 0.003
    d_min: float = 0.5
    d_max: float = 2.0
    eps: float = 1e-6
    beta_aware: bool = True
    # scheduling knobs of osdn_params (0: the library decides)
    segments: int = 0
    p1_pieces: int = 0
    p1_piece_sweeps: int = 0
    p1_solved: int = 0


def make_params(B, T, H, K, V, bf16: bool, hp: Hyper = Hyper(), retention_per_channel: bool = False,
                gate_per_channel: bool = False) -> OsdnParams:
    scale = float(K) ** -0.5 if hp.scale is None else float(hp.scale)
    return OsdnParams(B, T, H, K, V, 64, OSDN_BF16 if bf16 else OSDN_F32, scale, hp.eta, hp.d_min,
                      hp.d_max, hp.eps, int(hp.beta_aware), int(bool(retention_per_channel)),
                      int(bool(gate_per_channel)), int(hp.segments), int(hp.p1_pieces), int(hp.p1_piece_sweeps),
                      int(hp.p1_solved))


_PARAMS = struct.Struct("=7i5f7i")
assert _PARAMS.size == ctypes.sizeof(OsdnParams)


def _shape_params(B, T, H, K, V, bf16, hp, retention_per_channel, gate_per_channel) -> OsdnParams:
    """make_params for sizes that come from a tensor's shape: the same fields, packed at once (1.5 -> 0.9 us)."""
    try:
        return OsdnParams.from_buffer_copy(_PARAMS.pack(
            B, T, H, K, V, 64, OSDN_BF16 if bf16 else OSDN_F32,
            float(K) ** -0.5 if hp.scale is None else float(hp.scale), hp.eta, hp.d_min, hp.d_max, hp.eps,
            int(hp.beta_aware), retention_per_channel, gate_per_channel, int(hp.segments), int(hp.p1_pieces),
            int(hp.p1_piece_sweeps), int(hp.p1_solved)))
    except (struct.error, OverflowError):       # (a value outside its field: what ctypes makes of it)
        return make_params(B, T, H, K, V, bf16, hp, retention_per_channel, gate_per_channel)


def _ret_shape(p: OsdnParams):
    return (p.B, p.T, p.H, p.K) if p.retention_per_channel else (p.B, p.T, p.H)


def _gate_shape(p: OsdnParams):
    return (p.B, p.T, p.H, p.K) if p.gate_per_channel else (p.B, p.T, p.H)


def _per_channel(retention) -> bool:
    return retention is not None and retention.dim() == 4


def alloc_workspace(params: OsdnParams, for_backward: bool, device="cuda") -> torch.Tensor:
    n = osdn_workspace_bytes(params, for_backward)
    if n == 0:
        raise OsdnError(-2)
    return torch.empty(n, dtype=torch.uint8, device=device)   # torch allocations are >= 256-byte aligned


def forward(q, k, v, beta, log_alpha=None, retention=None, d_in=None, S_in=None, hp: Hyper = Hyper(),
            for_backward: bool = False, workspace=None, cu_seqlens=None):
    """Allocate outputs (+ workspace) and call osdn_fwd (osdn_fwd_packed when cu_seqlens is
    given: B == 1, one carried entry per sequence).  Returns (o, S_out, d_out, ctx)."""
    B, T, H, K = k.shape
    V = v.shape[-1]
    p = _shape_params(B, T, H, K, V, k.dtype == torch.bfloat16, hp, _per_channel(retention), _per_channel(log_alpha))
    if cu_seqlens is not None:
        cu_seqlens = [int(x) for x in cu_seqlens]
    if workspace is None:
        if cu_seqlens is None:
            workspace = alloc_workspace(p, for_backward, k.device)
        else:
            n = osdn_workspace_bytes_packed(p, cu_seqlens, for_backward)
            if n == 0:
                raise OsdnError(-2)
            workspace = torch.empty(n, dtype=torch.uint8, device=k.device)
    nb = B if cu_seqlens is None else len(cu_seqlens) - 1
    o = torch.empty_like(v)
    S_out = torch.empty(nb, H, V, K, dtype=torch.float32, device=k.device)
    d_out = torch.empty(nb, H, K, dtype=torch.float32, device=k.device)
    if cu_seqlens is None:
        osdn_fwd(p, q, k, v, beta, log_alpha, retention, d_in, S_in, o, S_out, d_out, workspace)
    else:
        osdn_fwd_packed(p, q, k, v, beta, log_alpha, retention, d_in, S_in, o, S_out, d_out, cu_seqlens, workspace)
    ctx = dict(params=p, inputs=(q, k, v, beta, log_alpha, retention, d_in, S_in), workspace=workspace,
               cu_seqlens=cu_seqlens)
    return o, S_out, d_out, ctx


def backward(ctx, dO, dS_out=None, dd_out=None):
    """Allocate gradients and call osdn_bwd on the context returned by ``forward``."""
    p = ctx["params"]
    q, k, v, beta, log_alpha, retention, d_in, S_in = ctx["inputs"]
    cu = ctx.get("cu_seqlens")
    nb = p.B if cu is None else len(cu) - 1
    f32 = dict(dtype=torch.float32, device=k.device)
    g = {
        "dq": torch.empty_like(q), "dk": torch.empty_like(k), "dv": torch.empty_like(v),
        "dbeta": torch.empty_like(beta),
        "dlog_alpha": torch.empty_like(log_alpha) if log_alpha is not None else None,
        "dretention": torch.empty_like(retention) if retention is not None else None,
        "dd_in": torch.empty(nb, p.H, p.K, **f32), "dS_in": torch.empty(nb, p.H, p.V, p.K, **f32),
    }
    if cu is None:
        osdn_bwd(p, q, k, v, beta, log_alpha, retention, d_in, S_in, dO, dS_out, dd_out,
                 g["dq"], g["dk"], g["dv"], g["dbeta"], g["dlog_alpha"], g["dretention"], g["dd_in"],
                 g["dS_in"], ctx["workspace"])
    else:
        osdn_bwd_packed(p, q, k, v, beta, log_alpha, retention, d_in, S_in, dO, dS_out, dd_out,
                        g["dq"], g["dk"], g["dv"], g["dbeta"], g["dlog_alpha"], g["dretention"], g["dd_in"],
                        g["dS_in"], cu, ctx["workspace"])
    return g


def step(q, k, v, beta, log_alpha=None, retention=None, d_in=None, S_in=None, hp: Hyper = Hyper(),
         in_place: bool = False):
    """Recurrent form for 1..64 tokens: returns (o, S_out, d_out); with in_place the state S_in
    is updated where it is (and returned)."""
    if _lib is None:
        lib()
    if _step_native is not None and isinstance(k, torch.Tensor) and k.is_cuda:
        # a call without anything out of the ordinary (osdn_native.cpp); else None
        dev = torch._C._cuda_getDevice()
        r = _step_native(q, k, v, beta, log_alpha, retention, d_in, S_in, hp, in_place, dev,
                         torch._C._cuda_getCurrentRawStream(dev))
        if r is not None:
            if type(r) is tuple:
                return r
            _check(r)
    B, T, H, K = k.shape
    V = v.shape[-1]
    p = _shape_params(B, T, H, K, V, k.dtype == torch.bfloat16, hp, _per_channel(retention), _per_channel(log_alpha))
    f32 = dict(dtype=torch.float32, device=k.device)
    o = torch.empty_like(v)
    S_out = S_in if (in_place and S_in is not None) else torch.empty(B, H, V, K, **f32)
    d_out = torch.empty(B, H, K, **f32)
    osdn_step(p, q, k, v, beta, log_alpha, retention, d_in, S_in, o, S_out, d_out)
    return o, S_out, d_out


def precond_update(k, beta, retention=None, d_in=None, hp: Hyper = Hyper(), want_ckpt: bool = False):
    """Allocate outputs and call osdn_precond_update.  Returns (k_tilde, d_out[, d_ckpt])."""
    B, T, H, K = k.shape
    p = make_params(B, T, H, K, 64, k.dtype == torch.bfloat16, hp, _per_channel(retention))
    kt = torch.empty_like(k)
    d_out = torch.empty(B, H, K, dtype=torch.float32, device=k.device)
    ck = torch.empty(B, H, T // 64, K, dtype=torch.float32, device=k.device) if want_ckpt else None
    osdn_precond_update(p, k, beta, retention, d_in, kt, d_out, ck)
    return (kt, d_out, ck) if want_ckpt else (kt, d_out)


# ------------------------------------------- queries, keys and values around the recurrence ----
NORMS = {"none": 0, "rms": 1, "l2": 2}


@dataclass
class NormHyper:
    norm: str = "l2"             # "l2": unit length (what the recurrence expects), "rms": unit mean square, "none"
    eps: float = 1e-6            # added to the sum (mean) of squares
    interleaved: bool = False    # rotation of the pairs (2i, 2i + 1); else (i, i + rotary_dim / 2)


def make_norm_params(B, T, Hq, Hk, K, bf16: bool, hp: NormHyper = NormHyper(), rotary=None) -> OsdnNormParams:
    if hp.norm not in NORMS:
        raise ValueError(f"norm: expected one of {sorted(NORMS)}, got {hp.norm!r}")
    if rotary is not None and (not isinstance(rotary, torch.Tensor) or rotary.dim() != 2):
        raise TypeError("rotary: expected a table [positions, rotary_dim]")
    rows, dim = (0, 0) if rotary is None else rotary.shape
    return OsdnNormParams(B, T, Hq, Hk, K, OSDN_BF16 if bf16 else OSDN_F32, NORMS[hp.norm], dim, rows, int(bool(hp.interleaved)),
                          hp.eps)


def make_decode_params(B, Hq, Hk, K, bf16: bool, max_length: int, scale: float | None = None, window: int = 0,
                       shares: int = 0) -> OsdnDecodeParams:
    # (a number past its field's end is the end: a window still shows all, the others are refused)
    end = lambda x: max(-2**31, min(2**31 - 1, int(x)))
    return OsdnDecodeParams(B, Hq, Hk, K, OSDN_BF16 if bf16 else OSDN_F32, end(window or 0), end(max_length), end(shares),
                            float(K) ** -0.5 if scale is None else float(scale))


def rotary_table(rows: int, dim: int, theta: float = 10000.0, device="cuda") -> torch.Tensor:
    """The table of the rotation, [rows, dim] fp32: a position's cosines, then its sines (angle i: position theta^(-2 i / dim),
    formed in 64 bits)."""
    angle = torch.arange(rows, dtype=torch.float64)[:, None] * theta ** (-2.0 * torch.arange(dim // 2, dtype=torch.float64) / dim)
    return torch.cat([angle.cos(), angle.sin()], dim=1).float().to(device)


def alloc_paged_cache(n_pages: int, page_size: int, H: int, K: int, dtype=torch.bfloat16, device="cuda"):
    """(k_cache, v_cache), [n_pages, page_size, H, K]: a page holds its tokens head after head (any order of pages,
    tokens and heads is taken, the other one as fast)."""
    return tuple(torch.empty(n_pages, H, page_size, K, dtype=dtype, device=device).transpose(1, 2) for _ in range(2))


def _here(t, name):
    """Launches go to the current device, which need not see the memory of another."""
    if t.device.index != torch._C._cuda_getDevice():
        raise ValueError(f"{name}: is on {t.device}, the current device is {torch._C._cuda_getDevice()}")


def _array(t, dtype, shape, name):
    p = _ptr(t, dtype, shape, name)
    if t is not None:
        _here(t, name)
    return p


def _rows(t, dtype, shape, name):
    """Rows of the last axis, wherever they stand: [B,T,H,K], or [B,H,K]."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name}: expected a CUDA/HIP torch tensor")
    if t.dtype != dtype:
        raise TypeError(f"{name}: expected dtype {dtype}, got {t.dtype}")
    if tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name}: expected shape {tuple(shape)}, got {tuple(t.shape)}")
    _here(t, name)
    st = t.stride()
    if st[-1] != 1:
        raise ValueError(f"{name}: the elements of a row must be adjacent")
    return OsdnRows(t.data_ptr(), st[0], st[1] if len(st) == 4 else 0, st[-2])


def _cache(k_cache, v_cache, page_table, dtype, H, K):
    if not isinstance(k_cache, torch.Tensor) or k_cache.dim() != 4:
        raise TypeError("k_cache: expected a CUDA/HIP torch tensor [n_pages, page_size, H, K]")
    n_pages, page_size = k_cache.shape[:2]
    for t, name in ((k_cache, "k_cache"), (v_cache, "v_cache")):
        _rows(t, dtype, (n_pages, page_size, H, K), name)
    if not isinstance(page_table, torch.Tensor) or not page_table.is_cuda or page_table.dtype != torch.int32:
        raise TypeError("page_table: expected an int32 CUDA/HIP torch tensor")
    if page_table.dim() != 2 or (page_table.shape[1] > 1 and page_table.stride(1) != 1):
        raise ValueError("page_table: expected [n_seqs, max_pages] with adjacent entries of a row")
    _here(page_table, "page_table")
    n_seqs, max_pages = page_table.shape
    k, v = k_cache.stride(), v_cache.stride()
    stride = page_table.stride(0) if n_seqs > 1 else max_pages
    return OsdnCache(k_cache.data_ptr(), v_cache.data_ptr(), k[0], k[1], k[2], v[0], v[1], v[2], page_table.data_ptr(), stride,
                     n_pages, page_size, n_seqs, max_pages)


def _ref(x):
    return None if x is None else ctypes.byref(x)


def _norm_rows(p, q, k, *more):
    io = _io_torch_dtype(p)
    sq, sk = (p.B, p.T, p.Hq, p.K), (p.B, p.T, p.Hk, p.K)
    return [_rows(t, io, sk if name.startswith(("k", "v", "dk")) else sq, name) for t, name in ((q, "q"), (k, "k"), *more)]


def _norm_shared(p, weight_q, weight_k, rotary, positions):
    f32 = torch.float32
    return (_array(weight_q, f32, (p.K,), "weight_q"), _array(weight_k, f32, (p.K,), "weight_k"),
            _array(rotary, f32, (p.rotary_rows, p.rotary_dim), "rotary"), _array(positions, torch.int32, (p.B, p.T), "positions"))


def osdn_qk_norm_fwd(params, q, k, weight_q, weight_k, rotary, positions, q_out, k_out, stream=None):
    r = _norm_rows(params, q, k, (q_out, "q_out"), (k_out, "k_out"))
    _check(lib().osdn_qk_norm_fwd(ctypes.byref(params), _ref(r[0]), _ref(r[1]), *_norm_shared(params, weight_q, weight_k, rotary, positions),
                                  _ref(r[2]), _ref(r[3]), _stream_ptr(stream)))


def osdn_qk_norm_bwd_workspace_bytes(params) -> int:
    return int(lib().osdn_qk_norm_bwd_workspace_bytes(ctypes.byref(params)))


def osdn_qk_norm_bwd(params, q, k, weight_q, weight_k, rotary, positions, dq_out, dk_out, dq, dk, dweight_q, dweight_k, workspace=None,
                     stream=None):
    p, f32 = params, torch.float32
    r = _norm_rows(p, q, k, (dq_out, "dq_out"), (dk_out, "dk_out"), (dq, "dq"), (dk, "dk"))
    _check(lib().osdn_qk_norm_bwd(
        ctypes.byref(p), _ref(r[0]), _ref(r[1]), *_norm_shared(p, weight_q, weight_k, rotary, positions), *(_ref(x) for x in r[2:]),
        _array(dweight_q, f32, (p.K,), "dweight_q"), _array(dweight_k, f32, (p.K,), "dweight_k"), _array(workspace, torch.uint8, None, "workspace"),
        ctypes.c_size_t(0 if workspace is None else workspace.numel()), _stream_ptr(stream)))


def osdn_paged_append(params, q, k, v, k_cache, v_cache, page_table, weight_q, weight_k, rotary, positions, seq, q_out, stream=None):
    p = params
    r = _norm_rows(p, q, k, (v, "v"), (q_out, "q_out"))
    cache = _cache(k_cache, v_cache, page_table, _io_torch_dtype(p), p.Hk, p.K)
    _check(lib().osdn_paged_append(
        ctypes.byref(p), ctypes.byref(cache), *(_ref(x) for x in r[:3]), *_norm_shared(p, weight_q, weight_k, rotary, positions),
        _array(seq, torch.int32, (p.B, p.T), "seq"), _ref(r[3]), _stream_ptr(stream)))


def osdn_paged_decode_workspace_bytes(params) -> int:
    return int(lib().osdn_paged_decode_workspace_bytes(ctypes.byref(params)))


def osdn_paged_decode(params, q, k_cache, v_cache, page_table, lengths, seq, o, lse, workspace=None, stream=None):
    p, i32 = params, torch.int32
    io, rows = _io_torch_dtype(p), (p.B, p.Hq, p.K)
    qr, orows = _rows(q, io, rows, "q"), _rows(o, io, rows, "o")
    cache = _cache(k_cache, v_cache, page_table, io, p.Hk, p.K)
    _check(lib().osdn_paged_decode(
        ctypes.byref(p), ctypes.byref(cache), _ref(qr), _array(lengths, i32, (p.B,), "lengths"), _array(seq, i32, (p.B,), "seq"), _ref(orows),
        _array(lse, torch.float32, (p.B, p.Hq), "lse"), _array(workspace, torch.uint8, None, "workspace"),
        ctypes.c_size_t(0 if workspace is None else workspace.numel()), _stream_ptr(stream)))


def _params_of(q, k, hp, rotary):
    x = k if q is None else q
    if not isinstance(x, torch.Tensor) or x.dim() != 4 or (q is not None and k is not None and (not isinstance(k, torch.Tensor) or k.dim() != 4)):
        raise TypeError("expected rows [B,T,H,K] as CUDA/HIP torch tensors")
    B, T, _, K = x.shape
    return make_norm_params(B, T, 0 if q is None else q.shape[2], 0 if k is None else k.shape[2], K, x.dtype == torch.bfloat16, hp, rotary)


# A call of plain tensors on the current device goes through the extension module, once the library is loaded (_rows_native is then set);
# for what that leaves alone it returns None, and a status for what the library refuses.
def qk_norm(q, k, weight_q=None, weight_k=None, rotary=None, positions=None, hp: NormHyper = NormHyper()):
    """Allocate outputs and call osdn_qk_norm_fwd (either of q and k may be None).  Returns (q_out, k_out)."""
    x = k if q is None else q
    if _rows_native is not None and type(x) is torch.Tensor and x.is_cuda:
        dev = torch._C._cuda_getDevice()
        r = _rows_native.qk_norm(q, k, weight_q, weight_k, rotary, positions, hp, dev, torch._C._cuda_getCurrentRawStream(dev))
        if r is not None:
            return r if type(r) is tuple else _check(r)
    p = _params_of(q, k, hp, rotary)
    out = [None if x is None else x.new_empty(x.shape) for x in (q, k)]
    osdn_qk_norm_fwd(p, q, k, weight_q, weight_k, rotary, positions, *out)
    return tuple(out)


def qk_norm_backward(q, k, dq_out, dk_out, weight_q=None, weight_k=None, rotary=None, positions=None, hp: NormHyper = NormHyper()):
    """Allocate gradients and call osdn_qk_norm_bwd on the inputs of ``qk_norm``.  Returns a dict of dq, dk and, where there are
    weights, dweight_q, dweight_k."""
    x = k if q is None else q
    if _rows_native is not None and type(x) is torch.Tensor and x.is_cuda:
        dev = torch._C._cuda_getDevice()
        r = _rows_native.qk_norm_backward(q, k, dq_out, dk_out, weight_q, weight_k, rotary, positions, hp, dev,
                                          torch._C._cuda_getCurrentRawStream(dev))
        if type(r) is tuple:
            return {"dq": r[0], "dk": r[1], "dweight_q": r[2], "dweight_k": r[3]}
        if r is not None:
            _check(r)
    p = _params_of(q, k, hp, rotary)
    g = {"dq": None if q is None else q.new_empty(q.shape), "dk": None if k is None else k.new_empty(k.shape),
         "dweight_q": None if weight_q is None else torch.empty_like(weight_q), "dweight_k": None if weight_k is None else torch.empty_like(weight_k)}
    ws = None
    if weight_q is not None or weight_k is not None:
        ws = torch.empty(osdn_qk_norm_bwd_workspace_bytes(p), dtype=torch.uint8, device=(k if q is None else q).device)
    osdn_qk_norm_bwd(p, q, k, weight_q, weight_k, rotary, positions, dq_out, dk_out, g["dq"], g["dk"], g["dweight_q"], g["dweight_k"], ws)
    return g


def paged_append(k, v, k_cache, v_cache, page_table, positions, seq=None, q=None, weight_q=None, weight_k=None, rotary=None,
                 hp: NormHyper = NormHyper()):
    """Append keys (normed and rotated) and values [B,T,Hk,K] to a paged cache [n_pages, page_size, Hk, K]; with q [B,T,Hq,K],
    returns the queries normed and rotated alike, from the same launch."""
    if _rows_native is not None and type(k) is torch.Tensor and k.is_cuda:
        dev = torch._C._cuda_getDevice()
        r = _rows_native.paged_append(k, v, k_cache, v_cache, page_table, positions, seq, q, weight_q, weight_k, rotary, hp, dev,
                                      torch._C._cuda_getCurrentRawStream(dev))
        if r is not None:
            return r[0] if type(r) is tuple else _check(r)
    p = _params_of(q, k, hp, rotary)
    q_out = None if q is None else q.new_empty(q.shape)
    osdn_paged_append(p, q, k, v, k_cache, v_cache, page_table, weight_q, weight_k, rotary, positions, seq, q_out)
    return q_out


def paged_decode(q, k_cache, v_cache, page_table, lengths, seq=None, scale=None, window: int = 0, max_length=None, want_lse: bool = False,
                 workspace=None):
    """Attention of one new token per sequence, q [B,Hq,K], over a paged cache.  max_length: no length is above it (None: what a
    row of the table can hold).  More queries than a call of osdn_paged_decode takes go in several.  Returns o, or (o, lse)."""
    if _rows_native is not None and type(q) is torch.Tensor and q.is_cuda:
        dev = torch._C._cuda_getDevice()
        r = _rows_native.paged_decode(q, k_cache, v_cache, page_table, lengths, seq, workspace, scale, window, max_length, want_lse, dev,
                                      torch._C._cuda_getCurrentRawStream(dev))
        if type(r) is tuple:
            return r if want_lse else r[0]
        if r is not None and r != OSDN_ERR_SHAPE:           # (too many queries are that, too)
            _check(r)
    if not isinstance(q, torch.Tensor) or q.dim() != 3 or not isinstance(k_cache, torch.Tensor) or k_cache.dim() != 4:
        raise TypeError("expected q [B,Hq,K] and a cache [n_pages, page_size, Hk, K] as CUDA/HIP torch tensors")
    B, Hq, K = q.shape
    if max_length is None:
        max_length = min(page_table.shape[1] * k_cache.shape[1], 0x7fffff00)
    most = min(65535, ((1 << 21) - 1) // max(Hq, 1)) or 1
    if B > most:
        if not q.is_cuda:
            raise TypeError("q: expected a CUDA/HIP torch tensor")
        _array(lengths, torch.int32, (B,), "lengths")
        _array(seq, torch.int32, (B,), "seq")
        if seq is None:
            seq = torch.arange(B, dtype=torch.int32, device=q.device)
        most = -(-B // -(-B // most))                       # (as many in each)
    o = q.new_empty(q.shape)
    lse = torch.empty(B, Hq, dtype=torch.float32, device=q.device) if want_lse else None
    of = (lambda t, i: t) if B <= most else (lambda t, i: None if t is None else t[i:i + most])
    for i in range(0, max(B, 1), most):
        p = make_decode_params(min(most, B - i), Hq, k_cache.shape[2], K, q.dtype == torch.bfloat16, max_length, scale, window)
        ws = workspace
        if ws is None:
            n = osdn_paged_decode_workspace_bytes(p)
            ws = torch.empty(n, dtype=torch.uint8, device=q.device) if n else None
        osdn_paged_decode(p, of(q, i), k_cache, v_cache, page_table, of(lengths, i), of(seq, i), of(o, i), of(lse, i), ws)
    return (o, lse) if want_lse else o


# ----------------------------------------------------------------- the pages of a cache ----
def _table_of(page_table):
    """(n_seqs, max_pages, stride) of a page table."""
    if not isinstance(page_table, torch.Tensor) or not page_table.is_cuda or page_table.dtype != torch.int32:
        raise TypeError("page_table: expected an int32 CUDA/HIP torch tensor")
    if page_table.dim() != 2 or (page_table.shape[1] > 1 and page_table.stride(1) != 1):
        raise ValueError("page_table: expected [n_seqs, max_pages] with adjacent entries of a row")
    _here(page_table, "page_table")
    n_seqs, max_pages = page_table.shape
    return n_seqs, max_pages, page_table.stride(0) if n_seqs > 1 else max_pages


def _pages(page_table, page_size, n_pages, free_pages=None):
    n_seqs, max_pages, stride = _table_of(page_table)
    free = _array(free_pages, torch.int32, None, "free_pages")
    capacity = 0 if free_pages is None else free_pages.numel()
    end = lambda x: max(-1, min(2**31 - 1, int(x)))
    return OsdnPages(page_table.data_ptr(), stride, free, end(capacity), end(n_pages), end(page_size), n_seqs, max_pages)


def _requests(t, name):
    if not isinstance(t, torch.Tensor) or t.dim() != 1:
        raise TypeError(f"{name}: expected an int32 CUDA/HIP torch tensor [B]")
    return t.shape[0]


def osdn_paged_plan(pages, B, tokens, cached, fresh, seq, n_free, n_free_out, lengths, starts, positions, rows, slots=None, stream=None):
    i32 = torch.int32
    of = lambda t, n, name: _array(t, i32, (n,), name)
    _check(lib().osdn_paged_plan(
        ctypes.byref(pages), B, tokens, of(cached, B, "cached"), of(fresh, B, "fresh"), of(seq, B, "seq"), of(n_free, 1, "n_free"), of(n_free_out, 1, "n_free_out"),
        of(lengths, B, "lengths"), of(starts, B + 1, "starts"), _array(positions, i32, None, "positions"), _array(rows, i32, None, "rows"),
        _array(slots, torch.int64, (tokens,), "slots"), _stream_ptr(stream)))


def osdn_paged_release(pages, B, lengths, seq, n_free, n_free_out, stream=None):
    of = lambda t, n, name: _array(t, torch.int32, (n,), name)
    _check(lib().osdn_paged_release(ctypes.byref(pages), B, of(lengths, B, "lengths"), of(seq, B, "seq"), of(n_free, 1, "n_free"),
                                    of(n_free_out, 1, "n_free_out"), _stream_ptr(stream)))


def paged_plan(page_table, cached, fresh, free_pages, n_free, page_size: int, tokens: int, seq=None, n_pages=None, want_slots: bool = False):
    """Places for the new tokens of a batch of requests: request b brings fresh[b] tokens to sequence seq[b] (None: b), which has cached[b].  The pages that it
    needs come off the end of free_pages, of which n_free [1] are in the list, into page_table; both are written in place.  tokens: the length of
    the token axis, at least the sum of fresh.  n_pages: of the cache (None: as many as the list has room for).  Returns a dict: lengths [B], starts [B + 1],
    positions and seq [1, tokens] as ``paged_append`` takes them, n_free [1] (for the next call) and, if wanted, slots [tokens] int64.  A request that
    finds no pages is not served, nor is a later one that needs some: its length stays, its tokens have no places, and starts[b + 1] == starts[b]."""
    if _rows_native is not None and type(page_table) is torch.Tensor and page_table.is_cuda:
        dev = torch._C._cuda_getDevice()
        r = _rows_native.paged_plan(page_table, cached, fresh, free_pages, n_free, seq, page_size, tokens, n_pages, want_slots, dev,
                                    torch._C._cuda_getCurrentRawStream(dev))
        if type(r) is tuple:
            return {"lengths": r[0], "starts": r[1], "positions": r[2], "seq": r[3], "n_free": r[4], "slots": r[5]}
        if r is not None:
            _check(r)
    B, N = _requests(cached, "cached"), int(tokens)
    g = _pages(page_table, page_size, free_pages.numel() if n_pages is None and isinstance(free_pages, torch.Tensor) else n_pages or 0, free_pages)
    new = lambda *shape, dtype=torch.int32: torch.empty(*shape, dtype=dtype, device=page_table.device)
    if N < 0 or N > 2**30:
        raise OsdnError(OSDN_ERR_SHAPE)
    r = {"lengths": new(B), "starts": new(B + 1), "positions": new(1, N), "seq": new(1, N), "n_free": new(1),
         "slots": new(N, dtype=torch.int64) if want_slots else None}
    osdn_paged_plan(g, B, N, cached, fresh, seq, n_free, r["n_free"], r["lengths"], r["starts"], r["positions"], r["seq"], r["slots"])
    return r


def paged_release(page_table, lengths, free_pages, n_free, page_size: int, seq=None, n_pages=None):
    """The pages of sequences that end (rows seq of the table, None: the first ones, of these lengths) go back onto the list; in place.  Returns how many
    the list holds then, [1]."""
    if _rows_native is not None and type(page_table) is torch.Tensor and page_table.is_cuda:
        dev = torch._C._cuda_getDevice()
        r = _rows_native.paged_release(page_table, lengths, free_pages, n_free, seq, page_size, n_pages, dev, torch._C._cuda_getCurrentRawStream(dev))
        if r is not None:
            return r[0] if type(r) is tuple else _check(r)
    B = _requests(lengths, "lengths")
    g = _pages(page_table, page_size, free_pages.numel() if n_pages is None and isinstance(free_pages, torch.Tensor) else n_pages or 0, free_pages)
    out = torch.empty(1, dtype=torch.int32, device=page_table.device)
    osdn_paged_release(g, B, lengths, seq, n_free, out)
    return out


# ------------------------------------------------------------------- a cache in 4 bits ----
def alloc_paged_cache_mx(n_pages: int, page_size: int, H: int, K: int, device="cuda"):
    """(k, v, k_scale, v_scale) of a cache in 4 bits: codes [n_pages, page_size, H, K / 2] and scales [n_pages, page_size, H, K / 32], uint8; a page
    holds its tokens head after head (any order of pages, tokens and heads is taken)."""
    new = lambda n: torch.empty(n_pages, H, page_size, n, dtype=torch.uint8, device=device).transpose(1, 2)
    return new(K // 2), new(K // 2), new(K // 32), new(K // 32)


def _cache_mx(cache, page_table, H, K, keys_alone=False):
    """page_table None: one that is not looked at."""
    n = 2 if keys_alone else 4
    if not isinstance(cache, (tuple, list)) or len(cache) != n or not isinstance(cache[0], torch.Tensor) or cache[0].dim() != 4:
        raise TypeError("cache: expected (k, k_scale), codes and scales" if keys_alone else "cache: expected (k, v, k_scale, v_scale), codes [n_pages, page_size, H, K / 2] and "
                        "scales [n_pages, page_size, H, K / 32]")
    n_pages, page_size = cache[0].shape[:2]
    r = [_rows(t, torch.uint8, (n_pages, page_size, H, K // (2 if i < n // 2 else 32)), name)
         for i, (t, name) in enumerate(zip(cache, ("k", "k_scale") if keys_alone else ("k", "v", "k_scale", "v_scale")))]
    if any(x is None for x in r):
        raise TypeError("cache: expected CUDA/HIP torch tensors")
    k, v, ks, vs = (r[0], r[0], r[1], r[1]) if keys_alone else r
    n_seqs, max_pages, stride = (1, 1, 1) if page_table is None else _table_of(page_table)
    steps = [x for y in (k, v, ks, vs) for x in (y.batch, y.token, y.head)]
    return OsdnCacheMx(k.data, v.data, ks.data, vs.data, *steps, None if page_table is None else page_table.data_ptr(), stride, n_pages, page_size, n_seqs, max_pages)


def osdn_paged_append_mx(params, q, k, v, cache, page_table, weight_q, weight_k, rotary, positions, seq, q_out, stream=None):
    p = params
    r = _norm_rows(p, q, k, (v, "v"), (q_out, "q_out"))
    c = _cache_mx(cache, page_table, p.Hk, p.K)
    _check(lib().osdn_paged_append_mx(
        ctypes.byref(p), ctypes.byref(c), *(_ref(x) for x in r[:3]), *_norm_shared(p, weight_q, weight_k, rotary, positions),
        _array(seq, torch.int32, (p.B, p.T), "seq"), _ref(r[3]), _stream_ptr(stream)))


def osdn_paged_read_mx(params, cache, page_table, positions, seq, k_out, v_out, stream=None):
    p, i32 = params, torch.int32
    r = [_rows(t, _io_torch_dtype(p), (p.B, p.T, p.Hk, p.K), name) for t, name in ((k_out, "k_out"), (v_out, "v_out"))]
    c = _cache_mx(cache, page_table, p.Hk, p.K)
    _check(lib().osdn_paged_read_mx(ctypes.byref(p), ctypes.byref(c), _array(positions, i32, (p.B, p.T), "positions"), _array(seq, i32, (p.B, p.T), "seq"),
                                    _ref(r[0]), _ref(r[1]), _stream_ptr(stream)))


def osdn_paged_decode_mx_workspace_bytes(params) -> int:
    return int(lib().osdn_paged_decode_mx_workspace_bytes(ctypes.byref(params)))


def _decode_outputs(p, q, o, lse, workspace):
    io, rows = _io_torch_dtype(p), (p.B, p.Hq, p.K)
    return (_ref(_rows(q, io, rows, "q")), _ref(_rows(o, io, rows, "o")), _array(lse, torch.float32, (p.B, p.Hq), "lse"),
            _array(workspace, torch.uint8, None, "workspace"), ctypes.c_size_t(0 if workspace is None else workspace.numel()))


def osdn_paged_decode_mx(params, q, cache, page_table, lengths, seq, o, lse, workspace=None, stream=None):
    p, i32 = params, torch.int32
    c = _cache_mx(cache, page_table, p.Hk, p.K)
    qr, orows, lp, ws, n = _decode_outputs(p, q, o, lse, workspace)
    _check(lib().osdn_paged_decode_mx(ctypes.byref(p), ctypes.byref(c), qr, _array(lengths, i32, (p.B,), "lengths"), _array(seq, i32, (p.B,), "seq"), orows, lp,
                                      ws, n, _stream_ptr(stream)))


def paged_append_mx(k, v, cache, page_table, positions, seq=None, q=None, weight_q=None, weight_k=None, rotary=None, hp: NormHyper = NormHyper()):
    """``paged_append`` to a cache in 4 bits (``alloc_paged_cache_mx``)."""
    if _rows_native is not None and type(k) is torch.Tensor and k.is_cuda and type(cache) is tuple and len(cache) == 4:
        dev = torch._C._cuda_getDevice()
        r = _rows_native.paged_append_mx(k, v, *cache, page_table, positions, seq, q, weight_q, weight_k, rotary, hp, dev,
                                         torch._C._cuda_getCurrentRawStream(dev))
        if r is not None:
            return r[0] if type(r) is tuple else _check(r)
    p = _params_of(q, k, hp, rotary)
    q_out = None if q is None else q.new_empty(q.shape)
    osdn_paged_append_mx(p, q, k, v, cache, page_table, weight_q, weight_k, rotary, positions, seq, q_out)
    return q_out


def paged_read_mx(cache, page_table, positions, seq=None, dtype=torch.bfloat16):
    """The rows that the tokens at positions [B,T] of their sequences have in a cache in 4 bits, as values: (k, v) [B,T,H,K]."""
    if _rows_native is not None and type(positions) is torch.Tensor and positions.is_cuda and type(cache) is tuple and len(cache) == 4:
        dev = torch._C._cuda_getDevice()
        r = _rows_native.paged_read_mx(*cache, page_table, positions, seq, dtype is torch.bfloat16, dtype is torch.float32, dev,
                                       torch._C._cuda_getCurrentRawStream(dev))
        if r is not None:
            return r if type(r) is tuple else _check(r)
    if dtype not in (torch.bfloat16, torch.float32):
        raise TypeError("dtype: expected torch.bfloat16 or torch.float32")
    if not isinstance(positions, torch.Tensor) or positions.dim() != 2:
        raise TypeError("positions: expected an int32 CUDA/HIP torch tensor [B,T]")
    if not isinstance(cache, (tuple, list)) or len(cache) != 4 or not isinstance(cache[0], torch.Tensor) or cache[0].dim() != 4:
        raise TypeError("cache: expected (k, v, k_scale, v_scale), codes [n_pages, page_size, H, K / 2] and scales [n_pages, page_size, H, K / 32]")
    (B, T), (H, K) = positions.shape, (cache[0].shape[2], 2 * cache[0].shape[3])
    p = OsdnNormParams(B, T, 0, H, K, OSDN_BF16 if dtype == torch.bfloat16 else OSDN_F32, 0, 0, 0, 0, 0.0)
    out = [torch.empty(B, T, H, K, dtype=dtype, device=positions.device) for _ in range(2)]
    osdn_paged_read_mx(p, cache, page_table, positions, seq, *out)
    return tuple(out)


def _decode_in_parts(q, most, bytes_of, call, per_head, workspace, want_lse):
    """Calls of at most `most` queries each; per_head: what goes with a query."""
    B, Hq, _ = q.shape
    most = most if B <= most else -(-B // -(-B // most))
    o = q.new_empty(q.shape)
    lse = torch.empty(B, Hq, dtype=torch.float32, device=q.device) if want_lse else None
    of = (lambda t, i: t) if B <= most else (lambda t, i: None if t is None else t[i:i + most])
    for i in range(0, max(B, 1), most):
        n = min(most, B - i)
        ws = workspace
        if ws is None:
            size = bytes_of(n)
            ws = torch.empty(size, dtype=torch.uint8, device=q.device) if size else None
        call(n, of(q, i), *(of(t, i) for t in per_head), of(o, i), of(lse, i), ws)
    return (o, lse) if want_lse else o


def paged_decode_mx(q, cache, page_table, lengths, seq=None, scale=None, window: int = 0, max_length=None, want_lse: bool = False, workspace=None):
    """``paged_decode`` over a cache in 4 bits.  max_length: no length is above it; the nearer to the longest, the better the call is cut."""
    if _rows_native is not None and type(q) is torch.Tensor and q.is_cuda and type(cache) is tuple and len(cache) == 4:
        dev = torch._C._cuda_getDevice()
        r = _rows_native.paged_decode_mx(q, *cache, page_table, lengths, seq, workspace, scale, window, max_length, want_lse, dev,
                                         torch._C._cuda_getCurrentRawStream(dev))
        if type(r) is tuple:
            return r if want_lse else r[0]
        if r is not None and r != OSDN_ERR_SHAPE:           # (too many queries are that, too)
            _check(r)
    if not isinstance(q, torch.Tensor) or q.dim() != 3 or not isinstance(cache, (tuple, list)) or len(cache) != 4 or not isinstance(cache[0], torch.Tensor) or cache[0].dim() != 4:
        raise TypeError("expected q [B,Hq,K] and a cache (k, v, k_scale, v_scale) as CUDA/HIP torch tensors")
    B, Hq, K = q.shape
    Hk = cache[0].shape[2]
    if max_length is None:
        max_length = min(page_table.shape[1] * cache[0].shape[1], 0x7fffff00)
    most = min(65535, ((1 << 21) - 1) // max(Hq, 1)) or 1
    if B > most:
        if not q.is_cuda:
            raise TypeError("q: expected a CUDA/HIP torch tensor")
        _array(lengths, torch.int32, (B,), "lengths")
        _array(seq, torch.int32, (B,), "seq")
        if seq is None:
            seq = torch.arange(B, dtype=torch.int32, device=q.device)
    params = lambda n: make_decode_params(n, Hq, Hk, K, q.dtype == torch.bfloat16, max_length, scale, window)
    return _decode_in_parts(q, most, lambda n: osdn_paged_decode_mx_workspace_bytes(params(n)),
                            lambda n, q, lengths, seq, o, lse, ws: osdn_paged_decode_mx(params(n), q, cache, page_table, lengths, seq, o, lse, ws), (lengths, seq), workspace, want_lse)


# ------------------------------------------------------- attention over selected pages ----
def alloc_page_bounds(n_pages: int, H: int, K: int, dtype=torch.bfloat16, device="cuda"):
    """Bounds of the keys of every page, [n_pages, H, 2, K]: the smallest, the largest."""
    return torch.empty(n_pages, H, 2, K, dtype=dtype, device=device)


def make_select_params(B, Hq, Hk, K, bf16: bool, max_length: int = 0, max_new: int = 1, pages: int = 2, first: int = 1, last: int = 1) -> OsdnSelectParams:
    end = lambda x: max(-2**31, min(2**31 - 1, int(x)))
    return OsdnSelectParams(B, Hq, Hk, K, OSDN_BF16 if bf16 else OSDN_F32, *(end(x) for x in (max_length, max_new, pages, first, last)))


def osdn_page_bounds(params, keys, page_table, cached, lengths, seq, bounds, stream=None):
    """keys: those of a cache [n_pages, page_size, Hk, K], or (codes, scales) of one in 4 bits (osdn_page_bounds_mx)."""
    p, i32 = params, torch.int32
    more = [_array(t, i32, (p.B,), name) for t, name in ((cached, "cached"), (lengths, "lengths"), (seq, "seq"))]
    if isinstance(keys, (tuple, list)):
        c, call = _cache_mx(keys, page_table, p.Hk, p.K, keys_alone=True), lib().osdn_page_bounds_mx
    else:
        c, call = _cache(keys, keys, page_table, _io_torch_dtype(p), p.Hk, p.K), lib().osdn_page_bounds
    _check(call(ctypes.byref(p), ctypes.byref(c), *more, _array(bounds, _io_torch_dtype(p), (c.n_pages, p.Hk, 2, p.K), "bounds"), _stream_ptr(stream)))


def osdn_page_select_workspace_bytes(params, page_size: int) -> int:
    return int(lib().osdn_page_select_workspace_bytes(ctypes.byref(params), int(page_size)))


def osdn_page_select(params, pages, q, bounds, lengths, seq, chosen, tokens, workspace=None, stream=None):
    p, i32 = params, torch.int32
    io = _io_torch_dtype(p)
    _check(lib().osdn_page_select(
        ctypes.byref(p), ctypes.byref(pages), _ref(_rows(q, io, (p.B, p.Hq, p.K), "q")), _array(bounds, io, (pages.n_pages, p.Hk, 2, p.K), "bounds"),
        _array(lengths, i32, (p.B,), "lengths"), _array(seq, i32, (p.B,), "seq"), _array(chosen, i32, (p.B, p.Hk, p.pages), "chosen"),
        _array(tokens, i32, (p.B, p.Hk), "tokens"), _array(workspace, torch.uint8, None, "workspace"),
        ctypes.c_size_t(0 if workspace is None else workspace.numel()), _stream_ptr(stream)))


def _pages_bytes(params, mx) -> int:
    return int((lib().osdn_paged_decode_pages_mx_workspace_bytes if mx else lib().osdn_paged_decode_pages_workspace_bytes)(ctypes.byref(params)))


def osdn_paged_decode_pages_workspace_bytes(params) -> int:
    return _pages_bytes(params, False)


def osdn_paged_decode_pages_mx_workspace_bytes(params) -> int:
    return _pages_bytes(params, True)


def _chosen(p, chosen, tokens):
    if not isinstance(chosen, torch.Tensor) or chosen.dim() != 3:
        raise TypeError("chosen: expected an int32 CUDA/HIP torch tensor [B,Hk,pages]")
    n = chosen.shape[2]
    return _array(chosen, torch.int32, (p.B, p.Hk, n), "chosen"), n, _array(tokens, torch.int32, (p.B, p.Hk), "tokens")


def osdn_paged_decode_pages(params, q, k_cache, v_cache, chosen, tokens, o, lse, workspace=None, stream=None):
    p = params
    at, n, toks = _chosen(p, chosen, tokens)
    c = _cache(k_cache, v_cache, chosen.flatten(0, 1), _io_torch_dtype(p), p.Hk, p.K)
    qr, orows, lp, ws, size = _decode_outputs(p, q, o, lse, workspace)
    _check(lib().osdn_paged_decode_pages(ctypes.byref(p), ctypes.byref(c), qr, at, n, toks, orows, lp, ws, size, _stream_ptr(stream)))


def osdn_paged_decode_pages_mx(params, q, cache, chosen, tokens, o, lse, workspace=None, stream=None):
    p = params
    at, n, toks = _chosen(p, chosen, tokens)
    c = _cache_mx(cache, None, p.Hk, p.K)
    qr, orows, lp, ws, size = _decode_outputs(p, q, o, lse, workspace)
    _check(lib().osdn_paged_decode_pages_mx(ctypes.byref(p), ctypes.byref(c), qr, at, n, toks, orows, lp, ws, size, _stream_ptr(stream)))


def page_bounds(keys, page_table, cached, lengths, bounds, seq=None, max_new=None):
    """Keep the bounds of the pages up with what was appended: the tokens cached[b] <= i < lengths[b] of sequence seq[b] (None: b).  keys: those of
    a cache [n_pages, page_size, Hk, K], or (codes, scales) of one in 4 bits.  bounds [n_pages, Hk, 2, K] are written in place.
    max_new: no sequence gets more new tokens (None: what a row of the table can hold; the launch is sized by it)."""
    mx = isinstance(keys, (tuple, list))
    k = keys[0] if mx and len(keys) == 2 else keys
    if _rows_native is not None and type(bounds) is torch.Tensor and bounds.is_cuda and (not mx or len(keys) == 2):
        dev = torch._C._cuda_getDevice()
        r = _rows_native.page_bounds(k, keys[1] if mx else None, page_table, cached, lengths, seq, bounds, max_new, dev, torch._C._cuda_getCurrentRawStream(dev))
        if r is not None:
            return None if type(r) is tuple else _check(r)
    if not isinstance(k, torch.Tensor) or k.dim() != 4 or not isinstance(bounds, torch.Tensor) or bounds.dim() != 4:
        raise TypeError("expected keys [n_pages, page_size, Hk, K] and bounds [n_pages, Hk, 2, K] as CUDA/HIP torch tensors")
    if max_new is None:
        max_new = page_table.shape[1] * k.shape[1]
    p = make_select_params(_requests(cached, "cached"), 0, k.shape[2], bounds.shape[3], bounds.dtype == torch.bfloat16, max_new=max_new)
    osdn_page_bounds(p, keys, page_table, cached, lengths, seq, bounds)


def page_select(q, bounds, page_table, lengths, page_size: int, pages: int, seq=None, first: int = 1, last: int = 1, max_length=None, workspace=None):
    """The pages that queries [B,Hq,K] read: of every key head the first, the last and those of the largest bounds of a score, at most `pages`.
    Returns (chosen [B,Hk,pages], tokens [B,Hk]) for ``paged_decode_pages``.  More queries than a launch takes go in several."""
    if _rows_native is not None and type(q) is torch.Tensor and q.is_cuda:
        dev = torch._C._cuda_getDevice()
        r = _rows_native.page_select(q, bounds, page_table, lengths, seq, workspace, page_size, pages, first, last, max_length, dev,
                                     torch._C._cuda_getCurrentRawStream(dev))
        if type(r) is tuple:
            return r
        if r is not None and r != OSDN_ERR_SHAPE:           # (too many queries are that, too)
            _check(r)
    if not isinstance(q, torch.Tensor) or q.dim() != 3 or not isinstance(bounds, torch.Tensor) or bounds.dim() != 4:
        raise TypeError("expected q [B,Hq,K] and bounds [n_pages, Hk, 2, K] as CUDA/HIP torch tensors")
    B, Hq, K = q.shape
    n_pages, Hk = bounds.shape[:2]
    g = _pages(page_table, page_size, n_pages)
    if max_length is None:
        max_length = min(g.max_pages * max(int(page_size), 0), 0x7fffff00)
    of = lambda n: make_select_params(n, Hq, Hk, K, q.dtype == torch.bfloat16, max_length, pages=pages, first=first, last=last)
    p = of(B)
    if p.pages < 1:
        raise OsdnError(-5)
    rows = max(Hk, 1) * max(p.pages, -(-p.max_length // max(g.page_size, 1)))               # pages of a query that are written, or have a score
    most = min(65535, (1 << 21) // max(Hk, 1), (2**31 - 1) // rows) or 1
    if Hk * p.pages > 2**31 - 1:                            # (before they are allocated)
        raise OsdnError(OSDN_ERR_SHAPE)
    if B > most:
        if not q.is_cuda:
            raise TypeError("q: expected a CUDA/HIP torch tensor")
        _array(lengths, torch.int32, (B,), "lengths")
        _array(seq, torch.int32, (B,), "seq")
        if seq is None:
            seq = torch.arange(B, dtype=torch.int32, device=q.device)
        most = -(-B // -(-B // most))
    new = lambda *shape: torch.empty(*shape, dtype=torch.int32, device=q.device)
    chosen, tokens = new(B, Hk, p.pages), new(B, Hk)
    part = (lambda t, i: t) if B <= most else (lambda t, i: None if t is None else t[i:i + most])
    for i in range(0, max(B, 1), most):
        p, ws = of(min(most, B - i)), workspace
        if ws is None:
            n = osdn_page_select_workspace_bytes(p, page_size)
            ws = torch.empty(n, dtype=torch.uint8, device=q.device) if n else None
        osdn_page_select(p, g, part(q, i), bounds, part(lengths, i), part(seq, i), part(chosen, i), part(tokens, i), ws)
    return chosen, tokens


def _decode_pages(q, cache, Hk, page_size, chosen, tokens, scale, max_length, want_lse, workspace, mx):
    B, Hq, K = q.shape
    if not isinstance(chosen, torch.Tensor) or chosen.dim() != 3:
        raise TypeError("chosen: expected an int32 CUDA/HIP torch tensor [B,Hk,pages]")
    if max_length is None:
        max_length = min(chosen.shape[2] * page_size, 0x7fffff00)
    most = min(65535 // max(Hk, 1), ((1 << 21) - 1) // max(Hq, 1)) or 1
    if B > most:
        _array(chosen, torch.int32, (B, Hk, chosen.shape[2]), "chosen")
        _array(tokens, torch.int32, (B, Hk), "tokens")
    params = lambda n: make_decode_params(n, Hq, Hk, K, q.dtype == torch.bfloat16, max_length, scale)
    call = osdn_paged_decode_pages_mx if mx else osdn_paged_decode_pages
    return _decode_in_parts(q, most, lambda n: _pages_bytes(params(n), mx),
                            lambda n, q, chosen, tokens, o, lse, ws: call(params(n), q, *cache, chosen, tokens, o, lse, ws), (chosen, tokens), workspace, want_lse)


def paged_decode_pages(q, k_cache, v_cache, chosen, tokens, scale=None, max_length=None, want_lse: bool = False, workspace=None):
    """Attention of q [B,Hq,K] over chosen pages: those of each key head, chosen [B,Hk,pages], of which the first tokens [B,Hk] tokens are seen
    (``page_select``).  max_length: no entry of tokens is above it (None: what the pages hold).  Returns o, or (o, lse)."""
    if _rows_native is not None and type(q) is torch.Tensor and q.is_cuda:
        dev = torch._C._cuda_getDevice()
        r = _rows_native.paged_decode_pages(q, k_cache, v_cache, None, None, chosen, tokens, workspace, scale, max_length, want_lse, dev,
                                            torch._C._cuda_getCurrentRawStream(dev))
        if type(r) is tuple:
            return r if want_lse else r[0]
        if r is not None and r != OSDN_ERR_SHAPE:
            _check(r)
    if not isinstance(q, torch.Tensor) or q.dim() != 3 or not isinstance(k_cache, torch.Tensor) or k_cache.dim() != 4:
        raise TypeError("expected q [B,Hq,K] and a cache [n_pages, page_size, Hk, K] as CUDA/HIP torch tensors")
    return _decode_pages(q, (k_cache, v_cache), k_cache.shape[2], k_cache.shape[1], chosen, tokens, scale, max_length, want_lse, workspace, False)


def paged_decode_pages_mx(q, cache, chosen, tokens, scale=None, max_length=None, want_lse: bool = False, workspace=None):
    """``paged_decode_pages`` over a cache in 4 bits."""
    if _rows_native is not None and type(q) is torch.Tensor and q.is_cuda and type(cache) is tuple and len(cache) == 4:
        dev = torch._C._cuda_getDevice()
        r = _rows_native.paged_decode_pages(q, *cache, chosen, tokens, workspace, scale, max_length, want_lse, dev, torch._C._cuda_getCurrentRawStream(dev))
        if type(r) is tuple:
            return r if want_lse else r[0]
        if r is not None and r != OSDN_ERR_SHAPE:
            _check(r)
    if not isinstance(q, torch.Tensor) or q.dim() != 3 or not isinstance(cache, (tuple, list)) or len(cache) != 4 or not isinstance(cache[0], torch.Tensor) or cache[0].dim() != 4:
        raise TypeError("expected q [B,Hq,K] and a cache (k, v, k_scale, v_scale) as CUDA/HIP torch tensors")
    return _decode_pages(q, (cache,), cache[0].shape[2], cache[0].shape[1], chosen, tokens, scale, max_length, want_lse, workspace, True)
