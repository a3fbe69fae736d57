// The ways from Python to osdn_step and to the operators around the recurrence, for calls whose arguments are what they should be.
//
// A decode step of few sequences takes the device 4 us; checking eleven tensors, allocating two and marshalling fifteen
// arguments in Python took 12 (8 chains of 128 x 128, one token: 11.8 us a call, so 6.0; a token appended to a cache 19.4, so 5.9; attention over 1531 cached tokens 20.9, so 10.2).  Anything out of the
// ordinary (a subclass of Tensor, a torch function mode, another device, a wrong type, shape or layout, a value outside its field) is left
// to the Python code, which says what is wrong with it: then this returns None and has done nothing.
#include <Python.h>

#include <algorithm>
#include <cfloat>
#include <climits>
#include <cmath>
#include <cstring>

#include <ATen/PythonTorchFunctionTLS.h>
#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/osdn.h"

namespace {

typedef int (*StepFn)(const osdn_params *, const void *, const void *, const void *, const float *, const float *, const float *,
                      const float *, const float *, void *, float *, float *, void *);
StepFn g_step = nullptr;
PyObject *g_names[10];       // interned: the fields of Hyper, in the order of HyperField
enum HyperField { SCALE, ETA, D_MIN, D_MAX, EPS, BETA_AWARE, SEGMENTS, P1_PIECES, P1_PIECE_SWEEPS, P1_SOLVED };
const char *const kNames[10] = {"scale", "eta", "d_min", "d_max", "eps", "beta_aware", "segments", "p1_pieces", "p1_piece_sweeps", "p1_solved"};

// a plain dense tensor of this type and shape on device `dev`
bool plain(const at::Tensor &t, at::ScalarType type, int64_t dev, at::IntArrayRef shape) {
    return t.is_cuda() && t.layout() == at::kStrided && t.has_storage() && t.scalar_type() == type && t.device().index() == dev &&
           t.sizes() == shape && t.is_contiguous();
}
bool as_float(PyObject *hp, int f, float &out) {
    PyObject *o = PyObject_GetAttr(hp, g_names[f]);
    if (!o) { PyErr_Clear(); return false; }
    const bool ok = PyFloat_CheckExact(o);
    const double x = ok ? PyFloat_AS_DOUBLE(o) : 0.0;
    Py_DECREF(o);
    if (!ok || (std::isfinite(x) && std::fabs(x) > FLT_MAX)) return false;
    out = (float)x;
    return true;
}
bool as_int(PyObject *hp, int f, int32_t &out) {
    PyObject *o = PyObject_GetAttr(hp, g_names[f]);
    if (!o) { PyErr_Clear(); return false; }
    int over = 0;
    const bool ok = PyLong_CheckExact(o) || PyBool_Check(o);
    const long x = ok ? PyLong_AsLongAndOverflow(o, &over) : 0;
    Py_DECREF(o);
    if (!ok || over || x < INT_MIN || x > INT_MAX) return false;
    out = (int32_t)x;
    return true;
}

// step(q, k, v, beta, log_alpha, retention, d_in, S_in, hp, in_place, device, stream): (o, S_out, d_out), the status
// of a call that failed, or None
PyObject *step(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    if (!g_step || n != 12 || at::impl::PythonTorchFunctionTLS::stack_len() > 0) Py_RETURN_NONE;
    const at::Tensor *t[8];
    for (int i = 0; i < 8; ++i) {
        t[i] = nullptr;
        if (a[i] == Py_None) {
            if (i < 4) Py_RETURN_NONE;
        } else if (THPVariable_CheckExact(a[i])) {
            t[i] = &THPVariable_Unpack(a[i]);
        } else {
            Py_RETURN_NONE;
        }
    }
    const at::Tensor &q = *t[0], &k = *t[1], &v = *t[2];
    const long dev = PyLong_AsLong(a[10]);
    void *stream = PyLong_AsVoidPtr(a[11]);
    if (PyErr_Occurred()) { PyErr_Clear(); Py_RETURN_NONE; }
    if (!PyBool_Check(a[9]) || k.dim() != 4 || v.dim() != 4) Py_RETURN_NONE;
    const int64_t B = k.size(0), T = k.size(1), H = k.size(2), K = k.size(3), V = v.size(3);
    for (int64_t x : {B, T, H, K, V})
        if (x > INT_MAX) Py_RETURN_NONE;
    const at::ScalarType io = k.scalar_type() == at::kBFloat16 ? at::kBFloat16 : at::kFloat, f32 = at::kFloat;
    const bool gate_vec = t[4] && t[4]->dim() == 4, ret_vec = t[5] && t[5]->dim() == 4;
    const int64_t bthk[] = {B, T, H, K}, bthv[] = {B, T, H, V}, bhvk[] = {B, H, V, K}, bhk[] = {B, H, K};
    const at::IntArrayRef th(bthk, 3), thk(bthk, 4);
    if (!plain(q, io, dev, thk) || !plain(k, io, dev, thk) || !plain(v, io, dev, at::IntArrayRef(bthv, 4)) || !plain(*t[3], f32, dev, th) ||
        (t[4] && !plain(*t[4], f32, dev, gate_vec ? thk : th)) || (t[5] && !plain(*t[5], f32, dev, ret_vec ? thk : th)) ||
        (t[6] && !plain(*t[6], f32, dev, at::IntArrayRef(bhk, 3))) || (t[7] && !plain(*t[7], f32, dev, at::IntArrayRef(bhvk, 4))))
        Py_RETURN_NONE;
    osdn_params p{};
    p.B = (int32_t)B; p.T = (int32_t)T; p.H = (int32_t)H; p.K = (int32_t)K; p.V = (int32_t)V; p.chunk = 64;
    p.io_dtype = io == at::kBFloat16 ? OSDN_BF16 : OSDN_F32;
    PyObject *hp = a[8], *scale = PyObject_GetAttr(hp, g_names[SCALE]);
    if (!scale) { PyErr_Clear(); Py_RETURN_NONE; }
    const bool no_scale = scale == Py_None;
    Py_DECREF(scale);
    if (no_scale) p.scale = (float)std::pow((double)K, -0.5);
    else if (!as_float(hp, SCALE, p.scale)) Py_RETURN_NONE;
    if (!as_float(hp, ETA, p.eta) || !as_float(hp, D_MIN, p.d_min) || !as_float(hp, D_MAX, p.d_max) || !as_float(hp, EPS, p.eps) ||
        !as_int(hp, BETA_AWARE, p.beta_aware) || !as_int(hp, SEGMENTS, p.segments) || !as_int(hp, P1_PIECES, p.p1_pieces) ||
        !as_int(hp, P1_PIECE_SWEEPS, p.p1_piece_sweeps) || !as_int(hp, P1_SOLVED, p.p1_solved))
        Py_RETURN_NONE;
    p.retention_per_channel = ret_vec;
    p.gate_per_channel = gate_vec;

    const at::TensorOptions f32_on = k.options().dtype(f32);
    const bool in_place = a[9] == Py_True && t[7];
    at::Tensor o = at::empty_like(v), d = at::empty(at::IntArrayRef(bhk, 3), f32_on);
    at::Tensor S = in_place ? *t[7] : at::empty(at::IntArrayRef(bhvk, 4), f32_on);
    auto ptr = [](const at::Tensor *x) { return x ? static_cast<const float *>(x->data_ptr()) : nullptr; };
    const void *qp = q.data_ptr(), *kp = k.data_ptr(), *vp = v.data_ptr();
    const float *bp = ptr(t[3]), *gp = ptr(t[4]), *rp = ptr(t[5]), *dp = ptr(t[6]), *sp = ptr(t[7]);
    void *op = o.data_ptr();
    float *So = static_cast<float *>(S.data_ptr()), *d_out = static_cast<float *>(d.data_ptr());
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_step(&p, qp, kp, vp, bp, gp, rp, dp, sp, op, So, d_out, stream);
    Py_END_ALLOW_THREADS
    if (rc != OSDN_OK) return PyLong_FromLong(rc);
    PyObject *out = PyTuple_New(3);
    if (!out) return nullptr;
    PyTuple_SET_ITEM(out, 0, THPVariable_Wrap(o));
    if (in_place) {
        Py_INCREF(a[7]);
        PyTuple_SET_ITEM(out, 1, a[7]);
    } else {
        PyTuple_SET_ITEM(out, 1, THPVariable_Wrap(S));
    }
    PyTuple_SET_ITEM(out, 2, THPVariable_Wrap(d));
    return out;
    END_HANDLE_TH_ERRORS
}

// ---- queries, keys and values around the recurrence ----------------------------------------
typedef decltype(&osdn_qk_norm_fwd) NormFwdFn;
typedef decltype(&osdn_qk_norm_bwd) NormBwdFn;
typedef decltype(&osdn_qk_norm_bwd_workspace_bytes) NormBwdBytesFn;
typedef decltype(&osdn_paged_append) AppendFn;
typedef decltype(&osdn_paged_decode) DecodeFn;
typedef decltype(&osdn_paged_decode_workspace_bytes) DecodeBytesFn;
struct {
    NormFwdFn norm_fwd;
    NormBwdFn norm_bwd;
    NormBwdBytesFn norm_bwd_bytes;
    AppendFn append;
    DecodeFn decode;
    DecodeBytesFn decode_bytes;
} g_rows{};
PyObject *g_norm_names[3];       // interned: the fields of NormHyper
const char *const kNormNames[3] = {"norm", "eps", "interleaved"};

// The arguments a[0 .. n) as tensors, null for None; false: something else among them
bool tensors(PyObject *const *a, int n, const at::Tensor **t) {
    for (int i = 0; i < n; ++i) {
        t[i] = nullptr;
        if (a[i] == Py_None) continue;
        if (!THPVariable_CheckExact(a[i])) return false;
        t[i] = &THPVariable_Unpack(a[i]);
    }
    return true;
}
bool device_and_stream(PyObject *dev, PyObject *stream, long &d, void *&s) {
    d = PyLong_AsLong(dev);
    s = PyLong_AsVoidPtr(stream);
    if (PyErr_Occurred()) { PyErr_Clear(); return false; }
    return true;
}
bool strided(const at::Tensor &t, at::ScalarType type, int64_t dev) {
    return t.is_cuda() && t.layout() == at::kStrided && t.has_storage() && t.scalar_type() == type && t.device().index() == dev;
}
// rows [B,T,H,K] (T < 0: [B,H,K]) wherever they stand; a tensor that is not there: H is 0
bool rows_of(const at::Tensor *t, at::ScalarType io, int64_t dev, int64_t B, int64_t T, int64_t H, int64_t K, osdn_rows &r) {
    if (!t) return H == 0;
    const int64_t want[] = {B, T, H, K}, short_want[] = {B, H, K};
    if (!strided(*t, io, dev) || t->sizes() != (T < 0 ? at::IntArrayRef(short_want, 3) : at::IntArrayRef(want, 4))) return false;
    const at::IntArrayRef st = t->strides();
    if (st.back() != 1) return false;
    r = osdn_rows{t->data_ptr(), st[0], T < 0 ? 0 : st[1], st[st.size() - 2]};
    return true;
}
bool cache_of(const at::Tensor *k, const at::Tensor *v, const at::Tensor *table, at::ScalarType io, int64_t dev, int64_t H, int64_t K, osdn_cache &c) {
    if (!k || !v || !table || k->dim() != 4 || table->dim() != 2 || !strided(*table, at::kInt, dev)) return false;
    osdn_rows kr, vr;
    const int64_t pages = k->size(0), page = k->size(1), seqs = table->size(0), most = table->size(1);
    if (!rows_of(k, io, dev, pages, page, H, K, kr) || !rows_of(v, io, dev, pages, page, H, K, vr) || (most > 1 && table->stride(1) != 1)) return false;
    for (int64_t x : {pages, page, seqs, most})
        if (x > INT_MAX) return false;
    c = osdn_cache{kr.data, vr.data, kr.batch, kr.token, kr.head, vr.batch, vr.token, vr.head, static_cast<const int32_t *>(table->data_ptr()),
                   seqs > 1 ? table->stride(0) : most, (int32_t)pages, (int32_t)page, (int32_t)seqs, (int32_t)most};
    return true;
}
// an array that the library reads as it lies; one that is not there is null
bool array(const at::Tensor *t, at::ScalarType type, int64_t dev, at::IntArrayRef shape, const void **p) {
    *p = nullptr;
    if (!t) return true;
    if (!plain(*t, type, dev, shape)) return false;
    *p = t->data_ptr();
    return true;
}

// What the three operators on rows share: sizes from q and k, NormHyper, weights, table and positions
struct NormCall {
    osdn_norm_params p;
    at::ScalarType io;
    const void *wq, *wk, *rotary, *positions;
    bool take(const at::Tensor *q, const at::Tensor *k, const at::Tensor *weight_q, const at::Tensor *weight_k, const at::Tensor *table, const at::Tensor *pos,
              PyObject *hp, long dev) {
        const at::Tensor *x = q ? q : k;
        if (!x || x->dim() != 4 || (k && k->dim() != 4)) return false;
        io = x->scalar_type() == at::kBFloat16 ? at::kBFloat16 : at::kFloat;
        const int64_t B = x->size(0), T = x->size(1), Hq = q ? q->size(2) : 0, Hk = k ? k->size(2) : 0, K = x->size(3);
        int64_t rows = 0, dim = 0;
        if (table) {
            if (table->dim() != 2) return false;
            rows = table->size(0);
            dim = table->size(1);
            if (dim == 0) return false;
        }
        for (int64_t n : {B, T, Hq, Hk, K, rows, dim})
            if (n > INT_MAX) return false;
        p = osdn_norm_params{(int32_t)B, (int32_t)T, (int32_t)Hq, (int32_t)Hk, (int32_t)K, io == at::kBFloat16 ? OSDN_BF16 : OSDN_F32, 0, (int32_t)dim, (int32_t)rows, 0, 0.f};
        const int64_t k1[] = {K}, tab[] = {rows, dim}, bt[] = {B, T};
        if (!array(weight_q, at::kFloat, dev, at::IntArrayRef(k1, 1), &wq) || !array(weight_k, at::kFloat, dev, at::IntArrayRef(k1, 1), &wk) ||
            !array(table, at::kFloat, dev, at::IntArrayRef(tab, 2), &rotary) || !array(pos, at::kInt, dev, at::IntArrayRef(bt, 2), &positions))
            return false;
        PyObject *o[3] = {};
        bool ok = true;
        for (int i = 0; i < 3 && ok; ++i) ok = (o[i] = PyObject_GetAttr(hp, g_norm_names[i])) != nullptr;
        if (!ok) PyErr_Clear();
        ok = ok && PyUnicode_CheckExact(o[0]) && PyFloat_CheckExact(o[1]) && PyBool_Check(o[2]);
        if (ok) {
            const double eps = PyFloat_AS_DOUBLE(o[1]);
            ok = !std::isfinite(eps) || std::fabs(eps) <= FLT_MAX;
            p.eps = ok ? (float)eps : 0.f;
            p.interleaved = o[2] == Py_True;
            if (PyUnicode_CompareWithASCIIString(o[0], "l2") == 0) p.norm = OSDN_NORM_L2;
            else if (PyUnicode_CompareWithASCIIString(o[0], "rms") == 0) p.norm = OSDN_NORM_RMS;
            else if (PyUnicode_CompareWithASCIIString(o[0], "none") == 0) p.norm = OSDN_NORM_NONE;
            else ok = false;
        }
        for (PyObject *x : o) Py_XDECREF(x);
        return ok;
    }
    const float *fwq() const { return static_cast<const float *>(wq); }
    const float *fwk() const { return static_cast<const float *>(wk); }
    const float *table() const { return static_cast<const float *>(rotary); }
    const int32_t *pos() const { return static_cast<const int32_t *>(positions); }
};
osdn_rows dense(const at::Tensor &t) { return osdn_rows{t.data_ptr(), t.stride(0), t.stride(1), t.stride(2)}; }
PyObject *wrapped(const at::Tensor &t) {
    if (t.defined()) return THPVariable_Wrap(t);
    Py_RETURN_NONE;
}

// qk_norm(q, k, weight_q, weight_k, rotary, positions, hp, device, stream): (q_out, k_out), a status, or None
PyObject *qk_norm(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const at::Tensor *t[6];
    long dev;
    void *stream;
    NormCall c;
    osdn_rows q{}, k{}, qo{}, ko{};
    if (!g_rows.norm_fwd || n != 9 || at::impl::PythonTorchFunctionTLS::stack_len() > 0 || !tensors(a, 6, t) || !device_and_stream(a[7], a[8], dev, stream) ||
        !c.take(t[0], t[1], t[2], t[3], t[4], t[5], a[6], dev) || !rows_of(t[0], c.io, dev, c.p.B, c.p.T, c.p.Hq, c.p.K, q) ||
        !rows_of(t[1], c.io, dev, c.p.B, c.p.T, c.p.Hk, c.p.K, k))
        Py_RETURN_NONE;
    at::Tensor out[2];
    for (int i = 0; i < 2; ++i)
        if (t[i]) {
            out[i] = at::empty(t[i]->sizes(), t[i]->options());
            (i == 0 ? qo : ko) = dense(out[i]);
        }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_rows.norm_fwd(&c.p, &q, &k, c.fwq(), c.fwk(), c.table(), c.pos(), &qo, &ko, stream);
    Py_END_ALLOW_THREADS
    if (rc != OSDN_OK) return PyLong_FromLong(rc);
    return Py_BuildValue("(NN)", wrapped(out[0]), wrapped(out[1]));
    END_HANDLE_TH_ERRORS
}

// qk_norm_backward(q, k, dq_out, dk_out, weight_q, weight_k, rotary, positions, hp, device, stream): (dq, dk, dweight_q, dweight_k), a status, or None
PyObject *qk_norm_backward(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const at::Tensor *t[8];
    long dev;
    void *stream;
    NormCall c;
    osdn_rows r[6] = {};
    if (!g_rows.norm_bwd || n != 11 || at::impl::PythonTorchFunctionTLS::stack_len() > 0 || !tensors(a, 8, t) || !device_and_stream(a[9], a[10], dev, stream) ||
        !c.take(t[0], t[1], t[4], t[5], t[6], t[7], a[8], dev))
        Py_RETURN_NONE;
    for (int i = 0; i < 4; ++i)
        if ((i % 2 ? c.p.Hk : c.p.Hq) > 0 && (!t[i] || !rows_of(t[i], c.io, dev, c.p.B, c.p.T, i % 2 ? c.p.Hk : c.p.Hq, c.p.K, r[i]))) Py_RETURN_NONE;
    at::Tensor out[4], ws;
    for (int i = 0; i < 2; ++i) {
        if (t[i]) {
            out[i] = at::empty(t[i]->sizes(), t[i]->options());
            r[4 + i] = dense(out[i]);
        }
        if (t[4 + i]) out[2 + i] = at::empty(t[4 + i]->sizes(), t[4 + i]->options());
    }
    const size_t bytes = t[4] || t[5] ? g_rows.norm_bwd_bytes(&c.p) : 0;
    if (bytes) ws = at::empty({(int64_t)bytes}, (t[0] ? t[0] : t[1])->options().dtype(at::kByte));
    auto weight = [&](int i) { return out[i].defined() ? static_cast<float *>(out[i].data_ptr()) : nullptr; };
    float *dwq = weight(2), *dwk = weight(3);
    void *scratch = bytes ? ws.data_ptr() : nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_rows.norm_bwd(&c.p, &r[0], &r[1], c.fwq(), c.fwk(), c.table(), c.pos(), &r[2], &r[3], &r[4], &r[5], dwq, dwk, scratch, bytes, stream);
    Py_END_ALLOW_THREADS
    if (rc != OSDN_OK) return PyLong_FromLong(rc);
    return Py_BuildValue("(NNNN)", wrapped(out[0]), wrapped(out[1]), wrapped(out[2]), wrapped(out[3]));
    END_HANDLE_TH_ERRORS
}

// paged_append(k, v, k_cache, v_cache, page_table, positions, seq, q, weight_q, weight_k, rotary, hp, device, stream): (q_out,), a status, or None
PyObject *paged_append(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const at::Tensor *t[11];
    long dev;
    void *stream;
    NormCall c;
    osdn_cache cache;
    osdn_rows q{}, k{}, v{}, qo{};
    const void *seq;
    if (!g_rows.append || n != 14 || at::impl::PythonTorchFunctionTLS::stack_len() > 0 || !tensors(a, 11, t) || !device_and_stream(a[12], a[13], dev, stream) ||
        !t[0] || !c.take(t[7], t[0], t[8], t[9], t[10], t[5], a[11], dev) || !rows_of(t[7], c.io, dev, c.p.B, c.p.T, c.p.Hq, c.p.K, q) ||
        !rows_of(t[0], c.io, dev, c.p.B, c.p.T, c.p.Hk, c.p.K, k) || !rows_of(t[1], c.io, dev, c.p.B, c.p.T, c.p.Hk, c.p.K, v) ||
        !cache_of(t[2], t[3], t[4], c.io, dev, c.p.Hk, c.p.K, cache))
        Py_RETURN_NONE;
    const int64_t bt[] = {c.p.B, c.p.T};
    if (!array(t[6], at::kInt, dev, at::IntArrayRef(bt, 2), &seq)) Py_RETURN_NONE;
    at::Tensor out;
    if (t[7]) {
        out = at::empty(t[7]->sizes(), t[7]->options());
        qo = dense(out);
    }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_rows.append(&c.p, &cache, &q, &k, &v, c.fwq(), c.fwk(), c.table(), c.pos(), static_cast<const int32_t *>(seq), &qo, stream);
    Py_END_ALLOW_THREADS
    if (rc != OSDN_OK) return PyLong_FromLong(rc);
    return Py_BuildValue("(N)", wrapped(out));
    END_HANDLE_TH_ERRORS
}

// paged_decode(q, k_cache, v_cache, page_table, lengths, seq, workspace, scale, window, max_length, want_lse, device, stream): (o, lse or None), a status,
// or None
PyObject *paged_decode(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const at::Tensor *t[7];
    long dev;
    void *stream;
    if (!g_rows.decode || n != 13 || at::impl::PythonTorchFunctionTLS::stack_len() > 0 || !tensors(a, 7, t) || !device_and_stream(a[11], a[12], dev, stream) ||
        !t[0] || !t[1] || !t[4] || t[0]->dim() != 3 || t[1]->dim() != 4 || !PyBool_Check(a[10]) || !PyLong_CheckExact(a[8]) ||
        (a[9] != Py_None && !PyLong_CheckExact(a[9])) || (a[7] != Py_None && !PyFloat_CheckExact(a[7])))
        Py_RETURN_NONE;
    const int64_t B = t[0]->size(0), Hq = t[0]->size(1), K = t[0]->size(2), Hk = t[1]->size(2);
    const at::ScalarType io = t[0]->scalar_type() == at::kBFloat16 ? at::kBFloat16 : at::kFloat;
    osdn_rows q, o;
    osdn_cache cache;
    const void *lengths, *seq;
    if (!rows_of(t[0], io, dev, B, -1, Hq, K, q) || !cache_of(t[1], t[2], t[3], io, dev, Hk, K, cache) || !array(t[4], at::kInt, dev, at::IntArrayRef(&B, 1), &lengths) ||
        !array(t[5], at::kInt, dev, at::IntArrayRef(&B, 1), &seq))
        Py_RETURN_NONE;
    int over = 0, over2 = 0;
    const long window = PyLong_AsLongAndOverflow(a[8], &over);
    const int64_t capacity = (int64_t)cache.max_pages * cache.page_size;
    const long longest = a[9] == Py_None ? (capacity < 0x7fffff00 ? capacity : 0x7fffff00) : PyLong_AsLongAndOverflow(a[9], &over2);
    const double scale = a[7] == Py_None ? std::pow((double)K, -0.5) : PyFloat_AS_DOUBLE(a[7]);
    if (over || over2 || std::fabs(scale) > FLT_MAX) Py_RETURN_NONE;
    for (int64_t x : {B, Hq, K, Hk, (int64_t)window, (int64_t)longest})
        if (x > INT_MAX || x < INT_MIN) Py_RETURN_NONE;
    osdn_decode_params p{(int32_t)B, (int32_t)Hq, (int32_t)Hk, (int32_t)K, io == at::kBFloat16 ? OSDN_BF16 : OSDN_F32, (int32_t)window, (int32_t)longest, 0, (float)scale};
    at::Tensor ws, lse, out = at::empty(t[0]->sizes(), t[0]->options());
    size_t bytes = g_rows.decode_bytes(&p);
    void *scratch = nullptr;
    if (t[6]) {
        if (!plain(*t[6], at::kByte, dev, t[6]->sizes())) Py_RETURN_NONE;
        bytes = (size_t)t[6]->numel();
        scratch = t[6]->data_ptr();
    } else if (bytes) {
        ws = at::empty({(int64_t)bytes}, t[0]->options().dtype(at::kByte));
        scratch = ws.data_ptr();
    }
    if (a[10] == Py_True) lse = at::empty({B, Hq}, t[0]->options().dtype(at::kFloat));
    o = osdn_rows{out.data_ptr(), out.stride(0), 0, out.stride(1)};
    float *l = lse.defined() ? static_cast<float *>(lse.data_ptr()) : nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_rows.decode(&p, &cache, &q, static_cast<const int32_t *>(lengths), static_cast<const int32_t *>(seq), &o, l, scratch, bytes, stream);
    Py_END_ALLOW_THREADS
    if (rc != OSDN_OK) return PyLong_FromLong(rc);
    return Py_BuildValue("(NN)", wrapped(out), wrapped(lse));
    END_HANDLE_TH_ERRORS
}

// ---- the pages of a cache, the cache in 4 bits, attention over selected pages ----------------
struct {
    decltype(&osdn_paged_plan) plan;
    decltype(&osdn_paged_release) release;
    decltype(&osdn_paged_append_mx) append;
    decltype(&osdn_paged_read_mx) read;
    decltype(&osdn_paged_decode_mx) decode;
    decltype(&osdn_paged_decode_mx_workspace_bytes) decode_bytes;
    decltype(&osdn_page_bounds) bounds;
    decltype(&osdn_page_bounds_mx) bounds_mx;
    decltype(&osdn_page_select) select;
    decltype(&osdn_page_select_workspace_bytes) select_bytes;
    decltype(&osdn_paged_decode_pages) decode_pages;
    decltype(&osdn_paged_decode_pages_workspace_bytes) decode_pages_bytes;
    decltype(&osdn_paged_decode_pages_mx) decode_pages_mx;
    decltype(&osdn_paged_decode_pages_mx_workspace_bytes) decode_pages_mx_bytes;
} g_pages{};
constexpr int PAGES_ENTRIES = 14;
bool ordinary() { return g_pages.plan && at::impl::PythonTorchFunctionTLS::stack_len() == 0; }

// an int that its field holds
bool int_of(PyObject *o, int32_t &out) {
    if (!PyLong_CheckExact(o)) return false;
    int over = 0;
    const long x = PyLong_AsLongAndOverflow(o, &over);
    if (over || x < INT_MIN || x > INT_MAX) return false;
    out = (int32_t)x;
    return true;
}
// ... or None, for which another value stands
bool int_or(PyObject *o, int64_t other, int32_t &out) {
    if (o != Py_None) return int_of(o, out);
    if (other > INT_MAX) return false;
    out = (int32_t)other;
    return true;
}
bool table_of(const at::Tensor *t, int64_t dev, int64_t &seqs, int64_t &most, int64_t &stride) {
    if (!t || t->dim() != 2 || !strided(*t, at::kInt, dev) || (t->size(1) > 1 && t->stride(1) != 1)) return false;
    seqs = t->size(0);
    most = t->size(1);
    stride = seqs > 1 ? t->stride(0) : most;
    return seqs <= INT_MAX && most <= INT_MAX;
}
bool int_array(const at::Tensor *t, int64_t dev, at::IntArrayRef shape, const int32_t **p, bool needed = true) {
    const void *at = nullptr;
    if ((needed && !t) || !array(t, at::kInt, dev, shape, &at)) return false;
    *p = static_cast<const int32_t *>(at);
    return true;
}
int32_t *ints(const at::Tensor &t) { return static_cast<int32_t *>(t.data_ptr()); }
PyObject *tuple_of(std::initializer_list<at::Tensor> ts) {
    PyObject *out = PyTuple_New((Py_ssize_t)ts.size());
    if (!out) return nullptr;
    Py_ssize_t i = 0;
    for (const at::Tensor &t : ts) PyTuple_SET_ITEM(out, i++, wrapped(t));
    return out;
}
// A part of a buffer's memory as a tensor of its own, contiguous (several outputs in one allocation: each of its own costs a microsecond)
at::Tensor piece(const at::Tensor &buffer, at::ScalarType type, int64_t byte, at::IntArrayRef sizes) {
    const caffe2::TypeMeta meta = c10::scalarTypeToTypeMeta(type);
    at::Tensor t = at::detail::make_tensor<c10::TensorImpl>(c10::Storage(buffer.storage()), buffer.key_set(), meta);
    t.unsafeGetTensorImpl()->set_storage_offset(byte / (int64_t)meta.itemsize());
    t.unsafeGetTensorImpl()->set_sizes_contiguous(sizes);
    return t;
}
bool pages_of(const at::Tensor *table, const at::Tensor *free_pages, PyObject *page_size, PyObject *n_pages, int64_t dev, osdn_pages &g) {
    int64_t seqs, most, stride;
    const int32_t *list;
    if (!table_of(table, dev, seqs, most, stride) || !free_pages || free_pages->dim() != 1 || !int_array(free_pages, dev, free_pages->sizes(), &list)) return false;
    g = osdn_pages{static_cast<int32_t *>(table->data_ptr()), stride, const_cast<int32_t *>(list), 0, 0, 0, (int32_t)seqs, (int32_t)most};
    if (free_pages->numel() > INT_MAX) return false;
    g.free_capacity = (int32_t)free_pages->numel();
    return int_of(page_size, g.page_size) && int_or(n_pages, free_pages->numel(), g.n_pages);
}

// paged_plan(page_table, cached, fresh, free_pages, n_free, seq, page_size, tokens, n_pages, want_slots, device, stream): (lengths, starts, positions, rows, n_free,
// slots or None), a status, or None
PyObject *paged_plan(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const at::Tensor *t[6];
    long dev;
    void *stream;
    osdn_pages g;
    int32_t tokens;
    const int32_t *cached, *fresh, *seq, *n_free;
    if (n != 12 || !ordinary() || !tensors(a, 6, t) || !device_and_stream(a[10], a[11], dev, stream) || !t[1] || t[1]->dim() != 1 || !PyBool_Check(a[9]) ||
        !int_of(a[7], tokens) || tokens < 1 || tokens > 1 << 30 || !pages_of(t[0], t[3], a[6], a[8], dev, g))
        Py_RETURN_NONE;
    const int64_t B = t[1]->size(0), one = 1;
    const at::IntArrayRef b(&B, 1);
    if (B < 1 || B > 65535 || !int_array(t[1], dev, b, &cached) || !int_array(t[2], dev, b, &fresh) || !int_array(t[5], dev, b, &seq, false) ||
        !int_array(t[4], dev, at::IntArrayRef(&one, 1), &n_free))
        Py_RETURN_NONE;
    const int64_t N = tokens, line[] = {1, N}, b1 = B + 1, slot_bytes = a[9] == Py_True ? 8 * N : 0;
    // One allocation for all, but where there are many tokens: what a server keeps of a step (lengths, starts, n_free) then does not hold their places, too
    const int64_t of_tokens = slot_bytes + 8 * N, of_requests = 4 * (2 * B + 2);
    const bool apart = of_tokens > 1 << 16;
    const at::TensorOptions bytes = t[0]->options().dtype(at::kByte);
    const at::Tensor places = at::empty({of_tokens + (apart ? 0 : of_requests)}, bytes), kept = apart ? at::empty({of_requests}, bytes) : places;
    const auto take = [&](int64_t at, at::IntArrayRef sizes) { return piece(places, at::kInt, slot_bytes + 4 * at, sizes); };
    const auto keep = [&](int64_t at, at::IntArrayRef sizes) { return piece(kept, at::kInt, (apart ? 0 : of_tokens) + 4 * at, sizes); };
    const at::Tensor pos = take(0, at::IntArrayRef(line, 2)), rows = take(N, at::IntArrayRef(line, 2)), lengths = keep(0, b), starts = keep(B, at::IntArrayRef(&b1, 1));
    const at::Tensor left = keep(2 * B + 1, at::IntArrayRef(&one, 1));
    at::Tensor slots;
    if (slot_bytes) slots = piece(places, at::kLong, 0, at::IntArrayRef(&N, 1));
    int32_t *l = ints(lengths), *s = ints(starts), *p = ints(pos), *r = ints(rows), *f = ints(left);
    int64_t *sl = slots.defined() ? static_cast<int64_t *>(slots.data_ptr()) : nullptr;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_pages.plan(&g, (int32_t)B, tokens, cached, fresh, seq, n_free, f, l, s, p, r, sl, stream);
    Py_END_ALLOW_THREADS
    if (rc != OSDN_OK) return PyLong_FromLong(rc);
    return tuple_of({lengths, starts, pos, rows, left, slots});
    END_HANDLE_TH_ERRORS
}

// paged_release(page_table, lengths, free_pages, n_free, seq, page_size, n_pages, device, stream): (n_free,), a status, or None
PyObject *paged_release(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const at::Tensor *t[5];
    long dev;
    void *stream;
    osdn_pages g;
    const int32_t *lengths, *seq, *n_free;
    if (n != 9 || !ordinary() || !tensors(a, 5, t) || !device_and_stream(a[7], a[8], dev, stream) || !t[1] || t[1]->dim() != 1 || !pages_of(t[0], t[2], a[5], a[6], dev, g))
        Py_RETURN_NONE;
    const int64_t B = t[1]->size(0), one = 1;
    const at::IntArrayRef b(&B, 1);
    if (B < 1 || B > 65535 || !int_array(t[1], dev, b, &lengths) || !int_array(t[4], dev, b, &seq, false) || !int_array(t[3], dev, at::IntArrayRef(&one, 1), &n_free)) Py_RETURN_NONE;
    at::Tensor left = at::empty({1}, t[0]->options());
    int32_t *f = ints(left);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_pages.release(&g, (int32_t)B, lengths, seq, n_free, f, stream);
    Py_END_ALLOW_THREADS
    if (rc != OSDN_OK) return PyLong_FromLong(rc);
    return tuple_of({left});
    END_HANDLE_TH_ERRORS
}

// a cache in 4 bits: codes [pages, page, H, K / 2] and scales [.., K / 32] of keys and values (values null: the keys alone; table null: one that is not looked at)
bool cache_mx_of(const at::Tensor *k, const at::Tensor *v, const at::Tensor *ks, const at::Tensor *vs, const at::Tensor *table, int64_t dev, int64_t H, int64_t K, osdn_cache_mx &c) {
    if (!k || k->dim() != 4) return false;
    osdn_rows r[4];
    const int64_t pages = k->size(0), page = k->size(1);
    const at::Tensor *t[4] = {k, v, ks, vs};
    if (!ks || pages > INT_MAX || page > INT_MAX || H < 1) return false;
    for (int i = 0; i < 4; ++i)
        if (t[i] && !rows_of(t[i], at::kByte, dev, pages, page, H, i < 2 ? K / 2 : K / 32, r[i])) return false;
    if (!v || !vs) {
        if (v || vs) return false;
        r[1] = r[0];
        r[3] = r[2];
    }
    int64_t seqs = 1, most = 1, stride = 1;
    if (table && !table_of(table, dev, seqs, most, stride)) return false;
    c = osdn_cache_mx{r[0].data, r[1].data, static_cast<uint8_t *>(r[2].data), static_cast<uint8_t *>(r[3].data), r[0].batch, r[0].token, r[0].head, r[1].batch, r[1].token, r[1].head,
                      r[2].batch, r[2].token, r[2].head, r[3].batch, r[3].token, r[3].head, table ? static_cast<const int32_t *>(table->data_ptr()) : nullptr, stride,
                      (int32_t)pages, (int32_t)page, (int32_t)seqs, (int32_t)most};
    return true;
}

// paged_append_mx(k, v, codes of k, of v, scales of k, of v, page_table, positions, seq, q, weight_q, weight_k, rotary, hp, device, stream): (q_out,), a status, or None
PyObject *paged_append_mx(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const at::Tensor *t[13];
    long dev;
    void *stream;
    NormCall c;
    osdn_cache_mx cache;
    osdn_rows q{}, k{}, v{}, qo{};
    const int32_t *seq;
    if (n != 16 || !ordinary() || !tensors(a, 13, t) || !device_and_stream(a[14], a[15], dev, stream) || !t[0] || !c.take(t[9], t[0], t[10], t[11], t[12], t[7], a[13], dev) ||
        !rows_of(t[9], c.io, dev, c.p.B, c.p.T, c.p.Hq, c.p.K, q) || !rows_of(t[0], c.io, dev, c.p.B, c.p.T, c.p.Hk, c.p.K, k) ||
        !rows_of(t[1], c.io, dev, c.p.B, c.p.T, c.p.Hk, c.p.K, v) || !t[3] || !t[5] || !t[6] || !cache_mx_of(t[2], t[3], t[4], t[5], t[6], dev, c.p.Hk, c.p.K, cache))
        Py_RETURN_NONE;
    const int64_t bt[] = {c.p.B, c.p.T};
    if (!int_array(t[8], dev, at::IntArrayRef(bt, 2), &seq, false)) Py_RETURN_NONE;
    at::Tensor out;
    if (t[9]) {
        out = at::empty(t[9]->sizes(), t[9]->options());
        qo = dense(out);
    }
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_pages.append(&c.p, &cache, &q, &k, &v, c.fwq(), c.fwk(), c.table(), c.pos(), seq, &qo, stream);
    Py_END_ALLOW_THREADS
    if (rc != OSDN_OK) return PyLong_FromLong(rc);
    return tuple_of({out});
    END_HANDLE_TH_ERRORS
}

// paged_read_mx(codes of k, of v, scales of k, of v, page_table, positions, seq, bf16, f32, device, stream): (k, v), a status, or None
PyObject *paged_read_mx(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const at::Tensor *t[7];
    long dev;
    void *stream;
    osdn_cache_mx cache;
    const int32_t *pos, *seq;
    if (n != 11 || !ordinary() || !tensors(a, 7, t) || !device_and_stream(a[9], a[10], dev, stream) || !t[0] || t[0]->dim() != 4 || !t[1] || !t[3] || !t[4] || !t[5] || t[5]->dim() != 2 ||
        (a[7] != Py_True && a[8] != Py_True))
        Py_RETURN_NONE;
    const int64_t B = t[5]->size(0), T = t[5]->size(1), H = t[0]->size(2), K = 2 * t[0]->size(3);
    for (int64_t x : {B, T, H, K})
        if (x > INT_MAX) Py_RETURN_NONE;
    if (!cache_mx_of(t[0], t[1], t[2], t[3], t[4], dev, H, K, cache) || !int_array(t[5], dev, t[5]->sizes(), &pos) || !int_array(t[6], dev, t[5]->sizes(), &seq, false)) Py_RETURN_NONE;
    osdn_norm_params p{(int32_t)B, (int32_t)T, 0, (int32_t)H, (int32_t)K, a[7] == Py_True ? OSDN_BF16 : OSDN_F32, 0, 0, 0, 0, 0.f};
    const at::TensorOptions io = t[0]->options().dtype(a[7] == Py_True ? at::kBFloat16 : at::kFloat);
    const int64_t half = B * T * H * K, sizes[] = {B, T, H, K};
    at::Tensor k, v;
    if (half <= 1 << 17) {
        const at::Tensor both = at::empty({2 * half}, io);
        k = piece(both, both.scalar_type(), 0, at::IntArrayRef(sizes, 4));
        v = piece(both, both.scalar_type(), half * (int64_t)both.itemsize(), at::IntArrayRef(sizes, 4));
    } else {
        k = at::empty(at::IntArrayRef(sizes, 4), io);
        v = at::empty(at::IntArrayRef(sizes, 4), io);
    }
    osdn_rows ko = dense(k), vo = dense(v);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_pages.read(&p, &cache, pos, seq, &ko, &vo, stream);
    Py_END_ALLOW_THREADS
    if (rc != OSDN_OK) return PyLong_FromLong(rc);
    return tuple_of({k, v});
    END_HANDLE_TH_ERRORS
}

// What the calls of attention share: sizes, scale, window (null: none) and the outputs
struct DecodeCall {
    osdn_decode_params p;
    osdn_rows q, o;
    at::Tensor out, lse, ws;
    void *scratch = nullptr;
    bool take(const at::Tensor *query, int64_t Hk, PyObject *scale, PyObject *window, PyObject *longest, int64_t capacity, PyObject *want_lse, int64_t dev) {
        if (!query || query->dim() != 3 || !PyBool_Check(want_lse) || (scale != Py_None && !PyFloat_CheckExact(scale))) return false;
        const int64_t B = query->size(0), Hq = query->size(1), K = query->size(2);
        for (int64_t x : {B, Hq, Hk, K})
            if (x > INT_MAX) return false;
        const at::ScalarType io = query->scalar_type() == at::kBFloat16 ? at::kBFloat16 : at::kFloat;
        const double s = scale == Py_None ? std::pow((double)K, -0.5) : PyFloat_AS_DOUBLE(scale);
        p = osdn_decode_params{(int32_t)B, (int32_t)Hq, (int32_t)Hk, (int32_t)K, io == at::kBFloat16 ? OSDN_BF16 : OSDN_F32, 0, 0, 0, (float)s};
        return !(std::fabs(s) > FLT_MAX) && (!window || int_of(window, p.window)) && int_or(longest, capacity < 0x7fffff00 ? capacity : 0x7fffff00, p.max_length) &&
               rows_of(query, io, dev, B, -1, Hq, K, q);
    }
    bool outputs(const at::Tensor &query, const at::Tensor *workspace, size_t &bytes, bool want_lse, int64_t dev) {
        if (workspace) {
            if (!plain(*workspace, at::kByte, dev, workspace->sizes())) return false;
            bytes = (size_t)workspace->numel();
            scratch = workspace->data_ptr();
        } else if (bytes) {
            ws = at::empty({(int64_t)bytes}, query.options().dtype(at::kByte));
            scratch = ws.data_ptr();
        }
        out = at::empty(query.sizes(), query.options());
        if (want_lse) lse = at::empty({p.B, p.Hq}, query.options().dtype(at::kFloat));
        o = osdn_rows{out.data_ptr(), out.stride(0), 0, out.stride(1)};
        return true;
    }
    float *l() const { return lse.defined() ? static_cast<float *>(lse.data_ptr()) : nullptr; }
};

// paged_decode_mx(q, codes of k, of v, scales of k, of v, page_table, lengths, seq, workspace, scale, window, max_length, want_lse, device, stream): (o, lse or None),
// a status, or None
PyObject *paged_decode_mx(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const at::Tensor *t[9];
    long dev;
    void *stream;
    osdn_cache_mx cache;
    DecodeCall d;
    const int32_t *lengths, *seq;
    if (n != 15 || !ordinary() || !tensors(a, 9, t) || !device_and_stream(a[13], a[14], dev, stream) || !t[0] || t[0]->dim() != 3 || !t[1] || t[1]->dim() != 4 || !t[2] || !t[4] || !t[5])
        Py_RETURN_NONE;
    const int64_t B = t[0]->size(0), Hk = t[1]->size(2);
    if (!cache_mx_of(t[1], t[2], t[3], t[4], t[5], dev, Hk, t[0]->size(2), cache) ||
        !d.take(t[0], Hk, a[9], a[10], a[11], (int64_t)cache.max_pages * cache.page_size, a[12], dev) || !int_array(t[6], dev, at::IntArrayRef(&B, 1), &lengths) ||
        !int_array(t[7], dev, at::IntArrayRef(&B, 1), &seq, false))
        Py_RETURN_NONE;
    size_t bytes = g_pages.decode_bytes(&d.p);
    if (!d.outputs(*t[0], t[8], bytes, a[12] == Py_True, dev)) Py_RETURN_NONE;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_pages.decode(&d.p, &cache, &d.q, lengths, seq, &d.o, d.l(), d.scratch, bytes, stream);
    Py_END_ALLOW_THREADS
    if (rc != OSDN_OK) return PyLong_FromLong(rc);
    return tuple_of({d.out, d.lse});
    END_HANDLE_TH_ERRORS
}

// paged_decode_pages(q, k, v, scales of k, of v (both None: rows of q's type), chosen, tokens, workspace, scale, max_length, want_lse, device, stream): (o, lse or
// None), a status, or None
PyObject *paged_decode_pages(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const at::Tensor *t[8];
    long dev;
    void *stream;
    DecodeCall d;
    if (n != 13 || !ordinary() || !tensors(a, 8, t) || !device_and_stream(a[11], a[12], dev, stream) || !t[0] || t[0]->dim() != 3 || !t[1] || t[1]->dim() != 4 || !t[2] || !t[5] ||
        t[5]->dim() != 3)
        Py_RETURN_NONE;
    const bool mx = t[3] && t[4];
    const int64_t B = t[0]->size(0), Hk = t[1]->size(2), N = t[5]->size(2), bhn[] = {B, Hk, N};
    const int32_t *chosen, *tokens;
    if ((!mx && (t[3] || t[4])) || N > INT_MAX || !int_array(t[5], dev, at::IntArrayRef(bhn, 3), &chosen) || !int_array(t[6], dev, at::IntArrayRef(bhn, 2), &tokens) ||
        !d.take(t[0], Hk, a[8], nullptr, a[9], N * t[1]->size(1), a[10], dev))
        Py_RETURN_NONE;
    osdn_cache cache;
    osdn_cache_mx cache_mx;
    if (mx) {
        if (!cache_mx_of(t[1], t[2], t[3], t[4], nullptr, dev, Hk, d.p.K, cache_mx)) Py_RETURN_NONE;
    } else {
        const at::ScalarType io = d.p.io_dtype == OSDN_BF16 ? at::kBFloat16 : at::kFloat;
        const int64_t pages = t[1]->size(0), page = t[1]->size(1);
        osdn_rows k, v;
        if (pages > INT_MAX || page > INT_MAX || !rows_of(t[1], io, dev, pages, page, Hk, d.p.K, k) || !rows_of(t[2], io, dev, pages, page, Hk, d.p.K, v)) Py_RETURN_NONE;
        cache = osdn_cache{k.data, v.data, k.batch, k.token, k.head, v.batch, v.token, v.head, chosen, N, (int32_t)pages, (int32_t)page, 1, (int32_t)N};
    }
    size_t bytes = mx ? g_pages.decode_pages_mx_bytes(&d.p) : g_pages.decode_pages_bytes(&d.p);
    if (!d.outputs(*t[0], t[7], bytes, a[10] == Py_True, dev)) Py_RETURN_NONE;
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = mx ? g_pages.decode_pages_mx(&d.p, &cache_mx, &d.q, chosen, (int32_t)N, tokens, &d.o, d.l(), d.scratch, bytes, stream)
            : g_pages.decode_pages(&d.p, &cache, &d.q, chosen, (int32_t)N, tokens, &d.o, d.l(), d.scratch, bytes, stream);
    Py_END_ALLOW_THREADS
    if (rc != OSDN_OK) return PyLong_FromLong(rc);
    return tuple_of({d.out, d.lse});
    END_HANDLE_TH_ERRORS
}

// page_bounds(keys, their scales or None, page_table, cached, lengths, seq, bounds, max_new, device, stream): (), a status, or None
PyObject *page_bounds(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const at::Tensor *t[7];
    long dev;
    void *stream;
    const int32_t *cached, *lengths, *seq;
    const void *bounds;
    if (n != 10 || !ordinary() || !tensors(a, 7, t) || !device_and_stream(a[8], a[9], dev, stream) || !t[0] || t[0]->dim() != 4 || !t[2] || !t[3] || t[3]->dim() != 1 || !t[6] ||
        t[6]->dim() != 4)
        Py_RETURN_NONE;
    const int64_t B = t[3]->size(0), Hk = t[0]->size(2), K = t[6]->size(3), shape[] = {t[0]->size(0), Hk, 2, K};
    const at::ScalarType io = t[6]->scalar_type() == at::kBFloat16 ? at::kBFloat16 : at::kFloat;
    osdn_cache cache;
    osdn_cache_mx cache_mx;
    osdn_select_params p{};
    if (B > INT_MAX || Hk > INT_MAX || K > INT_MAX || !array(t[6], io, dev, at::IntArrayRef(shape, 4), &bounds) || !int_array(t[3], dev, at::IntArrayRef(&B, 1), &cached) ||
        !int_array(t[4], dev, at::IntArrayRef(&B, 1), &lengths) || !int_array(t[5], dev, at::IntArrayRef(&B, 1), &seq, false))
        Py_RETURN_NONE;
    if (t[1] ? !cache_mx_of(t[0], nullptr, t[1], nullptr, t[2], dev, Hk, K, cache_mx) : !cache_of(t[0], t[0], t[2], io, dev, Hk, K, cache)) Py_RETURN_NONE;
    p.B = (int32_t)B; p.Hk = (int32_t)Hk; p.K = (int32_t)K; p.io_dtype = io == at::kBFloat16 ? OSDN_BF16 : OSDN_F32;
    if (!int_or(a[7], t[2]->size(1) * t[0]->size(1), p.max_new)) Py_RETURN_NONE;
    void *to = const_cast<void *>(bounds);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = t[1] ? g_pages.bounds_mx(&p, &cache_mx, cached, lengths, seq, to, stream) : g_pages.bounds(&p, &cache, cached, lengths, seq, to, stream);
    Py_END_ALLOW_THREADS
    if (rc != OSDN_OK) return PyLong_FromLong(rc);
    return PyTuple_New(0);
    END_HANDLE_TH_ERRORS
}

// page_select(q, bounds, page_table, lengths, seq, workspace, page_size, pages, first, last, max_length, device, stream): (chosen, tokens), a status, or None
PyObject *page_select(PyObject *, PyObject *const *a, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    const at::Tensor *t[6];
    long dev;
    void *stream;
    const int32_t *lengths, *seq;
    const void *bounds;
    osdn_rows q;
    osdn_pages g{};
    osdn_select_params p{};
    int64_t seqs, most, stride;
    if (n != 13 || !ordinary() || !tensors(a, 6, t) || !device_and_stream(a[11], a[12], dev, stream) || !t[0] || t[0]->dim() != 3 || !t[1] || t[1]->dim() != 4 ||
        !table_of(t[2], dev, seqs, most, stride) || !int_of(a[6], g.page_size) || !int_of(a[7], p.pages) || !int_of(a[8], p.first) || !int_of(a[9], p.last) ||
        !int_or(a[10], std::min<int64_t>(most * std::max(g.page_size, 0), 0x7fffff00), p.max_length))
        Py_RETURN_NONE;
    const int64_t B = t[0]->size(0), Hq = t[0]->size(1), K = t[0]->size(2), pages = t[1]->size(0), Hk = t[1]->size(1), shape[] = {pages, Hk, 2, K};
    const at::ScalarType io = t[0]->scalar_type() == at::kBFloat16 ? at::kBFloat16 : at::kFloat;
    for (int64_t x : {B, Hq, Hk, K, pages})
        if (x > INT_MAX) Py_RETURN_NONE;
    if (p.pages < 1 || !rows_of(t[0], io, dev, B, -1, Hq, K, q) || !array(t[1], io, dev, at::IntArrayRef(shape, 4), &bounds) || !int_array(t[3], dev, at::IntArrayRef(&B, 1), &lengths) ||
        !int_array(t[4], dev, at::IntArrayRef(&B, 1), &seq, false))
        Py_RETURN_NONE;
    g.table = static_cast<int32_t *>(t[2]->data_ptr()); g.table_stride = stride; g.n_pages = (int32_t)pages; g.n_seqs = (int32_t)seqs; g.max_pages = (int32_t)most;
    p.B = (int32_t)B; p.Hq = (int32_t)Hq; p.Hk = (int32_t)Hk; p.K = (int32_t)K; p.io_dtype = io == at::kBFloat16 ? OSDN_BF16 : OSDN_F32;
    size_t bytes = g_pages.select_bytes(&p, g.page_size);
    at::Tensor ws;
    void *scratch = nullptr;
    if (t[5]) {
        if (!plain(*t[5], at::kByte, dev, t[5]->sizes())) Py_RETURN_NONE;
        bytes = (size_t)t[5]->numel();
        scratch = t[5]->data_ptr();
    } else if (bytes) {
        ws = at::empty({(int64_t)bytes}, t[0]->options().dtype(at::kByte));
        scratch = ws.data_ptr();
    }
    if (B * Hk > (1 << 21) || B * Hk * p.pages > INT_MAX) Py_RETURN_NONE;
    const int64_t bhn[] = {B, Hk, p.pages};
    const at::Tensor both = at::empty({B * Hk * (p.pages + 1)}, t[2]->options());
    const at::Tensor chosen = piece(both, at::kInt, 0, at::IntArrayRef(bhn, 3)), tokens = piece(both, at::kInt, 4 * B * Hk * (int64_t)p.pages, at::IntArrayRef(bhn, 2));
    int32_t *c = ints(chosen), *k = ints(tokens);
    int rc;
    Py_BEGIN_ALLOW_THREADS
    rc = g_pages.select(&p, &g, &q, bounds, lengths, seq, c, k, scratch, bytes, stream);
    Py_END_ALLOW_THREADS
    if (rc != OSDN_OK) return PyLong_FromLong(rc);
    return tuple_of({chosen, tokens});
    END_HANDLE_TH_ERRORS
}

// bind_pages(the addresses in the order of g_pages, as a tuple, sizes of the three structs): refused where the structs are not those this was built for
PyObject *bind_pages(PyObject *, PyObject *args) {
    PyObject *at;
    Py_ssize_t size[3];
    if (!PyArg_ParseTuple(args, "O!nnn", &PyTuple_Type, &at, &size[0], &size[1], &size[2])) return nullptr;
    const size_t want[] = {sizeof(osdn_pages), sizeof(osdn_cache_mx), sizeof(osdn_select_params)};
    for (int i = 0; i < 3; ++i)
        if ((size_t)size[i] != want[i]) return PyErr_Format(PyExc_ImportError, "built for a struct of %zd bytes, not %zd", (Py_ssize_t)want[i], size[i]);
    if (PyTuple_GET_SIZE(at) != PAGES_ENTRIES) return PyErr_Format(PyExc_TypeError, "expected %d addresses", PAGES_ENTRIES);
    void *p[PAGES_ENTRIES];
    for (int i = 0; i < PAGES_ENTRIES; ++i) {
        p[i] = PyLong_AsVoidPtr(PyTuple_GET_ITEM(at, i));
        if (PyErr_Occurred()) return nullptr;
    }
    static_assert(sizeof(g_pages) == sizeof(p), "one address for each");
    std::memcpy(&g_pages, p, sizeof(p));
    Py_RETURN_NONE;
}

// bind_rows(the six addresses in the order of g_rows, sizes of their four structs): refused where the structs are not those this was built for
PyObject *bind_rows(PyObject *, PyObject *args) {
    PyObject *at[6];
    Py_ssize_t size[4];
    if (!PyArg_ParseTuple(args, "OOOOOOnnnn", &at[0], &at[1], &at[2], &at[3], &at[4], &at[5], &size[0], &size[1], &size[2], &size[3])) return nullptr;
    const size_t want[] = {sizeof(osdn_rows), sizeof(osdn_norm_params), sizeof(osdn_cache), sizeof(osdn_decode_params)};
    for (int i = 0; i < 4; ++i)
        if ((size_t)size[i] != want[i]) return PyErr_Format(PyExc_ImportError, "built for a struct of %zd bytes, not %zd", (Py_ssize_t)want[i], size[i]);
    void *p[6];
    for (int i = 0; i < 6; ++i) {
        p[i] = PyLong_AsVoidPtr(at[i]);
        if (PyErr_Occurred()) return nullptr;
    }
    g_rows = {reinterpret_cast<NormFwdFn>(p[0]), reinterpret_cast<NormBwdFn>(p[1]), reinterpret_cast<NormBwdBytesFn>(p[2]), reinterpret_cast<AppendFn>(p[3]),
              reinterpret_cast<DecodeFn>(p[4]), reinterpret_cast<DecodeBytesFn>(p[5])};
    Py_RETURN_NONE;
}

// bind(address, size, version): where osdn_step is.  Refused where its struct or the tensor library are not those this was built for.
PyObject *bind(PyObject *, PyObject *args) {
    PyObject *addr;
    Py_ssize_t size;
    const char *version;
    if (!PyArg_ParseTuple(args, "Ons", &addr, &size, &version)) return nullptr;
    void *p = PyLong_AsVoidPtr(addr);
    if (PyErr_Occurred()) return nullptr;
    if (size != (Py_ssize_t)sizeof(osdn_params))
        return PyErr_Format(PyExc_ImportError, "built for an osdn_params of %zd bytes, not %zd", (Py_ssize_t)sizeof(osdn_params), size);
    if (std::strcmp(version, OSDN_TORCH_VERSION) != 0)
        return PyErr_Format(PyExc_ImportError, "built for torch " OSDN_TORCH_VERSION ", not %s", version);
    g_step = reinterpret_cast<StepFn>(p);
    Py_RETURN_NONE;
}

PyMethodDef kMethods[] = {
    {"step", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(step)), METH_FASTCALL, "osdn_step on plain tensors, or None"},
    {"qk_norm", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(qk_norm)), METH_FASTCALL, "osdn_qk_norm_fwd on tensors, or None"},
    {"qk_norm_backward", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(qk_norm_backward)), METH_FASTCALL, "osdn_qk_norm_bwd on tensors, or None"},
    {"paged_append", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_append)), METH_FASTCALL, "osdn_paged_append on tensors, or None"},
    {"paged_decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_decode)), METH_FASTCALL, "osdn_paged_decode on tensors, or None"},
    {"paged_plan", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_plan)), METH_FASTCALL, "osdn_paged_plan on tensors, or None"},
    {"paged_release", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_release)), METH_FASTCALL, "osdn_paged_release on tensors, or None"},
    {"paged_append_mx", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_append_mx)), METH_FASTCALL, "osdn_paged_append_mx on tensors, or None"},
    {"paged_read_mx", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_read_mx)), METH_FASTCALL, "osdn_paged_read_mx on tensors, or None"},
    {"paged_decode_mx", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_decode_mx)), METH_FASTCALL, "osdn_paged_decode_mx on tensors, or None"},
    {"paged_decode_pages", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(paged_decode_pages)), METH_FASTCALL, "osdn_paged_decode_pages(_mx) on tensors, or None"},
    {"page_bounds", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(page_bounds)), METH_FASTCALL, "osdn_page_bounds(_mx) on tensors, or None"},
    {"page_select", reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(page_select)), METH_FASTCALL, "osdn_page_select on tensors, or None"},
    {"bind_pages", bind_pages, METH_VARARGS, "addresses of the entry points of pages and the cache in 4 bits, sizes of their structs"},
    {"bind_rows", bind_rows, METH_VARARGS, "addresses of the entry points around the recurrence, sizes of their structs"},
    {"bind", bind, METH_VARARGS, "address of osdn_step, size of osdn_params, version of the tensor library"},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef kModule = {PyModuleDef_HEAD_INIT, "_native", nullptr, -1, kMethods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__native(void) {
    for (int i = 0; i < 10; ++i) {
        g_names[i] = PyUnicode_InternFromString(kNames[i]);
        if (!g_names[i]) return nullptr;
    }
    for (int i = 0; i < 3; ++i) {
        g_norm_names[i] = PyUnicode_InternFromString(kNormNames[i]);
        if (!g_norm_names[i]) return nullptr;
    }
    return PyModule_Create(&kModule);
}
