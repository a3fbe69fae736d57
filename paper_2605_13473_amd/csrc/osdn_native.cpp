// The ways from Python to osdn_step and to the operators around the recurrence, for calls whose arguments are what they should be.
//
// A decode step of few sequences takes the device 4 us; checking eleven tensors, allocating two and marshalling fifteen
// arguments in Python took 12 (8 chains of 128 x 128, one token: 11.8 us a call, so 6.0; a token appended to a cache 19.4, so 5.9; attention over 1531 cached tokens 20.9, so 10.2).  Anything out of the
// ordinary (a subclass of Tensor, a torch function mode, another device, a wrong type, shape or layout, a value outside its field) is left
// to the Python code, which says what is wrong with it: then this returns None and has done nothing.
#include <Python.h>

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
