// Python extension module: the hot path of binding.py's wrappers in native code.
//
// A wrapper in Python spends 5-10 us on attribute lookups, torch.empty and ctypes conversions before the library
// is called -- more than a small kernel takes.  The functions here do the same checks and allocations on the C++ tensors
// and call the C ABI of libsage.so through the addresses that init() is given (one copy of the library, the
// one binding.load() opened).  They handle the calls that are in order: anything else (a wrong type or shape, an argument
// that is not a plain number) returns None, and the Python wrapper then takes its own path, which raises the error.
// Return values: the outputs; an int, the status of a call that the library refused; or None.
// The interpreter lock is released around the library calls, as ctypes does.
#include <Python.h>
#include <ATen/core/Tensor.h>
#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <torch/csrc/autograd/python_variable.h>
#include <cmath>
#include <cstring>

#include "../../include/sage.h"

#ifndef SAGE_NATIVE_HASH
#define SAGE_NATIVE_HASH "unknown"
#endif

namespace {

const char tagged_hash[] = "SAGE_NATIVE_HASH=" SAGE_NATIVE_HASH;

struct Api {
    decltype(&sage_quant_q) quant_q;
    decltype(&sage_rope_quant_q) rope_quant_q;
    decltype(&sage_smooth_quant_k_workspace) k_workspace;
    decltype(&sage_smooth_quant_k) smooth_quant_k;
    decltype(&sage_rope_smooth_quant_k) rope_smooth_quant_k;
    decltype(&sage_quant_qk) quant_qk;
    decltype(&sage_quant_v_workspace) v_workspace;
    decltype(&sage_quant_v) quant_v;
    decltype(&sage_attn_split_workspace) split_workspace;
    decltype(&sage_attn_cross_fwd) attn_cross;
    decltype(&sage_attn_cross_split_fwd) attn_split;
    decltype(&sage_attn_pv_int8_cross_fwd) pv8_cross;
    decltype(&sage_attn_pv_int8_cross_split_fwd) pv8_split;
    decltype(&sage_attention_workspace) attention_workspace;
    decltype(&sage_attention_fwd) attention;
    decltype(&sage_rope) rope;
    decltype(&sage_rope_bwd) rope_bwd;
    decltype(&sage_cache4_block_bytes) cache4_block_bytes;
    decltype(&sage_cache4_append) cache4_append;
    decltype(&sage_cache4_load) cache4_load;
    decltype(&sage_cache4_attn_workspace) cache4_attn_workspace;
    decltype(&sage_cache4_attn) cache4_attn;
    decltype(&sage_cache4_weights) cache4_weights;
    decltype(&sage_cache4_evict) cache4_evict;
} api;
PyObject *get_device, *get_stream;          // torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream

constexpr auto F16 = at::kHalf, F32 = at::kFloat, I8 = at::kChar, U8 = at::kByte;

const at::Tensor* tensor(PyObject* o) { return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr; }
bool on_device(const at::Tensor& t) { return t.is_cuda() && t.is_contiguous(); }

// Arguments of one call, read in order; ok turns false where one is not what the fast path handles.
struct Args {
    PyObject* const* a;
    bool ok = true, elsewhere = false;       // elsewhere: a stream was named that is not the current one
    explicit Args(PyObject* const* args) : a(args) {}
    // a contiguous device tensor of this type
    const at::Tensor* in(at::ScalarType type, int dims) {
        const at::Tensor* t = tensor(*a++);
        ok = ok && t && on_device(*t) && t->scalar_type() == type && (dims == 0 || t->dim() == dims);
        return t;
    }
    // the same or None
    PyObject* given(at::ScalarType type) {
        PyObject* o = *a++;
        if (o == Py_None) return nullptr;
        const at::Tensor* t = tensor(o);
        ok = ok && t && on_device(*t) && t->scalar_type() == type;
        return o;
    }
    // any device tensor or None (scratch of unstated type)
    PyObject* scratch() {
        PyObject* o = *a++;
        if (o == Py_None) return nullptr;
        const at::Tensor* t = tensor(o);
        ok = ok && t && on_device(*t);
        return o;
    }
    int integer() {
        PyObject* o = *a++;
        if (!PyLong_Check(o)) { ok = false; return 0; }        // (a bool is an int here too)
        int overflow = 0;
        const long v = PyLong_AsLongAndOverflow(o, &overflow);
        ok = ok && !overflow && v >= -0x7fffffffL && v <= 0x7fffffffL;
        return (int)v;
    }
    float real() {
        PyObject* o = *a++;
        if (!PyFloat_Check(o)) { ok = false; return 0.0f; }
        return (float)PyFloat_AS_DOUBLE(o);
    }
    // the current stream's handle, or null and false where it cannot be told
    static bool current(void*& p) {
        PyObject* dev = PyObject_CallNoArgs(get_device);
        PyObject* s = dev ? PyObject_CallOneArg(get_stream, dev) : nullptr;
        Py_XDECREF(dev);
        p = s ? PyLong_AsVoidPtr(s) : nullptr;
        Py_XDECREF(s);
        const bool told = !PyErr_Occurred();
        PyErr_Clear();
        return told;
    }
    void* stream() {
        PyObject* o = *a++;
        if (!ok) return nullptr;
        void *p = nullptr, *now = nullptr;
        if (o == Py_None) {
            ok = current(p);
            return p;
        }
        p = PyLong_Check(o) ? PyLong_AsVoidPtr(o) : nullptr;
        if (!PyLong_Check(o) || PyErr_Occurred()) { PyErr_Clear(); ok = false; }
        elsewhere = ok && current(now) && p != now;
        return p;
    }
    // Memory allocated here is the current stream's: a call on another one is taken only with every buffer given.
    bool take(bool all_given) const { return ok && (all_given || !elsewhere); }
};

// An output or scratch tensor: the caller's, or a new one on the device of `like`.
struct Buffer {
    at::Tensor own;
    const at::Tensor* t = nullptr;
    PyObject* from = nullptr;
    void take(PyObject* given, const at::Tensor& like, at::IntArrayRef sizes, at::ScalarType type) {
        from = given;
        if (given) { t = &THPVariable_Unpack(given); return; }
        own = at::empty(sizes, at::TensorOptions().device(like.device()).dtype(type));
        t = &own;
    }
    void bytes(PyObject* given, const at::Tensor& like, size_t need) {
        if (given || need > 0) take(given, like, {(int64_t)need}, U8);
    }
    void* p() const { return t ? t->data_ptr() : nullptr; }
    size_t size() const { return t ? (size_t)t->nbytes() : 0; }
    PyObject* out() const { return from ? (Py_INCREF(from), from) : THPVariable_Wrap(own); }
};

PyObject* none() { Py_RETURN_NONE; }
template <class F> int call(F&& f) {
    int st;
    Py_BEGIN_ALLOW_THREADS
    st = f();
    Py_END_ALLOW_THREADS
    return st;
}
// What the interpreter calls.  No C++ exception may pass through it: what throws here -- an allocation that fails, the
// sizes of a tensor that has none in numbers (symbolic, nested) -- the Python path meets again and reports.
using Entry = PyObject* (*)(PyObject* const*, Py_ssize_t);
template <Entry F> PyObject* guarded(PyObject*, PyObject* const* argv, Py_ssize_t n) {
    try {
        return F(argv, n);
    } catch (const std::exception&) {
        PyErr_Clear();
        return none();
    }
}
PyObject* result(int st, std::initializer_list<const Buffer*> outs) {
    if (st != 0) return PyLong_FromLong(st);
    if (outs.size() == 1) return (*outs.begin())->out();
    PyObject* t = PyTuple_New((Py_ssize_t)outs.size());
    Py_ssize_t i = 0;
    for (const Buffer* b : outs) PyTuple_SET_ITEM(t, i++, b->out());
    return t;
}
int64_t blocks(int64_t n, int block) { return block > 0 ? (n + block - 1) / block : 0; }
bool fits(const at::Tensor& t) {
    for (int i = 0; i < 4; ++i)
        if (t.size(i) > 0x7fffffff) return false;
    return true;
}

// (q, cos, sin, sm_scale, block_q, q_i8 | None, q_scale | None, stream | None); the tables both None unless ROPE: the call is
// named by its entry, so that a missing table does not turn it into the other one
template <bool ROPE> PyObject* py_quant_q(PyObject* const* argv, Py_ssize_t n) {
    if (n != 8) return none();
    Args a(argv);
    const at::Tensor* q = a.in(F16, 4);
    PyObject *cs = a.given(F32), *sn = a.given(F32);
    const float sm = a.real();
    const int block = a.integer();
    PyObject *gi = a.given(I8), *gs = a.given(F32);
    void* st = a.stream();
    if (!a.take(gi && gs) || block < 1 || !fits(*q) || ROPE != (cs != nullptr) || ROPE != (sn != nullptr)) return none();
    const int64_t B = q->size(0), H = q->size(1), N = q->size(2), D = q->size(3);
    const at::Tensor *c = cs ? tensor(cs) : nullptr, *s = sn ? tensor(sn) : nullptr;
    if (c && (c->dim() != 2 || c->size(0) != N || c->size(1) != D / 2 || s->dim() != 2 || s->size(0) != N || s->size(1) != D / 2)) return none();
    Buffer i8, sc;
    i8.take(gi, *q, {B, H, N, D}, I8);
    sc.take(gs, *q, {B, H, blocks(N, block)}, F32);
    void *pq = q->data_ptr(), *pi = i8.p(), *ps = sc.p();
    const void *pc = c ? c->data_ptr() : nullptr, *pn = s ? s->data_ptr() : nullptr;
    const int e = call([&] {
        return ROPE ? api.rope_quant_q(pq, (const float*)pc, (const float*)pn, (int8_t*)pi, (float*)ps, B, H, N, D, sm, block, st)
                    : api.quant_q(pq, (int8_t*)pi, (float*)ps, B, H, N, D, sm, block, st);
    });
    return result(e, {&i8, &sc});
}

// (k, cos, sin, block_k, k_i8 | None, k_scale | None, k_mean | None, workspace | None, stream | None); tables as above
template <bool ROPE> PyObject* py_smooth_quant_k(PyObject* const* argv, Py_ssize_t n) {
    if (n != 9) return none();
    Args a(argv);
    const at::Tensor* k = a.in(F16, 4);
    PyObject *cs = a.given(F32), *sn = a.given(F32);
    const int block = a.integer();
    PyObject *gi = a.given(I8), *gs = a.given(F32), *gm = a.given(F32), *gw = a.scratch();
    void* st = a.stream();
    if (!a.take(gi && gs && gm && gw) || block < 1 || !fits(*k) || ROPE != (cs != nullptr) || ROPE != (sn != nullptr)) return none();
    const int64_t B = k->size(0), H = k->size(1), N = k->size(2), D = k->size(3);
    const at::Tensor *c = cs ? tensor(cs) : nullptr, *s = sn ? tensor(sn) : nullptr;
    if (c && (c->dim() != 2 || c->size(0) != N || c->size(1) != D / 2 || s->dim() != 2 || s->size(0) != N || s->size(1) != D / 2)) return none();
    Buffer i8, sc, mean, ws;
    i8.take(gi, *k, {B, H, N, D}, I8);
    sc.take(gs, *k, {B, H, blocks(N, block)}, F32);
    mean.take(gm, *k, {B, H, D}, F32);
    ws.bytes(gw, *k, api.k_workspace(B, H, N, D));
    void *pk = k->data_ptr(), *pi = i8.p(), *ps = sc.p(), *pm = mean.p(), *pw = ws.p();
    const void *pc = c ? c->data_ptr() : nullptr, *pn = s ? s->data_ptr() : nullptr;
    const size_t wb = ws.size();
    const int e = call([&] {
        return ROPE ? api.rope_smooth_quant_k(pk, (const float*)pc, (const float*)pn, (int8_t*)pi, (float*)ps, (float*)pm, pw, wb, B, H, N, D, block, st)
                    : api.smooth_quant_k(pk, (int8_t*)pi, (float*)ps, (float*)pm, pw, wb, B, H, N, D, block, st);
    });
    return result(e, {&i8, &sc, &mean});
}

// (q, k, sm_scale, block_q, block_k, q_i8, q_scale, k_i8, k_scale, k_mean, workspace, stream), the last seven | None
PyObject* py_quant_qk(PyObject* const* argv, Py_ssize_t n) {
    if (n != 12) return none();
    Args a(argv);
    const at::Tensor *q = a.in(F16, 4), *k = a.in(F16, 4);
    const float sm = a.real();
    const int bq = a.integer(), bk = a.integer();
    PyObject *gqi = a.given(I8), *gqs = a.given(F32), *gki = a.given(I8), *gks = a.given(F32), *gm = a.given(F32), *gw = a.scratch();
    void* st = a.stream();
    if (!a.take(gqi && gqs && gki && gks && gm && gw) || bq < 1 || bk < 1 || !fits(*q) || !fits(*k)) return none();
    const int64_t B = q->size(0), H = q->size(1), Nq = q->size(2), D = q->size(3), Nkv = k->size(2);
    if (k->size(0) != B || k->size(1) != H || k->size(3) != D) return none();
    Buffer qi, qs, ki, ks, mean, ws;
    qi.take(gqi, *q, {B, H, Nq, D}, I8);
    qs.take(gqs, *q, {B, H, blocks(Nq, bq)}, F32);
    ki.take(gki, *q, {B, H, Nkv, D}, I8);
    ks.take(gks, *q, {B, H, blocks(Nkv, bk)}, F32);
    mean.take(gm, *q, {B, H, D}, F32);
    ws.bytes(gw, *q, api.k_workspace(B, H, Nkv, D));
    void *pq = q->data_ptr(), *pk = k->data_ptr(), *p0 = qi.p(), *p1 = qs.p(), *p2 = ki.p(), *p3 = ks.p(), *p4 = mean.p(), *pw = ws.p();
    const size_t wb = ws.size();
    const int e = call([&] {
        return api.quant_qk(pq, pk, (int8_t*)p0, (float*)p1, (int8_t*)p2, (float*)p3, (float*)p4, pw, wb, B, H, Nq, Nkv, D, sm, bq, bk, st);
    });
    return result(e, {&qi, &qs, &ki, &ks, &mean});
}

// (v, v_i8t | None, v_scale | None, workspace | None, stream | None)
PyObject* py_quant_v(PyObject* const* argv, Py_ssize_t n) {
    if (n != 5) return none();
    Args a(argv);
    const at::Tensor* v = a.in(F16, 4);
    PyObject *gi = a.given(I8), *gs = a.given(F32), *gw = a.scratch();
    void* st = a.stream();
    if (!a.take(gi && gs && gw) || !fits(*v)) return none();
    const int64_t B = v->size(0), H = v->size(1), N = v->size(2), D = v->size(3), Np = blocks(N, 64) * 64;
    if (gi) {
        const at::Tensor& t = *tensor(gi);
        if (t.dim() != 4 || t.size(0) != B || t.size(1) != H || t.size(2) != D || t.size(3) != Np) return none();
    }
    Buffer i8, sc, ws;
    i8.take(gi, *v, {B, H, D, Np}, I8);
    sc.take(gs, *v, {B, H, D}, F32);
    ws.bytes(gw, *v, api.v_workspace(B, H, N, D));
    void *pv = v->data_ptr(), *pi = i8.p(), *ps = sc.p(), *pw = ws.p();
    const size_t wb = ws.size();
    return result(call([&] { return api.quant_v(pv, (int8_t*)pi, (float*)ps, pw, wb, B, H, N, D, st); }), {&i8, &sc});
}

// (kind, q_i8, q_scale, k_i8, k_scale, v, v_scale, causal, sm_scale, block_q, block_k, n_splits, out | None, workspace | None,
// stream | None); PV8: v the INT8 codes, with their scales, else v fp16 and v_scale None; kind: 0 equal lengths, 1 any lengths,
// 2 keys split
template <bool PV8> PyObject* py_attn(PyObject* const* argv, Py_ssize_t n) {
    if (n != 15) return none();
    Args a(argv);
    const int kind = a.integer();
    const at::Tensor *qi = a.in(I8, 4), *qs = a.in(F32, 0), *ki = a.in(I8, 4), *ks = a.in(F32, 0), *v = a.in(PV8 ? I8 : F16, 4);
    PyObject* gvs = a.given(F32);
    const int causal = a.integer();
    const float sm = a.real();
    const int bq = a.integer(), bk = a.integer(), splits = a.integer();
    PyObject *go = a.given(F16), *gw = a.given(U8);
    void* st = a.stream();
    if (!a.take(go && (gw || kind != 2)) || PV8 != (gvs != nullptr) || !fits(*qi) || !fits(*ki) || !fits(*v)) return none();
    const int64_t B = ki->size(0), H = ki->size(1), Nkv = ki->size(2), D = ki->size(3), Nq = qi->size(2);
    if (qi->size(0) != B || qi->size(1) != H || qi->size(3) != D || v->size(0) != B || v->size(1) != H) return none();
    if (kind == 0 && Nq != Nkv) return none();
    if (PV8 ? v->size(2) != D || v->size(3) != blocks(Nkv, 64) * 64 : v->size(2) != Nkv || v->size(3) != D) return none();
    Buffer o, ws;
    o.take(go, *v, {B, H, Nq, D}, F16);
    if (kind == 2) ws.bytes(gw, *v, api.split_workspace(B, H, Nq, Nkv, D, causal != 0, splits));
    void *p0 = qi->data_ptr(), *p1 = qs->data_ptr(), *p2 = ki->data_ptr(), *p3 = ks->data_ptr(), *p4 = v->data_ptr(), *po = o.p(), *pw = ws.p();
    void* pvs = gvs ? tensor(gvs)->data_ptr() : nullptr;
    const size_t wb = ws.size();
    const int c = causal != 0;
    const int e = call([&] {
        const int8_t *q8 = (const int8_t*)p0, *k8 = (const int8_t*)p2, *v8 = (const int8_t*)p4;
        const float *qsc = (const float*)p1, *ksc = (const float*)p3, *vsc = (const float*)pvs;
        if (PV8)
            return kind != 2 ? api.pv8_cross(q8, qsc, k8, ksc, v8, vsc, po, B, H, Nq, Nkv, D, c, sm, bq, bk, st)
                              : api.pv8_split(q8, qsc, k8, ksc, v8, vsc, po, pw, wb, B, H, Nq, Nkv, D, c, sm, bq, bk, splits, st);
        return kind != 2 ? api.attn_cross(q8, qsc, k8, ksc, p4, po, B, H, Nq, Nkv, D, c, sm, bq, bk, st)
                          : api.attn_split(q8, qsc, k8, ksc, p4, po, pw, wb, B, H, Nq, Nkv, D, c, sm, bq, bk, splits, st);
    });
    return result(e, {&o});
}

// (q, k, v, causal, sm_scale, block_q, block_k, pv_int8, out | None, workspace | None, stream | None)
PyObject* py_attention(PyObject* const* argv, Py_ssize_t n) {
    if (n != 11) return none();
    Args a(argv);
    const at::Tensor *q = a.in(F16, 4), *k = a.in(F16, 4), *v = a.in(F16, 4);
    const int causal = a.integer();
    const float sm = a.real();
    const int bq = a.integer(), bk = a.integer(), pv8 = a.integer();
    PyObject *go = a.given(F16), *gw = a.given(U8);
    void* st = a.stream();
    if (!a.take(go && gw) || !fits(*q) || !fits(*k) || v->sizes() != k->sizes()) return none();
    const int64_t B = q->size(0), H = q->size(1), Nq = q->size(2), D = q->size(3), Nkv = k->size(2);
    if (k->size(0) != B || k->size(1) != H || k->size(3) != D) return none();
    if (go && tensor(go)->sizes() != q->sizes()) return none();
    Buffer o, ws;
    o.take(go, *q, {B, H, Nq, D}, F16);
    ws.bytes(gw, *q, api.attention_workspace(B, H, Nq, Nkv, D, causal != 0, bq, bk, pv8 != 0));
    void *pq = q->data_ptr(), *pk = k->data_ptr(), *pv = v->data_ptr(), *po = o.p(), *pw = ws.p();
    const size_t wb = ws.size();
    return result(call([&] { return api.attention(pq, pk, pv, po, pw, wb, B, H, Nq, Nkv, D, causal != 0, sm, bq, bk, pv8 != 0, st); }), {&o});
}

// ---- the serving calls (serving.py): tensors on the current device; the rows of [B, H, N, D] ones lie anywhere
constexpr auto BF16 = at::kBFloat16, I32 = at::kInt, F64 = at::kDouble;

struct ServingArgs : Args {
    int device = -1;
    explicit ServingArgs(PyObject* const* args) : Args(args) {
        PyObject* d = PyObject_CallNoArgs(get_device);
        device = d ? (int)PyLong_AsLong(d) : -1;
        Py_XDECREF(d);
        if (PyErr_Occurred()) { PyErr_Clear(); ok = false; }
    }
    bool here(const at::Tensor& t) const { return t.is_cuda() && t.get_device() == device; }
    // [B, H, N, D] with neighbouring channels, of a type of these calls
    const at::Tensor* rows(bool fp32 = false) {
        const at::Tensor* t = tensor(*a++);
        ok = ok && t && here(*t) && t->dim() == 4 && (t->scalar_type() == F16 || t->scalar_type() == BF16 || (fp32 && t->scalar_type() == F32)) &&
             (t->stride(3) == 1 || t->size(3) == 1) && fits(*t);
        return ok ? t : nullptr;
    }
    const at::Tensor* rows_or_none(bool fp32 = false) { return *a == Py_None ? (++a, nullptr) : rows(fp32); }
    // contiguous, of this type and these sizes (-1: any); null where None is allowed and given
    const at::Tensor* flat(at::ScalarType type, std::initializer_list<int64_t> sizes, bool optional = false) {
        PyObject* o = *a++;
        if (optional && o == Py_None) return nullptr;
        const at::Tensor* t = tensor(o);
        ok = ok && t && here(*t) && t->scalar_type() == type && t->dim() == (int64_t)sizes.size() && t->is_contiguous();
        if (!ok) return nullptr;
        int i = 0;
        for (int64_t n : sizes) {
            const int64_t m = t->size(i++);
            ok = ok && (n < 0 || n == m) && m <= 0x7fffffff;
        }
        return ok ? t : nullptr;
    }
    float real_or(float otherwise) {
        if (*a == Py_None) return ++a, otherwise;
        return real();
    }
};
struct RowsOf {                 // pointer and strides of a rows() tensor, as the library takes them
    void* p = nullptr;
    int64_t s[3] = {0, 0, 0};
    const int64_t* strides = nullptr;
    RowsOf() = default;
    explicit RowsOf(const at::Tensor* t) {
        if (!t) return;
        p = t->data_ptr();
        if (t->is_contiguous()) return;
        for (int i = 0; i < 3; ++i) s[i] = t->stride(i);
        strides = s;
    }
};
const void* at_or_null(const at::Tensor* t) { return t ? t->data_ptr() : nullptr; }
int type_of(const at::Tensor& t) { return t.scalar_type() == F16 ? SAGE_F16 : t.scalar_type() == BF16 ? SAGE_BF16 : SAGE_F32; }
// an output: the caller's, or a new tensor laid out as `like` is
struct LikeBuffer : Buffer {
    bool take_like(const at::Tensor* given, PyObject* object, const at::Tensor& like) {
        if (given) {
            from = object;
            t = given;
            return given->scalar_type() == like.scalar_type() && given->sizes() == like.sizes();
        }
        own = at::empty_like(like);
        t = &own;
        return true;
    }
};
// A pool and the table of its pages: (cache, pages), B sequences, checked against the form
struct CacheOf {
    const at::Tensor *cache, *pages;
    bool read(ServingArgs& a, int64_t B) {
        cache = a.flat(U8, {-1, -1, -1});
        pages = a.flat(I32, {B, -1});
        return a.ok;
    }
    int num_pages() const { return (int)cache->size(0); }
    int heads() const { return (int)cache->size(1); }
    int sequences() const { return (int)pages->size(0); }
    int columns() const { return (int)pages->size(1); }
    bool form(int64_t D, int page, int group) const {
        const size_t need = D > 0 && D < 4096 ? api.cache4_block_bytes((int)D, page, group) : 0;
        return need != 0 && cache->size(2) == (int64_t)need;
    }
};

// (q, k | None, positions, inv_freq, interleaved, amplitude, q_out | None, k_out | None, stream | None)
template <bool BWD> PyObject* py_rope(PyObject* const* argv, Py_ssize_t n) {
    if (n != 9) return none();
    ServingArgs a(argv);
    const at::Tensor *q = a.rows(true), *k = a.rows_or_none(true);
    if (!a.ok) return none();
    const int64_t B = q->size(0), Hq = q->size(1), N = q->size(2), D = q->size(3), Hk = k ? k->size(1) : 0;
    if (k && (k->scalar_type() != q->scalar_type() || k->size(0) != B || k->size(2) != N || k->size(3) != D)) return none();
    const at::Tensor* at_pos = tensor(argv[2]);
    const bool own_positions = at_pos && at_pos->dim() == 2;
    const at::Tensor* pos = own_positions ? a.flat(I32, {B, N}) : a.flat(I32, {N});
    const at::Tensor* freq = a.flat(F64, {-1});
    const int interleaved = a.integer();
    const float amplitude = a.real();
    const at::Tensor *gq = a.rows_or_none(true), *gk = a.rows_or_none(true);
    void* st = a.stream();
    // (calls that autograd takes note of are serving.py's)
    if (at::GradMode::is_enabled() && a.ok && (q->requires_grad() || (k && k->requires_grad()) || freq->requires_grad())) return none();
    if (!a.take(gq && (gk || !k)) || (gk && !k)) return none();
    LikeBuffer oq, ok;
    if (!oq.take_like(gq, argv[6], *q) || (k && !ok.take_like(gk, argv[7], *k))) return none();
    const RowsOf xq(q), yq(oq.t), xk(k), yk(k ? ok.t : nullptr);
    const int type = type_of(*q), rotated = 2 * (int)freq->size(0);
    const int32_t* pp = (const int32_t*)pos->data_ptr();
    const double* pf = (const double*)freq->data_ptr();
    const int e = call([&] {
        return (BWD ? api.rope_bwd : api.rope)(xq.p, xq.strides, yq.p, yq.strides, xk.p, xk.strides, yk.p, yk.strides, pp, own_positions ? N : 0, pf,
                                               amplitude, B, Hq, Hk, N, D, rotated, type, interleaved, st);
    });
    return k ? result(e, {&oq, &ok}) : result(e, {&oq});
}

// (k, v, cache, pages, start, count | None, k_mean | None, page, group, stream | None) -> cache
PyObject* py_cache4_append(PyObject* const* argv, Py_ssize_t n) {
    if (n != 10) return none();
    ServingArgs a(argv);
    const at::Tensor *k = a.rows(), *v = a.rows();
    if (!a.ok || k->scalar_type() != v->scalar_type() || k->sizes() != v->sizes()) return none();
    const int64_t B = k->size(0), H = k->size(1), N = k->size(2), D = k->size(3);
    CacheOf c;
    if (!c.read(a, B)) return none();
    const at::Tensor *start = a.flat(I32, {B}), *count = a.flat(I32, {B}, true), *mean = a.flat(F32, {B, H, D}, true);
    const int page = a.integer(), group = a.integer();
    void* st = a.stream();
    if (!a.take(true) || c.heads() != H || !c.form(D, page, group)) return none();
    const RowsOf rk(k), rv(v);
    const int type = type_of(*k);
    const void *pm = at_or_null(mean), *pt = c.pages->data_ptr(), *ps = start->data_ptr(), *pn = at_or_null(count);
    void* pc = c.cache->data_ptr();
    const int e = call([&] {
        return api.cache4_append(rk.p, rk.strides, rv.p, rv.strides, (const float*)pm, pc, (const int32_t*)pt, (const int32_t*)ps, (const int32_t*)pn, B, H, N, D,
                                 type, c.num_pages(), c.columns(), page, group, st);
    });
    return e != 0 ? PyLong_FromLong(e) : (Py_INCREF(argv[2]), argv[2]);
}

// (cache, pages, start | None, N, D, count | None, k_mean | None, bf16, page, group, k | None, v | None, stream | None)
PyObject* py_cache4_load(PyObject* const* argv, Py_ssize_t n) {
    if (n != 13) return none();
    ServingArgs a(argv);
    CacheOf c;
    if (!c.read(a, -1)) return none();
    const int64_t B = c.sequences(), H = c.heads();
    const at::Tensor* start = a.flat(I32, {B}, true);
    const int N = a.integer(), D = a.integer();
    const at::Tensor *count = a.flat(I32, {B}, true), *mean = a.flat(F32, {B, H, D}, true);
    const auto type = a.integer() ? BF16 : F16;
    const int page = a.integer(), group = a.integer();
    const at::Tensor *gk = a.flat(type, {B, H, N, D}, true), *gv = a.flat(type, {B, H, N, D}, true);
    void* st = a.stream();
    if (!a.take(gk && gv) || N <= 0 || !c.form(D, page, group)) return none();
    Buffer k, v;
    k.take(gk ? argv[10] : nullptr, *c.cache, {B, H, N, D}, type);
    v.take(gv ? argv[11] : nullptr, *c.cache, {B, H, N, D}, type);
    const void *pc = c.cache->data_ptr(), *pt = c.pages->data_ptr(), *ps = at_or_null(start), *pn = at_or_null(count), *pm = at_or_null(mean);
    void *pk = k.p(), *pv = v.p();
    return result(call([&] {
                      return api.cache4_load(pc, (const int32_t*)pt, (const int32_t*)ps, (const int32_t*)pn, (const float*)pm, pk, pv, B, H, N, D,
                                             type == BF16 ? SAGE_BF16 : SAGE_F16, c.num_pages(), c.columns(), page, group, st);
                  }),
                  {&k, &v});
}

// (q, cache, pages, lengths, count | None, causal, sm_scale | None, page, group, n_splits, return_lse, out | None, lse | None,
// workspace | None, stream | None)
PyObject* py_cache4_attn(PyObject* const* argv, Py_ssize_t n) {
    if (n != 15) return none();
    ServingArgs a(argv);
    const at::Tensor* q = a.rows();
    if (!a.ok) return none();
    const int64_t B = q->size(0), Hq = q->size(1), Nq = q->size(2), D = q->size(3);
    CacheOf c;
    if (!c.read(a, B)) return none();
    const at::Tensor *lengths = a.flat(I32, {B}), *count = a.flat(I32, {B}, true);
    const int causal = a.integer();
    const bool no_scale = argv[6] == Py_None;
    const float sm = a.real_or(0.0f);
    const int page = a.integer(), group = a.integer(), splits = a.integer(), with_lse = a.integer();
    const at::Tensor *go = a.rows_or_none(), *gl = a.flat(F32, {B, Hq, Nq}, true), *gw = a.flat(U8, {-1}, true);
    void* st = a.stream();
    if (!a.take(go && (gl || !with_lse) && gw) || splits < 0 || !c.form(D, page, group)) return none();
    LikeBuffer o;
    if (!o.take_like(go, argv[11], *q)) return none();
    Buffer lse, ws;
    if (gl || with_lse) lse.take(gl ? argv[12] : nullptr, *q, {B, Hq, Nq}, F32);
    ws.bytes(gw ? argv[13] : nullptr, *q, api.cache4_attn_workspace(B, Hq, c.heads(), Nq, D, c.columns(), page, splits));
    const RowsOf rq(q), ro(o.t);
    const int type = type_of(*q);
    const float scale = no_scale ? 1.0f / std::sqrt((float)D) : sm;
    const void *pc = c.cache->data_ptr(), *pt = c.pages->data_ptr(), *pl = lengths->data_ptr(), *pn = at_or_null(count);
    void *ps = lse.p(), *pw = ws.p();
    const size_t wb = ws.size();
    const int e = call([&] {
        return api.cache4_attn(rq.p, rq.strides, pc, (const int32_t*)pt, (const int32_t*)pl, (const int32_t*)pn, ro.p, ro.strides, (float*)ps, pw, wb, B, Hq,
                               c.heads(), Nq, D, type, c.num_pages(), c.columns(), page, group, causal != 0, scale, splits, st);
    });
    return lse.t ? result(e, {&o, &lse}) : result(e, {&o});
}

// (q, cache, pages, lengths, lse, weights | None, count | None, causal, sm_scale | None, page, group, out | None, stream | None)
PyObject* py_cache4_weights(PyObject* const* argv, Py_ssize_t n) {
    if (n != 13) return none();
    ServingArgs a(argv);
    const at::Tensor* q = a.rows();
    if (!a.ok) return none();
    const int64_t B = q->size(0), Hq = q->size(1), Nq = q->size(2), D = q->size(3);
    CacheOf c;
    if (!c.read(a, B)) return none();
    const at::Tensor *lengths = a.flat(I32, {B}), *lse = a.flat(F32, {B, Hq, Nq});
    const int64_t H = c.heads();
    const at::Tensor *had = a.flat(F32, {B, H, -1}, true), *count = a.flat(I32, {B}, true);
    const int causal = a.integer();
    const bool no_scale = argv[8] == Py_None;
    const float sm = a.real_or(0.0f);
    const int page = a.integer(), group = a.integer();
    const at::Tensor* go = a.flat(F32, {B, H, had ? had->size(2) : -1}, true);
    void* st = a.stream();
    if (!a.take(go != nullptr) || !c.form(D, page, group)) return none();
    const int64_t width = had ? had->size(2) : go ? go->size(2) : (int64_t)c.columns() * page;
    if (width > 0x7fffffff) return none();
    Buffer o;
    o.take(go ? argv[11] : nullptr, *q, {B, H, width}, F32);
    const RowsOf rq(q);
    const int type = type_of(*q);
    const float scale = no_scale ? 1.0f / std::sqrt((float)D) : sm;
    const void *pc = c.cache->data_ptr(), *pt = c.pages->data_ptr(), *pl = lengths->data_ptr(), *pn = at_or_null(count), *ps = lse->data_ptr(), *ph = at_or_null(had);
    void* po = o.p();
    return result(call([&] {
                      return api.cache4_weights(rq.p, rq.strides, pc, (const int32_t*)pt, (const int32_t*)pl, (const int32_t*)pn, (const float*)ps, (const float*)ph,
                                                (float*)po, (int)width, B, Hq, H, Nq, D, type, c.num_pages(), c.columns(), page, group, causal != 0, scale, st);
                  }),
                  {&o});
}

// (cache, pages, lengths, weights, out_cache, out_pages, keep, recent, D, page, group, out_weights | None, kept | None, out_lengths | None,
// stream | None)
PyObject* py_cache4_evict(PyObject* const* argv, Py_ssize_t n) {
    if (n != 15) return none();
    ServingArgs a(argv);
    CacheOf c, to;
    if (!c.read(a, -1)) return none();
    const int64_t B = c.sequences(), H = c.heads();
    const at::Tensor *lengths = a.flat(I32, {B}), *weights = a.flat(F32, {B, H, -1});
    if (!to.read(a, B)) return none();
    const int keep = a.integer(), recent = a.integer(), D = a.integer(), page = a.integer(), group = a.integer();
    if (!a.ok || keep < 1 || to.heads() != H || !c.form(D, page, group) || !to.form(D, page, group)) return none();
    const at::Tensor *gw = a.flat(F32, {B, H, -1}, true), *gk = a.flat(I32, {B, H, keep}, true), *gl = a.flat(I32, {B}, true);
    void* st = a.stream();
    if (!a.take(gw && gk && gl)) return none();
    const int64_t out_width = gw ? gw->size(2) : (int64_t)to.columns() * page;
    if (out_width > 0x7fffffff) return none();
    Buffer ow, kept, ol;
    ow.take(gw ? argv[11] : nullptr, *c.cache, {B, H, out_width}, F32);
    kept.take(gk ? argv[12] : nullptr, *c.cache, {B, H, keep}, I32);
    ol.take(gl ? argv[13] : nullptr, *c.cache, {B}, I32);
    const int width = (int)weights->size(2);
    const void *pc = c.cache->data_ptr(), *pt = c.pages->data_ptr(), *pl = lengths->data_ptr(), *pw = weights->data_ptr(), *qt = to.pages->data_ptr();
    void *qc = to.cache->data_ptr(), *qw = ow.p(), *qk = kept.p(), *ql = ol.p();
    return result(call([&] {
                      return api.cache4_evict(pc, c.num_pages(), (const int32_t*)pt, c.columns(), (const int32_t*)pl, (const float*)pw, width, qc, to.num_pages(),
                                              (const int32_t*)qt, to.columns(), (float*)qw, (int)out_width, (int32_t*)qk, (int32_t*)ql, B, H, D, page, group, keep,
                                              recent, st);
                  }),
                  {&kept, &ol, &ow});
}

// (torch._C._cuda_getDevice, torch._C._cuda_getCurrentRawStream, the addresses in Api's order)
PyObject* py_init(PyObject* const* argv, Py_ssize_t n) {
    constexpr int COUNT = sizeof(Api) / sizeof(void*);
    if (n != 2 + COUNT) {
        PyErr_SetString(PyExc_ValueError, "init: wrong number of addresses");
        return nullptr;
    }
    void* p[COUNT];
    for (int i = 0; i < COUNT; ++i) {
        p[i] = PyLong_AsVoidPtr(argv[2 + i]);
        if (PyErr_Occurred()) return nullptr;
    }
    static_assert(sizeof p == sizeof api, "Api is function pointers only");
    memcpy(&api, p, sizeof api);
    Py_INCREF(argv[0]);
    Py_INCREF(argv[1]);
    get_device = argv[0];
    get_stream = argv[1];
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {
    {"init", (PyCFunction)(void (*)(void))guarded<py_init>, METH_FASTCALL, nullptr},
    {"quant_q", (PyCFunction)(void (*)(void))guarded<py_quant_q<false>>, METH_FASTCALL, nullptr},
    {"rope_quant_q", (PyCFunction)(void (*)(void))guarded<py_quant_q<true>>, METH_FASTCALL, nullptr},
    {"smooth_quant_k", (PyCFunction)(void (*)(void))guarded<py_smooth_quant_k<false>>, METH_FASTCALL, nullptr},
    {"rope_smooth_quant_k", (PyCFunction)(void (*)(void))guarded<py_smooth_quant_k<true>>, METH_FASTCALL, nullptr},
    {"quant_qk", (PyCFunction)(void (*)(void))guarded<py_quant_qk>, METH_FASTCALL, nullptr},
    {"quant_v", (PyCFunction)(void (*)(void))guarded<py_quant_v>, METH_FASTCALL, nullptr},
    {"attn", (PyCFunction)(void (*)(void))guarded<py_attn<false>>, METH_FASTCALL, nullptr},
    {"attn_pv_int8", (PyCFunction)(void (*)(void))guarded<py_attn<true>>, METH_FASTCALL, nullptr},
    {"attention", (PyCFunction)(void (*)(void))guarded<py_attention>, METH_FASTCALL, nullptr},
    {"rope", (PyCFunction)(void (*)(void))guarded<py_rope<false>>, METH_FASTCALL, nullptr},
    {"rope_bwd", (PyCFunction)(void (*)(void))guarded<py_rope<true>>, METH_FASTCALL, nullptr},
    {"cache4_append", (PyCFunction)(void (*)(void))guarded<py_cache4_append>, METH_FASTCALL, nullptr},
    {"cache4_load", (PyCFunction)(void (*)(void))guarded<py_cache4_load>, METH_FASTCALL, nullptr},
    {"cache4_attn", (PyCFunction)(void (*)(void))guarded<py_cache4_attn>, METH_FASTCALL, nullptr},
    {"cache4_weights", (PyCFunction)(void (*)(void))guarded<py_cache4_weights>, METH_FASTCALL, nullptr},
    {"cache4_evict", (PyCFunction)(void (*)(void))guarded<py_cache4_evict>, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_sage_native", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

extern "C" __attribute__((visibility("default"))) PyObject* PyInit__sage_native(void) {
    PyObject* m = PyModule_Create(&module);
    if (m) PyModule_AddStringConstant(m, "source_hash", tagged_hash + sizeof("SAGE_NATIVE_HASH=") - 1);
    return m;
}
