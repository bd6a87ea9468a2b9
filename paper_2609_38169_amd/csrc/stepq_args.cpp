// Python module _stepq_args: the argument checks of the binding's device calls
// (stepq.py) in native code, followed by the C call.
//
// A small decode step is bound by its launch: checking eight tensors from
// Python and marshalling twelve arguments through ctypes took 9 of the 12 us
// of a one-request step (the kernel 5): 12.4 -> 5.2 us here; export + import
// with FP16 rows of 32 requests (four calls) 35.2 -> 26.4 us.  Each function here checks what
// stepq.py's own path checks (device, dtype, shape, contiguity) and makes the
// call, or returns -1 without calling anything when an argument is not plainly
// what the call takes: stepq.py then goes through its own path, which raises
// the error or handles the case.  Nothing is kept between calls.
#include <Python.h>

#include <cmath>
#include <type_traits>

#include <ATen/core/Tensor.h>
#include <ATen/ops/empty.h>
#include <torch/csrc/autograd/python_variable.h>

#include "stepq.h"

namespace {

struct Entry {
    decltype(&stepq_decode_step_ex) step;
    decltype(&stepq_pool_load) load;
    decltype(&stepq_pool_import) import;
    decltype(&stepq_pool_export) exprt;
    decltype(&stepq_pool_dequant) dequant;
    decltype(&stepq_pool_export_pivots) export_pivots;
    decltype(&stepq_pool_import_pivots) import_pivots;
    int (*get_device)(int *);                  // the runtime's current device
    PyObject *raw_stream, *stream_type;        // torch's raw current-stream query and stream class
    decltype(&stepq_state_step) state_step;
    decltype(&stepq_prompt_workspace) prompt_workspace;
    decltype(&stepq_prompt) prompt;
    decltype(&stepq_prefix_attention_workspace) attention_workspace;
    decltype(&stepq_prefix_attention) attention;
    decltype(&stepq_cache_write) cache_write;
    decltype(&stepq_cache_read) cache_read;
    decltype(&stepq_cache_attention_workspace) cache_attention_workspace;
    decltype(&stepq_cache_attention) cache_attention;
    decltype(&stepq_cache_bounds) cache_bounds;
    decltype(&stepq_cache_select_workspace) cache_select_workspace;
    decltype(&stepq_cache_select) cache_select;
} g{};

struct Plain {
    stepq_pool *pool;
    int device;
    int64_t Hv, Hqk, dk, dv;
};

// The tensor's data if it is a plain tensor of this device, type and shape.
bool take(PyObject *o, const Plain &p, at::ScalarType dt, at::IntArrayRef shape, void **out)
{
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (!t.is_cuda() || t.get_device() != p.device || t.scalar_type() != dt || t.layout() != at::kStrided ||
        t.sizes() != shape || !t.is_contiguous())
        return false;
    *out = t.data_ptr();
    return true;
}

bool take_ids(PyObject *o, const Plain &p, int64_t *n, void **out)
{
    if (!THPVariable_CheckExact(o)) return false;
    const at::Tensor &t = THPVariable_Unpack(o);
    if (t.dim() != 1) return false;
    *n = t.size(0);
    return *n <= INT32_MAX && take(o, p, at::kInt, {*n}, out);
}

// None: torch's current stream, which is the current device's (not the pool's);
// an int: the stream itself; a torch stream.
bool take_stream(PyObject *o, void **out)
{
    PyObject *v = nullptr;
    if (o == Py_None) {
        int device;
        if (g.get_device(&device) != 0) return false;
        if (PyObject *d = PyLong_FromLong(device)) {
            v = PyObject_CallOneArg(g.raw_stream, d);
            Py_DECREF(d);
        }
    } else if (PyLong_CheckExact(o)) {
        v = o;
        Py_INCREF(v);
    } else {
        const int is = PyObject_IsInstance(o, g.stream_type);
        if (is == 0) return false;
        if (is > 0) v = PyObject_GetAttrString(o, "cuda_stream");
    }
    if (!v) {
        PyErr_Clear();
        return false;
    }
    *out = PyLong_AsVoidPtr(v);
    Py_DECREF(v);
    if (PyErr_Occurred()) {
        PyErr_Clear();
        return false;
    }
    return true;
}

const Plain *plain_of(PyObject *o)
{
    if (!PyCapsule_CheckExact(o)) return nullptr;
    return static_cast<const Plain *>(PyCapsule_GetPointer(o, "stepq.plain"));
}

void free_plain(PyObject *cap) { delete static_cast<Plain *>(PyCapsule_GetPointer(cap, "stepq.plain")); }

// plain(handle, device, Hv, Hqk, dk, dv): what the checks compare with.
PyObject *py_plain(PyObject *, PyObject *args)
{
    unsigned long long handle;
    int device;
    long long Hv, Hqk, dk, dv;
    if (!PyArg_ParseTuple(args, "KiLLLL", &handle, &device, &Hv, &Hqk, &dk, &dv)) return nullptr;
    auto *p = new Plain{reinterpret_cast<stepq_pool *>(handle), device, Hv, Hqk, dk, dv};
    return PyCapsule_New(p, "stepq.plain", free_plain);
}

// bind(step_ex, load, import, export, dequant, export_pivots, import_pivots, get_device, raw_stream, stream_type)
PyObject *py_bind(PyObject *, PyObject *args)
{
    unsigned long long f[8];
    PyObject *rs, *st;
    if (!PyArg_ParseTuple(args, "KKKKKKKKOO", &f[0], &f[1], &f[2], &f[3], &f[4], &f[5], &f[6], &f[7], &rs, &st))
        return nullptr;
    auto set = [&f](auto &fn, int i) { fn = reinterpret_cast<std::remove_reference_t<decltype(fn)>>(f[i]); };
    set(g.step, 0);
    set(g.load, 1);
    set(g.import, 2);
    set(g.exprt, 3);
    set(g.dequant, 4);
    set(g.export_pivots, 5);
    set(g.import_pivots, 6);
    set(g.get_device, 7);
    Py_INCREF(rs);
    Py_XSETREF(g.raw_stream, rs);
    Py_INCREF(st);
    Py_XSETREF(g.stream_type, st);
    Py_RETURN_NONE;
}

template <class F>
PyObject *guarded(F &&f)
{
    long st = -1;
    try {
        st = f();
    } catch (...) {
        st = -1;      // e.g. a tensor without data: the binding's own path says so
    }
    return PyLong_FromLong(st);
}

// decode(plain, slot_ids, q, k, v, gate, beta, o, stream, flags) -> status or -1
PyObject *py_decode(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded([&]() -> long {
        const Plain *p = n_args == 10 ? plain_of(a[0]) : nullptr;
        if (!p || !g.step || !PyLong_CheckExact(a[9]) || !THPVariable_CheckExact(a[2])) return -1;
        const unsigned long flags = PyLong_AsUnsignedLong(a[9]);
        if (PyErr_Occurred()) {
            PyErr_Clear();
            return -1;
        }
        const at::ScalarType dt = THPVariable_Unpack(a[2]).scalar_type();
        if (dt != at::kFloat && dt != at::kBFloat16) return -1;
        int64_t n;
        void *ids, *q, *k, *v, *gate, *beta, *o, *s;
        if (!take_ids(a[1], *p, &n, &ids) || !take(a[2], *p, dt, {n, p->Hqk, p->dk}, &q) ||
            !take(a[3], *p, dt, {n, p->Hqk, p->dk}, &k) || !take(a[4], *p, dt, {n, p->Hv, p->dv}, &v) ||
            !((flags & STEPQ_STEP_KDA_GATE) ? take(a[5], *p, dt, {n, p->Hv, p->dk}, &gate)
                                            : take(a[5], *p, dt, {n, p->Hv}, &gate)) ||
            !take(a[6], *p, dt, {n, p->Hv}, &beta) || !take(a[7], *p, at::kFloat, {n, p->Hv, p->dv}, &o) ||
            !take_stream(a[8], &s))
            return -1;
        stepq_status st;
        Py_BEGIN_ALLOW_THREADS;
        st = g.step(p->pool, static_cast<const int32_t *>(ids), static_cast<int32_t>(n), q, k, v, gate, beta,
                    dt == at::kFloat ? STEPQ_F32 : STEPQ_BF16, static_cast<uint32_t>(flags), static_cast<float *>(o), s);
        Py_END_ALLOW_THREADS;
        return st;
    });
}

enum { kLoad, kImport, kExport };

// scaled(op, plain, slot_ids, rows, r, c, stream): load (0), import (1), export (2)
PyObject *py_scaled(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded([&]() -> long {
        const Plain *p = n_args == 7 ? plain_of(a[1]) : nullptr;
        if (!p || !g.load || !PyLong_CheckExact(a[0])) return -1;
        const long op = PyLong_AsLong(a[0]);
        int64_t n;
        void *ids, *x, *r, *c, *s;
        if (!take_ids(a[2], *p, &n, &ids) ||
            !take(a[3], *p, op == kLoad ? at::kFloat : at::kChar, {n, p->Hv, p->dk, p->dv}, &x) ||
            !take(a[4], *p, at::kFloat, {n, p->Hv, p->dk}, &r) || !take(a[5], *p, at::kFloat, {n, p->Hv, p->dv}, &c) ||
            !take_stream(a[6], &s))
            return -1;
        const auto *id = static_cast<const int32_t *>(ids);
        const auto m = static_cast<int32_t>(n);
        auto *rf = static_cast<float *>(r), *cf = static_cast<float *>(c);
        stepq_status st;
        Py_BEGIN_ALLOW_THREADS;
        st = op == kLoad     ? g.load(p->pool, id, m, static_cast<const float *>(x), rf, cf, s)
             : op == kImport ? g.import(p->pool, id, m, static_cast<const int8_t *>(x), rf, cf, s)
                             : g.exprt(p->pool, id, m, static_cast<int8_t *>(x), rf, cf, s);
        Py_END_ALLOW_THREADS;
        return st;
    });
}

enum { kDequant, kExportPivots, kImportPivots };

// tiles(op, plain, slot_ids, rows, stream): dequant (0), export (1) and import (2) of the pivot rows
PyObject *py_tiles(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded([&]() -> long {
        const Plain *p = n_args == 5 ? plain_of(a[1]) : nullptr;
        if (!p || !g.dequant || !PyLong_CheckExact(a[0])) return -1;
        const long op = PyLong_AsLong(a[0]);
        int64_t n;
        void *ids, *x, *s;
        if (!take_ids(a[2], *p, &n, &ids)) return -1;
        const int64_t shape[4] = {n, p->Hv, p->dk, p->dv};
        const bool ok = op == kDequant ? take(a[3], *p, at::kFloat, shape, &x)
                                       : take(a[3], *p, at::kShort, shape, &x) || take(a[3], *p, at::kUInt16, shape, &x);
        if (!ok || !take_stream(a[4], &s)) return -1;
        const auto *id = static_cast<const int32_t *>(ids);
        const auto m = static_cast<int32_t>(n);
        stepq_status st;
        Py_BEGIN_ALLOW_THREADS;
        st = op == kDequant        ? g.dequant(p->pool, id, m, static_cast<float *>(x), s)
             : op == kExportPivots ? g.export_pivots(p->pool, id, m, static_cast<uint16_t *>(x), s)
                                   : g.import_pivots(p->pool, id, m, static_cast<const uint16_t *>(x), s);
        Py_END_ALLOW_THREADS;
        return st;
    });
}

// ---------------------------------------------------------------------------
// The calls without a pool: everything is on the current device, sizes follow
// from the tensors, workspaces from torch (on the current stream).  One token
// of a small model 14 -> 4 us, attention of 4 requests 19 -> 11 us a call.

// bind_calls(state_step, prompt_workspace, prompt, attention_workspace, attention)
PyObject *py_bind_calls(PyObject *, PyObject *args)
{
    unsigned long long f[5];
    if (!PyArg_ParseTuple(args, "KKKKK", &f[0], &f[1], &f[2], &f[3], &f[4])) return nullptr;
    auto set = [&f](auto &fn, int i) { fn = reinterpret_cast<std::remove_reference_t<decltype(fn)>>(f[i]); };
    set(g.state_step, 0);
    set(g.prompt_workspace, 1);
    set(g.prompt, 2);
    set(g.attention_workspace, 3);
    set(g.attention, 4);
    Py_RETURN_NONE;
}

bool take_long(PyObject *o, int64_t *out)
{
    if (!PyLong_CheckExact(o)) return false;
    *out = PyLong_AsLongLong(o);
    if (!PyErr_Occurred()) return true;
    PyErr_Clear();
    return false;
}

// a whole number of 32 bits
bool take_int(PyObject *o, int64_t *out) { return take_long(o, out) && *out == static_cast<int32_t>(*out); }

const at::Tensor *tensor_of(PyObject *o, int64_t dims)
{
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor &t = THPVariable_Unpack(o);
    return t.dim() == dims && t.layout() == at::kStrided ? &t : nullptr;
}

bool known(at::ScalarType t) { return t == at::kFloat || t == at::kBFloat16; }
int code_of(at::ScalarType t) { return t == at::kFloat ? STEPQ_F32 : STEPQ_BF16; }

// The device that q lies on, if it is the current one.
bool take_device(const at::Tensor &q, Plain *p)
{
    int device;
    if (!q.is_cuda() || !known(q.scalar_type()) || g.get_device(&device) != 0 || q.get_device() != device) return false;
    p->device = device;
    return true;
}

// Tokens whose heads are contiguous: their data and the elements from one to the next.
bool take_tokens(PyObject *o, const Plain &p, at::ScalarType dt, at::IntArrayRef shape, void **out, int64_t *stride)
{
    const at::Tensor *t = tensor_of(o, 3);
    if (!t || !t->is_cuda() || t->get_device() != p.device || t->scalar_type() != dt || t->sizes() != shape) return false;
    const auto st = t->strides();
    const int64_t n = shape[0], h = shape[1], d = shape[2];
    if (n && ((d > 1 && st[2] != 1) || (h > 1 && st[1] != d) || (n > 1 && st[0] < h * d))) return false;
    *out = t->data_ptr();
    *stride = n > 1 ? st[0] : 0;
    return true;
}

// alpha, and beta or None
bool take_gates(PyObject *alpha, PyObject *beta, const Plain &p, at::IntArrayRef shape, void **a, void **b, int *code)
{
    const at::Tensor *t = tensor_of(alpha, static_cast<int64_t>(shape.size()));
    if (!t || !known(t->scalar_type())) return false;
    *code = code_of(t->scalar_type());
    *b = nullptr;
    return take(alpha, p, t->scalar_type(), shape, a) && (beta == Py_None || take(beta, p, t->scalar_type(), shape, b));
}

// Memory of the current stream for one call (the next owner there comes after it).
at::Tensor space(size_t bytes, int device)
{
    return at::empty({static_cast<int64_t>(bytes)},
                     at::TensorOptions().dtype(at::kByte).device(at::Device(at::kCUDA, static_cast<at::DeviceIndex>(device))));
}

// state_step(state, ids, q, k, v, alpha, beta, o, rule, stream) -> status or -1
PyObject *py_state_step(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded([&]() -> long {
        if (n_args != 10 || !g.state_step) return -1;
        const at::Tensor *S = tensor_of(a[0], 4), *q = tensor_of(a[2], 3), *v = tensor_of(a[4], 3);
        Plain p{};
        int64_t rule;
        if (!S || !q || !v || !take_device(*q, &p) || !take_int(a[8], &rule)) return -1;
        const int64_t B = q->size(0), Hqk = q->size(1), dk = q->size(2), Hv = v->size(1), dv = v->size(2), n = S->size(0);
        const at::ScalarType dt = q->scalar_type();
        void *sp, *ip, *qp, *kp, *vp, *ap, *bp, *op, *st;
        int gate;
        if (B > INT32_MAX || n > INT32_MAX || !take(a[0], p, at::kFloat, {n, Hv, dk, dv}, &sp) ||
            !take(a[1], p, at::kInt, {B}, &ip) || !take(a[2], p, dt, {B, Hqk, dk}, &qp) ||
            !take(a[3], p, dt, {B, Hqk, dk}, &kp) || !take(a[4], p, dt, {B, Hv, dv}, &vp) ||
            !take_gates(a[5], a[6], p, {B, Hv}, &ap, &bp, &gate) || !take(a[7], p, at::kFloat, {B, Hv, dv}, &op) ||
            !take_stream(a[9], &st))
            return -1;
        const stepq_state_desc d{static_cast<int32_t>(n),  static_cast<int32_t>(Hv), static_cast<int32_t>(Hqk),
                                 static_cast<int32_t>(dk), static_cast<int32_t>(dv), code_of(dt), gate,
                                 static_cast<int32_t>(rule)};
        stepq_status e;
        Py_BEGIN_ALLOW_THREADS;
        e = g.state_step(&d, static_cast<float *>(sp), static_cast<const int32_t *>(ip), static_cast<int32_t>(B), qp, kp, vp,
                         ap, bp, static_cast<float *>(op), st);
        Py_END_ALLOW_THREADS;
        return e;
    });
}

// prompt(q, k, v, alpha, beta, o, state_out, rule, cu_seqlens, state_in, in_ids): on the current stream, in torch's memory
PyObject *py_prompt(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded([&]() -> long {
        if (n_args != 11 || !g.prompt) return -1;
        const at::Tensor *q = tensor_of(a[0], 3), *v = tensor_of(a[2], 3), *cu = a[8] == Py_None ? nullptr : tensor_of(a[8], 1);
        Plain p{};
        int64_t rule;
        if (!q || !v || (a[8] != Py_None && (!cu || cu->size(0) < 1)) || !take_device(*q, &p) || !take_int(a[7], &rule)) return -1;
        const int64_t T = q->size(0), Hqk = q->size(1), dk = q->size(2), Hv = v->size(1), dv = v->size(2);
        const int64_t n = cu ? cu->size(0) - 1 : 1;
        const at::ScalarType dt = q->scalar_type();
        stepq_prompt_desc d{};
        void *qp, *kp, *vp, *op, *ap, *bp, *cp = nullptr, *out, *in = nullptr, *ids = nullptr, *st;
        int gate;
        int64_t m = 0;
        if (n > INT32_MAX || !take_tokens(a[0], p, dt, {T, Hqk, dk}, &qp, &d.q_stride) ||
            !take_tokens(a[1], p, dt, {T, Hqk, dk}, &kp, &d.k_stride) ||
            !take_tokens(a[2], p, dt, {T, Hv, dv}, &vp, &d.v_stride) ||
            !take_tokens(a[5], p, dt, {T, Hv, dv}, &op, &d.o_stride) ||
            !take_gates(a[3], a[4], p, {T, Hv}, &ap, &bp, &gate) || (cu && !take(a[8], p, at::kInt, {n + 1}, &cp)) ||
            !take(a[6], p, at::kFloat, {n, Hv, dk, dv}, &out))
            return -1;
        if (a[9] != Py_None) {
            const at::Tensor *s = tensor_of(a[9], 4);
            if (!s) return -1;
            m = a[10] == Py_None ? n : s->size(0);
            if (m > INT32_MAX || !take(a[9], p, at::kFloat, {m, Hv, dk, dv}, &in) ||
                (a[10] != Py_None && !take(a[10], p, at::kInt, {n}, &ids)))
                return -1;
            const auto lo = reinterpret_cast<uintptr_t>(in), hi = reinterpret_cast<uintptr_t>(out);
            const uintptr_t each = static_cast<uintptr_t>(Hv * dk * dv) * sizeof(float);
            if ((ids || lo != hi) && lo < hi + n * each && hi < lo + m * each) return -1;
        } else if (a[10] != Py_None) {
            return -1;
        }
        d.n_tokens = T, d.n_seq = static_cast<int32_t>(n);
        d.n_v_heads = static_cast<int32_t>(Hv), d.n_qk_heads = static_cast<int32_t>(Hqk);
        d.d_k = static_cast<int32_t>(dk), d.d_v = static_cast<int32_t>(dv);
        d.act_dtype = code_of(dt), d.gate_dtype = gate, d.rule = static_cast<int32_t>(rule);
        d.n_states_in = static_cast<int32_t>(m);
        size_t bytes = 0;
        stepq_status e = g.prompt_workspace(&d, &bytes);
        if (e != STEPQ_OK) return e;
        if (!take_stream(Py_None, &st)) return -1;
        const at::Tensor ws = space(bytes, p.device);
        void *wp = bytes ? ws.data_ptr() : nullptr;
        Py_BEGIN_ALLOW_THREADS;
        e = g.prompt(&d, static_cast<const int32_t *>(cp), qp, kp, vp, ap, bp, op, static_cast<const float *>(in),
                     static_cast<const int32_t *>(ids), static_cast<float *>(out), wp, bytes, st);
        Py_END_ALLOW_THREADS;
        return e;
    });
}

// attention(q, k_cache, v_cache, prefix_pages, prefix_len, page_table, lengths, o, lse, scale): as prompt
PyObject *py_attention(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded([&]() -> long {
        if (n_args != 10 || !g.attention) return -1;
        const at::Tensor *q = tensor_of(a[0], 3), *kc = tensor_of(a[1], 4), *table = tensor_of(a[5], 2);
        Plain p{};
        int64_t prefix;
        if (!q || !kc || !table || !take_device(*q, &p) || !take_long(a[4], &prefix) || prefix < 0 || !(a[9] == Py_None || PyFloat_CheckExact(a[9])))
            return -1;
        const int64_t B = q->size(0), Hq = q->size(1), D = q->size(2), M = table->size(1);
        const int64_t pages = kc->size(0), Hkv = kc->size(1), page = kc->size(2);
        const at::ScalarType dt = q->scalar_type();
        if (page < 1 || B > INT32_MAX || M > INT32_MAX || pages > INT32_MAX || page > INT32_MAX) return -1;
        const int64_t P = (prefix + page - 1) / page;
        void *qp, *kp, *vp, *pp = nullptr, *tp, *lp, *op, *ep = nullptr, *st;
        if (P) {
            const at::Tensor *t = tensor_of(a[3], 1);
            if (!t || t->size(0) < P || !take(a[3], p, at::kInt, t->sizes(), &pp)) return -1;
        }
        if (!take(a[0], p, dt, {B, Hq, D}, &qp) || !take(a[1], p, dt, {pages, Hkv, page, D}, &kp) ||
            !take(a[2], p, dt, {pages, Hkv, page, D}, &vp) || !take(a[5], p, at::kInt, {B, M}, &tp) ||
            !take(a[6], p, at::kInt, {B}, &lp) || !take(a[7], p, dt, {B, Hq, D}, &op) ||
            (a[8] != Py_None && !take(a[8], p, at::kFloat, {B, Hq}, &ep)))
            return -1;
        const stepq_attn_desc d{static_cast<int32_t>(B),     static_cast<int32_t>(Hq),   static_cast<int32_t>(Hkv),
                                static_cast<int32_t>(D),     static_cast<int32_t>(pages), static_cast<int32_t>(page), prefix,
                                static_cast<int32_t>(M),     code_of(dt),
                                static_cast<float>(a[9] == Py_None ? std::pow(static_cast<double>(D), -0.5) : PyFloat_AS_DOUBLE(a[9]))};
        size_t bytes = 0;
        stepq_status e = g.attention_workspace(&d, &bytes);
        if (e != STEPQ_OK) return e;
        if (!take_stream(Py_None, &st)) return -1;
        const at::Tensor ws = space(bytes, p.device);
        void *wp = bytes ? ws.data_ptr() : nullptr;
        Py_BEGIN_ALLOW_THREADS;
        e = g.attention(&d, qp, kp, vp, static_cast<const int32_t *>(pp), static_cast<const int32_t *>(tp),
                        static_cast<const int32_t *>(lp), op, static_cast<float *>(ep), wp, bytes, st);
        Py_END_ALLOW_THREADS;
        return e;
    });
}

// ---------------------------------------------------------------------------
// Calls on quantized caches, as above; the cache is on the current device.  Writing one token of 4 requests takes 3.5 us
// here, 13.4 through the binding's own path.

struct CachePlain {
    stepq_cache_desc desc;
    int device;
    void *memory;
};

void free_cache(PyObject *cap) { delete static_cast<CachePlain *>(PyCapsule_GetPointer(cap, "stepq.cache")); }

// cache(n_pages, n_kv_heads, page_size, head_dim, bits, device, memory): what the checks compare with
PyObject *py_cache(PyObject *, PyObject *args)
{
    int n, h, p, d, b, device;
    unsigned long long memory;
    if (!PyArg_ParseTuple(args, "iiiiiiK", &n, &h, &p, &d, &b, &device, &memory)) return nullptr;
    auto *c = new CachePlain{{n, h, p, d, b}, device, reinterpret_cast<void *>(memory)};
    return PyCapsule_New(c, "stepq.cache", free_cache);
}

// bind_caches(write, read, attention_workspace, attention, bounds, select_workspace, select)
PyObject *py_bind_caches(PyObject *, PyObject *args)
{
    unsigned long long f[7];
    if (!PyArg_ParseTuple(args, "KKKKKKK", &f[0], &f[1], &f[2], &f[3], &f[4], &f[5], &f[6])) return nullptr;
    auto set = [&f](auto &fn, int i) { fn = reinterpret_cast<std::remove_reference_t<decltype(fn)>>(f[i]); };
    set(g.cache_write, 0);
    set(g.cache_read, 1);
    set(g.cache_attention_workspace, 2);
    set(g.cache_attention, 3);
    set(g.cache_bounds, 4);
    set(g.cache_select_workspace, 5);
    set(g.cache_select, 6);
    Py_RETURN_NONE;
}

// The cache's description, if its memory is on the current device.
const CachePlain *cache_of(PyObject *o, Plain *p)
{
    if (!PyCapsule_CheckExact(o)) return nullptr;
    const auto *c = static_cast<const CachePlain *>(PyCapsule_GetPointer(o, "stepq.cache"));
    int device;
    if (!c) {
        PyErr_Clear();
        return nullptr;
    }
    if (!g.cache_write || g.get_device(&device) != 0 || device != c->device) return nullptr;
    p->device = device;
    return c;
}

// page_table [requests][pages]
bool take_table(PyObject *o, const Plain &p, int64_t *n, int64_t *m, void **out)
{
    const at::Tensor *t = tensor_of(o, 2);
    if (!t || t->size(0) > INT32_MAX || t->size(1) > INT32_MAX) return false;
    *n = t->size(0), *m = t->size(1);
    return take(o, p, at::kInt, {*n, *m}, out);
}

// cache_rows(op, cache, k, v, page_table, starts, cu_seqlens, stream): write (0), read (1)
PyObject *py_cache_rows(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded([&]() -> long {
        Plain p{};
        const CachePlain *c = n_args == 8 ? cache_of(a[1], &p) : nullptr;
        int64_t op, n, m;
        const at::Tensor *k = c ? tensor_of(a[2], 3) : nullptr;
        if (!k || !take_long(a[0], &op) || !known(k->scalar_type())) return -1;
        const int64_t T = k->size(0);
        const at::ScalarType dt = k->scalar_type();
        stepq_cache_tokens d{};
        void *kp, *vp, *tp, *sp, *cp = nullptr, *st;
        if (!take_tokens(a[2], p, dt, {T, c->desc.n_kv_heads, c->desc.head_dim}, &kp, &d.k_stride) ||
            !take_tokens(a[3], p, dt, {T, c->desc.n_kv_heads, c->desc.head_dim}, &vp, &d.v_stride) ||
            !take_table(a[4], p, &n, &m, &tp) || !take(a[5], p, at::kInt, {n}, &sp) ||
            !(a[6] == Py_None ? T == n : take(a[6], p, at::kInt, {n + 1}, &cp)) || !take_stream(a[7], &st))
            return -1;
        d.n_tokens = T, d.n_seq = static_cast<int32_t>(n), d.max_pages = static_cast<int32_t>(m), d.act_dtype = code_of(dt);
        const auto *table = static_cast<const int32_t *>(tp), *starts = static_cast<const int32_t *>(sp),
                   *cu = static_cast<const int32_t *>(cp);
        stepq_status e;
        Py_BEGIN_ALLOW_THREADS;
        e = op == 0 ? g.cache_write(&c->desc, &d, c->memory, table, starts, cu, kp, vp, st)
                    : g.cache_read(&c->desc, &d, c->memory, table, starts, cu, kp, vp, st);
        Py_END_ALLOW_THREADS;
        return e;
    });
}

// The query [requests][heads][d] of a cache's head_dim.
bool take_query(PyObject *o, const Plain &p, const CachePlain &c, int64_t n, int64_t *heads, at::ScalarType *dt, void **out)
{
    const at::Tensor *q = tensor_of(o, 3);
    if (!q || !known(q->scalar_type()) || q->size(1) > INT32_MAX) return false;
    *heads = q->size(1), *dt = q->scalar_type();
    return take(o, p, *dt, {n, *heads, c.desc.head_dim}, out);
}

// selected [requests][key/value heads][pages]
bool take_selected(PyObject *o, const Plain &p, const CachePlain &c, int64_t n, int64_t *pages, void **out)
{
    const at::Tensor *t = tensor_of(o, 3);
    if (!t || t->size(2) < 1 || t->size(2) > INT32_MAX) return false;
    *pages = t->size(2);
    return take(o, p, at::kInt, {n, c.desc.n_kv_heads, *pages}, out);
}

// cache_attention(cache, q, page_table, lengths, o, lse, selected, scale): on the current stream, in torch's memory
PyObject *py_cache_attention(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded([&]() -> long {
        Plain p{};
        const CachePlain *c = n_args == 8 ? cache_of(a[0], &p) : nullptr;
        if (!c || !(a[7] == Py_None || PyFloat_CheckExact(a[7]))) return -1;
        int64_t n, m, Hq, S = 0;
        at::ScalarType dt;
        void *tp, *qp, *lp, *op, *ep = nullptr, *sp = nullptr, *st;
        if (!take_table(a[2], p, &n, &m, &tp) || !take_query(a[1], p, *c, n, &Hq, &dt, &qp) || !take(a[3], p, at::kInt, {n}, &lp) ||
            !take(a[4], p, dt, {n, Hq, c->desc.head_dim}, &op) || (a[5] != Py_None && !take(a[5], p, at::kFloat, {n, Hq}, &ep)) ||
            (a[6] != Py_None && !take_selected(a[6], p, *c, n, &S, &sp)))
            return -1;
        const double scale = a[7] == Py_None ? std::pow(static_cast<double>(c->desc.head_dim), -0.5) : PyFloat_AS_DOUBLE(a[7]);
        const stepq_cache_attn_desc d{static_cast<int32_t>(n), static_cast<int32_t>(Hq), static_cast<int32_t>(m), code_of(dt),
                                      static_cast<int32_t>(S), static_cast<float>(scale)};
        size_t bytes = 0;
        stepq_status e = g.cache_attention_workspace(&c->desc, &d, &bytes);
        if (e != STEPQ_OK) return e;
        if (!take_stream(Py_None, &st)) return -1;
        const at::Tensor ws = bytes ? space(bytes, p.device) : at::Tensor();
        void *wp = bytes ? ws.data_ptr() : nullptr;
        Py_BEGIN_ALLOW_THREADS;
        e = g.cache_attention(&c->desc, &d, c->memory, qp, static_cast<const int32_t *>(tp), static_cast<const int32_t *>(lp),
                              static_cast<const int32_t *>(sp), op, static_cast<float *>(ep), wp, bytes, st);
        Py_END_ALLOW_THREADS;
        return e;
    });
}

// cache_bounds(cache, page_table, starts, lengths, bounds, stream)
PyObject *py_cache_bounds(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded([&]() -> long {
        Plain p{};
        const CachePlain *c = n_args == 6 ? cache_of(a[0], &p) : nullptr;
        int64_t n, m;
        void *tp, *sp, *lp, *bp, *st;
        if (!c || !take_table(a[1], p, &n, &m, &tp) || !take(a[2], p, at::kInt, {n}, &sp) || !take(a[3], p, at::kInt, {n}, &lp) ||
            !take(a[4], p, at::kBFloat16, {c->desc.n_pages, c->desc.n_kv_heads, 2, c->desc.head_dim}, &bp) ||
            !take_stream(a[5], &st))
            return -1;
        stepq_status e;
        Py_BEGIN_ALLOW_THREADS;
        e = g.cache_bounds(&c->desc, c->memory, static_cast<int32_t>(n), static_cast<int32_t>(m), static_cast<const int32_t *>(tp),
                           static_cast<const int32_t *>(sp), static_cast<const int32_t *>(lp), bp, st);
        Py_END_ALLOW_THREADS;
        return e;
    });
}

// cache_select(cache, q, bounds, page_table, lengths, selected, n_first, n_last): on the current stream, in torch's memory
PyObject *py_cache_select(PyObject *, PyObject *const *a, Py_ssize_t n_args)
{
    return guarded([&]() -> long {
        Plain p{};
        const CachePlain *c = n_args == 8 ? cache_of(a[0], &p) : nullptr;
        int64_t n, m, Hq, S, first, last;
        at::ScalarType dt;
        void *tp, *qp, *lp, *bp, *sp, *st;
        if (!c || !take_table(a[3], p, &n, &m, &tp) || !take_query(a[1], p, *c, n, &Hq, &dt, &qp) ||
            !take(a[2], p, at::kBFloat16, {c->desc.n_pages, c->desc.n_kv_heads, 2, c->desc.head_dim}, &bp) ||
            !take(a[4], p, at::kInt, {n}, &lp) || !take_selected(a[5], p, *c, n, &S, &sp) || !take_int(a[6], &first) ||
            !take_int(a[7], &last))
            return -1;
        const stepq_cache_select_desc d{static_cast<int32_t>(n), static_cast<int32_t>(Hq), static_cast<int32_t>(m), code_of(dt),
                                        static_cast<int32_t>(S), static_cast<int32_t>(first), static_cast<int32_t>(last)};
        size_t bytes = 0;
        stepq_status e = g.cache_select_workspace(&c->desc, &d, &bytes);
        if (e != STEPQ_OK) return e;
        if (!take_stream(Py_None, &st)) return -1;
        const at::Tensor ws = bytes ? space(bytes, p.device) : at::Tensor();
        void *wp = bytes ? ws.data_ptr() : nullptr;
        Py_BEGIN_ALLOW_THREADS;
        e = g.cache_select(&c->desc, &d, bp, qp, static_cast<const int32_t *>(tp), static_cast<const int32_t *>(lp),
                           static_cast<int32_t *>(sp), wp, bytes, st);
        Py_END_ALLOW_THREADS;
        return e;
    });
}

PyMethodDef methods[] = {
    {"bind", py_bind, METH_VARARGS, "addresses of the C calls, torch's raw stream query and stream class"},
    {"plain", py_plain, METH_VARARGS, "a pool's handle, device and sizes"},
    {"decode", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(py_decode)), METH_FASTCALL, "one decode step"},
    {"scaled", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(py_scaled)), METH_FASTCALL,
     "load, import or export"},
    {"tiles", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(py_tiles)), METH_FASTCALL,
     "dequant, export or import of pivot rows"},
    {"bind_calls", py_bind_calls, METH_VARARGS, "addresses of the C calls that need no pool"},
    {"state_step", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(py_state_step)), METH_FASTCALL,
     "one token on full-precision states"},
    {"prompt", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(py_prompt)), METH_FASTCALL, "packed prompts"},
    {"attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(py_attention)), METH_FASTCALL,
     "attention over a shared prefix"},
    {"bind_caches", py_bind_caches, METH_VARARGS, "addresses of the C calls on quantized caches"},
    {"cache", py_cache, METH_VARARGS, "a cache's sizes, device and memory"},
    {"cache_rows", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(py_cache_rows)), METH_FASTCALL,
     "tokens written or read back"},
    {"cache_attention", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(py_cache_attention)), METH_FASTCALL,
     "attention over a cache"},
    {"cache_bounds", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(py_cache_bounds)), METH_FASTCALL,
     "bounds of pages' keys"},
    {"cache_select", reinterpret_cast<PyCFunction>(reinterpret_cast<void *>(py_cache_select)), METH_FASTCALL,
     "pages by their scores"},
    {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_stepq_args", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__stepq_args(void) { return PyModule_Create(&module); }
