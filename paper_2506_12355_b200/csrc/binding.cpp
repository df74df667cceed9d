// CPython module `_binding`: argument marshalling of the small, latency-bound entry points in C++.
//
// The operators around the attention kernels run for a few microseconds in a serving step, and marshalling a call's dozen
// tensors in Python costs several times that (17 - 24 us of host time a call; 6 - 10 us through this module).  A function here
// handles the plain case: CUDA tensors of the current device with the expected types, shapes and layouts.  It returns the
// outputs, or the status code of the C entry point as an int, or NotImplemented for anything that is not the plain case;
// api.py then goes through its own checks, which say what is wrong or make the call all the same.
// Nothing is computed here: the C entry points of libattn_fwd.so, whose addresses api.py hands over in bind(), do the work.
#define PY_SSIZE_T_CLEAN
#include <Python.h>
#include <ATen/ATen.h>
#include <c10/cuda/CUDAFunctions.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "../../include/attn_fwd.h"

namespace {

struct Entries {
    decltype(&attn_qk_norm_rope) norm_rope;
    decltype(&attn_qk_norm_rope_bwd) norm_rope_bwd;
    decltype(&attn_qk_norm_rope_bwd_workspace_bytes) norm_rope_bwd_bytes;
    decltype(&attn_paged_append) append;
    decltype(&attn_paged_decode) decode;
    decltype(&attn_paged_decode_workspace_bytes) decode_bytes;
    decltype(&attn_fwd_window) fwd_window;
    decltype(&attn_bwd_window) bwd_window;
    decltype(&attn_bwd_window_workspace_bytes) bwd_window_bytes;
} fn = {};

using at::Tensor;

// Thrown (and caught in guarded() below) where a call is not the plain case.
struct NotPlain {};

void need(bool ok) {
    if (!ok) throw NotPlain();
}

// An argument that is a tensor, or None.
const Tensor* tensor(PyObject* o) {
    if (o == Py_None) return nullptr;
    need(THPVariable_Check(o));
    return &THPVariable_Unpack(o);
}

const Tensor& required(PyObject* o) {
    const Tensor* t = tensor(o);
    need(t != nullptr);
    return *t;
}

int integer(PyObject* o) {
    need(PyLong_Check(o));
    int overflow = 0;
    const long v = PyLong_AsLongAndOverflow(o, &overflow);
    need(!overflow && v >= INT32_MIN && v <= INT32_MAX);
    return static_cast<int>(v);
}

float number(PyObject* o) {
    need(PyFloat_Check(o) || PyLong_Check(o));
    const double v = PyFloat_AsDouble(o);
    if (v == -1.0 && PyErr_Occurred()) {
        PyErr_Clear();
        throw NotPlain();
    }
    return static_cast<float>(v);
}

// An argument's truth value; one that has none (an array of several) goes to the Python path, which raises what Python raises.
int truth(PyObject* o) {
    const int v = PyObject_IsTrue(o);
    if (v < 0) {
        PyErr_Clear();
        throw NotPlain();
    }
    return v;
}

// What the tensors of one call have in common.
struct Call {
    c10::DeviceIndex device;
    at::ScalarType type;
    int dtype;
    void* stream;
    explicit Call(const Tensor& x) {
        need(x.is_cuda());
        device = x.get_device();
        need(device == c10::cuda::current_device());
        type = x.scalar_type();
        need(type == at::kHalf || type == at::kBFloat16);
        dtype = type == at::kHalf ? ATTN_DTYPE_FP16 : ATTN_DTYPE_BF16;
        stream = c10::cuda::getCurrentCUDAStream(device).stream();
    }
    void check(const Tensor& t, at::IntArrayRef shape, at::ScalarType want, bool dense) const {
        need(t.is_cuda() && t.get_device() == device && t.scalar_type() == want && t.sizes() == shape);
        need(dense ? t.is_contiguous() : (shape.empty() || shape.back() <= 1 || t.strides().back() == 1));
    }
    void check(const Tensor& t, at::IntArrayRef shape, bool dense) const { check(t, shape, type, dense); }
    Tensor make(at::IntArrayRef shape, at::ScalarType want) const {
        return at::empty(shape, at::TensorOptions().dtype(want).device(at::kCUDA, device));
    }
    Tensor make(at::IntArrayRef shape) const { return make(shape, type); }
    // the caller's output, checked, or a new one
    Tensor output(const Tensor* t, at::IntArrayRef shape, at::ScalarType want, bool dense = true) const {
        if (!t) return make(shape, want);
        check(*t, shape, want, dense);
        return *t;
    }
    Tensor output(const Tensor* t, at::IntArrayRef shape, bool dense = true) const { return output(t, shape, type, dense); }
    Tensor workspace(const Tensor* t, size_t bytes) const {
        if (!t) return make({static_cast<int64_t>(bytes < 256 ? 256 : bytes)}, at::kByte);
        need(t->is_cuda() && t->get_device() == device && t->is_contiguous());
        return *t;
    }
};

void* ptr(const Tensor* t) { return t ? t->data_ptr() : nullptr; }

int small(int64_t v) {
    need(v >= 0 && v <= INT32_MAX);
    return static_cast<int>(v);
}

// Weights [D] of one type and the table [positions, R].
struct Rope {
    const Tensor *qw, *kw, *table;
    int f32 = 0, len = 0, R = 0;
    Rope(const Call& c, int64_t D, PyObject* q_weight, PyObject* k_weight, PyObject* cos_sin)
        : qw(tensor(q_weight)), kw(tensor(k_weight)), table(tensor(cos_sin)) {
        const Tensor* any = qw ? qw : kw;
        f32 = any && any->scalar_type() == at::kFloat;
        const at::ScalarType want = f32 ? at::kFloat : c.type;
        if (qw) c.check(*qw, {D}, want, true);
        if (kw) c.check(*kw, {D}, want, true);
        if (table) {
            need(table->dim() == 2);
            c.check(*table, table->sizes(), at::kFloat, true);
            len = small(table->size(0));
            R = small(table->size(1));
        }
    }
};

void strides3(long long* to, const Tensor* t) {
    for (int i = 0; i < 3; ++i) to[i] = t ? t->stride(i) : 0;
}

// Caches [pages, Hkv, page_size, D], block table [n, width] and lengths [n].
struct Cache {
    const Tensor &k, &v, &table, &lens;
    long long strides[6];
    int pages, heads, page_size, n, width;
    Cache(const Call& c, int64_t D, PyObject* k_cache, PyObject* v_cache, PyObject* block_table, PyObject* seq_lens)
        : k(required(k_cache)), v(required(v_cache)), table(required(block_table)), lens(required(seq_lens)) {
        need(k.dim() == 4 && k.size(3) == D && table.dim() == 2 && lens.dim() == 1);
        c.check(k, k.sizes(), false);
        c.check(v, k.sizes(), false);
        c.check(table, {lens.size(0), table.size(1)}, at::kInt, false);
        c.check(lens, {lens.size(0)}, at::kInt, true);
        strides3(strides, &k);
        strides3(strides + 3, &v);
        pages = small(k.size(0));
        heads = small(k.size(1));
        page_size = small(k.size(2));
        n = small(lens.size(0));
        width = small(table.size(1));
    }
};

PyObject* status(int rc) { return PyLong_FromLong(rc); }

PyObject* wrap(const Tensor& t) { return THPVariable_Wrap(t); }

PyObject* tuple(std::initializer_list<const Tensor*> ts) {
    PyObject* r = PyTuple_New(static_cast<Py_ssize_t>(ts.size()));
    if (!r) return nullptr;
    Py_ssize_t i = 0;
    for (const Tensor* t : ts) {
        PyObject* o = t ? wrap(*t) : Py_NewRef(Py_None);
        if (!o) {
            Py_DECREF(r);
            return nullptr;
        }
        PyTuple_SET_ITEM(r, i++, o);
    }
    return r;
}

// attn_qk_norm_rope(q, k, v, q_weight, k_weight, cos_sin, positions, eps, interleaved, q_out, k_out, v_out)
PyObject* norm_rope(PyObject* const* a) {
    const Tensor &q = required(a[0]), &k = required(a[1]);
    const Tensor *v = tensor(a[2]), *pos = tensor(a[6]);
    need(q.dim() == 4 && k.dim() == 4);
    const int64_t B = q.size(0), S = q.size(1), H = q.size(2), D = q.size(3), Hkv = k.size(2);
    const Call c(q);
    c.check(q, q.sizes(), false);
    c.check(k, {B, S, Hkv, D}, false);
    if (v) c.check(*v, {B, S, Hkv, D}, false);
    const Rope r(c, D, a[3], a[4], a[5]);
    if (pos) c.check(*pos, {B, S}, at::kInt, true);
    const Tensor qo = c.output(tensor(a[9]), {B, H, S, D}), ko = c.output(tensor(a[10]), {B, Hkv, S, D});
    Tensor vo;
    if (v) vo = c.output(tensor(a[11]), {B, Hkv, S, D});
    long long st[9];
    strides3(st, &q);
    strides3(st + 3, &k);
    strides3(st + 6, v);
    const int rc = fn.norm_rope(q.data_ptr(), k.data_ptr(), ptr(v), st, ptr(r.qw), ptr(r.kw), r.f32, static_cast<const float*>(ptr(r.table)), r.len,
                                r.R, truth(a[8]), static_cast<const int*>(ptr(pos)), number(a[7]), qo.data_ptr(), ko.data_ptr(),
                                v ? vo.data_ptr() : nullptr, small(B), small(S), small(H), small(Hkv), small(D), c.dtype, c.stream);
    return rc ? status(rc) : tuple({&qo, &ko, v ? &vo : nullptr});
}

// attn_qk_norm_rope_bwd(dq, dk, dv, q, k, q_weight, k_weight, cos_sin, positions, eps, interleaved, dq_in, dk_in, dv_in, workspace)
PyObject* norm_rope_bwd(PyObject* const* a) {
    const Tensor &dq = required(a[0]), &dk = required(a[1]), &q = required(a[3]), &k = required(a[4]);
    const Tensor *dv = tensor(a[2]), *pos = tensor(a[8]);
    need(q.dim() == 4 && k.dim() == 4);
    const int64_t B = q.size(0), S = q.size(1), H = q.size(2), D = q.size(3), Hkv = k.size(2);
    const Call c(q);
    c.check(q, q.sizes(), false);
    c.check(k, {B, S, Hkv, D}, false);
    c.check(dq, {B, H, S, D}, true);
    c.check(dk, {B, Hkv, S, D}, true);
    if (dv) c.check(*dv, {B, Hkv, S, D}, true);
    const Rope r(c, D, a[5], a[6], a[7]);
    if (pos) c.check(*pos, {B, S}, at::kInt, true);
    const Tensor qi = c.output(tensor(a[11]), {B, S, H, D}, false), ki = c.output(tensor(a[12]), {B, S, Hkv, D}, false);
    Tensor vi, qw, kw;
    if (dv) vi = c.output(tensor(a[13]), {B, S, Hkv, D}, false);
    if (r.qw) qw = c.make({D}, at::kFloat);
    if (r.kw) kw = c.make({D}, at::kFloat);
    const Tensor ws = c.workspace(tensor(a[14]), fn.norm_rope_bwd_bytes(small(D)));
    long long in[6], out[9];
    strides3(in, &q);
    strides3(in + 3, &k);
    strides3(out, &qi);
    strides3(out + 3, &ki);
    strides3(out + 6, dv ? &vi : nullptr);
    const int rc = fn.norm_rope_bwd(dq.data_ptr(), dk.data_ptr(), ptr(dv), q.data_ptr(), k.data_ptr(), in, ptr(r.qw), ptr(r.kw), r.f32,
                                    static_cast<const float*>(ptr(r.table)), r.len, r.R, truth(a[10]),
                                    static_cast<const int*>(ptr(pos)), number(a[9]), qi.data_ptr(), ki.data_ptr(),
                                    dv ? vi.data_ptr() : nullptr, out, r.qw ? qw.data_ptr<float>() : nullptr,
                                    r.kw ? kw.data_ptr<float>() : nullptr, small(B), small(S), small(H), small(Hkv), small(D), c.dtype,
                                    ws.data_ptr(), ws.nbytes(), c.stream);
    return rc ? status(rc) : tuple({&qi, &ki, dv ? &vi : nullptr, r.qw ? &qw : nullptr, r.kw ? &kw : nullptr});
}

// attn_paged_append(q, k, v, k_cache, v_cache, block_table, seq_lens, q_weight, k_weight, cos_sin, cu_seqlens, eps, interleaved, q_out)
PyObject* append(PyObject* const* a) {
    const Tensor &k = required(a[1]), &v = required(a[2]);
    const Tensor *q = tensor(a[0]), *cu = tensor(a[10]);
    need(q && k.dim() == 3 && q->dim() == 3);
    const int64_t T = k.size(0), Hkv = k.size(1), D = k.size(2), H = q->size(1);
    const Call c(k);
    c.check(k, k.sizes(), false);
    c.check(v, k.sizes(), false);
    c.check(*q, {T, H, D}, false);
    const Rope r(c, D, a[7], a[8], a[9]);
    const Cache m(c, D, a[3], a[4], a[5], a[6]);
    need(m.heads == Hkv && (cu || T == m.n));
    if (cu) c.check(*cu, {m.n + 1}, at::kInt, true);
    const Tensor qo = c.output(tensor(a[13]), {T, H, D});
    const long long st[6] = {q->stride(0), q->stride(1), k.stride(0), k.stride(1), v.stride(0), v.stride(1)};
    const int rc = fn.append(q->data_ptr(), k.data_ptr(), v.data_ptr(), st, ptr(r.qw), ptr(r.kw), r.f32, static_cast<const float*>(ptr(r.table)),
                             r.len, r.R, truth(a[12]), number(a[11]), qo.data_ptr(), m.k.data_ptr(), m.v.data_ptr(), m.strides,
                             m.pages, m.page_size, m.table.data_ptr<int>(), m.table.stride(0), m.width, m.lens.data_ptr<int>(),
                             static_cast<const int*>(ptr(cu)), m.n, small(T), small(H), small(Hkv), small(D), c.dtype, c.stream);
    return rc ? status(rc) : wrap(qo);
}

// attn_paged_decode(q, k_cache, v_cache, block_table, seq_lens, scale, window, sinks, out, lse, workspace)
PyObject* decode(PyObject* const* a) {
    const Tensor& q = required(a[0]);
    need(q.dim() == 3);
    const int64_t B = q.size(0), H = q.size(1), D = q.size(2);
    const Call c(q);
    c.check(q, q.sizes(), true);
    const Cache m(c, D, a[1], a[2], a[3], a[4]);
    need(m.n == B);
    const Tensor o = c.output(tensor(a[8]), {B, H, D}), lse = c.output(tensor(a[9]), {B, H}, at::kFloat);
    const Tensor ws = c.workspace(tensor(a[10]), fn.decode_bytes(small(H), m.heads, small(D)));
    const int rc = fn.decode(q.data_ptr(), m.k.data_ptr(), m.v.data_ptr(), m.strides, m.pages, m.page_size, m.table.data_ptr<int>(),
                             m.table.stride(0), m.width, m.lens.data_ptr<int>(), o.data_ptr(), lse.data_ptr<float>(), small(B), small(H),
                             m.heads, small(D), number(a[5]), integer(a[6]), integer(a[7]), c.dtype, ws.data_ptr(), ws.nbytes(), c.stream);
    return rc ? status(rc) : tuple({&o, &lse});
}

struct Heads {
    int64_t B, H, Hkv, Sq, Sk, D;
    Heads(const Call& c, const Tensor& q, const Tensor& k, const Tensor& v) {
        need(q.dim() == 4 && k.dim() == 4);
        B = q.size(0); H = q.size(1); Sq = q.size(2); D = q.size(3); Hkv = k.size(1); Sk = k.size(2);
        c.check(q, q.sizes(), true);
        c.check(k, {B, Hkv, Sk, D}, true);
        c.check(v, {B, Hkv, Sk, D}, true);
    }
};

// attn_fwd_window(q, k, v, scale, window, sinks, q_offset, out, lse)
PyObject* fwd_window(PyObject* const* a) {
    const Tensor &q = required(a[0]), &k = required(a[1]), &v = required(a[2]);
    const Call c(q);
    const Heads h(c, q, k, v);
    const Tensor o = c.output(tensor(a[7]), {h.B, h.H, h.Sq, h.D}), lse = c.output(tensor(a[8]), {h.B, h.H, h.Sq}, at::kFloat);
    const int rc = fn.fwd_window(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr<float>(), small(h.B), small(h.H),
                                 small(h.Hkv), small(h.Sq), small(h.Sk), small(h.D), number(a[3]), integer(a[4]), integer(a[5]),
                                 integer(a[6]), c.dtype, c.stream);
    return rc ? status(rc) : tuple({&o, &lse});
}

// attn_bwd_window(q, k, v, o, lse, dout, scale, window, sinks, q_offset, dq, dk, dv, workspace)
PyObject* bwd_window(PyObject* const* a) {
    const Tensor &q = required(a[0]), &k = required(a[1]), &v = required(a[2]), &o = required(a[3]), &lse = required(a[4]), &dout = required(a[5]);
    const Call c(q);
    const Heads h(c, q, k, v);
    c.check(o, q.sizes(), true);
    c.check(dout, q.sizes(), true);
    c.check(lse, {h.B, h.H, h.Sq}, at::kFloat, true);
    const int W = integer(a[7]), sinks = integer(a[8]), off = integer(a[9]);
    const Tensor dq = c.output(tensor(a[10]), q.sizes()), dk = c.output(tensor(a[11]), k.sizes()), dv = c.output(tensor(a[12]), k.sizes());
    const Tensor ws = c.workspace(tensor(a[13]), fn.bwd_window_bytes(small(h.B), small(h.H), small(h.Hkv), small(h.Sq), small(h.Sk), small(h.D),
                                                                     W, sinks, off));
    const int rc = fn.bwd_window(q.data_ptr(), k.data_ptr(), v.data_ptr(), o.data_ptr(), lse.data_ptr<float>(), dout.data_ptr(), dq.data_ptr(),
                                 dk.data_ptr(), dv.data_ptr(), small(h.B), small(h.H), small(h.Hkv), small(h.Sq), small(h.Sk), small(h.D),
                                 number(a[6]), W, sinks, off, c.dtype, ws.data_ptr(), ws.nbytes(), c.stream);
    return rc ? status(rc) : tuple({&dq, &dk, &dv});
}

// No C++ exception crosses into the interpreter: a call that is not plain, and one in which torch raised something (an
// allocation that failed, say), both go to the Python path, which meets the same condition and reports it.
template <PyObject* (*F)(PyObject* const*), int N>
PyObject* guarded(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != N || !fn.norm_rope) return Py_NewRef(Py_NotImplemented);
    try {
        return F(args);
    } catch (...) {
        return Py_NewRef(Py_NotImplemented);
    }
}

// bind(addresses): the C entry points, in the order of Entries.
PyObject* bind(PyObject*, PyObject* list) {
    constexpr Py_ssize_t count = sizeof(Entries) / sizeof(void*);
    if (!PyList_Check(list) || PyList_GET_SIZE(list) != count) {
        PyErr_SetString(PyExc_ValueError, "bind() takes the list of entry points");
        return nullptr;
    }
    void* address[count];
    for (Py_ssize_t i = 0; i < count; ++i) {
        address[i] = PyLong_AsVoidPtr(PyList_GET_ITEM(list, i));
        if (!address[i]) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "bind(): a missing entry point");
            return nullptr;
        }
    }
    memcpy(&fn, address, sizeof(fn));
    Py_RETURN_NONE;
}

template <PyObject* (*F)(PyObject* const*), int N>
PyCFunction fast() {
    return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(&guarded<F, N>));
}

PyMethodDef methods[] = {
    {"bind", bind, METH_O, nullptr},
    {"attn_qk_norm_rope", fast<norm_rope, 12>(), METH_FASTCALL, nullptr},
    {"attn_qk_norm_rope_bwd", fast<norm_rope_bwd, 15>(), METH_FASTCALL, nullptr},
    {"attn_paged_append", fast<append, 14>(), METH_FASTCALL, nullptr},
    {"attn_paged_decode", fast<decode, 11>(), METH_FASTCALL, nullptr},
    {"attn_fwd_window", fast<fwd_window, 9>(), METH_FASTCALL, nullptr},
    {"attn_bwd_window", fast<bwd_window, 14>(), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_binding", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__binding() { return PyModule_Create(&module); }
