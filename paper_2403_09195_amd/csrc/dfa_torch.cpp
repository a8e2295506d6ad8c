// The host side of one call of the library on torch tensors (dfa_forward, dfa_backward, the operators on 8-bit operands), in native code: checks, allocation of
// the results and the workspace, the current stream.  Small launches wait for their host side: one 256^2 image took 10.9 us a call in Python and ctypes (two
// torch.empty 3.5 us, marshalling 2.3, the ctypes call's own conversions 1) around 2.4 us of launch and 6.6 us on the GPU; its backward
// 16.0 (four torch.empty, six checked tensors), 9.1 this way, which is the GPU's time (forward and backward 21.0 / 15.8).
//
// Only the ordinary call goes this way: 4-d GPU tensors of one dtype with contiguous last dimension, lists of Python integers.  Anything else
// is handed back (None) to the binding's function of that name, which converts it or names what is wrong with it.
// The operators on 8-bit operands: us a call on the host, in Python / here: one row projected 13.1 / 5.0, gradients of a projection 31.5 / 10.4, a token
// appended 12.9 / 5.0, one row's attention 20.9 / 9.1.
#include <Python.h>
#include <pybind11/pybind11.h>
#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>
#include <ATen/ATen.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include "../../include/dfa.h"

namespace {

using ForwardAlloc = decltype(&dfa_forward_alloc);
using Backward = decltype(&dfa_backward);
ForwardAlloc g_forward = nullptr;
Backward g_backward = nullptr;

struct Library {                               // of the operators on 8-bit operands
    decltype(&dfa_quantized_linear) linear;
    decltype(&dfa_quantized_linear_workspace_bytes) linear_bytes;
    decltype(&dfa_quantized_linear_backward) linear_backward;
    decltype(&dfa_quantized_linear_backward_workspace_bytes) linear_backward_bytes;
    decltype(&dfa_cache_append) append;
    decltype(&dfa_cache_attention) attention;
    decltype(&dfa_cache_attention_workspace_bytes) attention_bytes;
};
Library g_lib = {};

constexpr int kMaxOffsets = 1024;

// A Python list or tuple; the items are borrowed.
struct Sequence {
    PyObject** items = nullptr;
    Py_ssize_t n = -1;
    explicit Sequence(PyObject* o) {
        if (PyList_CheckExact(o) || PyTuple_CheckExact(o)) {
            items = PySequence_Fast_ITEMS(o);
            n = PySequence_Fast_GET_SIZE(o);
        }
    }
};

bool as_int32(PyObject* o, int32_t* out) {
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    const long x = PyLong_AsLongAndOverflow(o, &overflow);
    if (overflow || x != (int32_t)x) return false;
    *out = (int32_t)x;
    return true;
}

// What the workspace callback needs, and what it leaves: the tensor lives until the call has enqueued its launches.
// (Allocated on the current stream: the allocator gives its memory to later work of this stream only.)
struct Workspace {
    const at::TensorOptions options;
    at::Tensor tensor;
    std::exception_ptr error;
};
void* allocate(void* context, size_t bytes) {
    Workspace* w = static_cast<Workspace*>(context);
    try {
        w->tensor = at::empty({(int64_t)bytes}, w->options);
        return w->tensor.data_ptr();
    } catch (...) {
        w->error = std::current_exception();
        return nullptr;
    }
}

// What both calls take, as the library reads it.
struct Call {
    const at::Tensor* t[3];                    // q, k, v
    dfa_strides_t s[3];
    dfa_dtype_t dtype;
    int64_t B, N, H, D;
    dfa_branch_t branches[DFA_MAX_BRANCHES];
    int32_t nb;
    float scale;
    int32_t table[kMaxOffsets];
    const int32_t* offsets;                    // table or NULL
};

// Reads q, k, v and branches, scale, head_offsets; false: not the ordinary call.
bool read_call(PyObject* const* qkv, PyObject* const* rest, Call* c) {
    for (int i = 0; i < 3; ++i) {
        if (!THPVariable_CheckExact(qkv[i])) return false;
        c->t[i] = &THPVariable_Unpack(qkv[i]);
        if (!c->t[i]->is_cuda() || c->t[i]->dim() != 4 || c->t[i]->stride(3) != 1) return false;
        c->s[i] = dfa_strides_t{c->t[i]->stride(0), c->t[i]->stride(1), c->t[i]->stride(2)};
    }
    const at::Tensor& q = *c->t[0];
    const at::ScalarType type = q.scalar_type();
    if (type != at::kBFloat16 && type != at::kFloat) return false;
    c->dtype = type == at::kFloat ? DFA_F32 : DFA_BF16;
    for (int i = 1; i < 3; ++i) {              // nor less than q, which the kernels would read past (the binding refuses it)
        if (c->t[i]->scalar_type() != type) return false;
        for (int d = 0; d < 4; ++d)
            if (c->t[i]->size(d) < q.size(d)) return false;
    }
    c->B = q.size(0), c->N = q.size(1), c->H = q.size(2), c->D = q.size(3);
    if (c->B > INT32_MAX || c->N > INT32_MAX || c->H > INT32_MAX || c->D > INT32_MAX) return false;

    const Sequence list(rest[0]);
    if (list.n < 1 || list.n > DFA_MAX_BRANCHES) return false;
    c->nb = (int32_t)list.n;
    for (Py_ssize_t i = 0; i < list.n; ++i) {
        const Sequence pair(list.items[i]);
        if (pair.n != 2 || !as_int32(pair.items[0], &c->branches[i].w) || !as_int32(pair.items[1], &c->branches[i].r)) return false;
    }
    if (!PyFloat_CheckExact(rest[1])) return false;
    c->scale = (float)PyFloat_AS_DOUBLE(rest[1]);

    c->offsets = nullptr;
    if (rest[2] != Py_None) {
        const Sequence rows(rest[2]);
        if (rows.n != list.n || list.n * c->H > kMaxOffsets) return false;
        for (Py_ssize_t i = 0; i < rows.n; ++i) {
            const Sequence row(rows.items[i]);
            if (row.n != c->H) return false;
            for (Py_ssize_t h = 0; h < row.n; ++h)
                if (!as_int32(row.items[h], &c->table[i * c->H + h])) return false;
        }
        c->offsets = c->table;
    }
    return true;
}

// Whether contiguous t, read as a contiguous array of the n sizes `want`, has the elements of t[:want[0], :want[1], ...]; with another number of
// dimensions, as many elements in this order.  (The kernels would read past the end of less.)
bool holds(const at::Tensor& t, const int64_t* want, int64_t n) {
    int64_t stride = 1;
    bool same = t.dim() == n;
    for (int64_t d = n - 1; d >= 0; --d) {
        same = same && t.size(d) >= want[d] && (want[d] == 1 || t.stride(d) == stride);
        stride *= want[d];
    }
    return t.dim() == n ? same : t.numel() >= stride;
}

// A tuple of tensors, which are given up.
template <size_t n>
PyObject* as_tuple(at::Tensor (&t)[n]) {
    PyObject* const tuple = PyTuple_New((Py_ssize_t)n);
    if (!tuple) return nullptr;
    for (size_t i = 0; i < n; ++i) {
        PyObject* const o = THPVariable_Wrap(std::move(t[i]));
        if (!o) {
            Py_DECREF(tuple);
            return nullptr;
        }
        PyTuple_SET_ITEM(tuple, (Py_ssize_t)i, o);
    }
    return tuple;
}

// forward(q, k, v, branches, scale, head_offsets) -> (out, lse), a negative status, or None
PyObject* forward(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    Call c;
    if (nargs != 6 || !g_forward || !read_call(args, args + 3, &c)) Py_RETURN_NONE;
    const at::Tensor& q = *c.t[0];
    at::Tensor res[2] = {at::empty({c.B, c.N, c.H, c.D}, q.options()), at::empty({c.B, c.H, c.N}, q.options().dtype(at::kFloat))};
    Workspace ws{q.options().dtype(at::kByte), at::Tensor(), nullptr};
    const void *const qp = q.data_ptr(), *const kp = c.t[1]->data_ptr(), *const vp = c.t[2]->data_ptr();
    int rc;
    {
        // Other threads run meanwhile: a shape's first call builds and uploads its plan, a dropped plan waits for the device, a
        // launch may wait for the queue.  (No Python object is touched; the workspace callback needs none either.)
        pybind11::gil_scoped_release release;
        rc = g_forward(qp, kp, vp, c.s[0], c.s[1], c.s[2], (int32_t)c.B, (int32_t)c.H, (int32_t)c.N, (int32_t)c.D, c.dtype, c.scale, c.branches, c.nb,
                       c.offsets, res[0].data_ptr(), res[1].data_ptr<float>(), allocate, &ws, c10::hip::getCurrentHIPStream().stream());
    }
    if (ws.error) std::rethrow_exception(ws.error);
    if (rc != DFA_OK) return PyLong_FromLong(rc);
    return as_tuple(res);
    END_HANDLE_TH_ERRORS
}

// backward(q, k, v, out, lse, dout, branches, scale, head_offsets) -> (dq, dk, dv), a negative status, or None
PyObject* backward(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    Call c;
    if (nargs != 9 || !g_backward || !read_call(args, args + 6, &c)) Py_RETURN_NONE;
    const at::Tensor& q = *c.t[0];
    const at::Tensor* x[3];                    // out, lse, dout
    const int64_t rows[4] = {c.B, c.N, c.H, c.D}, stats[3] = {c.B, c.H, c.N};
    for (int i = 0; i < 3; ++i) {
        if (!THPVariable_CheckExact(args[3 + i])) Py_RETURN_NONE;
        x[i] = &THPVariable_Unpack(args[3 + i]);
        if (!x[i]->is_cuda() || !x[i]->is_contiguous() || x[i]->scalar_type() != (i == 1 ? at::kFloat : q.scalar_type())) Py_RETURN_NONE;
        if (!(i == 1 ? holds(*x[i], stats, 3) : holds(*x[i], rows, 4))) Py_RETURN_NONE;
    }
    at::Tensor res[3];
    for (at::Tensor& r : res) r = at::empty({c.B, c.N, c.H, c.D}, q.options());
    // (allocated on the current stream: the allocator gives its memory to later work of this stream only)
    at::Tensor delta = at::empty({2, c.B, c.H, c.N}, q.options().dtype(at::kFloat));
    const void *const qp = q.data_ptr(), *const kp = c.t[1]->data_ptr(), *const vp = c.t[2]->data_ptr();
    int rc;
    {
        pybind11::gil_scoped_release release;  // as in forward
        rc = g_backward(qp, kp, vp, x[0]->data_ptr(), x[1]->data_ptr<float>(), x[2]->data_ptr(), c.s[0], c.s[1], c.s[2], (int32_t)c.B, (int32_t)c.H,
                        (int32_t)c.N, (int32_t)c.D, c.dtype, c.scale, c.branches, c.nb, c.offsets, delta.data_ptr<float>(), res[0].data_ptr(),
                        res[1].data_ptr(), res[2].data_ptr(), c10::hip::getCurrentHIPStream().stream());
    }
    if (rc != DFA_OK) return PyLong_FromLong(rc);
    return as_tuple(res);
    END_HANDLE_TH_ERRORS
}

// ---- the operators on 8-bit operands ----------------------------------------------------------------------------------------

// A tensor on the current device, or nullptr.
const at::Tensor* device_tensor(PyObject* o) {
    if (!THPVariable_CheckExact(o)) return nullptr;
    const at::Tensor& t = THPVariable_Unpack(o);
    return t.is_cuda() && t.get_device() == c10::hip::current_device() ? &t : nullptr;
}

bool float_type(const at::Tensor& t, dfa_dtype_t* dt) {
    const at::ScalarType type = t.scalar_type();
    *dt = type == at::kFloat ? DFA_F32 : DFA_BF16;
    return type == at::kFloat || type == at::kBFloat16;
}

int64_t up(int64_t n, int64_t of) { return (n + of - 1) / of * of; }

// A binding.QuantizedMatrix whose arrays hold what its shape says.
struct Matrix {
    dfa_quantized_t q;
    int64_t rows, cols;
};
bool read_matrix(PyObject* o, Matrix* m) {
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 3) return false;
    const at::Tensor *v = device_tensor(PyTuple_GET_ITEM(o, 0)), *s = device_tensor(PyTuple_GET_ITEM(o, 1));
    int32_t cols;
    if (!v || !s || !as_int32(PyTuple_GET_ITEM(o, 2), &cols)) return false;
    if (v->scalar_type() != at::kFloat8_e4m3fn || s->scalar_type() != at::kByte || v->dim() != 2 || s->dim() != 2) return false;
    if (!v->is_contiguous() || !s->is_contiguous() || cols < 1) return false;
    m->rows = v->size(0), m->cols = cols;
    const int64_t need = up(cols, 128);
    if (v->size(1) < need || s->size(0) < need / 128 || s->size(1) < up(m->rows, 16)) return false;
    m->q = dfa_quantized_t{v->data_ptr(), s->data_ptr(), v->size(1), s->size(1)};
    return true;
}

// A tensor read as a matrix of its last dimension: contiguous.
bool read_rows(const at::Tensor& t, int64_t* rows, int64_t* cols) {
    if (t.dim() < 1 || !t.is_contiguous() || t.numel() == 0) return false;
    *cols = t.size(t.dim() - 1);
    *rows = t.numel() / *cols;
    return true;
}

at::Tensor with_last(const at::Tensor& t, int64_t cols) {
    c10::SmallVector<int64_t, 5> sizes(t.sizes().begin(), t.sizes().end());
    sizes.back() = cols;
    return at::empty(sizes, t.options());
}

// Room of this many bytes, allocated on the current stream: the allocator gives its memory to later work of this stream only.
struct Room {
    at::Tensor tensor;
    void* ptr = nullptr;
    Room(size_t bytes, const at::Tensor& like) {
        if (!bytes) return;
        tensor = at::empty({(int64_t)bytes}, like.options().dtype(at::kByte));
        ptr = tensor.data_ptr();
    }
};

// quantized_linear(x, w) -> y, a negative status, or None
PyObject* quantized_linear(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    Matrix w;
    dfa_dtype_t dt;
    int64_t M, K;
    const at::Tensor* const x = nargs == 2 ? device_tensor(args[0]) : nullptr;
    if (!x || !g_lib.linear || !float_type(*x, &dt) || !read_rows(*x, &M, &K) || !read_matrix(args[1], &w) || w.cols != K || w.rows < 1) Py_RETURN_NONE;
    at::Tensor y = with_last(*x, w.rows);
    const size_t bytes = g_lib.linear_bytes(dt, M, w.rows, K);
    const Room room(bytes, *x);
    int rc;
    {
        pybind11::gil_scoped_release release;  // as in forward
        rc = g_lib.linear(x->data_ptr(), dt, K, w.q, y.data_ptr(), M, w.rows, K, w.rows, room.ptr, bytes, c10::hip::getCurrentHIPStream().stream());
    }
    return rc != DFA_OK ? PyLong_FromLong(rc) : THPVariable_Wrap(std::move(y));
    END_HANDLE_TH_ERRORS
}

// quantized_linear_backward(dy, x, w_t) -> (dx, dw), a negative status, or None
PyObject* quantized_linear_backward(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    Matrix w;
    dfa_dtype_t dt;
    int64_t M, N, rows, K;
    const at::Tensor *const dy = nargs == 3 ? device_tensor(args[0]) : nullptr, *const x = dy ? device_tensor(args[1]) : nullptr;
    if (!x || !g_lib.linear_backward || !float_type(*dy, &dt) || x->scalar_type() != dy->scalar_type() || !read_rows(*dy, &M, &N) || !read_rows(*x, &rows, &K))
        Py_RETURN_NONE;
    if (rows != M || !read_matrix(args[2], &w) || w.cols != N || w.rows != K) Py_RETURN_NONE;
    at::Tensor res[2] = {with_last(*dy, K), at::empty({N, K}, dy->options().dtype(at::kFloat))};
    const size_t bytes = g_lib.linear_backward_bytes(dt, M, N, K);
    const Room room(bytes, *dy);
    int rc;
    {
        pybind11::gil_scoped_release release;
        rc = g_lib.linear_backward(dy->data_ptr(), N, x->data_ptr(), K, dt, w.q, res[0].data_ptr(), K, res[1].data_ptr<float>(), K, M, N, K, room.ptr, bytes,
                                   c10::hip::getCurrentHIPStream().stream());
    }
    return rc != DFA_OK ? PyLong_FromLong(rc) : as_tuple(res);
    END_HANDLE_TH_ERRORS
}

// A binding.KvCache and what names a call's sequences in it.
struct Sequences {
    dfa_cache_t cache;
    const int32_t *table, *lengths, *counts;
    int32_t width;
    int64_t ld_table;
};
bool read_sequences(PyObject* o, PyObject* table, PyObject* lengths, PyObject* counts, int64_t B, Sequences* s) {
    if (!PyTuple_Check(o) || PyTuple_GET_SIZE(o) != 3) return false;
    const at::Tensor* t[3];
    for (int i = 0; i < 3; ++i) {
        t[i] = device_tensor(PyTuple_GET_ITEM(o, i));
        if (!t[i] || t[i]->scalar_type() != (i < 2 ? at::kFloat8_e4m3fn : at::kByte) || t[i]->dim() != (i < 2 ? 4 : 3) || !t[i]->is_contiguous()) return false;
    }
    for (int d = 0; d < 4; ++d)
        if (t[0]->size(d) > INT32_MAX || t[1]->size(d) != t[0]->size(d < 2 ? d : 5 - d) || (d < 3 && t[2]->size(d) != (d < 2 ? t[0]->size(d) : 2))) return false;
    s->cache = dfa_cache_t{t[0]->data_ptr(), t[1]->data_ptr(), t[2]->data_ptr(), (int32_t)t[0]->size(0), (int32_t)t[0]->size(1), (int32_t)t[0]->size(2),
                           (int32_t)t[0]->size(3)};
    const at::Tensor *const at = device_tensor(table), *const ln = device_tensor(lengths), *const cn = counts == Py_None ? nullptr : device_tensor(counts);
    if (!at || !ln || (counts != Py_None && !cn)) return false;
    if (at->scalar_type() != at::kInt || at->dim() != 2 || at->size(0) != B || at->size(1) < 1 || at->size(1) > INT32_MAX || !at->is_contiguous()) return false;
    for (const at::Tensor* x : {ln, cn})
        if (x && (x->scalar_type() != at::kInt || x->dim() != 1 || x->size(0) != B || !x->is_contiguous())) return false;
    s->table = at->data_ptr<int32_t>(), s->width = (int32_t)at->size(1), s->ld_table = at->size(1);
    s->lengths = ln->data_ptr<int32_t>(), s->counts = cn ? cn->data_ptr<int32_t>() : nullptr;
    return true;
}

// A [B, N, H, D] tensor with contiguous last dimension.
const at::Tensor* row_tensor(PyObject* o, dfa_dtype_t* dt, dfa_strides_t* s) {
    const at::Tensor* const t = device_tensor(o);
    if (!t || !float_type(*t, dt) || t->dim() != 4 || t->stride(3) != 1 || t->numel() == 0) return nullptr;
    for (int d = 0; d < 4; ++d)
        if (t->size(d) > INT32_MAX) return nullptr;
    *s = dfa_strides_t{t->stride(0), t->stride(1), t->stride(2)};
    return t;
}

// cache_append(k, v, cache, table, lengths, counts) -> True, a negative status, or None
PyObject* cache_append(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    dfa_dtype_t dt, other;
    dfa_strides_t sk, sv;
    Sequences s;
    const at::Tensor *const k = nargs == 6 ? row_tensor(args[0], &dt, &sk) : nullptr, *const v = k ? row_tensor(args[1], &other, &sv) : nullptr;
    if (!v || !g_lib.append || dt != other || v->sizes() != k->sizes() || !read_sequences(args[2], args[3], args[4], args[5], k->size(0), &s)) Py_RETURN_NONE;
    if (k->size(2) != s.cache.heads || k->size(3) != s.cache.D) Py_RETURN_NONE;
    int rc;
    {
        pybind11::gil_scoped_release release;
        rc = g_lib.append(k->data_ptr(), v->data_ptr(), sk, sv, dt, (int32_t)k->size(0), (int32_t)k->size(1), s.cache, s.table, s.width, s.ld_table, s.lengths,
                          s.counts, c10::hip::getCurrentHIPStream().stream());
    }
    if (rc != DFA_OK) return PyLong_FromLong(rc);
    Py_RETURN_TRUE;
    END_HANDLE_TH_ERRORS
}

// cache_attention(q, cache, table, lengths, scale, causal, counts, max_length) -> (out, lse), a negative status, or None
PyObject* cache_attention(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    HANDLE_TH_ERRORS
    dfa_dtype_t dt;
    dfa_strides_t sq;
    Sequences s;
    const at::Tensor* const q = nargs == 8 ? row_tensor(args[0], &dt, &sq) : nullptr;
    if (!q || !g_lib.attention || !PyFloat_CheckExact(args[4]) || !PyBool_Check(args[5])) Py_RETURN_NONE;
    const int64_t B = q->size(0), M = q->size(1), H = q->size(2);
    if (!read_sequences(args[1], args[2], args[3], args[6], B, &s) || q->size(3) != s.cache.D) Py_RETURN_NONE;
    int64_t limit = (int64_t)s.width * s.cache.page;
    if (args[7] != Py_None) {
        int32_t given;
        if (!as_int32(args[7], &given)) Py_RETURN_NONE;
        if (given < limit) limit = given;
    }
    at::Tensor res[2] = {at::empty({B, M, H, q->size(3)}, q->options()), at::empty({B, H, M}, q->options().dtype(at::kFloat))};
    const size_t bytes = g_lib.attention_bytes((int32_t)B, (int32_t)M, (int32_t)H, s.cache.heads, s.cache.D, dt, limit);
    const Room room(bytes, *q);
    int rc;
    {
        pybind11::gil_scoped_release release;
        rc = g_lib.attention(q->data_ptr(), sq, dt, (int32_t)B, (int32_t)M, (int32_t)H, s.cache, s.table, s.width, s.ld_table, s.lengths, s.counts,
                             args[5] == Py_True, (float)PyFloat_AS_DOUBLE(args[4]), limit, res[0].data_ptr(), res[1].data_ptr<float>(), room.ptr, bytes,
                             c10::hip::getCurrentHIPStream().stream());
    }
    return rc != DFA_OK ? PyLong_FromLong(rc) : as_tuple(res);
    END_HANDLE_TH_ERRORS
}

// bind(addresses in the loaded libdfa.so of dfa_forward_alloc, dfa_backward and Library's functions in order)
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t nargs) {
    if (nargs != 9) {
        PyErr_SetString(PyExc_TypeError, "bind takes nine addresses");
        return nullptr;
    }
    void* at[9];
    for (int i = 0; i < 9; ++i) at[i] = PyLong_AsVoidPtr(args[i]);
    if (PyErr_Occurred()) return nullptr;
    g_forward = reinterpret_cast<ForwardAlloc>(at[0]);
    g_backward = reinterpret_cast<Backward>(at[1]);
    g_lib = Library{reinterpret_cast<decltype(Library::linear)>(at[2]), reinterpret_cast<decltype(Library::linear_bytes)>(at[3]),
                    reinterpret_cast<decltype(Library::linear_backward)>(at[4]), reinterpret_cast<decltype(Library::linear_backward_bytes)>(at[5]),
                    reinterpret_cast<decltype(Library::append)>(at[6]), reinterpret_cast<decltype(Library::attention)>(at[7]),
                    reinterpret_cast<decltype(Library::attention_bytes)>(at[8])};
    Py_RETURN_NONE;
}

using FastCall = PyObject* (*)(PyObject*, PyObject* const*, Py_ssize_t);
PyCFunction method(FastCall f) { return reinterpret_cast<PyCFunction>(reinterpret_cast<void (*)()>(f)); }

PyMethodDef g_methods[] = {
    {"forward", method(forward), METH_FASTCALL, nullptr},
    {"backward", method(backward), METH_FASTCALL, nullptr},
    {"quantized_linear", method(quantized_linear), METH_FASTCALL, nullptr},
    {"quantized_linear_backward", method(quantized_linear_backward), METH_FASTCALL, nullptr},
    {"cache_append", method(cache_append), METH_FASTCALL, nullptr},
    {"cache_attention", method(cache_attention), METH_FASTCALL, nullptr},
    {"bind", method(bind), METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef g_module = {PyModuleDef_HEAD_INIT, "_dfa_torch", nullptr, -1, g_methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__dfa_torch() { return PyModule_Create(&g_module); }
