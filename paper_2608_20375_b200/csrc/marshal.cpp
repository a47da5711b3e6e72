// Arguments of the calls whose checks and conversions in Python take longer than their work on the GPU.  One tree's append, 3.4 us on the GPU: 15.1 us a call
// in a loop with the checks in Python, 4.2 with these.  Each function takes what the binding's method of the same name takes, checks it as the method does and makes the call: the call's status, or
// None when a check fails (nothing has been done then, and the method finds the reason).
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>
#include <cstdint>

#include "../../include/graft.h"

namespace {

decltype(&graft_cache_write) call_write = nullptr;
decltype(&graft_cache_read) call_read = nullptr;
decltype(&graft_cache_append) call_append = nullptr;
decltype(&graft_window_attention) call_window = nullptr;

using Shape = at::IntArrayRef;

const at::Tensor* tensor(PyObject* o) { return THPVariable_Check(o) ? &THPVariable_Unpack(o) : nullptr; }

struct Checks {
    int64_t dev;
    bool ok = true;

    bool is(const at::Tensor* t, at::ScalarType type) { return ok = ok && t && t->is_cuda() && t->get_device() == dev && t->scalar_type() == type; }
    // a dense tensor of this type and shape, or (if it may be None) nothing
    template <typename T>
    T* dense(PyObject* o, at::ScalarType type, Shape shape, bool optional = false) {
        if (optional && o == Py_None) return nullptr;
        const at::Tensor* t = tensor(o);
        if (is(t, type)) ok = t->sizes() == shape && t->is_contiguous();
        return ok ? (T*)t->data_ptr() : nullptr;
    }
    // [batch, rows, heads, dim] bf16 whose tokens may stand further apart than dense
    const void* rows(const at::Tensor* t, int64_t heads, int64_t dim, int64_t& stride) {
        if (!is(t, at::kBFloat16) || !(ok = t->dim() == 4 && t->size(2) == heads && t->size(3) == dim)) return nullptr;
        const int64_t batch = t->size(0), n = t->size(1);
        stride = heads * dim;
        if (!t->is_contiguous()) {
            stride = n > 1 ? t->stride(1) : batch > 1 ? t->stride(0) : heads * dim;
            ok = t->stride(3) == 1 && (heads == 1 || t->stride(2) == dim) && (batch == 1 || t->stride(0) == n * stride);
        }
        return ok ? t->data_ptr() : nullptr;
    }
    int64_t number(PyObject* o, int64_t lo, int64_t hi) {
        int over = 0;
        const int64_t x = PyLong_Check(o) ? PyLong_AsLongLongAndOverflow(o, &over) : 0;
        ok = ok && PyLong_Check(o) && !over && x >= lo && x <= hi;
        return x;
    }
    // k, v, k_exp, v_exp, table
    graft_cache cache(PyObject* const* a, int64_t batch) {
        graft_cache c = {};
        const at::Tensor *k = tensor(a[0]), *table = tensor(a[4]);
        ok = ok && k && table && k->dim() == 5 && table->dim() == 2;
        if (!ok) return c;
        const bool q8 = k->scalar_type() == at::kFloat8_e4m3fn;
        const at::ScalarType type = q8 ? at::kFloat8_e4m3fn : at::kBFloat16;
        const Shape shape = k->sizes();
        for (const int64_t n : shape) ok = ok && n <= INT32_MAX;
        ok = ok && table->size(1) <= INT32_MAX && q8 == (a[2] != Py_None) && q8 == (a[3] != Py_None);
        c.layers = (int32_t)shape[0], c.n_pages = (int32_t)shape[1], c.kv_heads = (int32_t)shape[2], c.page_size = (int32_t)shape[3];
        c.head_dim = (int32_t)shape[4], c.dtype = q8 ? GRAFT_E4M3 : GRAFT_BF16, c.table_width = (int32_t)table->size(1);
        c.d_k = dense<void>(a[0], type, shape), c.d_v = dense<void>(a[1], type, shape);
        c.d_k_exp = dense<uint8_t>(a[2], at::kByte, shape.slice(0, 4), true), c.d_v_exp = dense<uint8_t>(a[3], at::kByte, shape.slice(0, 4), true);
        c.d_table = dense<int32_t>(a[4], at::kInt, {batch, table->size(1)});
        return c;
    }
};

PyObject* none() { Py_RETURN_NONE; }

template <typename Call>
PyObject* status(Call call) {
    graft_status s;
    Py_BEGIN_ALLOW_THREADS;
    s = call();
    Py_END_ALLOW_THREADS;
    return PyLong_FromLong((long)s);
}

// bind(addresses of graft_cache_write, graft_cache_read, graft_cache_append, graft_window_attention)
PyObject* bind(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 4) return none();
    call_write = (decltype(call_write))PyLong_AsVoidPtr(a[0]);
    call_read = (decltype(call_read))PyLong_AsVoidPtr(a[1]);
    call_append = (decltype(call_append))PyLong_AsVoidPtr(a[2]);
    call_window = (decltype(call_window))PyLong_AsVoidPtr(a[3]);
    return PyErr_Occurred() ? nullptr : none();
}

// (context, device, stream, layer, k, v, k_exp, v_exp, table, prefix_len, count, key, value, status), written or read
PyObject* cache_rows(bool write, PyObject* const* a, Py_ssize_t n) try {
    if (n != 14 || !call_write || !call_read || !PyLong_Check(a[0]) || !PyLong_Check(a[2])) return none();
    Checks x{0};
    x.dev = x.number(a[1], INT32_MIN, INT32_MAX);
    const int32_t layer = (int32_t)x.number(a[3], INT32_MIN, INT32_MAX);
    const at::Tensor *key = tensor(a[11]), *value = tensor(a[12]);
    if (!x.ok || !key || !value || key->dim() != 4 || value->sizes() != key->sizes()) return none();
    const int64_t batch = key->size(0), rows = key->size(1);
    if (batch > INT32_MAX || rows > INT32_MAX) return none();
    const graft_cache c = x.cache(a + 4, batch);
    int64_t k_stride = 0, v_stride = 0;
    void* const kp = (void*)x.rows(key, c.kv_heads, c.head_dim, k_stride);
    void* const vp = (void*)x.rows(value, c.kv_heads, c.head_dim, v_stride);
    const int32_t* const prefix = x.dense<const int32_t>(a[9], at::kInt, {batch});
    const int32_t* const count = x.dense<const int32_t>(a[10], at::kInt, {batch});
    int32_t* const st = x.dense<int32_t>(a[13], at::kInt, {batch}, true);
    if (!x.ok || k_stride != v_stride || (!write && !(key->is_contiguous() && value->is_contiguous()))) return none();
    graft_ctx* const ctx = (graft_ctx*)PyLong_AsVoidPtr(a[0]);
    void* const stream = PyLong_AsVoidPtr(a[2]);
    if (PyErr_Occurred()) return nullptr;
    return status([&] {
        return write ? call_write(ctx, (int32_t)batch, &c, layer, prefix, count, (int32_t)rows, k_stride, kp, vp, st, stream)
                     : call_read(ctx, (int32_t)batch, &c, layer, prefix, count, (int32_t)rows, kp, vp, st, stream);
    });
} catch (...) {
    return none();
}
PyObject* cache_write(PyObject*, PyObject* const* a, Py_ssize_t n) { return cache_rows(true, a, n); }
PyObject* cache_read(PyObject*, PyObject* const* a, Py_ssize_t n) { return cache_rows(false, a, n); }

// (context, device, stream, layer, k, v, k_exp, v_exp, table, prefix_len, count, freq, interleaved, gain, shift, q, key, value, q_out, position, status)
PyObject* cache_append(PyObject*, PyObject* const* a, Py_ssize_t n) try {
    if (n != 21 || !call_append || !PyLong_Check(a[0]) || !PyLong_Check(a[2])) return none();
    Checks x{0};
    x.dev = x.number(a[1], INT32_MIN, INT32_MAX);
    const int32_t layer = (int32_t)x.number(a[3], INT32_MIN, INT32_MAX);
    const at::Tensor *key = tensor(a[16]), *value = tensor(a[17]), *freq = tensor(a[11]);
    if (!x.ok || !key || !value || !freq || key->dim() != 4 || freq->dim() != 2 || !PyBool_Check(a[12]) || !PyFloat_Check(a[13])) return none();
    const int64_t batch = key->size(0), rows = key->size(1);
    if (batch > INT32_MAX || rows > INT32_MAX || freq->size(0) > INT32_MAX || freq->size(1) > INT32_MAX / 2) return none();
    const graft_cache c = x.cache(a + 4, batch);
    int64_t kv_stride = 0, v_stride = 0, q_stride = 0, out_stride = 0;
    const void* const kp = x.rows(key, c.kv_heads, c.head_dim, kv_stride);
    const void* const vp = x.rows(value, c.kv_heads, c.head_dim, v_stride);
    if (!x.ok || value->size(0) != batch || value->size(1) != rows || v_stride != kv_stride) return none();
    const void* qp = nullptr;
    void* op = nullptr;
    int64_t heads = 0;
    if (a[15] != Py_None) {
        const at::Tensor* q = tensor(a[15]);
        if (!q || q->dim() != 4 || q->size(0) != batch || q->size(1) != rows || q->size(2) > INT32_MAX) return none();
        heads = q->size(2);
        qp = x.rows(q, heads, c.head_dim, q_stride);
        op = (void*)qp, out_stride = q_stride;
        if (a[18] != Py_None) {
            const at::Tensor* out = tensor(a[18]);
            if (!out || out->sizes() != q->sizes()) return none();
            op = (void*)x.rows(out, heads, c.head_dim, out_stride);
        }
    } else if (a[18] != Py_None)
        return none();
    graft_rope r = {};
    r.rot_dim = (int32_t)(2 * freq->size(1)), r.interleaved = a[12] == Py_True, r.axes = (int32_t)freq->size(0);
    r.gain = (float)PyFloat_AS_DOUBLE(a[13]);
    r.d_freq = x.dense<const float>(a[11], at::kFloat, freq->sizes());
    r.d_shift = x.dense<const int32_t>(a[14], at::kInt, {batch}, true);
    if (a[19] != Py_None) {
        const at::Tensor* at = tensor(a[19]);
        if (!at || (at->dim() != 2 && at->dim() != 3) || at->size(0) != batch || at->size(1) < rows || at->size(1) > INT32_MAX) return none();
        r.pos_axes = at->dim() == 2 ? 1 : (int32_t)at->size(2), r.pos_rows = (int32_t)at->size(1);
        if (at->dim() == 3 && at->size(2) != 1 && at->size(2) != freq->size(0)) return none();
        r.d_position = x.dense<const int32_t>(a[19], at::kInt, at->sizes());
    }
    const int32_t* const prefix = x.dense<const int32_t>(a[9], at::kInt, {batch});
    const int32_t* const count = x.dense<const int32_t>(a[10], at::kInt, {batch});
    int32_t* const st = x.dense<int32_t>(a[20], at::kInt, {batch}, true);
    graft_ctx* const ctx = (graft_ctx*)PyLong_AsVoidPtr(a[0]);
    void* const stream = PyLong_AsVoidPtr(a[2]);
    if (PyErr_Occurred()) return nullptr;
    if (!x.ok) return none();
    return status([&] {
        return call_append(ctx, (int32_t)batch, &c, layer, &r, (int32_t)heads, prefix, count, (int32_t)rows, q_stride, qp, kv_stride, kp, vp, out_stride, op, st,
                           stream);
    });
} catch (...) {
    return none();
}

// (context, device, stream, nmax, mask words, layer, k, v, k_exp, v_exp, table, q, prefix_len, count, mask, position, window, sinks, out, lse, scale, status)
PyObject* window_attention(PyObject*, PyObject* const* a, Py_ssize_t n) try {
    if (n != 22 || !call_window || !PyLong_Check(a[0]) || !PyLong_Check(a[2])) return none();
    Checks x{0};
    x.dev = x.number(a[1], INT32_MIN, INT32_MAX);
    const int64_t nmax = x.number(a[3], 0, INT32_MAX), words = x.number(a[4], 0, INT32_MAX);
    const int32_t layer = (int32_t)x.number(a[5], INT32_MIN, INT32_MAX), window = (int32_t)x.number(a[16], -1, INT32_MAX);
    const int32_t sinks = (int32_t)x.number(a[17], -1, INT32_MAX);
    const at::Tensor* q = tensor(a[11]);
    if (!x.ok || !q || q->dim() != 4 || (a[14] == Py_None) != (a[15] == Py_None) || (a[20] != Py_None && !PyFloat_Check(a[20]))) return none();
    const int64_t batch = q->size(0), rows = q->size(1), heads = q->size(2);
    if (batch > INT32_MAX || rows > INT32_MAX || heads > INT32_MAX) return none();
    const graft_cache c = x.cache(a + 6, batch);
    int64_t stride = 0;
    const void* const qp = x.rows(q, heads, c.head_dim, stride);
    const int32_t* const prefix = x.dense<const int32_t>(a[12], at::kInt, {batch});
    const int32_t* const count = x.dense<const int32_t>(a[13], at::kInt, {batch});
    const uint32_t* const mask = x.dense<const uint32_t>(a[14], at::kInt, {batch, nmax, words}, true);
    const int32_t* const position = x.dense<const int32_t>(a[15], at::kInt, {batch, nmax}, true);
    void* const out = x.dense<void>(a[18], at::kBFloat16, {batch, rows, heads, c.head_dim});
    float* const lse = x.dense<float>(a[19], at::kFloat, {batch, rows, heads}, true);
    int32_t* const st = x.dense<int32_t>(a[21], at::kInt, {batch}, true);
    if (!x.ok) return none();
    const float scale = (float)(a[20] == Py_None ? std::pow((double)c.head_dim, -0.5) : PyFloat_AS_DOUBLE(a[20]));
    graft_ctx* const ctx = (graft_ctx*)PyLong_AsVoidPtr(a[0]);
    void* const stream = PyLong_AsVoidPtr(a[2]);
    if (PyErr_Occurred()) return nullptr;
    return status([&] {
        return call_window(ctx, (int32_t)batch, &c, layer, (int32_t)heads, (int32_t)rows, stride, qp, scale, prefix, count, mask, position, window, sinks, out, lse,
                           st, stream);
    });
} catch (...) {
    return none();
}

PyMethodDef methods[] = {{"bind", (PyCFunction)(void*)bind, METH_FASTCALL, nullptr},
                         {"cache_write", (PyCFunction)(void*)cache_write, METH_FASTCALL, nullptr},
                         {"cache_read", (PyCFunction)(void*)cache_read, METH_FASTCALL, nullptr},
                         {"cache_append", (PyCFunction)(void*)cache_append, METH_FASTCALL, nullptr},
                         {"window_attention", (PyCFunction)(void*)window_attention, METH_FASTCALL, nullptr},
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods};

}  // namespace

PyMODINIT_FUNC PyInit__marshal() { return PyModule_Create(&module); }
