// The calls of a decoder's inner loop from Python without ctypes: arguments are read from the tensors themselves (address,
// type, sizes, strides) and passed to the C ABI.  A ctypes call of eight to thirteen arguments and the reading of shapes and
// strides through Python cost 3 to 5 us beside 1.9 us for the launch, more than the smallest kernels take
// (saem_block_norm of one row: 2.9 us a call against 7.2 us).  Each function returns the call's status, as the C ABI does.
// An address on the host, or of another GPU, would only be noticed by the kernel that reads it, as a fault that ends the
// context: every tensor of a call is looked at here, and the call goes to the GPU that they are on.
#include <Python.h>
#include <cstring>

#include <c10/cuda/CUDAGuard.h>
#include <c10/cuda/CUDAStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include "saem.h"

namespace {

struct Fault { const char* what; };          // a Python TypeError

const at::Tensor& tensor(PyObject* o) {
    if (!THPVariable_Check(o)) throw Fault{"a tensor is wanted"};
    return THPVariable_Unpack(o);
}
long long integer(PyObject* o) {
    const long long v = PyLong_AsLongLong(o);
    if (v == -1 && PyErr_Occurred()) throw Fault{nullptr};
    return v;
}
// What was given as `stream`: None (the device's current stream), a torch stream or its handle.
void* stream_of(PyObject* o, int device) {
    if (o == Py_None) return c10::cuda::getCurrentCUDAStream((c10::DeviceIndex)device).stream();
    if (PyLong_Check(o)) {
        void* p = PyLong_AsVoidPtr(o);
        if (!p && PyErr_Occurred()) throw Fault{nullptr};
        return p;
    }
    PyObject* h = PyObject_GetAttrString(o, "cuda_stream");
    if (!h) throw Fault{nullptr};
    void* p = PyLong_AsVoidPtr(h);
    Py_DECREF(h);
    if (!p && PyErr_Occurred()) throw Fault{nullptr};
    return p;
}

// A matrix on the GPU whose columns are consecutive, float32 or bfloat16.
struct Matrix {
    void* p;
    int dtype;
    int64_t rows, cols, stride;
    int device;
    int status;                             // SAEM_OK, or why it is none
};
int dtype_of(const at::Tensor& t) {
    return t.scalar_type() == at::kFloat ? SAEM_OUT_F32 : t.scalar_type() == at::kBFloat16 ? SAEM_OUT_BF16 : -1;
}
Matrix matrix(PyObject* o) {
    const at::Tensor& t = tensor(o);
    Matrix m = {};
    m.status = SAEM_ERR_INVALID_ARG;
    if (!t.is_cuda() || t.layout() != at::kStrided || t.dim() != 2 || (m.dtype = dtype_of(t)) < 0) return m;
    m.rows = t.size(0);
    m.cols = t.size(1);
    m.stride = t.stride(0);
    if (t.stride(1) != 1 && m.cols > 1) return m;
    m.device = t.get_device();
    m.p = t.data_ptr();
    m.status = SAEM_OK;
    return m;
}

// Heads [tokens, heads, dim] on the GPU whose elements are consecutive.  Strides of an extent of one are never used.
struct Heads {
    void* p;
    int dtype;
    int64_t tokens, heads, dim, token_stride, head_stride;
    int device;
    int status;
};
Heads heads_in(PyObject* o) {
    const at::Tensor& t = tensor(o);
    Heads h = {};
    h.status = SAEM_ERR_INVALID_ARG;
    if (!t.is_cuda() || t.layout() != at::kStrided || t.dim() != 3) return h;
    h.dtype = t.scalar_type() == at::kHalf ? SAEM_OUT_F16 : dtype_of(t);
    if (h.dtype < 0 || (t.stride(2) != 1 && t.size(2) > 1)) return h;
    h.tokens = t.size(0);
    h.heads = t.size(1);
    h.dim = t.size(2);
    h.token_stride = t.stride(0);
    h.head_stride = t.stride(1);
    h.device = t.get_device();
    h.p = t.data_ptr();
    h.status = h.tokens <= INT32_MAX && h.heads <= INT32_MAX ? SAEM_OK : SAEM_ERR_SHAPE;
    return h;
}

template <class F>
PyObject* guarded(F f) {
    try {
        return PyLong_FromLong(f());
    } catch (const Fault& e) {
        if (e.what) PyErr_SetString(PyExc_TypeError, e.what);
    } catch (const std::exception& e) {
        PyErr_SetString(PyExc_RuntimeError, e.what());
    }
    return nullptr;
}
// The launch with the interpreter free for other threads.
template <class F>
int unlocked(F f) {
    PyThreadState* s = PyEval_SaveThread();
    const int code = f();
    PyEval_RestoreThread(s);
    return code;
}
// The other tensors of a call whose first one is a matrix; the first that is refused decides the status.
struct Call {
    int device, status;
    explicit Call(const Matrix& first) : device(first.device), status(first.status) {}
    explicit Call(const Heads& first) : device(first.device), status(first.status) {}
    void refuse(int why) { if (status == SAEM_OK) status = why; }
    Matrix matrix_of(PyObject* o, int64_t rows, int64_t cols) {
        const Matrix m = matrix(o);
        if (m.status != SAEM_OK) refuse(m.status);
        else if (m.device != device) refuse(SAEM_ERR_INVALID_ARG);
        else if (m.rows != rows || m.cols != cols) refuse(SAEM_ERR_SHAPE);
        return m;
    }
    // n elements at least, one after the other
    void* array(PyObject* o, at::ScalarType type, size_t n) {
        if (o == Py_None) {
            refuse(SAEM_ERR_INVALID_ARG);
            return nullptr;
        }
        const at::Tensor& t = tensor(o);
        if (!t.is_cuda() || t.layout() != at::kStrided || t.get_device() != device || t.scalar_type() != type || !t.is_contiguous()) {
            refuse(SAEM_ERR_INVALID_ARG);
            return nullptr;
        }
        if ((size_t)t.numel() < n) refuse(SAEM_ERR_SHAPE);
        return t.data_ptr();
    }
    Heads heads_of(PyObject* o, int64_t tokens, int64_t heads, int64_t dim) {
        const Heads h = heads_in(o);
        if (h.status != SAEM_OK) refuse(h.status);
        else if (h.device != device) refuse(SAEM_ERR_INVALID_ARG);
        else if (h.tokens != tokens || h.heads != heads || h.dim != dim) refuse(SAEM_ERR_SHAPE);
        return h;
    }
    // a head's weights, float32 or bfloat16, or nullptr for None
    const void* weight(PyObject* o, int64_t dim, int* dtype) {
        if (o == Py_None) return nullptr;
        *dtype = dtype_of(tensor(o));
        return array(o, *dtype == SAEM_OUT_BF16 ? at::kBFloat16 : at::kFloat, (size_t)dim);
    }
    const uint64_t* turns(PyObject* o, int rotary_dim) {
        return rotary_dim ? static_cast<const uint64_t*>(array(o, at::kLong, (size_t)rotary_dim / 2)) : nullptr;
    }
    // [pages, kv_heads, page_size, dim], both alike
    saem_kv_cache cache(PyObject* k, PyObject* v) {
        saem_kv_cache c = {};
        const at::Tensor &a = tensor(k), &b = tensor(v);
        if (!a.is_cuda() || a.layout() != at::kStrided || a.dim() != 4) refuse(SAEM_ERR_INVALID_ARG);
        if (status != SAEM_OK) return c;
        c.dtype = a.scalar_type() == at::kHalf ? SAEM_OUT_F16 : dtype_of(a);
        c.k = array(k, a.scalar_type(), 0);
        c.v = array(v, a.scalar_type(), 0);
        if (b.sizes() != a.sizes() || a.size(1) > INT32_MAX || a.size(2) > INT32_MAX || a.size(3) > INT32_MAX) refuse(SAEM_ERR_SHAPE);
        if (status != SAEM_OK) return c;
        c.pages = a.size(0);
        c.kv_heads = (int32_t)a.size(1);
        c.page_size = (int32_t)a.size(2);
        c.head_dim = (int32_t)a.size(3);
        return c;
    }
    saem_batch batch(PyObject* offsets, PyObject* lengths, PyObject* table, PyObject* max_new, int64_t tokens) {
        saem_batch b = {};
        b.lengths = static_cast<const int32_t*>(array(lengths, at::kInt, 0));
        const at::Tensor &l = tensor(lengths), &t = tensor(table);
        const int64_t seqs = l.numel();
        b.offsets = static_cast<const int32_t*>(array(offsets, at::kInt, (size_t)seqs + 1));
        if (!t.is_cuda() || t.layout() != at::kStrided || t.get_device() != device || t.scalar_type() != at::kInt || t.dim() != 2 ||
            (t.size(1) > 1 && t.stride(1) != 1)) {
            refuse(SAEM_ERR_INVALID_ARG);
            return b;
        }
        const long long most = integer(max_new);
        if (l.dim() != 1 || t.size(0) < seqs || seqs > INT32_MAX || t.size(1) > INT32_MAX || most < 0) refuse(SAEM_ERR_SHAPE);
        b.table = static_cast<const int32_t*>(t.data_ptr());
        b.table_stride = t.stride(0);
        b.seqs = (int32_t)seqs;
        b.tokens = (int32_t)tokens;
        b.max_pages = (int32_t)t.size(1);
        b.max_new = (int32_t)(most < INT32_MAX ? most : INT32_MAX);
        return b;
    }
    void* codes(PyObject* o, int64_t rows, int64_t cols) { return array(o, at::kByte, saem_mx_codes_bytes(rows, cols)); }
    void* scales(PyObject* o, int64_t rows, int64_t cols) { return array(o, at::kByte, saem_mx_scales_bytes(rows, cols)); }
    template <class F>
    int launch(PyObject* stream, F f) {
        if (status != SAEM_OK) return status;
        c10::cuda::OptionalCUDAGuard guard;                                    // setting the device costs more than asking for it
        if (c10::cuda::current_device() != device) guard.set_index((c10::DeviceIndex)device);
        void* st = stream_of(stream, device);
        return unlocked([&] { return f(st); });
    }
};
PyObject* expect(Py_ssize_t n, Py_ssize_t want) {
    if (n != want) PyErr_Format(PyExc_TypeError, "%zd arguments are wanted, not %zd", want, n);
    return nullptr;
}

// quantize(x, rows, cols, codes, scales, stream)
PyObject* quantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 6) return expect(n, 6);
    return guarded([&] {
        const int64_t rows = integer(a[1]), cols = integer(a[2]);
        const Matrix x = matrix(a[0]);
        Call c(x);
        if (x.rows != rows || x.cols != cols) c.refuse(SAEM_ERR_SHAPE);
        void *codes = c.codes(a[3], rows, cols), *scales = c.scales(a[4], rows, cols);
        return c.launch(a[5], [&](void* st) { return saem_mx_quantize(x.p, x.dtype, rows, cols, x.stride, codes, scales, st); });
    });
}
// dequantize(codes, scales, rows, cols, out, stream)
PyObject* dequantize(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 6) return expect(n, 6);
    return guarded([&] {
        const int64_t rows = integer(a[2]), cols = integer(a[3]);
        const Matrix out = matrix(a[4]);
        Call c(out);
        if (out.rows != rows || out.cols != cols) c.refuse(SAEM_ERR_SHAPE);
        void *codes = c.codes(a[0], rows, cols), *scales = c.scales(a[1], rows, cols);
        return c.launch(a[5], [&](void* st) { return saem_mx_dequantize(codes, scales, rows, cols, out.p, out.dtype, out.stride, st); });
    });
}
// matmul(a_codes, a_scales, m, w_codes, w_scales, n, k, out, status, stream)
PyObject* matmul(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 10) return expect(n, 10);
    return guarded([&] {
        const int64_t m = integer(a[2]), rows = integer(a[5]), k = integer(a[6]);
        const Matrix out = matrix(a[7]);
        Call c(out);
        if (out.rows != m || out.cols != rows) c.refuse(SAEM_ERR_SHAPE);
        void *ac = c.codes(a[0], m, k), *as = c.scales(a[1], m, k), *wc = c.codes(a[3], rows, k), *ws = c.scales(a[4], rows, k);
        void* status = a[8] == Py_None ? nullptr : c.array(a[8], at::kInt, 1);
        return c.launch(a[9], [&](void* st) {
            return saem_mx_matmul(ac, as, m, wc, ws, rows, k, out.p, out.dtype, out.stride, (int32_t*)status, st);
        });
    });
}
// linear(x, w_codes, w_scales, n, k, out, workspace, max_rows, stream)
PyObject* linear(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 9) return expect(n, 9);
    return guarded([&] {
        const int64_t rows = integer(a[3]), k = integer(a[4]), most = integer(a[7]);
        const Matrix x = matrix(a[0]);
        Call c(x);
        if (x.cols != k || x.rows > most) c.refuse(SAEM_ERR_SHAPE);
        const Matrix out = c.matrix_of(a[5], x.rows, rows);
        void *wc = c.codes(a[1], rows, k), *ws = c.scales(a[2], rows, k), *work = c.array(a[6], at::kByte, 0);
        const size_t bytes = c.status == SAEM_OK ? tensor(a[6]).nbytes() : 0;
        return c.launch(a[8], [&](void* st) {
            return saem_mx_linear(x.p, x.dtype, x.rows, x.stride, wc, ws, rows, k, out.p, out.dtype, out.stride, work, bytes, st);
        });
    });
}
// block_norm(config, x, y, gate, w_post, w_pre, x_out, n_out, stream): what the config (bytes) says of rows, types and strides
// is taken from the tensors instead
PyObject* block_norm(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 9) return expect(n, 9);
    return guarded([&] {
        if (!PyBytes_Check(a[0]) || PyBytes_GET_SIZE(a[0]) != (Py_ssize_t)sizeof(saem_norm_config)) throw Fault{"a saem_norm_config is wanted"};
        saem_norm_config c;
        memcpy(&c, PyBytes_AS_STRING(a[0]), sizeof c);
        const Matrix x = matrix(a[1]);
        Call call(x);
        if (x.cols != c.cols) call.refuse(SAEM_ERR_SHAPE);
        c.rows = x.rows;
        c.x_dtype = x.dtype;
        c.x_stride = x.stride;
        Matrix y = {}, x_out = {}, n_out = {};
        if (a[2] != Py_None) {
            y = call.matrix_of(a[2], x.rows, x.cols);
            c.y_dtype = y.dtype;
            c.y_stride = y.stride;
        }
        if (a[6] != Py_None) {
            x_out = call.matrix_of(a[6], x.rows, x.cols);
            if (x_out.dtype != x.dtype) call.refuse(SAEM_ERR_INVALID_ARG);
            c.x_out_stride = x_out.stride;
        }
        if (a[7] != Py_None) {
            n_out = call.matrix_of(a[7], x.rows, x.cols);
            c.n_dtype = n_out.dtype;
            c.n_stride = n_out.stride;
        }
        void* gate = nullptr;
        if (a[3] != Py_None) {
            if (c.gate_mode == SAEM_GATE_FULL) {
                const Matrix g = call.matrix_of(a[3], x.rows, x.cols);
                c.gate_dtype = g.dtype;
                c.gate_stride = g.stride;
                gate = g.p;
            } else if (c.gate_mode == SAEM_GATE_NONE) {
                call.refuse(SAEM_ERR_SHAPE);
            } else {
                const at::Tensor& g = tensor(a[3]);
                if (!g.is_cuda() || g.layout() != at::kStrided || g.get_device() != call.device || (c.gate_dtype = dtype_of(g)) < 0) {
                    call.refuse(SAEM_ERR_INVALID_ARG);
                } else if (c.gate_mode == SAEM_GATE_TOKEN) {                   // [T] or [T, 1]
                    if (!(g.dim() == 1 || (g.dim() == 2 && g.size(1) == 1)) || g.size(0) != x.rows) call.refuse(SAEM_ERR_SHAPE);
                    else c.gate_stride = g.stride(0);
                } else {                                                       // [d] or [1, d]
                    if (!(g.dim() == 1 || (g.dim() == 2 && g.size(0) == 1)) || g.size(-1) != x.cols || (x.cols > 1 && g.stride(-1) != 1))
                        call.refuse(SAEM_ERR_SHAPE);
                }
                if (call.status == SAEM_OK) gate = g.data_ptr();
            }
        }
        const at::ScalarType w_type = c.w_dtype == SAEM_OUT_BF16 ? at::kBFloat16 : at::kFloat;
        void* post = a[4] == Py_None ? nullptr : call.array(a[4], w_type, (size_t)c.cols);
        void* pre = a[5] == Py_None ? nullptr : call.array(a[5], w_type, (size_t)c.cols);
        return call.launch(a[8], [&](void* st) { return saem_block_norm(&c, x.p, y.p, gate, post, pre, x_out.p, n_out.p, st); });
    });
}

template <class T>
T config_of(PyObject* o, const char* what) {
    T c;
    if (!PyBytes_Check(o) || PyBytes_GET_SIZE(o) != (Py_ssize_t)sizeof c) throw Fault{what};
    memcpy(&c, PyBytes_AS_STRING(o), sizeof c);
    return c;
}
// rotate(config, x, weight, turns, positions, out, stream): sizes, types and strides are the tensors'
PyObject* rotate(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 7) return expect(n, 7);
    return guarded([&] {
        saem_rotate_config c = config_of<saem_rotate_config>(a[0], "a saem_rotate_config is wanted");
        const Heads x = heads_in(a[1]);
        Call call(x);
        if (x.dim != c.rotary.head_dim) call.refuse(SAEM_ERR_SHAPE);
        const Heads out = call.heads_of(a[5], x.tokens, x.heads, x.dim);
        c.x_dtype = x.dtype;
        c.out_dtype = out.dtype;
        c.heads = (int32_t)x.heads;
        c.tokens = x.tokens;
        c.x_token_stride = x.token_stride;
        c.x_head_stride = x.head_stride;
        c.out_token_stride = out.token_stride;
        c.out_head_stride = out.head_stride;
        const void* w = call.weight(a[2], x.dim, &c.w_dtype);
        const uint64_t* turns = call.turns(a[3], c.rotary.rotary_dim);
        const auto* positions = static_cast<const int32_t*>(call.array(a[4], at::kInt, (size_t)x.tokens));
        return call.launch(a[6], [&](void* st) { return saem_rotate(&c, x.p, w, turns, positions, out.p, st); });
    });
}
// append(config, q, k, v, w_q, w_k, turns, positions, cache_k, cache_v, offsets, lengths, table, max_new, q_out, status, stream)
PyObject* append(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 17) return expect(n, 17);
    return guarded([&] {
        saem_append_config c = config_of<saem_append_config>(a[0], "a saem_append_config is wanted");
        const Heads k = heads_in(a[2]);
        Call call(k);
        const saem_kv_cache cache = call.cache(a[8], a[9]);
        if (k.dim != c.rotary.head_dim || k.dim != cache.head_dim || k.heads != cache.kv_heads) call.refuse(SAEM_ERR_SHAPE);
        const Heads v = call.heads_of(a[3], k.tokens, k.heads, k.dim);
        const saem_batch b = call.batch(a[10], a[11], a[12], a[13], k.tokens);
        Heads q = {}, out = {};
        if (a[1] != Py_None) {
            q = call.heads_of(a[1], k.tokens, c.q_heads, k.dim);
            out = call.heads_of(a[14], k.tokens, c.q_heads, k.dim);
            if (q.dtype != k.dtype || out.dtype != cache.dtype) call.refuse(SAEM_ERR_INVALID_ARG);
        }
        if (v.dtype != k.dtype) call.refuse(SAEM_ERR_INVALID_ARG);
        c.x_dtype = k.dtype;
        c.q_token_stride = q.token_stride;
        c.q_head_stride = q.head_stride;
        c.k_token_stride = k.token_stride;
        c.k_head_stride = k.head_stride;
        c.v_token_stride = v.token_stride;
        c.v_head_stride = v.head_stride;
        c.out_token_stride = out.token_stride;
        c.out_head_stride = out.head_stride;
        int wq_type = SAEM_OUT_F32, wk_type = SAEM_OUT_F32;
        const void *w_q = a[1] == Py_None ? nullptr : call.weight(a[4], k.dim, &wq_type), *w_k = call.weight(a[5], k.dim, &wk_type);
        if (w_q && w_k && wq_type != wk_type) call.refuse(SAEM_ERR_INVALID_ARG);
        c.w_dtype = w_q ? wq_type : wk_type;
        const uint64_t* turns = call.turns(a[6], c.rotary.rotary_dim);
        const auto* positions = a[7] == Py_None ? nullptr : static_cast<const int32_t*>(call.array(a[7], at::kInt, (size_t)k.tokens));
        auto* status = a[15] == Py_None ? nullptr : static_cast<int32_t*>(call.array(a[15], at::kInt, 1));
        return call.launch(a[16], [&](void* st) {
            return saem_kv_append(&c, &cache, &b, q.p, k.p, v.p, w_q, w_k, turns, positions, out.p, status, st);
        });
    });
}
// attend(config, q, cache_k, cache_v, offsets, lengths, table, max_new, out, lse, workspace, stream)
PyObject* attend(PyObject*, PyObject* const* a, Py_ssize_t n) {
    if (n != 12) return expect(n, 12);
    return guarded([&] {
        saem_attend_config c = config_of<saem_attend_config>(a[0], "a saem_attend_config is wanted");
        const Heads q = heads_in(a[1]);
        Call call(q);
        const saem_kv_cache cache = call.cache(a[2], a[3]);
        if (q.heads != c.q_heads || q.dim != cache.head_dim) call.refuse(SAEM_ERR_SHAPE);
        const Heads out = call.heads_of(a[8], q.tokens, q.heads, q.dim);
        if (q.dtype != cache.dtype || out.dtype != cache.dtype) call.refuse(SAEM_ERR_INVALID_ARG);
        const saem_batch b = call.batch(a[4], a[5], a[6], a[7], q.tokens);
        c.q_token_stride = q.token_stride;
        c.q_head_stride = q.head_stride;
        c.out_token_stride = out.token_stride;
        c.out_head_stride = out.head_stride;
        float* lse = nullptr;
        if (a[9] != Py_None) {
            lse = static_cast<float*>(call.array(a[9], at::kFloat, 0));
            const at::Tensor& t = tensor(a[9]);
            if (t.dim() != 2 || t.size(0) != q.tokens || t.size(1) != q.heads) call.refuse(SAEM_ERR_SHAPE);
        }
        void* work = call.array(a[10], at::kByte, 0);
        const size_t bytes = call.status == SAEM_OK ? tensor(a[10]).nbytes() : 0;
        return call.launch(a[11], [&](void* st) { return saem_attend(&c, &cache, &b, q.p, out.p, lse, work, bytes, st); });
    });
}

PyMethodDef methods[] = {
    {"quantize", (PyCFunction)(void (*)(void))quantize, METH_FASTCALL, nullptr},
    {"dequantize", (PyCFunction)(void (*)(void))dequantize, METH_FASTCALL, nullptr},
    {"matmul", (PyCFunction)(void (*)(void))matmul, METH_FASTCALL, nullptr},
    {"linear", (PyCFunction)(void (*)(void))linear, METH_FASTCALL, nullptr},
    {"block_norm", (PyCFunction)(void (*)(void))block_norm, METH_FASTCALL, nullptr},
    {"rotate", (PyCFunction)(void (*)(void))rotate, METH_FASTCALL, nullptr},
    {"append", (PyCFunction)(void (*)(void))append, METH_FASTCALL, nullptr},
    {"attend", (PyCFunction)(void (*)(void))attend, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
// what this file was built for, looked for in the built file
__attribute__((used)) const char built_for[] = SAEM_BUILT_FOR;

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host_calls(void) { return PyModule_Create(&module); }
