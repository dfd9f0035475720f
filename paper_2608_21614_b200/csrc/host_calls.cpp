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

PyMethodDef methods[] = {
    {"quantize", (PyCFunction)(void (*)(void))quantize, METH_FASTCALL, nullptr},
    {"dequantize", (PyCFunction)(void (*)(void))dequantize, METH_FASTCALL, nullptr},
    {"matmul", (PyCFunction)(void (*)(void))matmul, METH_FASTCALL, nullptr},
    {"linear", (PyCFunction)(void (*)(void))linear, METH_FASTCALL, nullptr},
    {"block_norm", (PyCFunction)(void (*)(void))block_norm, METH_FASTCALL, nullptr},
    {nullptr, nullptr, 0, nullptr},
};
// what this file was built for, looked for in the built file
__attribute__((used)) const char built_for[] = SAEM_BUILT_FOR;

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_host_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__host_calls(void) { return PyModule_Create(&module); }
