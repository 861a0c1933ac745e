// Turns torch tensors into the C ABI's matrices for the calls that are made once or more for every block and token, where
// marshalling through ctypes (about 1 us for each matrix) would take longer than the call itself.  A CPython module that
// binding.py hands the library's function addresses to; arguments are positional, None is a matrix that is left out.
// Every function returns the call's status.

#include <torch/csrc/Exceptions.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>

#include "flashoptim.h"

namespace {

template <typename F>
void take(PyObject* table, const char* name, F*& to) {
    PyObject* v = PyDict_GetItemString(table, name);      // (borrowed)
    if (v) to = reinterpret_cast<F*>(PyLong_AsVoidPtr(v));
}

decltype(&flashoptim_mx4_quantize) call_quantize;
decltype(&flashoptim_mx4_dequantize) call_dequantize;
decltype(&flashoptim_mx4_matmul) call_matmul;
decltype(&flashoptim_mx4_linear) call_linear;
decltype(&flashoptim_mx4_linear_backward) call_linear_backward;
decltype(&flashoptim_block_norm) call_norm;
decltype(&flashoptim_block_norm_backward) call_norm_backward;
PyObject *current_stream, *current_device;      // torch._C._cuda_getCurrentRawStream, _cuda_getDevice

// The arguments of one call, taken in order.  After the first failure a Python error is set and nothing more is taken.
struct Args {
    PyObject* const* at;
    Py_ssize_t n, i = 0;
    bool failed = false;

    Args(PyObject* const* args, Py_ssize_t count, Py_ssize_t expected) : at(args), n(count) {
        if (n != expected) fail(PyExc_TypeError, "%s", "wrong number of arguments");
    }
    template <typename... T>
    void fail(PyObject* type, const char* format, T... a) {
        if (!failed) PyErr_Format(type, format, a...);
        failed = true;
    }
    PyObject* next() { return failed ? Py_None : at[i++]; }

    const at::Tensor* tensor(const char* name) {
        PyObject* o = next();
        if (o == Py_None) return nullptr;
        if (!THPVariable_Check(o)) {
            fail(PyExc_TypeError, "%s: a tensor", name);
            return nullptr;
        }
        const at::Tensor* t = &THPVariable_Unpack(o);
        if (!t->is_cuda()) fail(PyExc_ValueError, "%s: not on the GPU", name);
        return failed ? nullptr : t;
    }
    // A two-dimensional tensor with neighbouring columns, whose rows may lie apart.
    const flashoptim_matrix* matrix(const char* name, flashoptim_matrix* m) {
        const at::Tensor* t = tensor(name);
        if (!t) return nullptr;
        const auto type = t->scalar_type();
        if (t->dim() != 2 || (type != at::kBFloat16 && type != at::kFloat)) {
            fail(PyExc_ValueError, "%s: a matrix of bfloat16 or float32 values", name);
            return nullptr;
        }
        const int64_t rows = t->size(0), cols = t->size(1);
        if (cols > 1 && t->stride(1) != 1) {
            fail(PyExc_ValueError, "%s: the values of a row must be neighbours in memory", name);
            return nullptr;
        }
        *m = {t->data_ptr(), rows, cols, rows > 1 ? t->stride(0) : cols, type == at::kFloat ? FLASHOPTIM_FP32 : FLASHOPTIM_BF16};
        return m;
    }
    // A contiguous tensor of this type and shape (any shape of `numel` values where rows < 0).
    void* plain(const char* name, at::ScalarType type, int64_t rows, int64_t cols, int64_t numel) {
        const at::Tensor* t = tensor(name);
        if (!t) return nullptr;
        const bool shaped = rows < 0 ? t->numel() == numel : t->dim() == 2 && t->size(0) == rows && t->size(1) == cols;
        if (t->scalar_type() != type || !shaped || !t->is_contiguous()) {
            fail(PyExc_ValueError, "%s: a contiguous tensor of another type or shape", name);
            return nullptr;
        }
        return t->data_ptr();
    }
    void workspace(void** p, int64_t* bytes) {
        const at::Tensor* t = tensor("workspace");
        *p = nullptr;
        *bytes = 0;
        if (!t) return;
        if (!t->is_contiguous()) return fail(PyExc_ValueError, "%s", "workspace: contiguous memory");
        *p = t->data_ptr();
        *bytes = (int64_t)t->nbytes();
    }
    // The address of a descriptor; 0 for one that is left out, negative for one that is not on the GPU.
    template <typename T>
    const T* address() {
        PyObject* o = next();
        if (o == Py_None) return nullptr;
        const long long v = PyLong_AsLongLong(o);
        if (v < 0) {
            if (!PyErr_Occurred()) PyErr_SetString(PyExc_ValueError, "a matrix in 4 bits that is not on the GPU");
            failed = true;
        }
        return failed ? nullptr : reinterpret_cast<const T*>((uintptr_t)v);
    }
    // A stream's handle, or None for the current stream of the current device.
    void* stream() {
        PyObject* o = next();
        if (failed) return nullptr;
        if (o != Py_None) {
            void* v = PyLong_AsVoidPtr(o);
            failed = PyErr_Occurred() != nullptr;
            return v;
        }
        PyObject* device = PyObject_CallNoArgs(current_device);
        PyObject* handle = device ? PyObject_CallOneArg(current_stream, device) : nullptr;
        Py_XDECREF(device);
        if (!handle) {
            failed = true;
            return nullptr;
        }
        void* v = PyLong_AsVoidPtr(handle);
        Py_DECREF(handle);
        return v;
    }
};

PyObject* status(const Args& a, int rc) { return a.failed ? nullptr : PyLong_FromLong(rc); }

PyObject* quantize(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n, 6);
    flashoptim_matrix mx;
    const flashoptim_matrix* x = a.matrix("x", &mx);
    const int64_t rows = x ? x->rows : 0, cols = x ? x->cols : 0;
    const auto* out = a.address<flashoptim_mx4>();
    const auto* out_t = a.address<flashoptim_mx4>();
    const void* rho = a.plain("rho", at::kChar, rows, cols, 0);
    const void* rand = a.plain("rand", at::kByte, rows, cols, 0);
    void* stream = a.stream();
    return status(a, a.failed ? 0 : call_quantize(x, (const int8_t*)rho, (const uint8_t*)rand, out, out_t, stream));
}

PyObject* dequantize(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n, 3);
    flashoptim_matrix mx;
    const auto* q = a.address<flashoptim_mx4>();
    const flashoptim_matrix* x = a.matrix("out", &mx);
    void* stream = a.stream();
    return status(a, a.failed ? 0 : call_dequantize(q, x, stream));
}

PyObject* matmul(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n, 5);
    flashoptim_matrix mc;
    void* ws;
    int64_t bytes;
    const auto* p = a.address<flashoptim_mx4>();
    const auto* q = a.address<flashoptim_mx4>();
    const flashoptim_matrix* c = a.matrix("out", &mc);
    a.workspace(&ws, &bytes);
    void* stream = a.stream();
    return status(a, a.failed ? 0 : call_matmul(p, q, c, ws, bytes, stream));
}

PyObject* linear(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n, 6);
    flashoptim_matrix mx, my;
    void* ws;
    int64_t bytes;
    const flashoptim_matrix* x = a.matrix("x", &mx);
    const auto* w = a.address<flashoptim_mx4>();
    const auto* xt = a.address<flashoptim_mx4>();
    const flashoptim_matrix* y = a.matrix("out", &my);
    a.workspace(&ws, &bytes);
    void* stream = a.stream();
    return status(a, a.failed ? 0 : call_linear(x, w, xt, y, ws, bytes, stream));
}

PyObject* linear_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n, 8);
    flashoptim_matrix mdy, mdx, mdw;
    void* ws;
    int64_t bytes;
    const flashoptim_matrix* dy = a.matrix("dy", &mdy);
    const void* rand = a.plain("rand", at::kByte, dy ? dy->rows : 0, dy ? dy->cols : 0, 0);
    const auto* wt = a.address<flashoptim_mx4>();
    const auto* xt = a.address<flashoptim_mx4>();
    const flashoptim_matrix* dx = a.matrix("dx", &mdx);
    const flashoptim_matrix* dw = a.matrix("dw", &mdw);
    a.workspace(&ws, &bytes);
    void* stream = a.stream();
    return status(a, a.failed ? 0 : call_linear_backward(dy, (const uint8_t*)rand, wt, xt, dx, dw, ws, bytes, stream));
}

PyObject* norm(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n, 8);
    flashoptim_matrix mx, mf, mg, mh, my;
    const auto* spec = a.address<flashoptim_block_norm_spec>();
    const flashoptim_matrix* x = a.matrix("x", &mx);
    const flashoptim_matrix* f = a.matrix("f", &mf);
    const flashoptim_matrix* gate = a.matrix("gate", &mg);
    const flashoptim_matrix* h = a.matrix("h", &mh);
    const flashoptim_matrix* y = a.matrix("y", &my);
    void* stats = a.plain("stats", at::kFloat, -1, 0, x ? 4 * x->rows : 0);
    void* stream = a.stream();
    return status(a, a.failed ? 0 : call_norm(spec, x, f, gate, h, y, (float*)stats, stream));
}

PyObject* norm_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n, 16);
    flashoptim_matrix mh, mf, mg, m[5];
    flashoptim_block_norm_grads g;
    void* ws;
    int64_t bytes;
    const auto* spec = a.address<flashoptim_block_norm_spec>();
    const flashoptim_matrix* h = a.matrix("h", &mh);
    const void* stats = a.plain("stats", at::kFloat, -1, 0, h ? 4 * h->rows : 0);
    const flashoptim_matrix* f = a.matrix("f", &mf);
    const flashoptim_matrix* gate = a.matrix("gate", &mg);
    g.dy = a.matrix("dy", &m[0]);
    g.dh = a.matrix("dh", &m[1]);
    g.dx = a.matrix("dx", &m[2]);
    g.df = a.matrix("df", &m[3]);
    g.dgate = a.matrix("dgate", &m[4]);
    const at::ScalarType type = spec && spec->param_dtype == FLASHOPTIM_FP32 ? at::kFloat : at::kBFloat16;
    const int64_t cols = spec ? spec->cols : 0;
    g.dpost_weight = a.plain("dpost_weight", type, -1, 0, cols);
    g.dpost_bias = a.plain("dpost_bias", type, -1, 0, cols);
    g.dpre_weight = a.plain("dpre_weight", type, -1, 0, cols);
    g.dpre_bias = a.plain("dpre_bias", type, -1, 0, cols);
    a.workspace(&ws, &bytes);
    void* stream = a.stream();
    return status(a, a.failed ? 0 : call_norm_backward(spec, h, f, gate, (const float*)stats, &g, ws, bytes, stream));
}

// bind(addresses by name, current_stream, current_device)
PyObject* bind(PyObject*, PyObject* const* args, Py_ssize_t n) {
    if (n != 3 || !PyDict_Check(args[0])) {
        PyErr_SetString(PyExc_TypeError, "bind(addresses, current_stream, current_device)");
        return nullptr;
    }
    take(args[0], "flashoptim_mx4_quantize", call_quantize);
    take(args[0], "flashoptim_mx4_dequantize", call_dequantize);
    take(args[0], "flashoptim_mx4_matmul", call_matmul);
    take(args[0], "flashoptim_mx4_linear", call_linear);
    take(args[0], "flashoptim_mx4_linear_backward", call_linear_backward);
    take(args[0], "flashoptim_block_norm", call_norm);
    take(args[0], "flashoptim_block_norm_backward", call_norm_backward);
    if (!call_quantize || !call_dequantize || !call_matmul || !call_linear || !call_linear_backward || !call_norm || !call_norm_backward) {
        PyErr_SetString(PyExc_RuntimeError, "bind: an entry point is missing");
        return nullptr;
    }
    Py_INCREF(args[1]);
    Py_INCREF(args[2]);
    Py_XSETREF(current_stream, args[1]);
    Py_XSETREF(current_device, args[2]);
    Py_RETURN_NONE;
}

// What torch throws on the way becomes a Python error: a tensor without memory (inside torch.vmap, a wrapper of torch.func) has no address to
// give, and one of a class of its own asks Python for its device.
template <PyObject* (*CALL)(PyObject*, PyObject* const*, Py_ssize_t)>
PyObject* guarded(PyObject* self, PyObject* const* args, Py_ssize_t n) {
    HANDLE_TH_ERRORS
    return CALL(self, args, n);
    END_HANDLE_TH_ERRORS
}

#define FO_METHOD(name) {#name, (PyCFunction)(void (*)(void))guarded<name>, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {FO_METHOD(bind),   FO_METHOD(quantize),        FO_METHOD(dequantize), FO_METHOD(matmul),
                         FO_METHOD(linear), FO_METHOD(linear_backward), FO_METHOD(norm),       FO_METHOD(norm_backward),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }
