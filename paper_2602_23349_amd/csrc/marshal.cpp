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
decltype(&flashoptim_token_logprob) call_logprob;
decltype(&flashoptim_token_logprob_backward) call_logprob_backward;
decltype(&flashoptim_policy_loss) call_policy;
decltype(&flashoptim_preference_loss) call_preference;
decltype(&flashoptim_grad_norm) call_grad_norm;
decltype(&flashoptim_clip_gradients) call_clip;
PyObject *current_stream, *current_device;      // torch._C._cuda_getCurrentRawStream, _cuda_getDevice

// The arguments of one call, taken in order.  After the first failure a Python error is set and nothing more is taken.
struct Args {
    PyObject* const* at;
    Py_ssize_t n, i = 0;
    bool failed = false;
    const bool one_device;               // all tensors lie on one device, the current one
    int64_t device = -1;

    Args(PyObject* const* args, Py_ssize_t count, Py_ssize_t expected, bool one_device_ = false) : at(args), n(count), one_device(one_device_) {
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
        if (one_device && !failed) {
            const int64_t on = t->get_device();      // (may run Python, so ahead of any error)
            if (device >= 0 && device != on) fail(PyExc_ValueError, "%s: on another device than the others", name);
            device = on;
        }
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
    float number() {
        PyObject* o = next();
        if (failed) return 0.0f;
        const double v = PyFloat_AsDouble(o);
        failed = v == -1.0 && PyErr_Occurred() != nullptr;
        return (float)v;
    }
    int64_t integer() {
        PyObject* o = next();
        if (failed) return 0;
        const long long v = PyLong_AsLongLong(o);
        failed = v == -1 && PyErr_Occurred() != nullptr;
        return (int64_t)v;
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
    // A stream's handle, or None for the current stream of the current device.  A call whose tensors lie on one device runs on that one only.
    void* stream() {
        PyObject* o = next();
        if (failed) return nullptr;
        PyObject* current = o == Py_None || (one_device && device >= 0) ? PyObject_CallNoArgs(current_device) : nullptr;
        if (current && one_device && device >= 0 && PyLong_AsLongLong(current) != device) fail(PyExc_ValueError, "%s", "the tensors lie on another device than the current one");
        PyObject* handle = o != Py_None ? Py_NewRef(o) : current && !failed ? PyObject_CallOneArg(current_stream, current) : nullptr;
        Py_XDECREF(current);
        if (!handle) {
            failed = true;
            return nullptr;
        }
        void* v = PyLong_AsVoidPtr(handle);
        failed = failed || PyErr_Occurred() != nullptr;
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

// Whether bind() has been given the call's address.
template <typename F>
void bound(Args& a, F* call) {
    if (!call) a.fail(PyExc_RuntimeError, "%s", "an entry point is missing");
}

PyObject* logprob(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n, 8, true);
    flashoptim_matrix mx;
    void* ws;
    int64_t bytes;
    const flashoptim_matrix* x = a.matrix("logits", &mx);
    const int64_t rows = x ? x->rows : 0;
    const void* tokens = a.plain("tokens", at::kLong, -1, 0, rows);
    const float temperature = a.number();
    void* logprob = a.plain("logprob", at::kFloat, -1, 0, rows);
    void* wide = a.plain("logprob64", at::kDouble, -1, 0, rows);
    void* lse = a.plain("lse", at::kFloat, -1, 0, rows);
    a.workspace(&ws, &bytes);
    void* stream = a.stream();
    bound(a, call_logprob);
    return status(a, a.failed ? 0 : call_logprob(x, (const int64_t*)tokens, temperature, (float*)logprob, (double*)wide, (float*)lse, ws, bytes, stream));
}

PyObject* logprob_backward(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n, 7, true);
    flashoptim_matrix mx, md;
    const flashoptim_matrix* x = a.matrix("logits", &mx);
    const int64_t rows = x ? x->rows : 0;
    const void* tokens = a.plain("tokens", at::kLong, -1, 0, rows);
    const float temperature = a.number();
    const void* lse = a.plain("lse", at::kFloat, -1, 0, rows);
    const void* d = a.plain("dlogprob", at::kFloat, -1, 0, rows);
    const flashoptim_matrix* dx = a.matrix("dlogits", &md);
    void* stream = a.stream();
    bound(a, call_logprob_backward);
    return status(a, a.failed ? 0 : call_logprob_backward(x, (const int64_t*)tokens, temperature, (const float*)lse, (const float*)d, dx, stream));
}

PyObject* policy(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n, 12, true);
    flashoptim_matrix mx, md;
    flashoptim_policy_inputs in;
    void* ws;
    int64_t bytes;
    const auto* spec = a.address<flashoptim_policy_spec>();
    const flashoptim_matrix* x = a.matrix("logits", &mx);
    const int64_t rows = x ? x->rows : 0;
    const void* tokens = a.plain("tokens", at::kLong, -1, 0, rows);
    in.advantages = (const float*)a.plain("advantages", at::kFloat, -1, 0, rows);
    in.old_logprob = (const float*)a.plain("old_logprob", at::kFloat, -1, 0, rows);
    in.ref_logprob = (const float*)a.plain("ref_logprob", at::kFloat, -1, 0, rows);
    in.weights = (const float*)a.plain("weights", at::kFloat, -1, 0, rows);
    void* stats = a.plain("stats", at::kFloat, -1, 0, 4);
    void* logprob = a.plain("logprob", at::kFloat, -1, 0, rows);
    const flashoptim_matrix* dx = a.matrix("dlogits", &md);
    a.workspace(&ws, &bytes);
    void* stream = a.stream();
    bound(a, call_policy);
    return status(a, a.failed ? 0 : call_policy(spec, x, (const int64_t*)tokens, &in, (float*)stats, (float*)logprob, dx, ws, bytes, stream));
}

PyObject* preference(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n, 9, true);
    const auto* spec = a.address<flashoptim_preference_spec>();
    const at::Tensor* first = a.tensor("logprob");
    const int64_t rows = first ? first->numel() : 0;
    const bool wide = first && first->scalar_type() == at::kDouble;
    if (!a.failed) --a.i;
    const void* logprob = a.plain("logprob", wide ? at::kDouble : at::kFloat, -1, 0, rows);
    const at::Tensor* cuts = a.tensor("offsets");
    const int64_t bounds = cuts ? cuts->numel() : 1;
    if (!a.failed) --a.i;
    const void* offsets = a.plain("offsets", at::kLong, -1, 0, bounds);
    if (bounds % 2 == 0) a.fail(PyExc_ValueError, "%s", "offsets: the bounds of an even number of sequences, one more than that");
    const int64_t pairs = bounds / 2;
    void* loss = a.plain("loss", at::kFloat, -1, 0, 1);
    const void* ref = a.plain("ref_logprob", at::kFloat, -1, 0, rows);
    const void* weights = a.plain("weights", at::kFloat, -1, 0, rows);
    void* margins = a.plain("margins", at::kFloat, -1, 0, pairs);
    void* d = a.plain("dlogprob", at::kFloat, -1, 0, rows);
    void* stream = a.stream();
    bound(a, call_preference);
    return status(a, a.failed ? 0 : call_preference(spec, wide ? nullptr : (const float*)logprob, wide ? (const double*)logprob : nullptr, (const float*)ref, (const float*)weights, rows,
                                                    (const int64_t*)offsets, pairs, (float*)loss, (float*)margins, (float*)d, stream));
}

// A list of gradients: its address, length, the types of what is read and of what is written, and the device that it and its factor lie on.
struct Gradients {
    const flashoptim_gradient* list;
    int64_t n;
    int src, dst;
    explicit Gradients(Args& a) {
        list = a.address<flashoptim_gradient>();
        n = a.integer();
        src = (int)a.integer();
        dst = (int)a.integer();
        a.device = a.integer();
    }
};

PyObject* grad_norm(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n, 9, true);
    void* ws;
    int64_t bytes;
    const Gradients g(a);
    const float max_norm = a.number();
    auto* factor = const_cast<flashoptim_clip_factor*>(a.address<flashoptim_clip_factor>());
    a.workspace(&ws, &bytes);
    void* stream = a.stream();
    bound(a, call_grad_norm);
    return status(a, a.failed ? 0 : call_grad_norm(g.list, g.n, g.src, max_norm, factor, ws, bytes, stream));
}

PyObject* clip(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n, 7, true);
    const Gradients g(a);
    const auto* factor = a.address<flashoptim_clip_factor>();
    void* stream = a.stream();
    bound(a, call_clip);
    return status(a, a.failed ? 0 : call_clip(g.list, g.n, g.src, g.dst, factor, stream));
}

// follow(gradients, tensors, count): each gradient is read and clipped where its tensor's descriptor has it now.
PyObject* follow(PyObject*, PyObject* const* args, Py_ssize_t n) {
    Args a(args, n, 3);
    auto* gradients = const_cast<flashoptim_gradient*>(a.address<flashoptim_gradient>());
    const auto* tensors = a.address<flashoptim_tensor>();
    const int64_t count = a.integer();
    if (a.failed) return nullptr;
    for (int64_t i = 0; i < count; ++i) gradients[i].src = gradients[i].dst = const_cast<void*>((const void*)tensors[i].grad);
    Py_RETURN_NONE;
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
    take(args[0], "flashoptim_token_logprob", call_logprob);
    take(args[0], "flashoptim_token_logprob_backward", call_logprob_backward);
    take(args[0], "flashoptim_policy_loss", call_policy);
    take(args[0], "flashoptim_preference_loss", call_preference);
    take(args[0], "flashoptim_grad_norm", call_grad_norm);
    take(args[0], "flashoptim_clip_gradients", call_clip);
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
                         FO_METHOD(logprob), FO_METHOD(logprob_backward), FO_METHOD(policy), FO_METHOD(preference),
                         FO_METHOD(grad_norm), FO_METHOD(clip), FO_METHOD(follow),
                         {nullptr, nullptr, 0, nullptr}};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "_marshal", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__marshal(void) { return PyModule_Create(&module); }
