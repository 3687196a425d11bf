// Argument marshalling of a policy's forwards, V-trace, the KL indicators and the operators of wide policies, as a CPython module: tensors are checked and taken to pointers here, and
// the library is called without the interpreter's lock.  A call of 32 states on the 64-unit MLP costs the host what the checks, the
// conversions of eight ctypes arguments and the launch cost; the kernel takes 2.5 us.
//
// Every function returns the library's status, or None for arguments that are not plain: tensors of another type than torch.Tensor itself,
// another dtype, device or layout than the call takes, shapes that do not match, an active torch-function mode, a stream object.  The
// caller then goes the general way (binding.py), which raises the error or finds the pointer.  The operators of wide policies also make their
// outputs here (a call of the loss through ctypes costs the host 25 us, its kernels take 9 for 32 rows of 18 actions), and return
// (status, outputs ..).
#define PY_SSIZE_T_CLEAN
#include <Python.h>

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <c10/hip/HIPFunctions.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <vector>

#include "accerl.h"

namespace {

PyTypeObject* handle_type = nullptr;      // ctypes.c_void_p
PyObject* value_name = nullptr;

// One argument after the other; `plain` turns false at the first one that is not.
struct Args {
    PyObject* const* at;
    bool plain;
    int device;                               // where all tensors lie; negative: anywhere

    explicit Args(PyObject* const* a, int device = -1) : at(a), plain(!at::impl::torch_function_mode_enabled()), device(device) {}

    bool here(const at::Tensor& t) const { return t.is_cuda() && (device < 0 || t.device().index() == device); }

    const at::Tensor* tensor() {
        PyObject* o = *at++;
        if (!plain || Py_TYPE(o) != (PyTypeObject*)THPVariableClass) { plain = false; return nullptr; }
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!here(t) || !t.is_contiguous()) plain = false;
        return &t;
    }
    void* pointer(c10::ScalarType type) {
        if (*at == Py_None) { ++at; return nullptr; }
        const at::Tensor* t = tensor();
        if (plain && t->scalar_type() != type) plain = false;
        return plain ? t->data_ptr() : nullptr;
    }
    // a tensor of this shape
    void* shaped(c10::ScalarType type, c10::IntArrayRef shape) {
        const at::Tensor* t = tensor();
        if (plain && (t->scalar_type() != type || t->sizes() != shape)) plain = false;
        return plain ? t->data_ptr() : nullptr;
    }
    float* f32() { return (float*)pointer(c10::kFloat); }
    accerl_policy* handle() {
        PyObject* o = *at++;
        if (!plain || Py_TYPE(o) != handle_type) { plain = false; return nullptr; }
        PyObject* v = PyObject_GetAttr(o, value_name);
        void* p = v && v != Py_None ? PyLong_AsVoidPtr(v) : nullptr;
        Py_XDECREF(v);
        return (accerl_policy*)p;
    }
    void* states(int64_t* B) {
        const at::Tensor* t = tensor();
        if (plain && t->dim() < 1) plain = false;
        if (!plain) return nullptr;
        *B = t->size(0);
        return t->data_ptr();
    }
    // a matrix whose rows are contiguous, of this type and shape unless they are to be found out (type Undefined, B < 0); `maybe`: or None
    void* rows(c10::ScalarType* type, int64_t* B, int64_t* A, int64_t* ld, bool maybe = false) {
        if (maybe && *at == Py_None) { ++at; *ld = 0; return nullptr; }
        PyObject* o = *at++;
        if (!plain || Py_TYPE(o) != (PyTypeObject*)THPVariableClass) { plain = false; return nullptr; }
        const at::Tensor& t = THPVariable_Unpack(o);
        if (!here(t) || t.dim() != 2 || (*type != c10::ScalarType::Undefined && t.scalar_type() != *type) || (*B >= 0 && t.size(0) != *B) ||
            (*A >= 0 && t.size(1) != *A)) { plain = false; return nullptr; }
        *type = t.scalar_type();
        *B = t.size(0);
        *A = t.size(1);
        *ld = *B > 1 ? t.stride(0) : *A;
        if ((*A > 1 && t.stride(1) != 1) || *ld < *A) { plain = false; return nullptr; }
        return t.data_ptr();
    }
    // a vector of n, or None
    void* vector(c10::ScalarType type, int64_t n) {
        if (*at == Py_None) { ++at; return nullptr; }
        const at::Tensor* t = tensor();
        if (plain && (t->scalar_type() != type || t->dim() != 1 || t->size(0) != n)) plain = false;
        return plain ? t->data_ptr() : nullptr;
    }
    // uint8 [B, A], or [1, A] with a row stride of 0
    uint8_t* mask(int64_t B, int64_t A, int64_t* ld) {
        c10::ScalarType type = c10::kByte;
        int64_t rows_of = -1;
        void* p = rows(&type, &rows_of, &A, ld, true);
        if (p && rows_of != 1 && rows_of != B) plain = false;
        if (p && rows_of == 1) *ld = 0;
        return (uint8_t*)p;
    }
    int64_t integer() {
        PyObject* o = *at++;
        if (!PyLong_CheckExact(o)) { plain = false; return 0; }
        return PyLong_AsLongLong(o);
    }
    void* stream() {
        PyObject* o = *at++;
        if (o == Py_None) return plain ? (void*)c10::hip::getCurrentHIPStream().stream() : nullptr;
        if (!PyLong_CheckExact(o)) { plain = false; return nullptr; }
        return PyLong_AsVoidPtr(o);
    }
    double number() {
        PyObject* o = *at++;
        if (!PyFloat_CheckExact(o)) { plain = false; return 0.0; }
        return PyFloat_AS_DOUBLE(o);
    }
};

// count arguments: parse(args) reads them in order and returns the call that is then made
template <class Parse>
PyObject* call(PyObject* const* argv, Py_ssize_t given, Py_ssize_t count, Parse&& parse) {
    if (given != count) { PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", count, given); return nullptr; }
    try {
        Args a(argv);
        auto made = parse(a);
        if (PyErr_Occurred()) { PyErr_Clear(); a.plain = false; }
        if (!a.plain) Py_RETURN_NONE;
        int rc = 0;
        bool threw = false;                      // (said only when the lock is held again, and never taken for arguments that are not plain)
        Py_BEGIN_ALLOW_THREADS
        try { rc = made(); } catch (...) { threw = true; }
        Py_END_ALLOW_THREADS
        if (threw) { PyErr_SetString(PyExc_RuntimeError, "the library threw an exception"); return nullptr; }
        return PyLong_FromLong(rc);
    } catch (const std::exception&) {            // a tensor without storage, for one: the general way says it
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

template <int (*F)(accerl_policy*, const void*, int64_t, const float*, float*, float*, int32_t*, void*)>
PyObject* forward(PyObject*, PyObject* const* argv, Py_ssize_t n) {
    return call(argv, n, 7, [](Args& a) {
        int64_t B = 0;
        accerl_policy* p = a.handle();
        void* x = a.states(&B);
        float *u = a.f32(), *l = a.f32(), *v = a.f32();
        int32_t* act = (int32_t*)a.pointer(c10::kInt);
        void* s = a.stream();
        return [=] { return F(p, x, B, u, l, v, act, s); };
    });
}

PyObject* recurrent(PyObject*, PyObject* const* argv, Py_ssize_t n) {
    return call(argv, n, 10, [](Args& a) {
        int64_t B = 0;
        accerl_policy* p = a.handle();
        void* x = a.states(&B);
        float* u = a.f32();
        uint8_t* done = (uint8_t*)a.pointer(c10::kByte);
        float *h = a.f32(), *c = a.f32(), *l = a.f32(), *v = a.f32();
        int32_t* act = (int32_t*)a.pointer(c10::kInt);
        void* s = a.stream();
        return [=] { return accerl_actor_forward_recurrent(p, x, B, u, done, h, c, l, v, act, s); };
    });
}

template <int (*F)(const float*, const float*, int64_t, int32_t, float*, float*, double*, void*)>
PyObject* monitor(PyObject*, PyObject* const* argv, Py_ssize_t n) {
    return call(argv, n, 6, [](Args& a) {
        const at::Tensor* o = a.tensor();
        if (a.plain && (o->scalar_type() != c10::kFloat || o->dim() != 2)) a.plain = false;
        const int64_t B = a.plain ? o->size(0) : 0, A = a.plain ? o->size(1) : 0;
        const float* po = a.plain ? (const float*)o->data_ptr() : nullptr;
        const float* ps = (const float*)a.shaped(c10::kFloat, {B, A});
        float *kl = a.f32(), *ent = a.f32();
        double* st = (double*)a.pointer(c10::kDouble);
        void* s = a.stream();
        return [=] { return F(po, ps, B, (int32_t)A, kl, ent, st, s); };
    });
}

PyObject* vtrace(PyObject*, PyObject* const* argv, Py_ssize_t n) {
    return call(argv, n, 13, [](Args& a) {
        const at::Tensor* o = a.tensor();
        if (a.plain && (o->scalar_type() != c10::kFloat || o->dim() != 3)) a.plain = false;
        const int64_t T = a.plain ? o->size(0) : 0, B = a.plain ? o->size(1) : 0, A = a.plain ? o->size(2) : 0;
        const float* po = a.plain ? (const float*)o->data_ptr() : nullptr;
        const float* ps = (const float*)a.shaped(c10::kFloat, {T, B, A});
        const int32_t* act = (const int32_t*)a.shaped(c10::kInt, {T, B});
        const float *rew = (const float*)a.shaped(c10::kFloat, {T, B}), *disc = (const float*)a.shaped(c10::kFloat, {T, B});
        const float* val = (const float*)a.shaped(c10::kFloat, {T, B});
        const float* boot = a.f32();
        const double rho_bar = a.number(), c_bar = a.number();
        float* vs = (float*)a.shaped(c10::kFloat, {T, B});
        float* adv = a.f32();
        float* rho = (float*)a.shaped(c10::kFloat, {T, B});
        void* s = a.stream();
        return [=] { return accerl_vtrace(po, ps, act, rew, disc, val, boot, T, B, (int32_t)A, (float)rho_bar, (float)c_bar, vs, adv, rho, s); };
    });
}

int dtype_code(c10::ScalarType t) { return t == c10::kFloat ? ACCERL_DT_F32 : t == c10::kBFloat16 ? ACCERL_DT_BF16 : t == c10::kHalf ? ACCERL_DT_F16 : -1; }
constexpr c10::ScalarType CODES[3] = {c10::kFloat, c10::kBFloat16, c10::kHalf};

at::Tensor made(c10::IntArrayRef shape, c10::ScalarType type) { return at::empty(shape, c10::TensorOptions(c10::kCUDA).dtype(type)); }

// Like call(), for functions that make their outputs: parse(args, outputs) reads the arguments, appends the outputs and returns the call.  Outputs are made
// on the current device, where the call's tensors must lie.
template <class Parse>
PyObject* call_out(PyObject* const* argv, Py_ssize_t given, Py_ssize_t count, Parse&& parse) {
    if (given != count) { PyErr_Format(PyExc_TypeError, "expected %zd arguments, got %zd", count, given); return nullptr; }
    try {
        Args a(argv, c10::hip::current_device());
        std::vector<at::Tensor> outs;
        auto run = parse(a, outs);
        if (PyErr_Occurred()) { PyErr_Clear(); a.plain = false; }
        if (!a.plain) Py_RETURN_NONE;
        int rc = 0;
        bool threw = false;
        Py_BEGIN_ALLOW_THREADS
        try { rc = run(); } catch (...) { threw = true; }
        Py_END_ALLOW_THREADS
        if (threw) { PyErr_SetString(PyExc_RuntimeError, "the library threw an exception"); return nullptr; }
        PyObject* t = PyTuple_New(1 + (Py_ssize_t)outs.size());
        if (!t) return nullptr;
        PyTuple_SET_ITEM(t, 0, PyLong_FromLong(rc));
        for (size_t i = 0; i < outs.size(); ++i) PyTuple_SET_ITEM(t, 1 + (Py_ssize_t)i, THPVariable_Wrap(outs[i]));
        return t;
    } catch (const std::exception&) {
        PyErr_Clear();
        Py_RETURN_NONE;
    }
}

// (x, N, K, w_packed, w_scale, bias, relu, type of the output or -1 for x's, workspace, stream) -> (status, out)
PyObject* dense_dynamic(PyObject*, PyObject* const* argv, Py_ssize_t n) {
    return call_out(argv, n, 10, [](Args& a, std::vector<at::Tensor>& outs) {
        c10::ScalarType type = c10::ScalarType::Undefined;
        int64_t M = -1, Kx = -1, ldx = 0, bytes = 0;
        const void* x = a.rows(&type, &M, &Kx, &ldx);
        const int code = dtype_code(type);
        const int64_t N = a.integer(), K = a.integer();
        const at::Tensor* w = a.tensor();
        const float *sw = (const float*)a.vector(c10::kFloat, N), *bias = (const float*)a.vector(c10::kFloat, N);
        const int64_t relu = a.integer();
        int64_t out = a.integer();
        const at::Tensor* ws = a.tensor();
        void* s = a.stream();
        if (out < 0) out = code;
        if (code < 0 || out > 2 || Kx != K || !sw) a.plain = false;
        if (a.plain && (w->scalar_type() != c10::kChar || w->numel() < accerl_packed_rows_bytes(N, K))) a.plain = false;
        const int8_t* pw = a.plain ? (const int8_t*)w->data_ptr() : nullptr;
        void *po = nullptr, *pws = nullptr;
        if (a.plain) {
            bytes = ws->numel();
            pws = ws->data_ptr();
            if (bytes < accerl_dense_i8_workspace(M, K)) a.plain = false;
            else {
                outs.push_back(made({M, N}, CODES[out]));
                po = outs[0].data_ptr();
            }
        }
        return [=] { return accerl_dense_i8_dynamic(x, code, ldx, pw, sw, bias, M, N, K, (int32_t)relu, po, (int32_t)out, N, pws, bytes, s); };
    });
}

// (logits, actions, mask, workspace, stream) -> (status, log-probabilities, entropies)
PyObject* action_logprob(PyObject*, PyObject* const* argv, Py_ssize_t n) {
    return call_out(argv, n, 5, [](Args& a, std::vector<at::Tensor>& outs) {
        c10::ScalarType type = c10::ScalarType::Undefined;
        int64_t B = -1, A = -1, ld = 0, ldm = 0, bytes = 0;
        const void* z = a.rows(&type, &B, &A, &ld);
        const int code = dtype_code(type);
        const int32_t* act = (const int32_t*)a.vector(c10::kInt, B);
        const uint8_t* mask = a.mask(B, A, &ldm);
        const at::Tensor* ws = a.tensor();
        void* s = a.stream();
        if (code < 0 || !act) a.plain = false;
        float *lp = nullptr, *ent = nullptr;
        void* pws = nullptr;
        if (a.plain) {
            bytes = ws->numel();
            pws = ws->data_ptr();
            outs.push_back(made({B}, c10::kFloat));
            outs.push_back(made({B}, c10::kFloat));
            lp = (float*)outs[0].data_ptr();
            ent = (float*)outs[1].data_ptr();
        }
        return [=] { return accerl_action_logprob(z, code, ld, mask, ldm, act, B, A, lp, ent, pws, bytes, s); };
    });
}

// (logits, actions, old_logp, advantages, mask, weights, ref_logits, ref_logp, gradient: 0 none, 1 a new one, kind of KL, clip_low, clip_high, kl_coef,
// entropy_coef, scale, workspace, stream) -> (status, loss, logp, kl, entropy, stats[, gradient])
PyObject* policy_loss(PyObject*, PyObject* const* argv, Py_ssize_t n) {
    return call_out(argv, n, 17, [](Args& a, std::vector<at::Tensor>& outs) {
        accerl_policy_loss_args p{};
        c10::ScalarType type = c10::ScalarType::Undefined;
        p.B = p.A = -1;
        p.logits = a.rows(&type, &p.B, &p.A, &p.ld_logits);
        p.dtype = dtype_code(type);
        p.actions = (const int32_t*)a.vector(c10::kInt, p.B);
        p.old_logp = (const float*)a.vector(c10::kFloat, p.B);
        p.advantages = (const float*)a.vector(c10::kFloat, p.B);
        p.mask = a.mask(p.B, p.A, &p.ld_mask);
        p.weights = (const float*)a.vector(c10::kFloat, p.B);
        p.ref_logits = a.rows(&type, &p.B, &p.A, &p.ld_ref, true);
        p.ref_logp = (const float*)a.vector(c10::kFloat, p.B);
        const int64_t grad = a.integer();
        p.kl_kind = (int32_t)a.integer();
        p.clip_low = a.number(); p.clip_high = a.number(); p.kl_coef = a.number(); p.entropy_coef = a.number(); p.scale = a.number();
        const at::Tensor* ws = a.tensor();
        void* s = a.stream();
        if (p.dtype < 0 || p.B < 1) a.plain = false;
        if (a.plain) {
            p.workspace = ws->data_ptr();
            p.workspace_bytes = ws->numel();
            float** to[4] = {&p.out_loss, &p.out_logp, &p.out_kl, &p.out_entropy};
            for (float** t : to) { outs.push_back(made({p.B}, c10::kFloat)); *t = (float*)outs.back().data_ptr(); }
            outs.push_back(made({4}, c10::kFloat));
            p.out_stats = (float*)outs.back().data_ptr();
            if (grad) {
                outs.push_back(made({p.B, p.A}, type));
                p.grad_logits = outs.back().data_ptr();
                p.ld_grad = p.A;
            }
        }
        return [=] { return accerl_policy_loss(&p, s); };
    });
}

PyObject* init(PyObject*, PyObject* type) {
    if (!PyType_Check(type)) { PyErr_SetString(PyExc_TypeError, "expected ctypes.c_void_p"); return nullptr; }
    Py_INCREF(type);
    handle_type = (PyTypeObject*)type;
    Py_RETURN_NONE;
}

#define FAST(f) (PyCFunction)(void (*)(void))(f), METH_FASTCALL, nullptr
PyMethodDef methods[] = {
    {"init", init, METH_O, nullptr},
    {"forward", FAST(forward<accerl_actor_forward>)},
    {"forward_teacher", FAST(forward<accerl_actor_forward_teacher>)},
    {"forward_recurrent", FAST(recurrent)},
    {"monitor_kl", FAST(monitor<accerl_monitor_kl>)},
    {"monitor_kl_noalloc", FAST(monitor<accerl_monitor_kl_noalloc>)},
    {"vtrace", FAST(vtrace)},
    {"dense_dynamic", FAST(dense_dynamic)},
    {"action_logprob", FAST(action_logprob)},
    {"policy_loss", FAST(policy_loss)},
    {nullptr, nullptr, 0, nullptr},
};
PyModuleDef module = {PyModuleDef_HEAD_INIT, "accerl_args", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit_accerl_args() {
    value_name = PyUnicode_InternFromString("value");
    return value_name ? PyModule_Create(&module) : nullptr;
}
