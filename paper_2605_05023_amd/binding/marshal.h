// marshal.h -- helpers of the native argument marshalling (fast.cpp, fast_cache.cpp).
#pragma once

#include <ATen/ATen.h>
#include <ATen/PythonTorchFunctionTLS.h>
#include <Python.h>
#include <c10/core/DeviceGuard.h>
#include <c10/core/impl/TorchDispatchModeTLS.h>
#include <c10/hip/HIPStream.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cmath>

#include "../../include/attn.h"

namespace attn_py {

// A plain device tensor: no subclass, no functional transform, no lazy bit.
inline bool plain(PyObject* o, at::Tensor* t)
{
    if (!THPVariable_CheckExact(o)) return false;
    *t = THPVariable_Unpack(o);
    if (!t->defined() || !t->is_cuda() || t->layout() != at::kStrided) return false;
    using c10::DispatchKey;
    const c10::DispatchKeySet odd({DispatchKey::Python, DispatchKey::Functionalize, DispatchKey::Conjugate,
                                   DispatchKey::Negative, DispatchKey::ZeroTensor,
                                   DispatchKey::FuncTorchBatched, DispatchKey::FuncTorchGradWrapper});
    return !t->key_set().has_any(odd);
}

// An axis of more than one entry with stride 0 (an expanded tensor): the
// descriptor takes a stride of 0 for the contiguous default.
inline bool broadcast(const at::Tensor& t)
{
    for (int64_t i = 0; i < t.dim(); ++i)
        if (t.stride(i) == 0 && t.size(i) > 1) return true;
    return false;
}

inline bool as_int(PyObject* o, int64_t* v)
{
    if (!PyLong_CheckExact(o)) return false;
    int overflow = 0;
    *v = PyLong_AsLongLongAndOverflow(o, &overflow);
    return overflow == 0;
}

inline bool as_i32(PyObject* o, int32_t* v)
{
    int64_t x;
    if (!as_int(o, &x) || x < INT32_MIN || x > INT32_MAX) return false;
    *v = (int32_t)x;
    return true;
}

inline bool as_float(PyObject* o, float* v)
{
    if (PyFloat_CheckExact(o)) {
        *v = (float)PyFloat_AS_DOUBLE(o);
        return true;
    }
    int32_t i;
    if (!as_i32(o, &i)) return false;
    *v = (float)i;
    return true;
}

inline bool is(PyObject* o, const char* s) { return PyUnicode_CompareWithASCIIString(o, s) == 0; }

// The value of a name in `names`, or of an exact int.
inline bool as_kind(PyObject* o, const char* const* names, int n, int32_t* v)
{
    if (PyUnicode_CheckExact(o)) {
        for (int i = 0; i < n; ++i)
            if (is(o, names[i])) {
                *v = i;
                return true;
            }
        return false;
    }
    return as_i32(o, v);
}

struct NoGil {
    PyThreadState* state = PyEval_SaveThread();
    ~NoGil() { PyEval_RestoreThread(state); }
};

// A mode of torch's that would see the calls made here.
inline bool modes()
{
    return at::impl::torch_function_mode_enabled() || c10::impl::TorchDispatchModeTLS::any_modes_set();
}

// Raise the AttnError of a status (returns NULL).
inline PyObject* raise_status(int status)
{
    PyObject* abi = PyImport_ImportModule("paper_2605_05023_amd._abi");
    PyObject* none = abi ? PyObject_CallMethod(abi, "check", "i", status) : nullptr;
    Py_XDECREF(abi);
    return none;
}

// out, or (out, lse): the caller's own objects where it passed them.
inline PyObject* outputs(PyObject* out_arg, const at::Tensor& out, PyObject* lse_arg, const at::Tensor& lse,
                         bool with_lse)
{
    PyObject* o = out_arg == Py_None ? THPVariable_Wrap(out) : Py_NewRef(out_arg);
    if (!o || !with_lse) return o;
    PyObject* l = lse_arg == Py_None ? THPVariable_Wrap(lse) : Py_NewRef(lse_arg);
    if (!l) {
        Py_DECREF(o);
        return nullptr;
    }
    PyObject* r = PyTuple_Pack(2, o, l);
    Py_DECREF(o);
    Py_DECREF(l);
    return r;
}

// fast_cache.cpp
PyObject* py_cache_plan(PyObject*, PyObject* const* a, Py_ssize_t n);
PyObject* py_cache_append(PyObject*, PyObject* const* a, Py_ssize_t n);
PyObject* py_cache_fwd(PyObject*, PyObject* const* a, Py_ssize_t n);
PyObject* py_bind_cache(PyObject*, PyObject* args);

}  // namespace attn_py
