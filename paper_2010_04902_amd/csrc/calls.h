// Shared by the Python modules of the worker operators' common calls (not part of the C-ABI): a call's tensors, checked, and its
// results.
#ifndef BYZ_CALLS_H
#define BYZ_CALLS_H

#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <torch/csrc/autograd/python_variable.h>

#include <cstring>
#include <vector>

#include "byzshield_worker.h"

namespace {

PyObject *get_device = nullptr, *get_stream = nullptr;  // torch's: the current GPU, the handle of its current stream
constexpr char no_graph[] =  // as in worker.py
    "outputs are not part of autograd's graph: gradients come from the operator's own backward call (no warning under torch.no_grad)";

// The tensors of a call: each is looked at once, and the first that is not as it has to be spoils the call.
struct Call {
    bool good = true, graph = false;  // graph: of a tensor that requires a gradient
    int device = -1;
    void need(bool b) { good = good && b; }
    // a tensor of torch's own class on the call's GPU; an empty one where the call is spoilt
    const at::Tensor &tensor(PyObject *o) {
        static const at::Tensor nothing;
        if (!good || !THPVariable_CheckExact(o)) return good = false, nothing;
        const at::Tensor &t = THPVariable_Unpack(o);
        if (!t.is_cuda() || t.layout() != c10::kStrided || t.numel() == 0) return good = false, nothing;
        graph = graph || t.requires_grad();
        if (device < 0)
            device = t.get_device();
        else
            need(t.get_device() == device);
        return t;
    }
    const at::Tensor &matrix(PyObject *o, c10::ScalarType type) {
        const at::Tensor &t = tensor(o);
        need(t.defined() && t.dim() == 2 && t.scalar_type() == type && t.is_contiguous());
        return t;
    }
    // contiguous fp32 of these sizes; None is no address where that is allowed
    const float *floats(PyObject *o, c10::IntArrayRef sizes, bool none = false) {
        if (none && o == Py_None) return nullptr;
        const at::Tensor &t = tensor(o);
        need(t.defined() && t.scalar_type() == at::kFloat && t.sizes() == sizes && t.is_contiguous());
        return good ? (const float *)t.data_ptr() : nullptr;
    }
    const int32_t *integers(PyObject *o, c10::IntArrayRef sizes) {
        const at::Tensor &t = tensor(o);
        need(t.defined() && t.scalar_type() == at::kInt && t.sizes() == sizes && t.is_contiguous());
        return good ? (const int32_t *)t.data_ptr() : nullptr;
    }
    uint64_t word(PyObject *o) {  // the low 64 bits
        if (!PyLong_CheckExact(o)) return good = false, 0;
        return PyLong_AsUnsignedLongLongMask(o);
    }
    int64_t integer64(PyObject *o) {
        int overflow = 0;
        const long long v = PyLong_CheckExact(o) ? PyLong_AsLongLongAndOverflow(o, &overflow) : (overflow = 1, 0LL);
        need(!overflow);
        return v;
    }
    int integer(PyObject *o) {
        int overflow = 0;
        const long v = PyLong_CheckExact(o) ? PyLong_AsLongAndOverflow(o, &overflow) : (overflow = 1, 0L);
        need(!overflow && v >= INT32_MIN && v <= INT32_MAX);
        return (int)v;
    }
    float real(PyObject *o) {
        if (PyLong_CheckExact(o)) return (float)integer(o);
        if (!PyFloat_CheckExact(o)) return good = false, 0.0f;
        return (float)PyFloat_AS_DOUBLE(o);
    }
    int dtype(const at::Tensor &t) {
        if (!good) return -1;
        const auto type = t.scalar_type();
        const int code = type == at::kFloat ? BYZ_F32 : type == at::kBFloat16 ? BYZ_BF16 : type == at::kHalf ? BYZ_F16 : -1;
        need(code >= 0);
        return code;
    }
    // A forward call whose outputs somebody may take for part of autograd's graph is worth a word; where warnings are
    // errors the Python path raises it.
    void outside_the_graph() {
        if (good && graph && at::GradMode::is_enabled()) good = PyErr_WarnEx(PyExc_RuntimeWarning, no_graph, 2) == 0;
    }
    // the handle of the current stream; spoils the call if its tensors are not on the current GPU
    void *stream() {
        if (!good) return nullptr;
        PyObject *now = PyObject_CallNoArgs(get_device);
        const long current = now ? PyLong_AsLong(now) : -1;
        PyObject *handle = now && current == device ? PyObject_CallOneArg(get_stream, now) : nullptr;
        Py_XDECREF(now);
        void *s = handle ? PyLong_AsVoidPtr(handle) : nullptr;
        if (!handle || PyErr_Occurred()) PyErr_Clear(), good = false;
        Py_XDECREF(handle);
        return s;
    }
};

at::Tensor fp32(c10::IntArrayRef sizes, const at::Tensor &like) { return at::empty(sizes, like.options().dtype(at::kFloat)); }
at::Tensor bytes(size_t n, const at::Tensor &like) {
    return n ? at::empty({(int64_t)n}, like.options().dtype(at::kByte)) : at::Tensor();
}
void *address(const at::Tensor &t) { return t.defined() ? t.data_ptr() : nullptr; }

// What a call gives back: its code where it failed, else the tensors.
struct Result {
    int rc;
    std::vector<at::Tensor> tensors;
};

// Allocates and enqueues by `work`, which can wait for the GPU: other threads go on meanwhile.
template <typename F>
PyObject *answer(F work) {
    struct Unlocked {
        PyThreadState *const state = PyEval_SaveThread();
        ~Unlocked() { PyEval_RestoreThread(state); }
    };
    const Result r = [&] {
        const Unlocked unlocked;
        return work();
    }();
    if (r.rc != BYZ_OK) return PyLong_FromLong(r.rc);
    if (r.tensors.size() == 1) return THPVariable_Wrap(r.tensors[0]);
    PyObject *out = PyTuple_New((Py_ssize_t)r.tensors.size());
    for (size_t i = 0; out && i < r.tensors.size(); i++) {
        PyObject *o = THPVariable_Wrap(r.tensors[i]);
        if (!o) {
            Py_DECREF(out);
            return nullptr;
        }
        PyTuple_SET_ITEM(out, (Py_ssize_t)i, o);
    }
    return out;
}

// Runs `body(args)` for `count` arguments; no C++ exception leaves: the Python path meets its cause again.
template <typename F>
PyObject *guarded(Py_ssize_t given, Py_ssize_t count, F body) {
    if (given == count) {
        try {
            if (PyObject *o = body()) return o;
        } catch (const std::exception &) {
        }
        PyErr_Clear();
    }
    Py_RETURN_NONE;
}

// torch's functions that calls ask; false where they are not there
inline bool find_torch() {
    PyObject *torch_c = PyImport_ImportModule("torch._C");
    if (!torch_c) return false;
    get_device = PyObject_GetAttrString(torch_c, "_cuda_getDevice");
    get_stream = get_device ? PyObject_GetAttrString(torch_c, "_cuda_getCurrentRawStream") : nullptr;
    Py_DECREF(torch_c);
    return get_stream != nullptr;
}

}  // namespace

#define BYZ_CALL(name) {#name, (PyCFunction)(void (*)())name, METH_FASTCALL, nullptr}

#endif
