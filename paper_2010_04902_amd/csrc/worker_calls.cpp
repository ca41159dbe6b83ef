// The worker operators' calls in their common form, for Python: dense tensors, nothing given to write to, the current stream.
//
// A small call is bound by the host.  Checked, allocated and enqueued here, a call takes half of what the same steps take
// in Python (figures in worker.py).  Whatever is not of the common form is answered with None and nothing done: the
// Python path behind it handles or refuses it, so every rule and every word about it stands there alone.  An
// int is the library's error code.
#include <Python.h>

#include <ATen/core/Tensor.h>
#include <ATen/core/grad_mode.h>
#include <ATen/ops/empty.h>
#include <ATen/ops/empty_like.h>
#include <torch/csrc/autograd/python_variable.h>

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

struct Features {
    int64_t n, p, c;
};

bool features(const at::Tensor &x, Features &f) {
    if (x.dim() == 4) {
        f = {x.size(0), x.size(2) * x.size(3), x.size(1)};
        return x.is_contiguous(at::MemoryFormat::ChannelsLast);
    }
    if (x.dim() != 3) return false;
    f = {x.size(0), x.size(1), x.size(2)};
    return x.is_contiguous();
}

// x, groups, gamma, beta, eps, act -> y, mean, rstd
PyObject *group_norm(PyObject *, PyObject *const *o, Py_ssize_t count) {
    return guarded(count, 6, [&]() -> PyObject * {
        Call call;
        Features f{};
        const at::Tensor &x = call.tensor(o[0]);
        call.need(x.defined() && features(x, f));
        const int groups = call.integer(o[1]), dtype = call.dtype(x), act = call.integer(o[5]);
        const float eps = call.real(o[4]);
        const float *gamma = call.floats(o[2], {f.c}, true), *beta = call.floats(o[3], {f.c}, true);
        void *const stream = call.stream();
        call.outside_the_graph();
        if (!call.good || groups < 1) return nullptr;
        return answer([&]() -> Result {
            at::Tensor y = at::empty_like(x), mean = fp32({f.n, groups}, x), rstd = fp32({f.n, groups}, x);
            const size_t need = byz_group_norm_workspace_bytes(f.n, f.p, f.c, groups, dtype);
            const at::Tensor ws = bytes(need, x);
            const int64_t sample = f.p * f.c;
            const int rc = byz_group_norm(x.data_ptr(), sample, f.c, f.n, f.p, f.c, groups, dtype, gamma, beta, eps, act, y.data_ptr(),
                                          sample, f.c, (float *)mean.data_ptr(), (float *)rstd.data_ptr(), address(ws), need, stream);
            return {rc, {y, mean, rstd}};
        });
    });
}

// dy, x, groups, mean, rstd, gamma, beta, act -> dx, dgamma, dbeta
PyObject *group_norm_backward(PyObject *, PyObject *const *o, Py_ssize_t count) {
    return guarded(count, 8, [&]() -> PyObject * {
        Call call;
        Features f{}, g{};
        const at::Tensor &x = call.tensor(o[1]), &dy = call.tensor(o[0]);
        call.need(x.defined() && dy.defined() && features(x, f) && features(dy, g) && x.sizes() == dy.sizes() &&
                  x.scalar_type() == dy.scalar_type());
        const int groups = call.integer(o[2]), dtype = call.dtype(x), act = call.integer(o[7]);
        const float *mean = call.floats(o[3], {f.n, groups}), *rstd = call.floats(o[4], {f.n, groups});
        const float *gamma = call.floats(o[5], {f.c}, true), *beta = call.floats(o[6], {f.c}, true);
        void *const stream = call.stream();
        if (!call.good) return nullptr;
        return answer([&]() -> Result {
            at::Tensor dx = at::empty_like(x), dgamma = fp32({f.c}, x), dbeta = fp32({f.c}, x);
            const size_t need = byz_group_norm_backward_workspace_bytes(f.n, f.p, f.c, groups, dtype);
            const at::Tensor ws = bytes(need, x);
            const int64_t sample = f.p * f.c;
            const int rc = byz_group_norm_backward(dy.data_ptr(), sample, f.c, x.data_ptr(), sample, f.c, f.n, f.p, f.c, groups, dtype, gamma,
                                                   beta, mean, rstd, act, dx.data_ptr(), sample, f.c, (float *)dgamma.data_ptr(),
                                                   (float *)dbeta.data_ptr(), address(ws), need, stream);
            return {rc, {dx, dgamma, dbeta}};
        });
    });
}

// The student's and the teacher's rows.
struct Distill {
    const at::Tensor &logits, &teacher, &index;
    int dtype;
    Distill(Call &call, PyObject *const *o)
        : logits(call.tensor(o[0])), teacher(call.matrix(o[1], at::kFloat)), index(call.matrix(o[2], at::kInt)), dtype(call.dtype(logits)) {
        call.need(call.good && logits.dim() == 2 && logits.is_contiguous() && teacher.sizes() == index.sizes() &&
                  teacher.size(0) == logits.size(0) && teacher.size(1) <= BYZ_MAX_TEACHER);
    }
};

// logits, teacher, index, temperature -> loss, lse
PyObject *distill_loss(PyObject *, PyObject *const *o, Py_ssize_t count) {
    return guarded(count, 4, [&]() -> PyObject * {
        Call call;
        const Distill d(call, o);
        const float temperature = call.real(o[3]);
        void *const stream = call.stream();
        call.outside_the_graph();
        if (!call.good) return nullptr;
        const int64_t rows = d.logits.size(0), vocab = d.logits.size(1), k = d.teacher.size(1);
        return answer([&]() -> Result {
            at::Tensor loss = fp32({rows}, d.logits), lse = fp32({rows}, d.logits);
            const int rc = byz_distill_loss(d.logits.data_ptr(), rows, vocab, vocab, d.dtype, (const float *)d.teacher.data_ptr(),
                                            (const int32_t *)d.index.data_ptr(), (int)k, k, temperature, (float *)loss.data_ptr(),
                                            (float *)lse.data_ptr(), stream);
            return {rc, {loss, lse}};
        });
    });
}

// logits, teacher, index, dloss, temperature -> loss, dlogits
PyObject *distill_loss_step(PyObject *, PyObject *const *o, Py_ssize_t count) {
    return guarded(count, 5, [&]() -> PyObject * {
        Call call;
        const Distill d(call, o);
        if (!call.good) return nullptr;
        const int64_t rows = d.logits.size(0), vocab = d.logits.size(1), k = d.teacher.size(1);
        const float *dloss = call.floats(o[3], {rows});
        const float temperature = call.real(o[4]);
        void *const stream = call.stream();
        if (!call.good) return nullptr;
        return answer([&]() -> Result {
            at::Tensor loss = fp32({rows}, d.logits), dlogits = at::empty_like(d.logits);
            const size_t need = byz_distill_loss_step_workspace_bytes(rows, vocab, (int)k, d.dtype);
            const at::Tensor ws = bytes(need, d.logits);
            const int rc = byz_distill_loss_step(d.logits.data_ptr(), rows, vocab, vocab, d.dtype, (const float *)d.teacher.data_ptr(),
                                                 (const int32_t *)d.index.data_ptr(), (int)k, k, dloss, temperature,
                                                 (float *)loss.data_ptr(), nullptr, dlogits.data_ptr(), vocab, address(ws), need, stream);
            return {rc, {loss, dlogits}};
        });
    });
}

// A block's tokens and weights; aligned: 16-byte rows, so that a forward call needs no workspace and the backward none for copies.
struct Block {
    const at::Tensor &x, &w_gate, &w_up;
    int dtype;
    Block(Call &call, PyObject *const *o, bool only_aligned) : x(call.tensor(o[0])), w_gate(call.tensor(o[1])), w_up(call.tensor(o[2])), dtype(call.dtype(x)) {
        call.need(call.good && dtype != BYZ_F32 && x.dim() == 2 && w_gate.dim() == 2 && w_up.sizes() == w_gate.sizes() &&
                  x.size(1) == w_gate.size(1) && w_gate.scalar_type() == x.scalar_type() && w_up.scalar_type() == x.scalar_type() &&
                  x.is_contiguous() && w_gate.is_contiguous() && w_up.is_contiguous());
        if (call.good && only_aligned && x.size(0) > 16) call.need(aligned());
    }
    bool aligned() const {
        return x.size(1) % 8 == 0 && (((uintptr_t)x.data_ptr() | (uintptr_t)w_gate.data_ptr() | (uintptr_t)w_up.data_ptr()) & 15) == 0;
    }
};

// x, w_gate, w_up, act, save -> h, or h, gate, up
PyObject *gated_ffn(PyObject *, PyObject *const *o, Py_ssize_t count) {
    return guarded(count, 5, [&]() -> PyObject * {
        Call call;
        const Block b(call, o, true);
        const int act = call.integer(o[3]);
        call.need(PyBool_Check(o[4]));
        const bool save = o[4] == Py_True;
        void *const stream = call.stream();
        call.outside_the_graph();
        if (!call.good) return nullptr;
        const int64_t m = b.x.size(0), k = b.x.size(1), n = b.w_gate.size(0);
        if (save && n % 4) return nullptr;  // rows of the saved products are padded
        return answer([&]() -> Result {
            at::Tensor h = at::empty({m, n}, b.x.options()), gate, up;
            if (save) gate = fp32({m, n}, b.x), up = fp32({m, n}, b.x);
            const int rc = byz_gated_ffn(b.x.data_ptr(), k, b.w_gate.data_ptr(), b.w_up.data_ptr(), k, m, k, n, b.dtype, act, h.data_ptr(), n,
                                         (float *)address(gate), (float *)address(up), n, nullptr, 0, stream);
            if (save) return {rc, {h, gate, up}};
            return {rc, {h}};
        });
    });
}

// dh, x, w_gate, w_up, gate, up, act -> dx, dw_gate, dw_up
PyObject *gated_ffn_backward(PyObject *, PyObject *const *o, Py_ssize_t count) {
    return guarded(count, 7, [&]() -> PyObject * {
        Call call;
        const Block b(call, o + 1, false);
        if (!call.good) return nullptr;
        const int64_t m = b.x.size(0), k = b.x.size(1), n = b.w_gate.size(0);
        const at::Tensor &dh = call.matrix(o[0], b.x.scalar_type());
        call.need(call.good && dh.size(0) == m && dh.size(1) == n);
        const float *gate = call.floats(o[4], {m, n}), *up = call.floats(o[5], {m, n});
        const int act = call.integer(o[6]);
        void *const stream = call.stream();
        if (!call.good) return nullptr;
        return answer([&]() -> Result {
            at::Tensor dx = at::empty({m, k}, b.x.options()), dw_gate = at::empty({n, k}, b.x.options()), dw_up = at::empty({n, k}, b.x.options());
            const size_t need = b.aligned() ? byz_gated_ffn_backward_aligned_workspace_bytes(m, k, n, b.dtype)
                                            : byz_gated_ffn_backward_workspace_bytes(m, k, n, b.dtype);
            const at::Tensor ws = bytes(need, b.x);
            const int rc = byz_gated_ffn_backward(dh.data_ptr(), n, b.x.data_ptr(), k, b.w_gate.data_ptr(), b.w_up.data_ptr(), k, gate, up, n, m,
                                                  k, n, b.dtype, act, dx.data_ptr(), k, dw_gate.data_ptr(), dw_up.data_ptr(), k, address(ws),
                                                  need, stream);
            return {rc, {dx, dw_gate, dw_up}};
        });
    });
}

#define BYZ_CALL(name) {#name, (PyCFunction)(void (*)())name, METH_FASTCALL, nullptr}
PyMethodDef methods[] = {BYZ_CALL(group_norm),        BYZ_CALL(group_norm_backward), BYZ_CALL(distill_loss), BYZ_CALL(distill_loss_step),
                         BYZ_CALL(gated_ffn),         BYZ_CALL(gated_ffn_backward),  {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_worker_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__worker_calls() {
    PyObject *torch_c = PyImport_ImportModule("torch._C");
    if (!torch_c) return nullptr;
    get_device = PyObject_GetAttrString(torch_c, "_cuda_getDevice");
    get_stream = get_device ? PyObject_GetAttrString(torch_c, "_cuda_getCurrentRawStream") : nullptr;
    Py_DECREF(torch_c);
    return get_stream ? PyModule_Create(&module) : nullptr;
}
