// The worker operators' calls in their common form, for Python: dense tensors, nothing given to write to, the current stream.
//
// A small call is bound by the host.  Checked, allocated and enqueued here, a call takes half of what the same steps take
// in Python (figures in worker.py).  Whatever is not of the common form is answered with None and nothing done: the
// Python path behind it handles or refuses it, so every rule and every word about it stands there alone.  An
// int is the library's error code.
#include "calls.h"

namespace {

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

PyMethodDef methods[] = {BYZ_CALL(group_norm),        BYZ_CALL(group_norm_backward), BYZ_CALL(distill_loss), BYZ_CALL(distill_loss_step),
                         BYZ_CALL(gated_ffn),         BYZ_CALL(gated_ffn_backward),  {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_worker_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__worker_calls() { return find_torch() ? PyModule_Create(&module) : nullptr; }
