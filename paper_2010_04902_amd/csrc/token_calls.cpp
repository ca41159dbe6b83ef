// The token operators' calls in their common form, for Python, as worker_calls.cpp has those of the other worker operators.
#include "calls.h"

namespace {

PyObject *form_class = nullptr;  // byz_residual_form's, a ctypes structure of the C struct

// x, p, seed, offset, first_row -> y
PyObject *dropout(PyObject *, PyObject *const *o, Py_ssize_t count) {
    return guarded(count, 5, [&]() -> PyObject * {
        Call call;
        const at::Tensor &x = call.tensor(o[0]);
        call.need(x.defined() && x.dim() == 2 && x.is_contiguous());
        const int dtype = call.dtype(x);
        const float p = call.real(o[1]);
        const uint64_t seed = call.word(o[2]), offset = call.word(o[3]);
        const int64_t first_row = call.integer64(o[4]);
        void *const stream = call.stream();
        call.outside_the_graph();
        if (!call.good) return nullptr;
        return answer([&]() -> Result {
            at::Tensor y = at::empty_like(x);
            const int64_t cols = x.size(1);
            return {byz_dropout(x.data_ptr(), x.size(0), cols, cols, dtype, p, seed, offset, nullptr, first_row, y.data_ptr(), cols, stream), {y}};
        });
    });
}

// A block, its residual and what joins them: x, h, form, post_weight, post_bias, gate, pre_weight, pre_bias.
struct Join {
    const at::Tensor &x;
    int64_t rows = 0, cols = 0, gate_rows = 1;
    int dtype;
    const void *h = nullptr;
    byz_residual_form form{};
    const float *w1 = nullptr, *b1 = nullptr, *gate = nullptr, *w2 = nullptr, *b2 = nullptr;
    Join(Call &call, PyObject *const *o) : x(call.tensor(o[0])), dtype(call.dtype(x)) {
        call.need(x.defined() && x.dim() == 2 && x.is_contiguous());
        if (!call.good) return;
        rows = gate_rows = x.size(0), cols = x.size(1);
        if (o[1] != Py_None) h = like_x(call, o[1]);
        Py_buffer view;
        if (!form_class || Py_TYPE(o[2]) != (PyTypeObject *)form_class || PyObject_GetBuffer(o[2], &view, PyBUF_SIMPLE) != 0) {
            call.good = false;
            return;
        }
        call.need(view.len == sizeof form);
        if (call.good) memcpy(&form, view.buf, sizeof form);
        PyBuffer_Release(&view);
        call.need(!form.offset_at);
        w1 = call.floats(o[3], {cols}, true), b1 = call.floats(o[4], {cols}, true);
        w2 = call.floats(o[6], {cols}, true), b2 = call.floats(o[7], {cols}, true);
        if (o[5] == Py_None || !call.good) return;
        const at::Tensor &g = call.tensor(o[5]);
        if (g.defined() && g.dim() == 2) {
            call.need(rows % g.size(0) == 0);
            if (call.good) gate_rows = rows / g.size(0), gate = call.floats(o[5], {g.size(0), cols});
        } else {
            gate = call.floats(o[5], {cols});
        }
    }
    const void *like_x(Call &call, PyObject *o) const {
        const at::Tensor &t = call.tensor(o);
        call.need(t.defined() && t.sizes() == x.sizes() && t.scalar_type() == x.scalar_type() && t.is_contiguous());
        return call.good ? t.data_ptr() : nullptr;
    }
};

// x, h, form, post_weight, post_bias, gate, pre_weight, pre_bias -> out (None without h), y (None without a pre norm), stats
PyObject *residual_norm(PyObject *, PyObject *const *o, Py_ssize_t count) {
    return guarded(count, 8, [&]() -> PyObject * {
        Call call;
        const Join j(call, o);
        void *const stream = call.stream();
        call.outside_the_graph();
        if (!call.good) return nullptr;
        return answer([&]() -> Result {
            at::Tensor out, y, stats = fp32({j.rows, 4}, j.x);
            if (j.h) out = at::empty_like(j.x);
            if (j.form.pre != BYZ_NORM_NONE) y = at::empty_like(j.x);
            const int rc = byz_residual_norm(j.x.data_ptr(), j.cols, j.h, j.cols, j.rows, j.cols, j.dtype, &j.form, j.w1, j.b1, j.gate, j.gate_rows,
                                             j.w2, j.b2, address(out), j.cols, address(y), j.cols, (float *)stats.data_ptr(), stream);
            return {rc, {out, y, stats}};
        });
    });
}

// dout, dy, stats, x, h, form, post_weight, post_bias, gate, pre_weight, pre_bias -> dx, dh, and the gradients of the last five but
// the form, in their order; None for what is not there
PyObject *residual_norm_backward(PyObject *, PyObject *const *o, Py_ssize_t count) {
    return guarded(count, 11, [&]() -> PyObject * {
        Call call;
        const Join j(call, o + 3);
        if (!call.good) return nullptr;
        const void *dout = o[0] == Py_None ? nullptr : j.like_x(call, o[0]), *dy = o[1] == Py_None ? nullptr : j.like_x(call, o[1]);
        const float *stats = call.floats(o[2], {j.rows, 4});
        void *const stream = call.stream();
        if (!call.good) return nullptr;
        return answer([&]() -> Result {
            at::Tensor dx = at::empty_like(j.x), dh, d[5];
            if (j.h) dh = at::empty_like(j.x);
            const float *given[5] = {j.w1, j.b1, j.gate, j.w2, j.b2};
            for (int i = 0; i < 5; i++)
                if (given[i]) d[i] = i == 2 && THPVariable_Unpack(o[8]).dim() == 2 ? fp32({j.rows / j.gate_rows, j.cols}, j.x) : fp32({j.cols}, j.x);
            const size_t need = byz_residual_norm_backward_workspace_bytes(j.rows, j.cols, j.dtype, j.gate_rows);
            const at::Tensor ws = bytes(need, j.x);
            const int rc = byz_residual_norm_backward(dout, j.cols, dy, j.cols, j.x.data_ptr(), j.cols, j.h, j.cols, stats, j.rows, j.cols, j.dtype,
                                                      &j.form, j.w1, j.b1, j.gate, j.gate_rows, j.w2, dx.data_ptr(), j.cols, address(dh), j.cols,
                                                      (float *)address(d[0]), (float *)address(d[1]), (float *)address(d[2]), (float *)address(d[3]),
                                                      (float *)address(d[4]), address(ws), need, stream);
            return {rc, {dx, dh, d[0], d[1], d[2], d[3], d[4]}};
        });
    });
}

// Logits and their tokens, and the workspace of the losses' calls.
struct Rows {
    const at::Tensor &logits;
    int dtype;
    int64_t rows = 0, vocab = 0;
    const int32_t *label = nullptr;
    size_t need = 0;
    Rows(Call &call, PyObject *const *o) : logits(call.tensor(o[0])), dtype(call.dtype(logits)) {
        call.need(logits.defined() && logits.dim() == 2 && logits.is_contiguous());
        if (!call.good) return;
        rows = logits.size(0), vocab = logits.size(1);
        label = call.integers(o[1], {rows});
        need = byz_token_loss_workspace_bytes(rows, vocab, dtype);
    }
    const float *floats(Call &call, PyObject *o, bool none = false) const { return call.floats(o, {rows}, none); }
    at::Tensor each() const { return fp32({rows}, logits); }
    at::Tensor stats() const { return fp32({rows, 2}, logits); }
    at::Tensor gradient() const { return at::empty_like(logits); }
    at::Tensor workspace() const { return bytes(need, logits); }
};
float *floats_of(const at::Tensor &t) { return (float *)t.data_ptr(); }

// logits, label, temperature -> logp, stats
PyObject *token_logp(PyObject *, PyObject *const *o, Py_ssize_t count) {
    return guarded(count, 3, [&]() -> PyObject * {
        Call call;
        const Rows r(call, o);
        const float temperature = call.real(o[2]);
        void *const stream = call.stream();
        call.outside_the_graph();
        if (!call.good) return nullptr;
        return answer([&]() -> Result {
            const at::Tensor logp = r.each(), stats = r.stats(), ws = r.workspace();
            const int rc = byz_token_logp(r.logits.data_ptr(), r.rows, r.vocab, r.vocab, r.dtype, r.label, temperature, floats_of(logp), floats_of(stats),
                                          address(ws), r.need, stream);
            return {rc, {logp, stats}};
        });
    });
}

// logits, label, dlogp, stats, temperature -> dlogits
PyObject *token_logp_backward(PyObject *, PyObject *const *o, Py_ssize_t count) {
    return guarded(count, 5, [&]() -> PyObject * {
        Call call;
        const Rows r(call, o);
        if (!call.good) return nullptr;
        const float *d = r.floats(call, o[2]), *stats = call.floats(o[3], {r.rows, 2}), temperature = call.real(o[4]);
        void *const stream = call.stream();
        if (!call.good) return nullptr;
        return answer([&]() -> Result {
            const at::Tensor dlogits = r.gradient(), ws = r.workspace();
            const int rc = byz_token_logp_backward(d, r.logits.data_ptr(), r.rows, r.vocab, r.vocab, r.dtype, r.label, stats, temperature,
                                                   dlogits.data_ptr(), r.vocab, address(ws), r.need, stream);
            return {rc, {dlogits}};
        });
    });
}

// old, advantage, ref, clip_low, clip_high, kl, temperature
struct Policy {
    const float *old, *advantage, *ref;
    float clip_low, clip_high, kl, temperature;
    Policy(Call &call, const Rows &r, PyObject *const *o)
        : old(r.floats(call, o[0])), advantage(r.floats(call, o[1])), ref(r.floats(call, o[2], true)), clip_low(call.real(o[3])),
          clip_high(call.real(o[4])), kl(call.real(o[5])), temperature(call.real(o[6])) {}
};

// logits, label, old, advantage, ref, clip_low, clip_high, kl, temperature -> loss, logp, stats
PyObject *policy_loss(PyObject *, PyObject *const *o, Py_ssize_t count) {
    return guarded(count, 9, [&]() -> PyObject * {
        Call call;
        const Rows r(call, o);
        if (!call.good) return nullptr;
        const Policy p(call, r, o + 2);
        void *const stream = call.stream();
        call.outside_the_graph();
        if (!call.good) return nullptr;
        return answer([&]() -> Result {
            const at::Tensor loss = r.each(), logp = r.each(), stats = r.stats(), ws = r.workspace();
            const int rc = byz_policy_loss(r.logits.data_ptr(), r.rows, r.vocab, r.vocab, r.dtype, r.label, p.old, p.advantage, p.ref, p.clip_low,
                                           p.clip_high, p.kl, p.temperature, floats_of(loss), floats_of(logp), floats_of(stats), address(ws), r.need,
                                           stream);
            return {rc, {loss, logp, stats}};
        });
    });
}

// logits, label, old, advantage, ref, clip_low, clip_high, kl, temperature, dloss, stats -> dlogits
PyObject *policy_loss_backward(PyObject *, PyObject *const *o, Py_ssize_t count) {
    return guarded(count, 11, [&]() -> PyObject * {
        Call call;
        const Rows r(call, o);
        if (!call.good) return nullptr;
        const Policy p(call, r, o + 2);
        const float *d = r.floats(call, o[9]), *stats = call.floats(o[10], {r.rows, 2});
        void *const stream = call.stream();
        if (!call.good) return nullptr;
        return answer([&]() -> Result {
            const at::Tensor dlogits = r.gradient(), ws = r.workspace();
            const int rc = byz_policy_loss_backward(d, r.logits.data_ptr(), r.rows, r.vocab, r.vocab, r.dtype, r.label, p.old, p.advantage, p.ref,
                                                    p.clip_low, p.clip_high, p.kl, p.temperature, stats, dlogits.data_ptr(), r.vocab, address(ws),
                                                    r.need, stream);
            return {rc, {dlogits}};
        });
    });
}

// logits, label, old, advantage, ref, clip_low, clip_high, kl, temperature, dloss -> loss, logp, dlogits
PyObject *policy_loss_step(PyObject *, PyObject *const *o, Py_ssize_t count) {
    return guarded(count, 10, [&]() -> PyObject * {
        Call call;
        const Rows r(call, o);
        if (!call.good) return nullptr;
        const Policy p(call, r, o + 2);
        const float *d = r.floats(call, o[9]);
        void *const stream = call.stream();
        if (!call.good) return nullptr;
        return answer([&]() -> Result {
            const at::Tensor loss = r.each(), logp = r.each(), dlogits = r.gradient(), ws = r.workspace();
            const int rc = byz_policy_loss_step(d, r.logits.data_ptr(), r.rows, r.vocab, r.vocab, r.dtype, r.label, p.old, p.advantage, p.ref, p.clip_low,
                                                p.clip_high, p.kl, p.temperature, floats_of(loss), floats_of(logp), dlogits.data_ptr(), r.vocab,
                                                address(ws), r.need, stream);
            return {rc, {loss, logp, dlogits}};
        });
    });
}

// Bounds of the sequences of pairs.
struct Pairs {
    const int32_t *bounds = nullptr;
    int64_t pairs = 0;
    Pairs(Call &call, PyObject *o) {
        const at::Tensor &t = call.tensor(o);
        call.need(t.defined() && t.dim() == 1 && t.size(0) % 2 == 1 && t.size(0) > 1);
        if (!call.good) return;
        pairs = t.size(0) / 2;
        bounds = call.integers(o, {t.size(0)});
    }
};

// logits, label, bounds, ref, beta, smoothing, temperature -> loss, sums, slope, stats
PyObject *preference_loss(PyObject *, PyObject *const *o, Py_ssize_t count) {
    return guarded(count, 7, [&]() -> PyObject * {
        Call call;
        const Rows r(call, o);
        if (!call.good) return nullptr;
        const Pairs p(call, o[2]);
        const float *ref = call.floats(o[3], {2 * p.pairs}, true);
        const float beta = call.real(o[4]), smoothing = call.real(o[5]), temperature = call.real(o[6]);
        void *const stream = call.stream();
        call.outside_the_graph();
        if (!call.good) return nullptr;
        return answer([&]() -> Result {
            const at::Tensor loss = fp32({p.pairs}, r.logits), sums = fp32({2 * p.pairs}, r.logits), slope = fp32({p.pairs}, r.logits);
            const at::Tensor stats = r.stats(), ws = r.workspace();
            const int rc = byz_preference_loss(r.logits.data_ptr(), r.rows, r.vocab, r.vocab, r.dtype, r.label, p.bounds, p.pairs, ref, beta, smoothing,
                                               temperature, floats_of(loss), floats_of(sums), floats_of(slope), floats_of(stats), address(ws), r.need,
                                               stream);
            return {rc, {loss, sums, slope, stats}};
        });
    });
}

// logits, label, bounds, dloss, slope, stats, beta, temperature -> dlogits
PyObject *preference_loss_backward(PyObject *, PyObject *const *o, Py_ssize_t count) {
    return guarded(count, 8, [&]() -> PyObject * {
        Call call;
        const Rows r(call, o);
        if (!call.good) return nullptr;
        const Pairs p(call, o[2]);
        const float *d = call.floats(o[3], {p.pairs}), *slope = call.floats(o[4], {p.pairs}), *stats = call.floats(o[5], {r.rows, 2});
        const float beta = call.real(o[6]), temperature = call.real(o[7]);
        void *const stream = call.stream();
        if (!call.good) return nullptr;
        return answer([&]() -> Result {
            const at::Tensor dlogits = r.gradient(), ws = r.workspace();
            const int rc = byz_preference_loss_backward(d, r.logits.data_ptr(), r.rows, r.vocab, r.vocab, r.dtype, r.label, p.bounds, p.pairs, slope, beta,
                                                        temperature, stats, dlogits.data_ptr(), r.vocab, address(ws), r.need, stream);
            return {rc, {dlogits}};
        });
    });
}

// logits, label, bounds, dloss, ref, beta, smoothing, temperature -> loss, sums, dlogits
PyObject *preference_loss_step(PyObject *, PyObject *const *o, Py_ssize_t count) {
    return guarded(count, 8, [&]() -> PyObject * {
        Call call;
        const Rows r(call, o);
        if (!call.good) return nullptr;
        const Pairs p(call, o[2]);
        const float *d = call.floats(o[3], {p.pairs}), *ref = call.floats(o[4], {2 * p.pairs}, true);
        const float beta = call.real(o[5]), smoothing = call.real(o[6]), temperature = call.real(o[7]);
        void *const stream = call.stream();
        if (!call.good) return nullptr;
        return answer([&]() -> Result {
            const at::Tensor loss = fp32({p.pairs}, r.logits), sums = fp32({2 * p.pairs}, r.logits), dlogits = r.gradient(), ws = r.workspace();
            const int rc = byz_preference_loss_step(d, r.logits.data_ptr(), r.rows, r.vocab, r.vocab, r.dtype, r.label, p.bounds, p.pairs, ref, beta,
                                                    smoothing, temperature, floats_of(loss), floats_of(sums), dlogits.data_ptr(), r.vocab, address(ws),
                                                    r.need, stream);
            return {rc, {loss, sums, dlogits}};
        });
    });
}

// The class of byz_residual_form.
PyObject *use_form(PyObject *, PyObject *cls) {
    Py_INCREF(cls);
    Py_XDECREF(form_class);
    form_class = cls;
    Py_RETURN_NONE;
}

PyMethodDef methods[] = {BYZ_CALL(dropout),
                         BYZ_CALL(residual_norm),
                         BYZ_CALL(residual_norm_backward),
                         BYZ_CALL(token_logp),
                         BYZ_CALL(token_logp_backward),
                         BYZ_CALL(policy_loss),
                         BYZ_CALL(policy_loss_backward),
                         BYZ_CALL(policy_loss_step),
                         BYZ_CALL(preference_loss),
                         BYZ_CALL(preference_loss_backward),
                         BYZ_CALL(preference_loss_step),
                         {"use_form", use_form, METH_O, nullptr},
                         {nullptr, nullptr, 0, nullptr}};

PyModuleDef module = {PyModuleDef_HEAD_INIT, "_token_calls", nullptr, -1, methods, nullptr, nullptr, nullptr, nullptr};

}  // namespace

PyMODINIT_FUNC PyInit__token_calls() { return find_torch() ? PyModule_Create(&module) : nullptr; }
