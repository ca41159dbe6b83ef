"""Operators of a worker that trains on tokens (include/byzshield_worker.h): dropout whose mask is made where it is used, the join of a
block's output with the residual and its norms, and losses of tokens' log-probabilities, each with its gradients.

In the manner of worker.py: torch CUDA tensors in, outputs allocated with torch where the caller gives none, work enqueued on
`stream` (the current one by default), nothing synchronised, explicit calls for gradients, the same bits from calls of the same
sizes and type on the same values.
"""
import ctypes

from . import binding as _b
from . import worker as _w

BYZ_NORM_NONE, BYZ_NORM_RMS, BYZ_NORM_LAYER = range(3)
BYZ_NORMS = {"none": BYZ_NORM_NONE, "rms": BYZ_NORM_RMS, "layer": BYZ_NORM_LAYER}
_WORD = 2 ** 64 - 1

_lib = None
_calls = None
_torch = None


class byz_residual_form(ctypes.Structure):
    """How byz_residual_norm joins a block to the residual: its norms (BYZ_NORM_*), the scale of what joins, and the dropout
    (byz_dropout's p, seed, offset, offset_at, first_row).  A program keeps one for each of its blocks; offset may be set anew
    for every step."""
    _fields_ = [("post", ctypes.c_int32), ("pre", ctypes.c_int32), ("eps", ctypes.c_float), ("scale", ctypes.c_float),
                ("p", ctypes.c_float), ("seed", ctypes.c_uint64), ("offset", ctypes.c_uint64), ("_offset_at", ctypes.c_void_p),
                ("first_row", ctypes.c_int64)]

    def __init__(self, post=BYZ_NORM_NONE, pre=BYZ_NORM_RMS, scale=1.0, eps=1e-5, p=0.0, seed=0, offset=0, offset_at=None,
                 first_row=0):
        super().__init__(post, pre, eps, scale, p, seed & _WORD, offset & _WORD, None, first_row)
        self.offset_at = offset_at

    def __setattr__(self, name, value):
        super().__setattr__(name, _row(value) if name == "first_row" else value)

    @property
    def offset_at(self):
        return self._counter

    @offset_at.setter
    def offset_at(self, t):
        self._offset_at = None if t is None else _counter(t)
        self._counter = t  # lives as long as the form


def _load():
    global _lib, _calls, _torch
    if _lib is not None:
        return _lib
    L = _w._load()
    _torch, _calls = _w._torch, _w._load_calls("_token_calls", "build_token_calls")
    _calls.use_form(byz_residual_form)
    vp, c_int, i64, u64, sz, f32 = (ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_uint64, ctypes.c_size_t,
                                    ctypes.c_float)
    form = ctypes.POINTER(byz_residual_form)
    rows = [vp, i64, i64, i64, c_int, vp]  # logits, rows, vocab, ld, dtype, label
    work = [vp, sz, vp]
    policy = [vp, vp, vp, f32, f32, f32, f32]
    sig = {
        "byz_dropout": (c_int, [vp, i64, i64, i64, c_int, f32, u64, u64, vp, i64, vp, i64, vp]),
        "byz_residual_norm": (c_int, [vp, i64, vp, i64, i64, i64, c_int, form, vp, vp, vp, i64, vp, vp, vp, i64, vp, i64, vp, vp]),
        "byz_residual_norm_backward_workspace_bytes": (sz, [i64, i64, c_int, i64]),
        "byz_residual_norm_backward": (c_int, [vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, i64, c_int, form, vp, vp, vp, i64, vp,
                                               vp, i64, vp, i64, vp, vp, vp, vp, vp] + work),
        "byz_token_loss_workspace_bytes": (sz, [i64, i64, c_int]),
        "byz_token_logp": (c_int, rows + [f32, vp, vp] + work),
        "byz_token_logp_backward": (c_int, [vp] + rows + [vp, f32, vp, i64] + work),
        "byz_policy_loss": (c_int, rows + policy + [vp, vp, vp] + work),
        "byz_policy_loss_backward": (c_int, [vp] + rows + policy + [vp, vp, i64] + work),
        "byz_policy_loss_step": (c_int, [vp] + rows + policy + [vp, vp, vp, i64] + work),
        "byz_preference_loss": (c_int, rows + [vp, i64, vp, f32, f32, f32, vp, vp, vp, vp] + work),
        "byz_preference_loss_backward": (c_int, [vp] + rows + [vp, i64, vp, f32, f32, vp, vp, i64] + work),
        "byz_preference_loss_step": (c_int, [vp] + rows + [vp, i64, vp, f32, f32, f32, vp, vp, vp, i64] + work),
    }
    for name, (res, args) in sig.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    _lib = L
    return L


# Calls of the common form go through csrc/token_calls.cpp first, as in worker.py; the Python below handles or refuses the rest.
# us of host time a call, Python / csrc/token_calls.cpp: dropout 8.2 / 4.0, residual 15.0 / 5.9, its backward 26.4 / 10.8, log-probabilities
# 10.8 / 5.4, policy loss 13.7 / 6.2, its step 14.4 / 6.5, preference step 19.3 / 11.3.


def _row(n):
    """n, if the library can be given it whole; which rows there are it says itself."""
    if not -2 ** 63 <= n < 2 ** 63:
        raise ValueError("first_row is %d, the last row there can be is 2^32 - 1" % n)
    return n


def _counter(t):
    """Address of an int64 of one element on the GPU."""
    if _lib is None:
        _load()
    if t.dtype is not _torch.int64 or t.numel() != 1 or t.get_device() < 0:
        raise ValueError("offset_at must be a CUDA tensor of one int64")
    return t.data_ptr()


def _empties(stream):
    return _torch.empty if stream is None else _b._empty_on(stream)


def _same_place(t, what, index):
    if t.get_device() != index:
        _w._refuse_device(t, what, index)


def _result(out, shape, dtype, what, empty, device, index):
    """(tensor, pitch) of a result: `out` if it is given."""
    if out is None:
        return empty(shape, dtype=dtype, device=device), shape[1]
    _same_place(out, what, index)
    return out, _w._matrix(out, what, shape, dtype)[2]


# ------------------------------------------------------------------ dropout


def byz_dropout(x, p, seed, offset=0, offset_at=None, first_row=0, out=None, stream=None):
    """x / (1 - p) where a value stays, else 0 -> y; the gradient is the same call on dy.

    x [rows, cols] float32, bfloat16 or float16.  What stays depends on seed, the sum of offset and offset_at (an int64 on
    the GPU, for captured calls), first_row + the row, and the column, and on nothing else.  out may be x."""
    if _lib is None:
        _load()
    if out is None and stream is None and offset_at is None:
        done = _calls.dropout(x, p, seed, offset, first_row)
        if done is not None:
            return _w._done(done, "byz_dropout")
    first_row = _row(first_row)
    _w._outside_the_graph(x)
    rows, cols, ld = _w._matrix(x, "x")
    index, dtype = _w._device(x, "x"), _w._dtype(x, "x")
    at = None
    if offset_at is not None:
        at = _counter(offset_at)
        _same_place(offset_at, "offset_at", index)
    out, out_ld = _result(out, x.shape, x.dtype, "out", _empties(stream), x.device, index)
    _b._check(_lib.byz_dropout(x.data_ptr(), rows, cols, ld, dtype, p, seed & _WORD, offset & _WORD, at, first_row,
                               out.data_ptr(), out_ld, _w._stream(stream, index)), "byz_dropout")
    return out


# ------------------------------------------------------------------ residual and norms


def _vectors(x, form, post_weight, post_bias, gate, pre_weight, pre_bias, index):
    """(addresses of the five, rows of x that share one of gate)"""
    rows, cols = x.shape
    shape = (cols,)
    gate_rows = rows if rows else 1
    gate_shape = shape
    if gate is not None and gate.dim() == 2:
        gate_shape = (gate.shape[0], cols)
        if gate.shape[0] < 1 or rows % gate.shape[0] or (rows == 0 and gate.shape[0] > 1):
            raise ValueError("gate has %d rows, x %d: no whole number to each" % (gate.shape[0], rows))
        gate_rows = max(1, rows // gate.shape[0])
    if form.offset_at is not None:
        _same_place(form.offset_at, "offset_at", index)
    return (_w._floats(post_weight, shape, "post_weight", index), _w._floats(post_bias, shape, "post_bias", index),
            _w._floats(gate, gate_shape, "gate", index), _w._floats(pre_weight, shape, "pre_weight", index),
            _w._floats(pre_bias, shape, "pre_bias", index)), gate_rows


def _like_x(t, what, x, index):
    """(address, pitch) of a matrix of x's shape and type, (None, 0) for None."""
    if t is None:
        return None, 0
    _same_place(t, what, index)
    return t.data_ptr(), _w._matrix(t, what, x.shape, x.dtype)[2]


def byz_residual_norm(x, h, form, post_weight=None, post_bias=None, gate=None, pre_weight=None, pre_bias=None, out=None,
                      stream=None):
    """out = x + scale * gate * dropout(norm_post(h) * post_weight + post_bias), y = norm_pre(out) * pre_weight + pre_bias
    -> (out, y, stats[rows, 4] float32).

    x, h: [rows, cols] float32, bfloat16 or float16.  form: a byz_residual_form.  Weights and biases: float32 [cols] or None.
    gate: float32 [cols], or [n, cols], a row for each of n equal parts of the rows, or None.  y is None without a pre norm.
    h None: y = norm_pre(x) alone, and out is x.  out may be x or h (the backward call needs both)."""
    if _lib is None:
        _load()
    if out is None and stream is None:
        done = _calls.residual_norm(x, h, form, post_weight, post_bias, gate, pre_weight, pre_bias)
        if done is not None:
            total, y, stats = _w._done(done, "byz_residual_norm")
            return x if h is None else total, y, stats
    _w._outside_the_graph(x, h, post_weight, post_bias, gate, pre_weight, pre_bias)
    rows, cols, x_ld = _w._matrix(x, "x")
    index, dtype = _w._device(x, "x"), _w._dtype(x, "x")
    device, empty = x.device, _empties(stream)
    h_at, h_ld = _like_x(h, "h", x, index)
    (w1, b1, g, w2, b2), gate_rows = _vectors(x, form, post_weight, post_bias, gate, pre_weight, pre_bias, index)
    if h is None:
        if out is not None:
            raise ValueError("out without a block's output h")
        total, total_at, total_ld = x, None, 0
    else:
        total, total_ld = _result(out, x.shape, x.dtype, "out", empty, device, index)
        total_at = total.data_ptr()
    y = empty(x.shape, dtype=x.dtype, device=device) if form.pre else None
    stats = empty((rows, 4), dtype=_torch.float32, device=device)
    _b._check(_lib.byz_residual_norm(x.data_ptr(), x_ld, h_at, h_ld, rows, cols, dtype, form, w1, b1, g, gate_rows, w2, b2,
                                     total_at, total_ld, y.data_ptr() if form.pre else None, cols, stats.data_ptr(),
                                     _w._stream(stream, index)), "byz_residual_norm")
    return total, y, stats


def byz_residual_norm_backward(dout, dy, x, h, stats, form, post_weight=None, post_bias=None, gate=None, pre_weight=None,
                               pre_bias=None, parameters=True, stream=None):
    """-> (dx, dh, (d_post_weight, d_post_bias, d_gate, d_pre_weight, d_pre_bias) float32) for dout and dy (either may be
    None: zeros), from byz_residual_norm's inputs and stats.

    A vector that was None has no gradient; parameters=False: none of them has.  dh is None without h."""
    if _lib is None:
        _load()
    if stream is None and parameters:
        done = _calls.residual_norm_backward(dout, dy, stats, x, h, form, post_weight, post_bias, gate, pre_weight, pre_bias)
        if done is not None:
            done = _w._done(done, "byz_residual_norm_backward")
            return done[0], done[1], done[2:]
    rows, cols, x_ld = _w._matrix(x, "x")
    index, dtype = _w._device(x, "x"), _w._dtype(x, "x")
    device, empty = x.device, _empties(stream)
    h_at, h_ld = _like_x(h, "h", x, index)
    dout_at, dout_ld = _like_x(dout, "dout", x, index)
    dy_at, dy_ld = _like_x(dy, "dy", x, index)
    s = _w._floats(stats, (rows, 4), "stats", index)
    vectors = (post_weight, post_bias, gate, pre_weight, pre_bias)
    (w1, b1, g, w2, _), gate_rows = _vectors(x, form, *vectors, index)
    dx = empty(x.shape, dtype=x.dtype, device=device)
    dh = empty(x.shape, dtype=x.dtype, device=device) if h is not None else None
    grads = tuple(empty(v.shape, dtype=_torch.float32, device=device) if parameters and v is not None else None for v in vectors)
    nbytes = _w._workspace_bytes("byz_residual_norm_backward_workspace_bytes", rows, cols, dtype, gate_rows)
    ws, at = _w._workspace(nbytes, empty, device)
    _b._check(_lib.byz_residual_norm_backward(
        dout_at, dout_ld, dy_at, dy_ld, x.data_ptr(), x_ld, h_at, h_ld, s, rows, cols, dtype, form, w1, b1, g, gate_rows, w2,
        dx.data_ptr(), cols, dh.data_ptr() if h is not None else None, cols,
        *(d.data_ptr() if d is not None else None for d in grads), at, nbytes, _w._stream(stream, index)),
        "byz_residual_norm_backward")
    return dx, dh, grads


# ------------------------------------------------------------------ losses of tokens


class _Rows:
    """Logits and their tokens, checked, and the call's surroundings."""
    __slots__ = ("rows", "vocab", "index", "device", "empty", "given", "ws", "work")

    def __init__(self, logits, label, stream):
        self.rows, self.vocab, ld = _w._matrix(logits, "logits")
        self.index, dtype = _w._device(logits, "logits"), _w._dtype(logits, "logits")
        self.device, self.empty = logits.device, _empties(stream)
        at = _integers(label, (self.rows,), "label", self.index)
        self.given = (logits.data_ptr(), self.rows, self.vocab, ld, dtype, at)
        nbytes = _w._workspace_bytes("byz_token_loss_workspace_bytes", self.rows, self.vocab, dtype)
        self.ws, at = _w._workspace(nbytes, self.empty, self.device)
        self.work = (at, nbytes, _w._stream(stream, self.index))

    def floats(self, t, what, count=None):
        return _w._floats(t, (self.rows if count is None else count,), what, self.index)

    def results(self, *shapes):
        return [self.empty(shape, dtype=_torch.float32, device=self.device) for shape in shapes]

    def gradient(self, out, logits):
        return _w._gradient_out(out, logits, self.empty, self.index)


def _integers(t, shape, what, index):
    if t.dtype is _torch.int32 and t.shape == shape and t.get_device() == index and t.is_contiguous():
        return t.data_ptr()
    _same_place(t, what, index)
    raise ValueError("%s is %s of shape %s%s, the call needs contiguous int32 of shape %s"
                     % (what, t.dtype, tuple(t.shape), "" if t.is_contiguous() else " with gaps", tuple(shape)))


def byz_token_logp(logits, label, temperature=1.0, stream=None):
    """Log-probability of each row's token -> (logp[rows] float32, stats[rows, 2] float32).

    logits [rows, vocab] float32, bfloat16 or float16; label int32 [rows], negative where there is no token: logp 0."""
    if _lib is None:
        _load()
    if stream is None:
        done = _calls.token_logp(logits, label, temperature)
        if done is not None:
            return _w._done(done, "byz_token_logp")
    _w._outside_the_graph(logits)
    r = _Rows(logits, label, stream)
    logp, stats = r.results(r.rows, (r.rows, 2))
    _b._check(_lib.byz_token_logp(*r.given, temperature, logp.data_ptr(), stats.data_ptr(), *r.work), "byz_token_logp")
    return logp, stats


def byz_token_logp_backward(dlogp, logits, label, stats, temperature=1.0, out=None, stream=None):
    """-> dlogits (type of logits) for dlogp[rows] float32, from byz_token_logp's stats.  out may be logits."""
    if _lib is None:
        _load()
    if out is None and stream is None:
        done = _calls.token_logp_backward(logits, label, dlogp, stats, temperature)
        if done is not None:
            return _w._done(done, "byz_token_logp_backward")
    r = _Rows(logits, label, stream)
    d, s = r.floats(dlogp, "dlogp"), _w._floats(stats, (r.rows, 2), "stats", r.index)
    out, ld = r.gradient(out, logits)
    _b._check(_lib.byz_token_logp_backward(d, *r.given, s, temperature, out.data_ptr(), ld, *r.work), "byz_token_logp_backward")
    return out


def byz_policy_loss(logits, label, old, advantage, ref=None, clip_low=0.2, clip_high=0.2, kl=0.0, temperature=1.0, stream=None):
    """The clipped policy loss of each token, with its KL term -> (loss[rows], logp[rows], stats[rows, 2]), all float32.

    logits and label as in byz_token_logp; old (log-probabilities when the tokens were drawn), advantage and ref (those of
    the reference model; None if kl is 0): float32 [rows]."""
    if _lib is None:
        _load()
    if stream is None:
        done = _calls.policy_loss(logits, label, old, advantage, ref, clip_low, clip_high, kl, temperature)
        if done is not None:
            return _w._done(done, "byz_policy_loss")
    _w._outside_the_graph(logits, old, advantage, ref)
    r = _Rows(logits, label, stream)
    o, a, f = r.floats(old, "old"), r.floats(advantage, "advantage"), r.floats(ref, "ref")
    loss, logp, stats = r.results(r.rows, r.rows, (r.rows, 2))
    _b._check(_lib.byz_policy_loss(*r.given, o, a, f, clip_low, clip_high, kl, temperature, loss.data_ptr(), logp.data_ptr(),
                                   stats.data_ptr(), *r.work), "byz_policy_loss")
    return loss, logp, stats


def byz_policy_loss_backward(dloss, logits, label, old, advantage, stats, ref=None, clip_low=0.2, clip_high=0.2, kl=0.0,
                             temperature=1.0, out=None, stream=None):
    """-> dlogits (type of logits) for dloss[rows] float32, from byz_policy_loss' stats.  out may be logits."""
    if _lib is None:
        _load()
    if out is None and stream is None:
        done = _calls.policy_loss_backward(logits, label, old, advantage, ref, clip_low, clip_high, kl, temperature, dloss, stats)
        if done is not None:
            return _w._done(done, "byz_policy_loss_backward")
    r = _Rows(logits, label, stream)
    d, o, a, f = r.floats(dloss, "dloss"), r.floats(old, "old"), r.floats(advantage, "advantage"), r.floats(ref, "ref")
    s = _w._floats(stats, (r.rows, 2), "stats", r.index)
    out, ld = r.gradient(out, logits)
    _b._check(_lib.byz_policy_loss_backward(d, *r.given, o, a, f, clip_low, clip_high, kl, temperature, s, out.data_ptr(), ld,
                                            *r.work), "byz_policy_loss_backward")
    return out


def byz_policy_loss_step(logits, label, old, advantage, dloss, ref=None, clip_low=0.2, clip_high=0.2, kl=0.0, temperature=1.0,
                         out=None, stream=None):
    """Loss and gradient in one call, for weights dloss[rows] float32 known beforehand
    -> (loss[rows] float32, logp[rows] float32, dlogits).  out (dlogits) may be logits."""
    if _lib is None:
        _load()
    if out is None and stream is None:
        done = _calls.policy_loss_step(logits, label, old, advantage, ref, clip_low, clip_high, kl, temperature, dloss)
        if done is not None:
            return _w._done(done, "byz_policy_loss_step")
    r = _Rows(logits, label, stream)
    d, o, a, f = r.floats(dloss, "dloss"), r.floats(old, "old"), r.floats(advantage, "advantage"), r.floats(ref, "ref")
    out, ld = r.gradient(out, logits)
    loss, logp = r.results(r.rows, r.rows)
    _b._check(_lib.byz_policy_loss_step(d, *r.given, o, a, f, clip_low, clip_high, kl, temperature, loss.data_ptr(),
                                        logp.data_ptr(), out.data_ptr(), ld, *r.work), "byz_policy_loss_step")
    return loss, logp, out


def _pairs(bounds, r):
    """(address of bounds, number of pairs)"""
    if bounds.dim() != 1 or bounds.shape[0] % 2 != 1:
        raise ValueError("bounds has shape %s, the call needs [2 * pairs + 1]" % (tuple(bounds.shape),))
    return _integers(bounds, bounds.shape, "bounds", r.index), bounds.shape[0] // 2


def byz_preference_loss(logits, label, bounds, ref=None, beta=0.1, smoothing=0.0, temperature=1.0, stream=None):
    """The preference loss of pairs of sequences -> (loss[pairs], sums[2 * pairs], slope[pairs], stats[rows, 2]), all float32.

    logits and label as in byz_token_logp; bounds int32 [2 * pairs + 1]: sequence s has the rows bounds[s] to bounds[s + 1] - 1,
    sequences 2 i and 2 i + 1 are pair i's chosen and rejected one.  ref: the reference model's sums, float32 [2 * pairs]."""
    if _lib is None:
        _load()
    if stream is None:
        done = _calls.preference_loss(logits, label, bounds, ref, beta, smoothing, temperature)
        if done is not None:
            return _w._done(done, "byz_preference_loss")
    _w._outside_the_graph(logits, ref)
    r = _Rows(logits, label, stream)
    at, pairs = _pairs(bounds, r)
    f = r.floats(ref, "ref", 2 * pairs)
    loss, sums, slope, stats = r.results(pairs, 2 * pairs, pairs, (r.rows, 2))
    _b._check(_lib.byz_preference_loss(*r.given, at, pairs, f, beta, smoothing, temperature, loss.data_ptr(), sums.data_ptr(),
                                       slope.data_ptr(), stats.data_ptr(), *r.work), "byz_preference_loss")
    return loss, sums, slope, stats


def byz_preference_loss_backward(dloss, logits, label, bounds, slope, stats, beta=0.1, temperature=1.0, out=None, stream=None):
    """-> dlogits (type of logits) for dloss[pairs] float32, from byz_preference_loss' slope and stats.  out may be logits."""
    if _lib is None:
        _load()
    if out is None and stream is None:
        done = _calls.preference_loss_backward(logits, label, bounds, dloss, slope, stats, beta, temperature)
        if done is not None:
            return _w._done(done, "byz_preference_loss_backward")
    r = _Rows(logits, label, stream)
    at, pairs = _pairs(bounds, r)
    d, l = r.floats(dloss, "dloss", pairs), r.floats(slope, "slope", pairs)
    s = _w._floats(stats, (r.rows, 2), "stats", r.index)
    out, ld = r.gradient(out, logits)
    _b._check(_lib.byz_preference_loss_backward(d, *r.given, at, pairs, l, beta, temperature, s, out.data_ptr(), ld, *r.work),
              "byz_preference_loss_backward")
    return out


def byz_preference_loss_step(logits, label, bounds, dloss, ref=None, beta=0.1, smoothing=0.0, temperature=1.0, out=None,
                             stream=None):
    """Loss and gradient in one call, for weights dloss[pairs] float32 known beforehand
    -> (loss[pairs] float32, sums[2 * pairs] float32, dlogits).  out (dlogits) may be logits."""
    if _lib is None:
        _load()
    if out is None and stream is None:
        done = _calls.preference_loss_step(logits, label, bounds, dloss, ref, beta, smoothing, temperature)
        if done is not None:
            return _w._done(done, "byz_preference_loss_step")
    r = _Rows(logits, label, stream)
    at, pairs = _pairs(bounds, r)
    d, f = r.floats(dloss, "dloss", pairs), r.floats(ref, "ref", 2 * pairs)
    out, ld = r.gradient(out, logits)
    loss, sums = r.results(pairs, 2 * pairs)
    _b._check(_lib.byz_preference_loss_step(d, *r.given, at, pairs, f, beta, smoothing, temperature, loss.data_ptr(),
                                            sums.data_ptr(), out.data_ptr(), ld, *r.work), "byz_preference_loss_step")
    return loss, sums, out
