"""Operators of a worker's training step (include/byzshield_worker.h): group norm with an activation,
the gated feed-forward block, distillation from a teacher's top logits, each with its gradients.

Same manner as the server's entry points: torch CUDA tensors in, outputs allocated with torch where
the caller gives none, work enqueued on `stream` (the current one by default), nothing synchronised.  Autograd knows nothing of
them: outputs are not part of its graph, gradients are explicit calls (a forward call warns where a tensor requires one).
A layout the kernels do not read is refused (the feed-forward's rows may be copied to a workspace).  Calls of the same sizes and type on
the same values give the same bits, wherever their tensors lie, which is what the server's vote over the copies of a file's gradient
needs: copies of a file have to be computed by calls alike, not once alone and once within a larger batch.
"""
import ctypes
import functools
import importlib
import subprocess
import warnings

from . import binding as _b

BYZ_ACT_NONE, BYZ_ACT_RELU, BYZ_ACT_SILU, BYZ_ACT_GELU, BYZ_ACT_SIGMOID = range(5)
BYZ_ACTS = {"none": BYZ_ACT_NONE, "relu": BYZ_ACT_RELU, "silu": BYZ_ACT_SILU, "gelu": BYZ_ACT_GELU,
            "sigmoid": BYZ_ACT_SIGMOID}
BYZ_MAX_TEACHER = 1024
BYZ_F32, BYZ_BF16, BYZ_F16 = range(3)

_NO_GRAPH = ("outputs are not part of autograd's graph: gradients come from the operator's own backward call "
             "(no warning under torch.no_grad)")

_lib = None
_calls = None
_torch = None
_dtypes = {}


class _NoCalls:
    """Stands in for the native module where there is none: every call is left to the Python below."""

    def __getattr__(self, name):
        return lambda *args: None


def _load_calls():
    """csrc/worker_calls.cpp's module; built once where it is missing or made for another torch, and done without, with a
    warning, where that fails."""
    for build in (False, True):
        try:
            if build:
                from . import build as _build
                _build.build_calls()
                importlib.invalidate_caches()
            return importlib.import_module("._worker_calls", __package__)
        except (ImportError, OSError, subprocess.CalledProcessError) as e:
            reason = e
    warnings.warn("the worker operators' native module is not there (%s): small calls take about twice the host's time" % reason,
                  RuntimeWarning, stacklevel=3)
    return _NoCalls()


def _load():
    global _lib, _torch, _calls
    if _lib is not None:
        return _lib
    L = _b._load()
    torch = _torch = _b._torch()
    _calls = _load_calls()
    _dtypes.update({torch.float32: BYZ_F32, torch.bfloat16: BYZ_BF16, torch.float16: BYZ_F16})
    vp, c_int, i64, sz, f32 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
    sig = {
        "byz_group_norm_workspace_bytes": (sz, [i64, i64, i64, c_int, c_int]),
        "byz_group_norm": (c_int, [vp, i64, i64, i64, i64, i64, c_int, c_int, vp, vp, f32, c_int, vp, i64, i64,
                                   vp, vp, vp, sz, vp]),
        "byz_group_norm_backward_workspace_bytes": (sz, [i64, i64, i64, c_int, c_int]),
        "byz_group_norm_backward": (c_int, [vp, i64, i64, vp, i64, i64, i64, i64, i64, c_int, c_int, vp, vp, vp, vp,
                                            c_int, vp, i64, i64, vp, vp, vp, sz, vp]),
        "byz_distill_loss": (c_int, [vp, i64, i64, i64, c_int, vp, vp, c_int, i64, f32, vp, vp, vp]),
        "byz_distill_loss_step_workspace_bytes": (sz, [i64, i64, c_int, c_int]),
        "byz_distill_loss_backward": (c_int, [vp, vp, i64, i64, i64, c_int, vp, vp, c_int, i64, vp, f32, vp, i64, vp]),
        "byz_distill_loss_step": (c_int, [vp, i64, i64, i64, c_int, vp, vp, c_int, i64, vp, f32, vp, vp, vp, i64,
                                          vp, sz, vp]),
        "byz_gated_ffn_workspace_bytes": (sz, [i64, i64, i64, c_int]),
        "byz_gated_ffn": (c_int, [vp, i64, vp, vp, i64, i64, i64, i64, c_int, c_int, vp, i64, vp, vp, i64, vp, sz, vp]),
        "byz_gated_ffn_backward_workspace_bytes": (sz, [i64, i64, i64, c_int]),
        "byz_gated_ffn_backward_aligned_workspace_bytes": (sz, [i64, i64, i64, c_int]),
        "byz_gated_ffn_backward": (c_int, [vp, i64, vp, i64, vp, vp, i64, vp, vp, i64, i64, i64, i64, c_int, c_int,
                                           vp, i64, vp, vp, i64, vp, sz, vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    _lib = L
    return L


# The small calls are bound by the host.  Calls of the common form (dense tensors, nothing given to write to, the current
# stream) are made by csrc/worker_calls.cpp; it answers None to any other, and an int where the library failed.  The Python
# below handles or refuses the rest: each argument is tested by one expression of cheap terms, and only where that is
# false a second function finds the words.
# us of host time a call, Python / csrc/worker_calls.cpp: group norm 12.6 / 6.6, its backward 17.8 / 10.2, loss 9.4 / 5.5, its step
# 11.3 / 5.9, feed-forward 8.8 / 4.7, its backward 21.3 / 13.5.


def _device(x, what):
    """Index of the GPU that x is on, which is the current one."""
    device = x.get_device()
    if device < 0:
        raise ValueError("%s must be a CUDA tensor" % what)
    if device != _torch.cuda.current_device():
        raise ValueError("%s is on cuda:%d, which is not the current device" % (what, device))
    return device


def _refuse_device(t, what, device):
    if t.get_device() < 0:
        raise ValueError("%s must be a CUDA tensor" % what)
    if t.get_device() != device:
        raise ValueError("%s is on cuda:%d, the call on cuda:%d" % (what, t.get_device(), device))


def _dtype(t, what):
    code = _dtypes.get(t.dtype)
    if code is None:
        raise ValueError("%s has dtype %s" % (what, t.dtype))
    return code


def _stream(stream, device):
    if stream is None and _b._raw_current_stream is not None:
        return _b._raw_current_stream(device)
    return _b._stream_ptr(stream)


def _floats(t, shape, what, device):
    """Address of a contiguous float32 tensor of this shape, None for None."""
    if t is None:
        return None
    if t.dtype is _torch.float32 and t.shape == shape and t.get_device() == device and t.is_contiguous():
        return t.data_ptr()
    _refuse_device(t, what, device)
    raise ValueError("%s is %s of shape %s%s, the call needs contiguous float32 of shape %s"
                     % (what, t.dtype, tuple(t.shape), "" if t.is_contiguous() else " with gaps", tuple(shape)))


def _matrix(t, what, shape=None, dtype=None):
    """(rows, columns, pitch) of a 2-D tensor whose columns are neighbours in memory."""
    if t.dim() != 2 or (shape is not None and t.shape != shape):
        raise ValueError("%s has shape %s%s" % (what, tuple(t.shape), "" if shape is None else
                                                ", the call needs %s" % (tuple(shape),)))
    if dtype is not None and t.dtype is not dtype:
        raise ValueError("%s has dtype %s, the call needs %s" % (what, t.dtype, dtype))
    rows, cols = t.shape
    pitch, step = t.stride()
    if rows <= 1 and pitch < cols:
        pitch = cols
    if (step != 1 and cols > 1) or pitch < cols:
        raise ValueError("%s must have neighbouring columns and rows that do not overlap" % what)
    return rows, cols, pitch


@functools.lru_cache(maxsize=256)
def _workspace_bytes(name, *sizes):
    return getattr(_lib, name)(*sizes)


def _workspace(nbytes, empty, device):
    """(tensor, its address): the tensor is to be held until the call has been enqueued."""
    if nbytes == 0:
        return None, None
    t = empty(nbytes, dtype=_torch.uint8, device=device)
    return t, t.data_ptr()


def _outside_the_graph(*tensors):
    if _torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors):
        warnings.warn(_NO_GRAPH, RuntimeWarning, stacklevel=3)


def _done(r, where):
    """A common call's outputs, or its error."""
    if r.__class__ is int:
        _b._check(r, where)
    return r


# ------------------------------------------------------------------ group norm


def _features(x, what):
    """(n, p, c, sample stride, pixel stride) of channels-last features: [n, c, h, w] as torch's channels_last
    lays them out, or [n, p, c]; channels may be a slice of wider pixels."""
    if x.dim() == 4:
        n, c, h, w = x.shape
        sn, sc, sh, sw = x.stride()
        p, pixel = h * w, sw if w > 1 else sh if h > 1 else c
        regular = w == 1 or h == 1 or sh == w * sw
    elif x.dim() == 3:
        n, p, c = x.shape
        sn, pixel, sc = x.stride()
        pixel = pixel if p > 1 else c
        regular = True
    else:
        raise ValueError("%s must be [n, c, h, w] or [n, p, c], has shape %s" % (what, tuple(x.shape)))
    if (c > 1 and sc != 1) or not regular or pixel < c:
        raise ValueError("%s must be channels last in memory" % what)
    return n, p, c, sn, pixel


def _features_like(x, dense, empty, device):
    if dense and empty is _torch.empty:
        return _torch.empty_like(x)  # the same strides
    if x.dim() == 4:
        n, c, h, w = x.shape
        return empty((n, h, w, c), dtype=x.dtype, device=device).permute(0, 3, 1, 2)
    return empty(x.shape, dtype=x.dtype, device=device)


def _strides_of(t, x, what, device, xs, xp):
    """(sample stride, pixel stride) of features with x's shape and type."""
    if t.shape != x.shape or t.dtype is not x.dtype:
        raise ValueError("%s is %s of shape %s, x is %s of shape %s"
                         % (what, t.dtype, tuple(t.shape), x.dtype, tuple(x.shape)))
    if t.get_device() != device:
        _refuse_device(t, what, device)
    return (xs, xp) if t.stride() == x.stride() else _features(t, what)[3:]


def byz_group_norm(x, groups, gamma=None, beta=None, eps=1e-5, act=BYZ_ACT_NONE, out=None, stream=None):
    """act(group norm of x * gamma + beta) -> (y, mean[n, groups] float32, rstd[n, groups] float32).

    x: [n, c, h, w] in torch's channels_last memory format or [n, p, c]; float32, bfloat16 or float16.
    gamma, beta: float32 [c] or None.  out may be x."""
    if _lib is None:
        _load()
    if out is None and stream is None:
        done = _calls.group_norm(x, groups, gamma, beta, eps, act)
        if done is not None:
            return _done(done, "byz_group_norm")
    _outside_the_graph(x, gamma, beta)
    n, p, c, xs, xp = _features(x, "x")
    index = _device(x, "x")
    device, dtype, groups = x.device, _dtype(x, "x"), int(groups)
    empty = _torch.empty if stream is None else _b._empty_on(stream)
    g, b = _floats(gamma, (c,), "gamma", index), _floats(beta, (c,), "beta", index)
    if out is None:
        out = _features_like(x, xp == c and (n <= 1 or xs == p * c), empty, device)
    ys, yp = _strides_of(out, x, "out", index, xs, xp)
    mean = empty((n, max(groups, 0)), dtype=_torch.float32, device=device)
    rstd = empty((n, max(groups, 0)), dtype=_torch.float32, device=device)
    nbytes = _workspace_bytes("byz_group_norm_workspace_bytes", n, p, c, groups, dtype)
    ws, at = _workspace(nbytes, empty, device)
    _b._check(_lib.byz_group_norm(x.data_ptr(), xs, xp, n, p, c, groups, dtype, g, b, eps, act, out.data_ptr(), ys, yp,
                                  mean.data_ptr(), rstd.data_ptr(), at, nbytes, _stream(stream, index)), "byz_group_norm")
    return out, mean, rstd


def byz_group_norm_backward(dy, x, groups, mean, rstd, gamma=None, beta=None, act=BYZ_ACT_NONE, out=None,
                            parameters=True, stream=None):
    """-> (dx, dgamma[c] float32, dbeta[c] float32) for dy, from x and byz_group_norm's mean and rstd.

    out (dx) may be dy.  parameters=False: dgamma and dbeta are None and not computed."""
    if _lib is None:
        _load()
    if out is None and stream is None and parameters:
        done = _calls.group_norm_backward(dy, x, groups, mean, rstd, gamma, beta, act)
        if done is not None:
            return _done(done, "byz_group_norm_backward")
    n, p, c, xs, xp = _features(x, "x")
    index = _device(x, "x")
    device, dtype, groups = x.device, _dtype(x, "x"), int(groups)
    empty = _torch.empty if stream is None else _b._empty_on(stream)
    ds, dp = _strides_of(dy, x, "dy", index, xs, xp)
    g, b = _floats(gamma, (c,), "gamma", index), _floats(beta, (c,), "beta", index)
    m, r = _floats(mean, (n, groups), "mean", index), _floats(rstd, (n, groups), "rstd", index)
    if out is None:
        out = _features_like(x, xp == c and (n <= 1 or xs == p * c), empty, device)
    os, op = _strides_of(out, x, "out", index, xs, xp)
    dgamma = dbeta = None
    if parameters:
        dgamma = empty(c, dtype=_torch.float32, device=device)
        dbeta = empty(c, dtype=_torch.float32, device=device)
    nbytes = _workspace_bytes("byz_group_norm_backward_workspace_bytes", n, p, c, groups, dtype)
    ws, at = _workspace(nbytes, empty, device)
    _b._check(_lib.byz_group_norm_backward(
        dy.data_ptr(), ds, dp, x.data_ptr(), xs, xp, n, p, c, groups, dtype, g, b, m, r, act, out.data_ptr(), os, op,
        dgamma.data_ptr() if parameters else None, dbeta.data_ptr() if parameters else None, at, nbytes,
        _stream(stream, index)), "byz_group_norm_backward")
    return out, dgamma, dbeta


# ------------------------------------------------------------------ distillation


def _distill_arguments(logits, teacher, index):
    """(rows, vocab, pitch, k, teacher's pitch, GPU)"""
    rows, vocab, ld = _matrix(logits, "logits")
    trows, k, tld = _matrix(teacher, "teacher", dtype=_torch.float32)
    _, _, ild = _matrix(index, "index", teacher.shape, _torch.int32)
    if trows != rows:
        raise ValueError("teacher has %d rows, logits %d" % (trows, rows))
    if tld != ild and rows > 1:
        raise ValueError("teacher and index must have one row pitch")
    device = _device(logits, "logits")
    if teacher.get_device() != device or index.get_device() != device:
        _refuse_device(teacher, "teacher", device)
        _refuse_device(index, "index", device)
    return rows, vocab, ld, k, tld, device


def _gradient_out(out, logits, empty, index):
    """(dlogits, pitch)"""
    if out is None:
        out = empty(logits.shape, dtype=logits.dtype, device=logits.device)
        return out, out.shape[1]
    if out.get_device() != index:
        _refuse_device(out, "out", index)
    return out, _matrix(out, "out", logits.shape, logits.dtype)[2]


def byz_distill_loss(logits, teacher, index, temperature=1.0, stream=None):
    """Loss of each row against a teacher's top logits -> (loss[rows] float32, lse[rows] float32).

    logits [rows, vocab] float32, bfloat16 or float16; teacher float32 and index int32 [rows, k]: the
    teacher's logits and their places, a negative place is no entry."""
    if _lib is None:
        _load()
    if stream is None:
        done = _calls.distill_loss(logits, teacher, index, temperature)
        if done is not None:
            return _done(done, "byz_distill_loss")
    _outside_the_graph(logits, teacher)
    rows, vocab, ld, k, tld, gpu = _distill_arguments(logits, teacher, index)
    device, dtype = logits.device, _dtype(logits, "logits")
    empty = _torch.empty if stream is None else _b._empty_on(stream)
    loss = empty(rows, dtype=_torch.float32, device=device)
    lse = empty(rows, dtype=_torch.float32, device=device)
    _b._check(_lib.byz_distill_loss(logits.data_ptr(), rows, vocab, ld, dtype, teacher.data_ptr(), index.data_ptr(), k, tld,
                                    temperature, loss.data_ptr(), lse.data_ptr(), _stream(stream, gpu)), "byz_distill_loss")
    return loss, lse


def byz_distill_loss_backward(dloss, logits, teacher, index, lse, temperature=1.0, out=None, stream=None):
    """-> dlogits (type of logits) for dloss[rows] float32, from byz_distill_loss' lse.  out may be logits."""
    if _lib is None:
        _load()
    rows, vocab, ld, k, tld, gpu = _distill_arguments(logits, teacher, index)
    dtype = _dtype(logits, "logits")
    empty = _torch.empty if stream is None else _b._empty_on(stream)
    d, l = _floats(dloss, (rows,), "dloss", gpu), _floats(lse, (rows,), "lse", gpu)
    out, old = _gradient_out(out, logits, empty, gpu)
    _b._check(_lib.byz_distill_loss_backward(d, logits.data_ptr(), rows, vocab, ld, dtype, teacher.data_ptr(),
                                             index.data_ptr(), k, tld, l, temperature, out.data_ptr(), old,
                                             _stream(stream, gpu)), "byz_distill_loss_backward")
    return out


def byz_distill_loss_step(logits, teacher, index, dloss, temperature=1.0, out=None, stream=None):
    """Loss and gradient in one call, for weights dloss[rows] float32 known beforehand
    -> (loss[rows] float32, dlogits).  out (dlogits) may be logits."""
    if _lib is None:
        _load()
    if out is None and stream is None:
        done = _calls.distill_loss_step(logits, teacher, index, dloss, temperature)
        if done is not None:
            return _done(done, "byz_distill_loss_step")
    rows, vocab, ld, k, tld, gpu = _distill_arguments(logits, teacher, index)
    device, dtype = logits.device, _dtype(logits, "logits")
    empty = _torch.empty if stream is None else _b._empty_on(stream)
    d = _floats(dloss, (rows,), "dloss", gpu)
    out, old = _gradient_out(out, logits, empty, gpu)
    loss = empty(rows, dtype=_torch.float32, device=device)
    nbytes = _workspace_bytes("byz_distill_loss_step_workspace_bytes", rows, vocab, k, dtype)
    ws, at = _workspace(nbytes, empty, device)
    _b._check(_lib.byz_distill_loss_step(logits.data_ptr(), rows, vocab, ld, dtype, teacher.data_ptr(), index.data_ptr(), k,
                                         tld, d, temperature, loss.data_ptr(), None, out.data_ptr(), old, at, nbytes,
                                         _stream(stream, gpu)), "byz_distill_loss_step")
    return loss, out


# ------------------------------------------------------------------ gated feed-forward


def _ffn_arguments(x, w_gate, w_up):
    """(m, k, n, x's pitch, the weights' pitch, GPU)"""
    m, k, x_ld = _matrix(x, "x")
    n, wk, w_ld = _matrix(w_gate, "w_gate", None, x.dtype)
    _, _, u_ld = _matrix(w_up, "w_up", w_gate.shape, x.dtype)
    if wk != k:
        raise ValueError("x has %d columns, the weights %d" % (k, wk))
    if u_ld != w_ld and n > 1:
        raise ValueError("w_gate and w_up must have one row pitch")
    device = _device(x, "x")
    if w_gate.get_device() != device or w_up.get_device() != device:
        _refuse_device(w_gate, "w_gate", device)
        _refuse_device(w_up, "w_up", device)
    return m, k, n, x_ld, w_ld, device


def _copied(k, x_ld, w_ld, xa, ga, ua):
    """Whether rows of x or the weights are such that the kernel cannot read them as they lie."""
    return (k | x_ld | w_ld) % 8 | (xa | ga | ua) % 16


def byz_gated_ffn(x, w_gate, w_up, act=BYZ_ACT_SILU, save=False, out=None, stream=None):
    """h = act(x w_gate^T) * (x w_up^T) -> h, or (h, gate, up) with save=True: both products, float32, for the
    backward pass.

    x [m, k], w_gate and w_up [n, k], bfloat16 or float16."""
    if _lib is None:
        _load()
    if out is None and stream is None:
        done = _calls.gated_ffn(x, w_gate, w_up, act, save)
        if done is not None:
            return _done(done, "byz_gated_ffn")
    _outside_the_graph(x, w_gate, w_up)
    m, k, n, x_ld, w_ld, gpu = _ffn_arguments(x, w_gate, w_up)
    device, dtype, kind = x.device, _dtype(x, "x"), x.dtype
    empty = _torch.empty if stream is None else _b._empty_on(stream)
    if out is None:
        out, h_ld = empty((m, n), dtype=kind, device=device), n
    else:
        if out.get_device() != gpu:
            _refuse_device(out, "out", gpu)
        h_ld = _matrix(out, "out", (m, n), kind)[2]
    gate = up = None
    wide = n
    if save:  # rows of whole 16 bytes: the backward pass reads them in pieces
        wide = (n + 3) // 4 * 4
        gate = empty((m, wide), dtype=_torch.float32, device=device)
        up = empty((m, wide), dtype=_torch.float32, device=device)
        if wide != n:
            gate, up = gate[:, :n], up[:, :n]
    xa, ga, ua = x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr()
    nbytes, ws, at = 0, None, None
    if m > 16 and _copied(k, x_ld, w_ld, xa, ga, ua):
        nbytes = _workspace_bytes("byz_gated_ffn_workspace_bytes", m, k, n, dtype)
        ws, at = _workspace(nbytes, empty, device)
    _b._check(_lib.byz_gated_ffn(xa, x_ld, ga, ua, w_ld, m, k, n, dtype, act, out.data_ptr(), h_ld,
                                 gate.data_ptr() if save else None, up.data_ptr() if save else None, wide, at, nbytes,
                                 _stream(stream, gpu)), "byz_gated_ffn")
    return (out, gate, up) if save else out


def byz_gated_ffn_backward(dh, x, w_gate, w_up, gate, up, act=BYZ_ACT_SILU, stream=None):
    """-> (dx, dw_gate, dw_up) for dh [m, n], from byz_gated_ffn's gate and up."""
    if _lib is None:
        _load()
    if stream is None:
        done = _calls.gated_ffn_backward(dh, x, w_gate, w_up, gate, up, act)
        if done is not None:
            return _done(done, "byz_gated_ffn_backward")
    m, k, n, x_ld, w_ld, gpu = _ffn_arguments(x, w_gate, w_up)
    device, dtype, kind = x.device, _dtype(x, "x"), x.dtype
    empty = _torch.empty if stream is None else _b._empty_on(stream)
    _, _, dh_ld = _matrix(dh, "dh", (m, n), kind)
    _, _, gate_ld = _matrix(gate, "gate", (m, n), _torch.float32)
    _, _, up_ld = _matrix(up, "up", (m, n), _torch.float32)
    if gate_ld != up_ld and m > 1:
        raise ValueError("gate and up must have one row pitch")
    for t, what in ((dh, "dh"), (gate, "gate"), (up, "up")):
        if t.get_device() != gpu:
            _refuse_device(t, what, gpu)
    dx = empty((m, k), dtype=kind, device=device)
    dw_gate = empty((n, k), dtype=kind, device=device)
    dw_up = empty((n, k), dtype=kind, device=device)
    xa, ga, ua = x.data_ptr(), w_gate.data_ptr(), w_up.data_ptr()
    nbytes = _workspace_bytes("byz_gated_ffn_backward_workspace_bytes" if _copied(k, x_ld, w_ld, xa, ga, ua) else
                              "byz_gated_ffn_backward_aligned_workspace_bytes", m, k, n, dtype)
    ws, at = _workspace(nbytes, empty, device)
    _b._check(_lib.byz_gated_ffn_backward(
        dh.data_ptr(), dh_ld, xa, x_ld, ga, ua, w_ld, gate.data_ptr(),
        up.data_ptr(), gate_ld, m, k, n, dtype, act, dx.data_ptr(), k, dw_gate.data_ptr(), dw_up.data_ptr(), k,
        at, nbytes, _stream(stream, gpu)), "byz_gated_ffn_backward")
    return dx, dw_gate, dw_up
