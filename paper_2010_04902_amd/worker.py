"""Operators of a worker's training step (include/byzshield_worker.h): group norm with an activation,
the gated feed-forward block, distillation from a teacher's top logits, each with its gradients.

Same manner as the server's entry points: torch CUDA tensors in, outputs allocated with torch where
the caller gives none, work enqueued on `stream` (the current one by default), nothing synchronised.
Inputs are never copied: a layout the kernels do not read is refused.  Results depend on the arguments
alone, bit for bit, which is what the server's vote over the copies of a file's gradient needs.
"""
import ctypes

from . import binding as _b

BYZ_ACT_NONE, BYZ_ACT_RELU, BYZ_ACT_SILU, BYZ_ACT_GELU, BYZ_ACT_SIGMOID = range(5)
BYZ_ACTS = {"none": BYZ_ACT_NONE, "relu": BYZ_ACT_RELU, "silu": BYZ_ACT_SILU, "gelu": BYZ_ACT_GELU,
            "sigmoid": BYZ_ACT_SIGMOID}
BYZ_MAX_TEACHER = 1024
BYZ_F32, BYZ_BF16, BYZ_F16 = range(3)

_lib = None
_dtypes = {}


def _load():
    global _lib
    if _lib is not None:
        return _lib
    L = _b._load()
    torch = _b._torch()
    _dtypes.update({torch.float32: BYZ_F32, torch.bfloat16: BYZ_BF16, torch.float16: BYZ_F16})
    vp, c_int, i64, sz, f32 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64, ctypes.c_size_t, ctypes.c_float
    sig = {
        "byz_group_norm_workspace_bytes": (sz, [i64, i64, i64, c_int, c_int]),
        "byz_group_norm": (c_int, [vp, i64, i64, i64, i64, i64, c_int, c_int, vp, vp, f32, c_int, vp, i64, i64,
                                   vp, vp, vp, sz, vp]),
        "byz_group_norm_backward_workspace_bytes": (sz, [i64, i64, i64, c_int, c_int]),
        "byz_group_norm_backward": (c_int, [vp, i64, i64, vp, i64, i64, i64, i64, i64, c_int, c_int, vp, vp, vp, vp,
                                            c_int, vp, i64, i64, vp, vp, vp, sz, vp]),
        "byz_distill_loss_workspace_bytes": (sz, [i64, i64, c_int, c_int]),
        "byz_distill_loss": (c_int, [vp, i64, i64, i64, c_int, vp, vp, c_int, i64, f32, vp, vp, vp, sz, vp]),
        "byz_distill_loss_backward": (c_int, [vp, vp, i64, i64, i64, c_int, vp, vp, c_int, i64, vp, f32, vp, i64, vp]),
        "byz_distill_loss_step": (c_int, [vp, i64, i64, i64, c_int, vp, vp, c_int, i64, vp, f32, vp, vp, vp, i64,
                                          vp, sz, vp]),
        "byz_gated_ffn": (c_int, [vp, i64, vp, vp, i64, i64, i64, i64, c_int, c_int, vp, i64, vp, vp, i64, vp]),
        "byz_gated_ffn_backward_workspace_bytes": (sz, [i64, i64, i64, c_int]),
        "byz_gated_ffn_backward": (c_int, [vp, i64, vp, i64, vp, vp, i64, vp, vp, i64, i64, i64, i64, c_int, c_int,
                                           vp, i64, vp, vp, i64, vp, sz, vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(L, name)
        fn.restype = res
        fn.argtypes = args
    _lib = L
    return L


def _on_gpu(tensors):
    """Every tensor on one GPU, the current one."""
    device = tensors[0][0].device
    for t, what in tensors:
        if not t.is_cuda:
            raise ValueError("%s must be a CUDA tensor" % what)
        if t.device != device:
            raise ValueError("%s is on %s, %s on %s" % (what, t.device, tensors[0][1], device))
    if device.index != _b._torch().cuda.current_device():
        raise ValueError("%s is not on the current device" % tensors[0][1])
    return device


def _dtype(t, what):
    code = _dtypes.get(t.dtype)
    if code is None:
        raise ValueError("%s has dtype %s" % (what, t.dtype))
    return code


def _vector(t, n, what, dtype="float32"):
    """Address of a contiguous 1-D tensor of n elements, None for None."""
    if t is None:
        return None
    at = _b._dev_ptr(t, (dtype,), what)
    if t.dim() != 1 or t.shape[0] != n:
        raise ValueError("%s has shape %s, the call needs (%d,)" % (what, tuple(t.shape), n))
    return at


def _matrix(t, what, shape=None, dtype=None):
    """(rows, columns, pitch) of a 2-D tensor whose columns are neighbours in memory."""
    if t.dim() != 2 or (shape is not None and tuple(t.shape) != shape):
        raise ValueError("%s has shape %s%s" % (what, tuple(t.shape), "" if shape is None else
                                                ", the call needs %s" % (shape,)))
    if dtype is not None and t.dtype != dtype:
        raise ValueError("%s has dtype %s, the call needs %s" % (what, t.dtype, dtype))
    rows, cols = t.shape
    pitch = t.stride(0) if rows > 1 else max(cols, t.stride(0))
    if cols > 1 and t.stride(1) != 1 or pitch < cols and rows > 1:
        raise ValueError("%s must have neighbouring columns and rows that do not overlap" % what)
    return rows, cols, pitch


def _workspace(nbytes, empty, device):
    if nbytes == 0:
        return None, None
    t = empty(nbytes, dtype=_b._torch().uint8, device=device)
    return t, t.data_ptr()


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


def _features_like(x, empty):
    if x.dim() == 4:
        n, c, h, w = x.shape
        return empty((n, h, w, c), dtype=x.dtype, device=x.device).permute(0, 3, 1, 2)
    return empty(tuple(x.shape), dtype=x.dtype, device=x.device)


def _same(t, x, what, like):
    if t.shape != x.shape or t.dtype != x.dtype:
        raise ValueError("%s is %s of shape %s, %s is %s of shape %s"
                         % (what, t.dtype, tuple(t.shape), like, x.dtype, tuple(x.shape)))


def byz_group_norm(x, groups, gamma=None, beta=None, eps=1e-5, act=BYZ_ACT_NONE, out=None, stream=None):
    """act(group norm of x * gamma + beta) -> (y, mean[n, groups] float32, rstd[n, groups] float32).

    x: [n, c, h, w] in torch's channels_last memory format or [n, p, c]; float32, bfloat16 or float16.
    gamma, beta: float32 [c] or None.  out may be x."""
    L = _load()
    torch = _b._torch()
    empty = torch.empty if stream is None else _b._empty_on(stream)
    n, p, c, xs, xp = _features(x, "x")
    device = _on_gpu([(t, w) for t, w in ((x, "x"), (gamma, "gamma"), (beta, "beta"), (out, "out")) if t is not None])
    dtype, groups = _dtype(x, "x"), int(groups)
    if out is None:
        out = _features_like(x, empty)
    else:
        _same(out, x, "out", "x")
    _, _, _, ys, yp = _features(out, "out")
    mean = empty((n, max(groups, 0)), dtype=torch.float32, device=device)
    rstd = empty((n, max(groups, 0)), dtype=torch.float32, device=device)
    nbytes = L.byz_group_norm_workspace_bytes(n, p, c, groups, dtype)
    ws, at = _workspace(nbytes, empty, device)
    _b._check(L.byz_group_norm(x.data_ptr(), xs, xp, n, p, c, groups, dtype, _vector(gamma, c, "gamma"),
                               _vector(beta, c, "beta"), float(eps), int(act), out.data_ptr(), ys, yp,
                               mean.data_ptr(), rstd.data_ptr(), at, nbytes, _b._stream_ptr(stream)), "byz_group_norm")
    return out, mean, rstd


def byz_group_norm_backward(dy, x, groups, mean, rstd, gamma=None, beta=None, act=BYZ_ACT_NONE, out=None,
                            parameters=True, stream=None):
    """-> (dx, dgamma[c] float32, dbeta[c] float32) for dy, from x and byz_group_norm's mean and rstd.

    out (dx) may be dy.  parameters=False: dgamma and dbeta are None and not computed."""
    L = _load()
    torch = _b._torch()
    empty = torch.empty if stream is None else _b._empty_on(stream)
    n, p, c, xs, xp = _features(x, "x")
    device = _on_gpu([(t, w) for t, w in ((x, "x"), (dy, "dy"), (mean, "mean"), (rstd, "rstd"), (gamma, "gamma"),
                                          (beta, "beta"), (out, "out")) if t is not None])
    dtype, groups = _dtype(x, "x"), int(groups)
    _same(dy, x, "dy", "x")
    _, _, _, ds, dp = _features(dy, "dy")
    if out is None:
        out = _features_like(x, empty)
    else:
        _same(out, x, "out", "x")
    _, _, _, os, op = _features(out, "out")
    for t, what in ((mean, "mean"), (rstd, "rstd")):
        if tuple(t.shape) != (n, groups) or t.dtype != torch.float32 or not t.is_contiguous():
            raise ValueError("%s must be contiguous float32 [%d, %d]" % (what, n, groups))
    dgamma = dbeta = None
    if parameters:
        dgamma = empty(c, dtype=torch.float32, device=device)
        dbeta = empty(c, dtype=torch.float32, device=device)
    nbytes = L.byz_group_norm_backward_workspace_bytes(n, p, c, groups, dtype)
    ws, at = _workspace(nbytes, empty, device)
    _b._check(L.byz_group_norm_backward(
        dy.data_ptr(), ds, dp, x.data_ptr(), xs, xp, n, p, c, groups, dtype, _vector(gamma, c, "gamma"),
        _vector(beta, c, "beta"), mean.data_ptr(), rstd.data_ptr(), int(act), out.data_ptr(), os, op,
        dgamma.data_ptr() if parameters else None, dbeta.data_ptr() if parameters else None, at, nbytes,
        _b._stream_ptr(stream)), "byz_group_norm_backward")
    return out, dgamma, dbeta


# ------------------------------------------------------------------ distillation


def _distill_arguments(logits, teacher, index, more=()):
    rows, vocab, ld = _matrix(logits, "logits")
    trows, k, tld = _matrix(teacher, "teacher", dtype=_b._torch().float32)
    _, _, ild = _matrix(index, "index", (trows, k), _b._torch().int32)
    if trows != rows:
        raise ValueError("teacher has %d rows, logits %d" % (trows, rows))
    if tld != ild and rows > 1:
        raise ValueError("teacher and index must have one row pitch")
    device = _on_gpu([(t, w) for t, w in ((logits, "logits"), (teacher, "teacher"), (index, "index")) + tuple(more)
                      if t is not None])
    return rows, vocab, ld, k, tld, device


def byz_distill_loss(logits, teacher, index, temperature=1.0, stream=None):
    """Loss of each row against a teacher's top logits -> (loss[rows] float32, lse[rows] float32).

    logits [rows, vocab] float32, bfloat16 or float16; teacher float32 and index int32 [rows, k]: the
    teacher's logits and their places, a negative place is no entry."""
    L = _load()
    torch = _b._torch()
    empty = torch.empty if stream is None else _b._empty_on(stream)
    rows, vocab, ld, k, tld, device = _distill_arguments(logits, teacher, index)
    dtype = _dtype(logits, "logits")
    loss = empty(rows, dtype=torch.float32, device=device)
    lse = empty(rows, dtype=torch.float32, device=device)
    nbytes = L.byz_distill_loss_workspace_bytes(rows, vocab, k, dtype)
    ws, at = _workspace(nbytes, empty, device)
    _b._check(L.byz_distill_loss(logits.data_ptr(), rows, vocab, ld, dtype, teacher.data_ptr(), index.data_ptr(), k, tld,
                                 float(temperature), loss.data_ptr(), lse.data_ptr(), at, nbytes,
                                 _b._stream_ptr(stream)), "byz_distill_loss")
    return loss, lse


def byz_distill_loss_backward(dloss, logits, teacher, index, lse, temperature=1.0, out=None, stream=None):
    """-> dlogits (type of logits) for dloss[rows] float32, from byz_distill_loss' lse.  out may be logits."""
    L = _load()
    torch = _b._torch()
    empty = torch.empty if stream is None else _b._empty_on(stream)
    rows, vocab, ld, k, tld, device = _distill_arguments(logits, teacher, index, ((dloss, "dloss"), (lse, "lse"),
                                                                                  (out, "out")))
    dtype = _dtype(logits, "logits")
    if out is None:
        out = empty((rows, vocab), dtype=logits.dtype, device=device)
    _, _, old = _matrix(out, "out", (rows, vocab), logits.dtype)
    _b._check(L.byz_distill_loss_backward(
        _vector(dloss, rows, "dloss"), logits.data_ptr(), rows, vocab, ld, dtype, teacher.data_ptr(), index.data_ptr(), k,
        tld, _vector(lse, rows, "lse"), float(temperature), out.data_ptr(), old, _b._stream_ptr(stream)),
        "byz_distill_loss_backward")
    return out


def byz_distill_loss_step(logits, teacher, index, dloss, temperature=1.0, out=None, stream=None):
    """Loss and gradient in one call, for weights dloss[rows] float32 known beforehand
    -> (loss[rows] float32, dlogits).  out (dlogits) may be logits."""
    L = _load()
    torch = _b._torch()
    empty = torch.empty if stream is None else _b._empty_on(stream)
    rows, vocab, ld, k, tld, device = _distill_arguments(logits, teacher, index, ((dloss, "dloss"), (out, "out")))
    dtype = _dtype(logits, "logits")
    if out is None:
        out = empty((rows, vocab), dtype=logits.dtype, device=device)
    _, _, old = _matrix(out, "out", (rows, vocab), logits.dtype)
    loss = empty(rows, dtype=torch.float32, device=device)
    nbytes = L.byz_distill_loss_workspace_bytes(rows, vocab, k, dtype)
    ws, at = _workspace(nbytes, empty, device)
    _b._check(L.byz_distill_loss_step(
        logits.data_ptr(), rows, vocab, ld, dtype, teacher.data_ptr(), index.data_ptr(), k, tld,
        _vector(dloss, rows, "dloss"), float(temperature), loss.data_ptr(), None, out.data_ptr(), old, at, nbytes,
        _b._stream_ptr(stream)), "byz_distill_loss_step")
    return loss, out


# ------------------------------------------------------------------ gated feed-forward


def _ffn_arguments(x, w_gate, w_up, more=()):
    m, k, x_ld = _matrix(x, "x")
    n, wk, w_ld = _matrix(w_gate, "w_gate", dtype=x.dtype)
    _, _, u_ld = _matrix(w_up, "w_up", (n, wk), x.dtype)
    if wk != k:
        raise ValueError("x has %d columns, the weights %d" % (k, wk))
    if u_ld != w_ld and n > 1:
        raise ValueError("w_gate and w_up must have one row pitch")
    device = _on_gpu([(t, w) for t, w in ((x, "x"), (w_gate, "w_gate"), (w_up, "w_up")) + tuple(more) if t is not None])
    return m, k, n, x_ld, w_ld, device


def byz_gated_ffn(x, w_gate, w_up, act=BYZ_ACT_SILU, save=False, out=None, stream=None):
    """h = act(x w_gate^T) * (x w_up^T) -> h, or (h, gate, up) with save=True: both products, float32, for the
    backward pass.

    x [m, k], w_gate and w_up [n, k], bfloat16 or float16."""
    L = _load()
    torch = _b._torch()
    empty = torch.empty if stream is None else _b._empty_on(stream)
    m, k, n, x_ld, w_ld, device = _ffn_arguments(x, w_gate, w_up, ((out, "out"),))
    dtype = _dtype(x, "x")
    if out is None:
        out = empty((m, n), dtype=x.dtype, device=device)
    _, _, h_ld = _matrix(out, "out", (m, n), x.dtype)
    gate = up = None
    if save:  # rows of whole 16 bytes: the backward pass reads them in pieces
        wide = (n + 3) // 4 * 4
        gate, up = (empty((m, wide), dtype=torch.float32, device=device)[:, :n] for _ in range(2))
    _b._check(L.byz_gated_ffn(x.data_ptr(), x_ld, w_gate.data_ptr(), w_up.data_ptr(), w_ld, m, k, n, dtype, int(act),
                              out.data_ptr(), h_ld, gate.data_ptr() if save else None, up.data_ptr() if save else None,
                              gate.stride(0) if save else 0, _b._stream_ptr(stream)), "byz_gated_ffn")
    return (out, gate, up) if save else out


def byz_gated_ffn_backward(dh, x, w_gate, w_up, gate, up, act=BYZ_ACT_SILU, stream=None):
    """-> (dx, dw_gate, dw_up) for dh [m, n], from byz_gated_ffn's gate and up."""
    L = _load()
    torch = _b._torch()
    empty = torch.empty if stream is None else _b._empty_on(stream)
    m, k, n, x_ld, w_ld, device = _ffn_arguments(x, w_gate, w_up, ((dh, "dh"), (gate, "gate"), (up, "up")))
    dtype = _dtype(x, "x")
    _, _, dh_ld = _matrix(dh, "dh", (m, n), x.dtype)
    _, _, gate_ld = _matrix(gate, "gate", (m, n), torch.float32)
    _, _, up_ld = _matrix(up, "up", (m, n), torch.float32)
    if gate_ld != up_ld and m > 1:
        raise ValueError("gate and up must have one row pitch")
    dx = empty((m, k), dtype=x.dtype, device=device)
    dw_gate = empty((n, k), dtype=x.dtype, device=device)
    dw_up = empty((n, k), dtype=x.dtype, device=device)
    nbytes = L.byz_gated_ffn_backward_workspace_bytes(m, k, n, dtype)
    ws, at = _workspace(nbytes, empty, device)
    _b._check(L.byz_gated_ffn_backward(
        dh.data_ptr(), dh_ld, x.data_ptr(), x_ld, w_gate.data_ptr(), w_up.data_ptr(), w_ld, gate.data_ptr(),
        up.data_ptr(), gate_ld, m, k, n, dtype, int(act), dx.data_ptr(), k, dw_gate.data_ptr(), dw_up.data_ptr(), k,
        at, nbytes, _b._stream_ptr(stream)), "byz_gated_ffn_backward")
    return dx, dw_gate, dw_up
