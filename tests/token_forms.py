"""Plain forms of the token operators in 64 bits, for their tests."""
import numpy as np
import torch

M32 = 0xFFFFFFFF
E = 2.0 ** -24


def philox(counter, key):
    """Philox 4x32-10 on arrays of four counter words (uint64 holding 32 bits), from the generator's definition."""
    c = [np.asarray(v, dtype=np.uint64) & np.uint64(M32) for v in counter]
    k = [key[0] & M32, key[1] & M32]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & np.uint64(M32),
             (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & np.uint64(M32)]
        k = [(k[0] + 0x9E3779B9) & M32, (k[1] + 0xBB67AE85) & M32]
    return c


def kept(rows, cols, p, seed, offset=0, first_row=0):
    """Which values of a dropout stay: bool [rows, cols]."""
    seed, offset = seed & (2 ** 64 - 1), offset & (2 ** 64 - 1)
    row = (np.arange(rows, dtype=np.uint64) + np.uint64(first_row))[:, None]
    group = np.arange((cols + 7) // 8, dtype=np.uint64)[None]
    row, group = np.broadcast_arrays(row, group)
    words = philox((group, row, np.full_like(group, offset & M32), np.full_like(group, offset >> 32)), (seed & M32, seed >> 32))
    halves = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=2)
    return torch.from_numpy(halves.reshape(rows, -1)[:, :cols] >= np.uint64(round(p * 65536)))


def kept_scale(p):
    taken = round(p * 65536)
    return 65536 / (65536 - taken) if taken < 65536 else 0.0


def norm(v, kind, eps):
    """(normalised, mean, 1 / deviation) of rows"""
    mean = v.mean(1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    rstd = ((v - mean).square().mean(1, keepdim=True) + eps) ** -0.5 if kind != "none" else torch.ones_like(v[:, :1])
    return (v - mean) * rstd, mean, rstd


def _norm_back(a, normal, rstd, kind):
    if kind == "none":
        return a
    mean = a.mean(1, keepdim=True) if kind == "layer" else 0.0
    return rstd * (a - mean - normal * (a * normal).mean(1, keepdim=True))


def _wide(v, shape, none):
    """A vector over the columns, or one for each part of the rows, as a matrix."""
    if v is None:
        return torch.full(shape, none, dtype=torch.float64)
    v = v.double()
    return v.expand(shape) if v.dim() == 1 else v.repeat_interleave(shape[0] // max(1, v.shape[0]), 0)


def residual(x, h, post, pre, scale, eps, mask, mask_scale, w1, b1, gate, w2, b2, dout=None, dy=None):
    """Outputs, stats and, with dout or dy, gradients by name, all on the CPU in 64 bits; and under name + "_scale" what fp32
    arithmetic's rounding acts on."""
    x = x.double()
    shape = x.shape
    W1, B1, G, W2, B2 = (_wide(v, shape, n) for v, n in ((w1, 1.0), (b1, 0.0), (gate, 1.0), (w2, 1.0), (b2, 0.0)))
    r, zero = {}, torch.zeros(shape, dtype=torch.float64)
    top = lambda v: v.abs().amax(1, keepdim=True) if v.shape[1] else v  # noqa: E731
    if h is not None:
        h = h.double()
        hn, mean1, rstd1 = norm(h, post, eps)
        factor = mask.double() * mask_scale
        v = torch.where(mask, hn * W1 + B1, 0.0) * mask_scale
        v_scale = (top(h) * rstd1 * W1.abs() + B1.abs()) * mask_scale
        t, t_scale = x + scale * G * v, x.abs() + (scale * G).abs() * v_scale
    else:
        hn, mean1, rstd1, t, t_scale = zero, zero[:, :1], zero[:, :1] + 1, x, x.abs()
    tn, mean2, rstd2 = norm(t, pre, eps)
    r["stats"] = torch.cat((mean1, rstd1, mean2, rstd2), 1)
    h_top, t_top = top(h) if h is not None else zero[:, :1], top(t_scale)
    xe1, xe2 = 1 + h_top * rstd1, 1 + t_top * rstd2
    r["stats_scale"] = torch.cat((h_top, rstd1 * xe1 ** 2, t_top, rstd2 * xe2 ** 2), 1)
    r["out"], r["out_scale"] = t, t_scale
    if pre != "none":
        r["y"], r["y_scale"] = tn * W2 + B2, (xe2 * (1 + tn.square())) * W2.abs() + B2.abs()
    if dout is None and dy is None:
        return r
    dout = dout.double() if dout is not None else zero
    dy = dy.double() if dy is not None else zero
    dt, dt_scale = dout, dout.abs()
    if pre != "none":
        a = dy * W2
        dt = dt + _norm_back(a, tn, rstd2, pre)
        dt_scale = dt_scale + rstd2 * top(a) * xe2 * (2 + tn.abs() + tn.square()) * xe2
        r["d_pre_weight"], r["d_pre_weight_scale"] = (dy * tn).sum(0), (dy.abs() * xe2 * (1 + tn.square())).sum(0)
        r["d_pre_bias"], r["d_pre_bias_scale"] = dy.sum(0), dy.abs().sum(0)
    r["dx"], r["dx_scale"] = dt, dt_scale
    if h is not None:
        each, each_scale = scale * v * dt, abs(scale) * (v.abs() * dt_scale + v_scale * dt.abs())
        parts = gate.shape[0] if gate is not None and gate.dim() == 2 else 1
        r["d_gate"] = each.view(parts, -1, shape[1]).sum(1)
        r["d_gate_scale"] = each_scale.view(parts, -1, shape[1]).sum(1)
        if gate is None or gate.dim() == 1:
            r["d_gate"], r["d_gate_scale"] = r["d_gate"][0], r["d_gate_scale"][0]
        du, du_scale = scale * G * factor * dt, (scale * G).abs() * factor * dt_scale
        r["d_post_weight"], r["d_post_weight_scale"] = (du * hn).sum(0), (du_scale * xe1 * (1 + hn.square())).sum(0)
        r["d_post_bias"], r["d_post_bias_scale"] = du.sum(0), du_scale.sum(0)
        b = du * W1
        r["dh"] = _norm_back(b, hn, rstd1, post)
        r["dh_scale"] = rstd1 * top(du_scale * W1) * xe1 * (2 + hn.abs() + hn.square()) * xe1 if post != "none" else du_scale * W1.abs()
    return r


def logp_terms(logits, label, temperature):
    """(logp, softmax, label's one-hot) of rows in 64 bits; rows without a token have zeros."""
    z = logits.double()
    top = z.amax(1, keepdim=True)
    top = torch.where(top == -np.inf, torch.zeros_like(top), top)
    d = (z - top) / temperature
    total = d.exp().sum(1, keepdim=True)
    log_sum = torch.where(total > 0, total, torch.ones_like(total)).log()
    hot = torch.zeros_like(z)
    here = label >= 0
    at = label.long().clamp_min(0)[:, None]
    hot.scatter_(1, at, here.double()[:, None])
    logp = torch.where(here, (d.gather(1, at) - log_sum)[:, 0], torch.zeros_like(log_sum[:, 0]))
    return logp, torch.where(here[:, None], (d - log_sum).exp(), torch.zeros_like(z)), hot


def policy(logp, old, advantage, ref, clip_low, clip_high, kl):
    """(loss, derivative by logp, what rounding acts on) in 64 bits"""
    old, advantage = old.double(), advantage.double()
    r = (logp - old).exp()
    low, high = float(np.float32(1) - np.float32(clip_low)), float(np.float32(1) + np.float32(clip_high))
    loss = -torch.minimum(r * advantage, r.clamp(low, high) * advantage)
    moving = torch.where(advantage >= 0, r <= high, r >= low)
    slope = torch.where(moving, -advantage * r, torch.zeros_like(r))
    scale = advantage.abs() * r
    if kl:
        g = ref.double() - logp
        loss = loss + kl * (torch.expm1(g) - g)
        slope = slope - kl * torch.expm1(g)
        scale = scale + kl * (g.exp() + 1)
    return loss, slope, scale


def preference(logp, bounds, ref, beta, smoothing):
    """(loss, sums, slope, sequence of each row or -1) in 64 bits"""
    edges = bounds.tolist()
    sums = torch.stack([logp[a:b].sum() for a, b in zip(edges, edges[1:])]) if len(edges) > 1 else logp.new_zeros(0)
    ratio = (sums - ref.double() if ref is not None else sums).view(-1, 2)
    margin = beta * (ratio[:, 0] - ratio[:, 1])
    softplus = torch.nn.functional.softplus
    loss = (1 - smoothing) * softplus(-margin, threshold=1e9) + smoothing * softplus(margin, threshold=1e9)
    slope = smoothing - torch.sigmoid(-margin)
    sequence = torch.full((logp.shape[0],), -1, dtype=torch.long)
    for s, (a, b) in enumerate(zip(edges, edges[1:])):
        sequence[a:b] = s
    return loss, sums, slope, sequence
