"""Operators of a worker that trains on tokens, for timing on a GPU.

A worker whose files are token sequences adds the branches of its network to a residual stream, drops
values of them, and learns from rewards or from pairs of answers.  Every case is one pass through one
of these operators:

    dropout     values dropped by a counter-based generator: forward, or forward and backward
    residual    a block's output normalised, dropped, gated, scaled and added to the residual stream,
                and the norm in front of the next block: forward, or forward and backward
    policy      the clipped policy loss of each token with its KL term, from logits: forward, or loss
                and gradient
    preference  the loss of pairs of sequences by their log ratios, from logits: forward, or loss and
                gradient

Sizes: 30 rows a file, 750 a batch of 25 files, 512 channels and 10 or 1000 outputs are those of the
workloads in synth/configs.py and of perf/operators.py; widths, token counts and vocabularies beyond
are generic.

    listed()  draw(rng)  prepare(case, seed)  run(state)  work(case)  exact(case, seed)
"""
import math
import random

import torch

own = False
DEV = "cuda:0"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
SIZE = {"f32": 4, "bf16": 2, "f16": 2}
EPS = 1e-5
LOW32 = 0xFFFFFFFF


def listed():
    return [
        # one file's pooled features: a short call, latency counts
        {"name": "dropout_step_file_30x512", "op": "dropout", "step": True, "dtype": "f32", "rows": 30, "cols": 512, "p": 0.1},
        # an odd batch of odd rows
        {"name": "dropout_forward_3333x1001", "op": "dropout", "step": False, "dtype": "f16", "rows": 3333, "cols": 1001,
         "p": 0.5},
        # the hidden values of 8192 tokens in a wide block, the largest
        {"name": "dropout_step_8192x16384", "op": "dropout", "step": True, "dtype": "bf16", "rows": 8192, "cols": 16384,
         "p": 0.1},
        # a single token answered: both norms, the gate of each channel
        {"name": "residual_forward_token", "op": "residual", "step": False, "dtype": "bf16", "post": "rms", "pre": "rms",
         "gate": 1, "p": 0.0, "rows": 1, "cols": 4096},
        # a training step on one file: 30 sequences of 64 tokens, a gate of each sequence
        {"name": "residual_step_file_1920x512", "op": "residual", "step": True, "dtype": "bf16", "post": "none",
         "pre": "layer", "gate": 30, "p": 0.1, "rows": 1920, "cols": 512},
        # a training step on an odd batch of odd width
        {"name": "residual_step_333x1000", "op": "residual", "step": True, "dtype": "f32", "post": "layer", "pre": "layer",
         "gate": 1, "p": 0.1, "rows": 333, "cols": 1000},
        # a training step on 8192 tokens of a wide block, the largest
        {"name": "residual_step_8192x4096", "op": "residual", "step": True, "dtype": "bf16", "post": "rms", "pre": "rms",
         "gate": 1, "p": 0.1, "rows": 8192, "cols": 4096},
        # one short answer over an odd vocabulary with banned entries, its loss alone
        {"name": "policy_forward_7x50021", "op": "policy", "step": False, "dtype": "f32", "masked": True, "rows": 7,
         "vocab": 50021, "kl": 0.05, "temperature": 0.7},
        # a batch of 750 tokens of a middling vocabulary
        {"name": "policy_step_750x32000", "op": "policy", "step": True, "dtype": "f16", "masked": False, "rows": 750,
         "vocab": 32000, "kl": 0.0, "temperature": 1.0},
        # a training step on 8192 tokens of a large vocabulary
        {"name": "policy_step_8192x131072", "op": "policy", "step": True, "dtype": "bf16", "masked": False, "rows": 8192,
         "vocab": 131072, "kl": 0.05, "temperature": 1.0},
        # one file: two pairs of short answers over a small vocabulary
        {"name": "preference_step_file_2x1000", "op": "preference", "step": True, "dtype": "f32", "pairs": 2, "rows": 61,
         "vocab": 1000, "smoothing": 0.0},
        # a batch of pairs of answers of ragged lengths
        {"name": "preference_step_16x50021", "op": "preference", "step": True, "dtype": "bf16", "pairs": 16, "rows": 6144,
         "vocab": 50021, "smoothing": 0.1},
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["dropout", "residual", "policy", "preference"])
    dtype = rng.choice(["f32", "bf16", "f16"])
    step = rng.random() < 0.6
    e = SIZE[dtype]
    if op == "dropout":
        cols = _log_uniform(rng, 1, 16384)
        rows = _log_uniform(rng, 1, max(1, min(65536, 8192 * 16384 * 2 // (cols * e))))
        return {"op": op, "step": step, "dtype": dtype, "rows": rows, "cols": cols, "p": rng.choice([0.05, 0.1, 0.25, 0.5])}
    if op == "residual":
        cols = _log_uniform(rng, 32, 16384)
        if rng.random() < 0.6:  # widths are round more often than not
            cols = min(16384, (cols + 63) // 64 * 64)
        rows = _log_uniform(rng, 1, max(1, min(32768, 8192 * 4096 * 2 // (cols * e))))
        gate = rng.choice([0, 1, 1, 2])
        if gate == 2:  # a gate for each of several sequences of one length
            gate = rng.randint(1, min(rows, 64))
            rows = rows // gate * gate
        post, pre = rng.choice(["none", "rms", "layer"]), rng.choice(["none", "rms", "rms", "layer", "layer"])
        return {"op": op, "step": step, "dtype": dtype, "post": post, "pre": pre, "gate": gate,
                "p": rng.choice([0.0, 0.1, 0.3]), "rows": rows, "cols": cols}
    if op == "policy":
        rows, vocab = _log_uniform(rng, 1, 8192), _log_uniform(rng, 10, 200000)
        rows = max(1, min(rows, 8192 * 131072 * 2 // (vocab * e)))
        return {"op": op, "step": step, "dtype": dtype, "masked": rng.random() < 0.25, "rows": rows, "vocab": vocab,
                "kl": rng.choice([0.0, 0.02, 0.1]), "temperature": rng.choice([0.7, 1.0, 1.5])}
    vocab, pairs = _log_uniform(rng, 10, 131072), _log_uniform(rng, 1, 64)
    rows = max(4 * pairs, min(_log_uniform(rng, 4, 8192), 6144 * 50021 * 2 // (vocab * e)))
    return {"op": op, "step": step, "dtype": dtype, "pairs": pairs, "rows": rows, "vocab": vocab,
            "smoothing": rng.choice([0.0, 0.0, 0.1])}


# ------------------------------------------------------------------------------- inputs


def _randn(gen, *shape, dtype=torch.float32, scale=1.0):
    return torch.randn(*shape, generator=gen, device=DEV, dtype=torch.float32).mul_(scale).to(dtype)


def _key(seed):
    """A generator's key and the number of the call, from anywhere in 64 bits."""
    rng = random.Random(seed)
    return rng.getrandbits(64), rng.getrandbits(64)


def _dropout_inputs(case, gen, seed):
    shape, dtype = (case["rows"], case["cols"]), DTYPES[case["dtype"]]
    s = {"p": case["p"], "step": case["step"], "key": _key(seed), "x": _randn(gen, *shape, dtype=dtype)}
    if case["step"]:
        s["dy"] = _randn(gen, *shape, dtype=dtype)
    return s


def _residual_inputs(case, gen, seed):
    m, d, dtype = case["rows"], case["cols"], DTYPES[case["dtype"]]
    s = {name: case[name] for name in ("post", "pre", "p", "step")}
    s["key"], s["scale"] = _key(seed), 0.5
    # a residual stream has a few channels far larger than the rest, and a mean
    channels = torch.where(torch.rand(d, generator=gen, device=DEV) < 1 / 64, 8.0, 1.0)
    s["x"] = (_randn(gen, m, d) * channels + 0.25).to(dtype)
    s["h"] = (_randn(gen, m, d, scale=0.7) + _randn(gen, d, scale=0.2)).to(dtype)
    for norm in ("post", "pre"):
        s[norm + "_weight"] = 1 + _randn(gen, d, scale=0.1) if case[norm] != "none" else None
        s[norm + "_bias"] = _randn(gen, d, scale=0.1) if case[norm] == "layer" else None
    s["gate"] = 1 + _randn(gen, case["gate"], d, scale=0.3) if case["gate"] else None
    if case["step"]:
        s["dout"] = _randn(gen, m, d, dtype=dtype)
        s["dy"] = _randn(gen, m, d, dtype=dtype) if case["pre"] != "none" else None
    return s


def _token_logits(rows, vocab, dtype, gen, masked):
    """Logits of a model that knows something of its tokens, and the tokens."""
    logits = torch.randn(rows, vocab, generator=gen, device=DEV, dtype=dtype).mul_(2)
    if masked:  # a tenth of the vocabulary is banned
        logits.masked_fill_(torch.rand(vocab, generator=gen, device=DEV) < 0.1, -math.inf)
    label = torch.randint(0, vocab, (rows, 1), generator=gen, device=DEV)
    logits.scatter_(1, label, (_randn(gen, rows, 1, scale=2.0) + math.log(vocab)).to(dtype))
    return logits, label.squeeze(1)


def _loss_scale(case):
    return 1024.0 if case["dtype"] == "f16" else 1.0


def _policy_rows(case):
    """Rows that have a token: the last sixteenth is padding."""
    return case["rows"] - case["rows"] // 16


def _policy_inputs(case, gen, seed):
    rows, counted = case["rows"], _policy_rows(case)
    s = {name: case[name] for name in ("kl", "temperature", "step")}
    s["logits"], label = _token_logits(rows, case["vocab"], DTYPES[case["dtype"]], gen, case["masked"])
    logp = torch.cat([torch.log_softmax(part.double() / case["temperature"], 1).gather(1, at[:, None]).squeeze(1)
                      for part, at in zip(s["logits"].split(512), label.split(512))])
    # the policy has moved since the tokens were drawn: most ratios are within the clipping range, some
    # beyond.  The loss has a kink at its ends: what lies within 0.002 of one is moved away
    moved = _randn(gen, rows, scale=0.15).double()
    for end in (0.8, 1.25):
        moved = torch.where((moved.exp() - end).abs() < 2e-3, moved + 0.01, moved)
    s["old"] = (logp - moved).float()
    s["ref"] = (logp + _randn(gen, rows, scale=0.3)).float() if case["kl"] else None
    # advantages of one sequence are one value; some have none
    advantage = _randn(gen, rows // 8 + 1).repeat_interleave(8)[:rows]
    s["advantage"] = torch.where(torch.arange(rows, device=DEV) // 8 % 8 == 5, 0.0, advantage).contiguous()
    s["label"] = torch.where(torch.arange(rows, device=DEV) < counted, label, -1).to(torch.int32)
    if case["step"]:  # the weight of each token in the mean (times a loss scale where the type needs one)
        s["dloss"] = torch.rand(rows, generator=gen, device=DEV).add_(0.5).mul_(_loss_scale(case) / rows)
    return s


def _sequences(case):
    """(bounds of the 2 * pairs sequences, their prompts' lengths): ragged, some rows of padding behind the last."""
    rng = random.Random(case["pairs"] * 1000003 + case["rows"])
    count, used = 2 * case["pairs"], case["rows"] - case["rows"] // 32
    share = [rng.uniform(0.25, 1.0) for _ in range(count)]
    lengths = [1 + int((used - count) * v / sum(share)) for v in share]
    bounds = [0]
    for length in lengths:
        bounds.append(bounds[-1] + length)
    return bounds, [length // 4 for length in lengths]


def _preference_inputs(case, gen, seed):
    rows, pairs = case["rows"], case["pairs"]
    s = {"beta": 0.1, "smoothing": case["smoothing"], "step": case["step"]}
    s["logits"], label = _token_logits(rows, case["vocab"], DTYPES[case["dtype"]], gen, False)
    bounds, prompts = _sequences(case)
    counted = torch.zeros(rows, dtype=torch.bool)
    for at, end, prompt in zip(bounds, bounds[1:], prompts):
        counted[at + prompt:end] = True  # a prompt's tokens are given, not learnt
    counted = counted.to(DEV)
    s["label"] = torch.where(counted, label, -1).to(torch.int32)
    s["bounds"] = torch.tensor(bounds, dtype=torch.int32, device=DEV)
    logp = torch.cat([torch.log_softmax(part.double(), 1).gather(1, at[:, None]).squeeze(1)
                      for part, at in zip(s["logits"].split(512), label.split(512))])
    total = torch.cat([torch.zeros(1, device=DEV, dtype=torch.float64), torch.where(counted, logp, 0.0).cumsum(0)])
    sums = total[s["bounds"][1:].long()] - total[s["bounds"][:-1].long()]
    # the reference model agrees but for some nats a sequence
    s["ref"] = (sums + _randn(gen, 2 * pairs, scale=4.0)).float()
    if case["step"]:
        s["dloss"] = torch.rand(pairs, generator=gen, device=DEV).add_(0.5).mul_(_loss_scale(case) / pairs)
    return s


INPUTS = {"dropout": _dropout_inputs, "residual": _residual_inputs, "policy": _policy_inputs,
          "preference": _preference_inputs}


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(int(seed))
    s = INPUTS[case["op"]](case, gen, int(seed))
    s["op"] = case["op"]
    return s


# --------------------------------------------------------------------------- plain forms


def _mul32(a, b):
    """(high, low) words of the 64-bit product of 32-bit words in int64, which wraps."""
    product = a * b
    return (product >> 32) & LOW32, product & LOW32


def _words(rows, groups, key):
    """Four 32-bit words for each of a row's groups of eight columns: Philox 4x32 of ten rounds (Salmon, Moraes, Dror
    and Shaw, 2011); the counter is (group, row, number of the call)."""
    seed, offset = key
    c0 = torch.arange(groups, device=DEV).expand(rows, groups)
    c1 = torch.arange(rows, device=DEV)[:, None].expand(rows, groups)
    c2 = torch.full((1, 1), offset & LOW32, device=DEV)
    c3 = torch.full((1, 1), offset >> 32, device=DEV)
    k0, k1 = seed & LOW32, seed >> 32
    for _ in range(10):
        high0, low0 = _mul32(c0, 0xD2511F53)
        high1, low1 = _mul32(c2, 0xCD9E8D57)
        c0, c1, c2, c3 = high1 ^ c1 ^ k0, low1, high0 ^ c3 ^ k1, low0
        k0, k1 = (k0 + 0x9E3779B9) & LOW32, (k1 + 0xBB67AE85) & LOW32
    return torch.stack(torch.broadcast_tensors(c0, c1, c2, c3), dim=2)


def _kept(rows, cols, p, key):
    """Which values stay: those whose 16 random bits are at least p * 2^16."""
    words = _words(rows, (cols + 7) // 8, key)
    halves = torch.stack((words & 0xFFFF, words >> 16), dim=3).reshape(rows, -1)[:, :cols]
    return halves >= round(p * 65536)


def _kept_scale(p):
    return 65536.0 / (65536 - round(p * 65536))


def _dropout_plain(s):
    x, p = s["x"], s["p"]
    kept, scale = _kept(*x.shape, p, s["key"]), _kept_scale(p)
    out = {"y": torch.where(kept, x.float() * scale, 0.0).to(x.dtype)}
    if s["step"]:
        out["dx"] = torch.where(kept, s["dy"].float() * scale, 0.0).to(x.dtype)
    return out


def _normal(v, kind):
    """(normalised, mean, 1 / deviation) of rows."""
    mean = v.mean(dim=1, keepdim=True) if kind == "layer" else torch.zeros_like(v[:, :1])
    v = v - mean
    rstd = torch.rsqrt(v.square().mean(dim=1, keepdim=True) + EPS) if kind != "none" else torch.ones_like(v[:, :1])
    return v * rstd, mean, rstd


def _normal_back(g, normal, rstd, kind):
    """Gradient of what was normalised, for that of the result."""
    if kind == "none":
        return g
    inner = normal * (g * normal).mean(dim=1, keepdim=True)
    return rstd * (g - inner - (g.mean(dim=1, keepdim=True) if kind == "layer" else 0.0))


def _affine(v, weight, bias):
    v = v * weight if weight is not None else v
    return v + bias if bias is not None else v


def _residual_plain(s):
    x, h, dtype = s["x"].float(), s["h"].float(), s["x"].dtype
    m, d = x.shape
    post, pre, gate, scale = s["post"], s["pre"], s["gate"], s["scale"]
    hn, mean1, rstd1 = _normal(h, post)
    factor = torch.where(_kept(m, d, s["p"], s["key"]), _kept_scale(s["p"]), 0.0) if s["p"] else torch.ones(1, 1, device=DEV)
    v = _affine(hn, s["post_weight"], s["post_bias"]) * factor
    wide = gate.repeat_interleave(m // gate.shape[0], dim=0) if gate is not None else torch.ones(1, 1, device=DEV)
    total = x + scale * wide * v
    tn, mean2, rstd2 = _normal(total, pre)
    out = {"out": total.to(dtype), "stats": torch.cat((mean1, rstd1, mean2, rstd2), dim=1)}
    if pre != "none":
        out["y"] = _affine(tn, s["pre_weight"], s["pre_bias"]).to(dtype)
    if s["step"]:
        dt = s["dout"].float()
        if pre != "none":
            dy = s["dy"].float()
            out["d_pre_weight"] = (dy * tn).sum(dim=0)
            if s["pre_bias"] is not None:
                out["d_pre_bias"] = dy.sum(dim=0)
            dt = dt + _normal_back(dy * s["pre_weight"], tn, rstd2, pre)
        out["dx"] = dt.to(dtype)
        if gate is not None:
            out["d_gate"] = (scale * v * dt).view(gate.shape[0], -1, d).sum(dim=1)
        du = scale * wide * dt * factor
        if post != "none":
            out["d_post_weight"] = (du * hn).sum(dim=0)
            if s["post_bias"] is not None:
                out["d_post_bias"] = du.sum(dim=0)
            du = _normal_back(du * s["post_weight"], hn, rstd1, post)
        out["dh"] = du.to(dtype)
    return out


def _row_terms(logits, label, temperature):
    """(rows that have a token, its column, logits over the temperature less their maximum, the logarithm of the sum of
    their exponentials, the token's log-probability): per-row terms in 64 bits."""
    here = (label >= 0)[:, None]
    at = label.long().clamp_min(0)[:, None]
    z = logits.float()
    z = (z - z.max(dim=1, keepdim=True).values) / temperature
    log_sum = torch.log(torch.exp(z).sum(dim=1, keepdim=True, dtype=torch.float64))
    logp = torch.where(here, z.gather(1, at).double() - log_sum, 0.0)
    return here, at, z, log_sum, logp


def _logits_gradient(s, here, at, z, log_sum, dlogp, temperature):
    w = torch.where(here, dlogp / temperature, 0.0).float()
    d = torch.exp(z - log_sum.float()).mul_(-w)
    return d.scatter_add_(1, at, w).to(s["logits"].dtype)


def _policy_plain(s):
    low, high, tau, advantage = 0.8, 1.25, s["temperature"], s["advantage"].double()[:, None]
    here, at, z, log_sum, logp = _row_terms(s["logits"], s["label"], tau)
    ratio = torch.exp(logp - s["old"].double()[:, None])
    loss = -torch.minimum(ratio * advantage, ratio.clamp(low, high) * advantage)
    if s["kl"]:
        gap = s["ref"].double()[:, None] - logp
        loss = loss + s["kl"] * (torch.expm1(gap) - gap)
    out = {"loss": torch.where(here, loss, 0.0).squeeze(1).float(), "logp": logp.squeeze(1).float()}
    if s["step"]:
        moving = torch.where(advantage >= 0, ratio <= high, ratio >= low)
        dlogp = torch.where(moving, -advantage * ratio, 0.0)
        if s["kl"]:
            dlogp = dlogp - s["kl"] * torch.expm1(gap)
        out["dlogits"] = _logits_gradient(s, here, at, z, log_sum, dlogp * s["dloss"].double()[:, None], tau)
    return out


def _preference_plain(s):
    beta, smoothing, bounds = s["beta"], s["smoothing"], s["bounds"].long()
    here, at, z, log_sum, logp = _row_terms(s["logits"], s["label"], 1.0)
    total = torch.cat([torch.zeros(1, device=DEV, dtype=torch.float64), logp.squeeze(1).cumsum(0)])
    sums = total[bounds[1:]] - total[bounds[:-1]]
    ratio = (sums - s["ref"].double()).view(-1, 2)
    margin = beta * (ratio[:, 0] - ratio[:, 1])
    # log(1 + exp(-margin)) and its mirror image, from the side that does not overflow
    small = torch.log1p(torch.exp(-margin.abs()))
    loss = (1 - smoothing) * (small + (-margin).clamp_min(0)) + smoothing * (small + margin.clamp_min(0))
    out = {"loss": loss.float(), "sums": sums.float()}
    if s["step"]:
        slope = smoothing - 1 / (1 + torch.exp(margin))
        each = beta * slope * s["dloss"].double()
        each = torch.stack((each, -each), dim=1).view(-1)
        sequence = torch.searchsorted(bounds, torch.arange(len(s["label"]), device=DEV), right=True) - 1
        dlogp = torch.cat((each, each.new_zeros(1)))[sequence][:, None]
        out["dlogits"] = _logits_gradient(s, here, at, z, log_sum, dlogp, 1.0)
    return out


PLAIN = {"dropout": _dropout_plain, "residual": _residual_plain, "policy": _policy_plain, "preference": _preference_plain}


# -------------------------------------------------------------------- the framework's own


def _dropout_own(B, s):
    seed, offset = s["key"]
    out = {"y": B.byz_dropout(s["x"], s["p"], seed, offset)}
    if s["step"]:
        out["dx"] = B.byz_dropout(s["dy"], s["p"], seed, offset)
    return out


def _residual_own(B, s):
    seed, offset = s["key"]
    form = B.byz_residual_form(post=B.BYZ_NORMS[s["post"]], pre=B.BYZ_NORMS[s["pre"]], scale=s["scale"], eps=EPS, p=s["p"],
                               seed=seed, offset=offset)
    parameters = (s["post_weight"], s["post_bias"], s["gate"], s["pre_weight"], s["pre_bias"])
    total, y, stats = B.byz_residual_norm(s["x"], s["h"], form, *parameters)
    out = {"out": total, "stats": stats}
    if y is not None:
        out["y"] = y
    if s["step"]:
        out["dx"], out["dh"], grads = B.byz_residual_norm_backward(s["dout"], s["dy"], s["x"], s["h"], stats, form, *parameters)
        for name, grad in zip(("post_weight", "post_bias", "gate", "pre_weight", "pre_bias"), grads):
            if grad is not None:
                out["d_" + name] = grad
    return out


def _policy_own(B, s):
    given = (s["logits"], s["label"], s["old"], s["advantage"])
    terms = {"ref": s["ref"], "kl": s["kl"], "clip_low": 0.2, "clip_high": 0.25, "temperature": s["temperature"]}
    if s["step"]:
        loss, logp, dlogits = B.byz_policy_loss_step(*given, s["dloss"], **terms)
        return {"loss": loss, "logp": logp, "dlogits": dlogits}
    loss, logp, _ = B.byz_policy_loss(*given, **terms)
    return {"loss": loss, "logp": logp}


def _preference_own(B, s):
    given = (s["logits"], s["label"], s["bounds"])
    terms = {"ref": s["ref"], "beta": s["beta"], "smoothing": s["smoothing"]}
    if s["step"]:
        loss, sums, dlogits = B.byz_preference_loss_step(*given, s["dloss"], **terms)
        return {"loss": loss, "sums": sums, "dlogits": dlogits}
    loss, sums, _, _ = B.byz_preference_loss(*given, **terms)
    return {"loss": loss, "sums": sums}


OWN = {"dropout": _dropout_own, "residual": _residual_own, "policy": _policy_own, "preference": _preference_own}


def run(state):
    if own:
        import paper_2010_04902_amd as B
        return OWN[state["op"]](B, state)
    return PLAIN[state["op"]](state)


# ------------------------------------------------------------------------ what a pass needs


def work(case):
    e = SIZE[case["dtype"]]
    if case["op"] == "dropout":
        size = case["rows"] * case["cols"]
        passes = 2 if case["step"] else 1
        return {"bytes": 2 * passes * size * e, "flops": 2 * passes * size}
    if case["op"] == "residual":
        m, d = case["rows"], case["cols"]
        vectors = case["gate"] + sum({"none": 0, "rms": 1, "layer": 2}[case[n]] for n in ("post", "pre"))
        tensors = 3 + (case["pre"] != "none")  # x, h in; the sum and y out
        if case["step"]:  # gradients of both in; of x and h out
            tensors += 3 + (case["pre"] != "none")
        return {"bytes": tensors * m * d * e + (2 if case["step"] else 1) * vectors * d * 4 + 16 * m,
                "flops": (44 if case["step"] else 14) * m * d}
    if case["op"] == "policy":
        counted, extra = _policy_rows(case), 24 * case["rows"]
    else:
        bounds, prompts = _sequences(case)
        counted, extra = bounds[-1] - sum(prompts), 4 * case["rows"] + 28 * case["pairs"]
    # rows that have a token are read; a step writes all
    byts = (counted + (case["rows"] if case["step"] else 0)) * case["vocab"] * e + extra
    return {"bytes": byts, "flops": (7 if case["step"] else 4) * counted * case["vocab"]}


# ------------------------------------------------------------ the definitions, in 64 bits


def _product64(a, m):
    """(high, low) words of a times the number m, from products of 16-bit parts."""
    a0, a1, m0, m1 = a % 65536, a // 65536, m % 65536, m // 65536
    middle = a0 * m1 + a1 * m0 + a0 * m0 // 65536
    return a1 * m1 + middle // 65536, (middle % 65536) * 65536 + a0 * m0 % 65536


def _kept64(rows, cols, p, key):
    groups = -(-cols // 8)
    number = torch.arange(rows * groups, device=DEV)
    word = [number % groups, number // groups, torch.full_like(number, key[1] % 2 ** 32), torch.full_like(number, key[1] // 2 ** 32)]
    for turn in range(10):
        k = [(key[0] % 2 ** 32 + turn * 0x9E3779B9) % 2 ** 32, (key[0] // 2 ** 32 + turn * 0xBB67AE85) % 2 ** 32]
        first, second = _product64(word[0], 0xD2511F53), _product64(word[2], 0xCD9E8D57)
        word = [second[0] ^ word[1] ^ k[0], second[1], first[0] ^ word[3] ^ k[1], first[1]]
    bits = torch.empty(rows * groups, 8, device=DEV, dtype=torch.float64)
    for i in range(8):
        bits[:, i] = (word[i // 2] // 65536 if i % 2 else word[i // 2] % 65536).double()
    return (bits.view(rows, groups * 8)[:, :cols] / 65536 >= round(p * 65536) / 65536).double()


def _dropout_exact(s):
    share = 1 - round(s["p"] * 65536) / 65536
    mask = _kept64(*s["x"].shape, s["p"], s["key"]) / share
    out = {"y": s["x"].double() * mask}
    if s["step"]:
        out["dx"] = s["dy"].double() * mask
    return out


def _norm64(v, kind, weight, bias):
    if kind == "none":
        return v, torch.tensor([0.0, 1.0], device=DEV, dtype=torch.float64).expand(v.shape[0], 2)
    mean = v.mean(1, keepdim=True) if kind == "layer" else 0.0 * v[:, :1]
    deviation = ((v - mean).pow(2).mean(1, keepdim=True) + EPS).sqrt()
    result = (v - mean) / deviation * weight
    return (result if bias is None else result + bias), torch.cat((mean, 1 / deviation), 1).detach()


def _residual_exact(s):
    names = [n for n in ("x", "h", "post_weight", "post_bias", "gate", "pre_weight", "pre_bias") if s[n] is not None]
    leaf = {n: s[n].double().requires_grad_(s["step"]) for n in names}
    m, d = s["x"].shape
    branch, stats1 = _norm64(leaf["h"], s["post"], leaf.get("post_weight"), leaf.get("post_bias"))
    if s["p"]:
        branch = branch * (_kept64(m, d, s["p"], s["key"]) / (1 - round(s["p"] * 65536) / 65536))
    if "gate" in leaf:
        branch = (branch.view(leaf["gate"].shape[0], -1, d) * leaf["gate"][:, None]).view(m, d)
    total = leaf["x"] + branch * s["scale"]
    y, stats2 = _norm64(total, s["pre"], leaf.get("pre_weight"), leaf.get("pre_bias"))
    out = {"out": total.detach(), "stats": torch.cat((stats1, stats2), 1)}
    if s["pre"] != "none":
        out["y"] = y.detach()
    if s["step"]:
        ends = [(total, s["dout"])] + ([(y, s["dy"])] if s["pre"] != "none" else [])
        grads = torch.autograd.grad([v for v, _ in ends], [leaf[n] for n in names], [g.double() for _, g in ends])
        out.update(zip(["dx" if n == "x" else "dh" if n == "h" else "d_" + n for n in names], grads))
    return out


def _logp64(logits, label, temperature):
    """Log-probabilities of the tokens of rows that have one, 0 for others."""
    logp = torch.log_softmax(logits / temperature, dim=1).gather(1, label.long().clamp_min(0)[:, None])[:, 0]
    return torch.where(label >= 0, logp, torch.zeros_like(logp))


def _from_logp64(s, temperature, loss_of):
    """(loss, log-probabilities, gradient of the logits or None), rows in parts."""
    parts = [slice(at, at + 512) for at in range(0, len(s["label"]), 512)]
    logp = torch.cat([_logp64(s["logits"][r].double(), s["label"][r], temperature) for r in parts]).requires_grad_(s["step"])
    loss, dlogits = loss_of(logp), None
    if s["step"]:
        dlogp = torch.autograd.grad(loss, logp, s["dloss"].double())[0]
        grads = []
        for r in parts:
            student = s["logits"][r].double().requires_grad_()
            grads.append(torch.autograd.grad(_logp64(student, s["label"][r], temperature), student, dlogp[r])[0])
        dlogits = torch.cat(grads)
    return loss.detach(), logp.detach(), dlogits


def _policy_exact(s):
    def loss_of(logp):
        ratio, advantage = (logp - s["old"].double()).exp(), s["advantage"].double()
        bounded = torch.where(advantage > 0, ratio.clamp(max=1.25), ratio.clamp(min=0.8))
        loss = -bounded * advantage
        if s["kl"]:
            log_ratio = s["ref"].double() - logp
            loss = loss + s["kl"] * (log_ratio.exp() - 1 - log_ratio)
        return torch.where(s["label"] >= 0, loss, torch.zeros_like(loss))

    loss, logp, dlogits = _from_logp64(s, s["temperature"], loss_of)
    out = {"loss": loss, "logp": logp}
    return {**out, "dlogits": dlogits} if s["step"] else out


def _preference_exact(s):
    edges = s["bounds"].tolist()

    def sums_of(logp):
        return torch.stack([logp[at:end].sum() for at, end in zip(edges, edges[1:])])

    def loss_of(logp):
        gap = sums_of(logp) - s["ref"].double()
        margin = s["beta"] * (gap[0::2] - gap[1::2])
        log_sigmoid = torch.nn.functional.logsigmoid
        return -(1 - s["smoothing"]) * log_sigmoid(margin) - s["smoothing"] * log_sigmoid(-margin)

    loss, logp, dlogits = _from_logp64(s, 1.0, loss_of)
    out = {"loss": loss, "sums": sums_of(logp)}
    return {**out, "dlogits": dlogits} if s["step"] else out


EXACT = {"dropout": _dropout_exact, "residual": _residual_exact, "policy": _policy_exact, "preference": _preference_exact}


def exact(case, seed):
    return EXACT[case["op"]](prepare(case, seed))
