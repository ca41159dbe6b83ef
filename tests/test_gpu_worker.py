"""The operators of a worker's training step against their definitions in 64 bits.

Tolerances.  u = finfo(type).eps / 2 is what one rounding can be off, relative to the value; fp32 arithmetic
is allowed some dozens of 2^-24 of the largest term that enters a result (the terms are written at each test).
"""
import math

import pytest
import torch

import paper_2010_04902_amd as B

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
E = 2.0 ** -24


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _randn(gen, *shape, dtype=F32, scale=1.0):
    return (torch.randn(*shape, generator=gen, device=DEV) * scale).to(dtype)


def _u(dtype):
    return torch.finfo(dtype).eps / 2


def _act(z, act):
    return {"none": lambda v: v, "relu": lambda v: torch.where(v < 0, torch.zeros_like(v), v),
            "silu": lambda v: v * torch.sigmoid(v), "gelu": lambda v: v * torch.special.ndtr(v),
            "sigmoid": torch.sigmoid}[act](z)


def _near(got, want, tol, what):
    assert got.shape == want.shape, what
    bad = ~((got.double() - want).abs() <= tol)
    assert not bool(bad.any()), "%s: %d of %d off, worst by %.3g of what is allowed" % (
        what, int(bad.sum()), bad.numel(), float(((got.double() - want).abs() / tol).nan_to_num(nan=math.inf).max()))


def _same_bits(a, b):
    view = torch.int32 if a.dtype == F32 else torch.int16
    return torch.equal(a.contiguous().view(view), b.contiguous().view(view))


# ------------------------------------------------------------------ group norm


def _norm_reference(x, groups, gamma, beta, eps, act, dy=None):
    """x [n, p, c] -> y, mean, rstd and, with dy, dx, dgamma, dbeta: all in 64 bits; scales of their terms."""
    n, p, c = x.shape
    X = x.double().view(n, p, groups, c // groups)
    mean = X.mean(dim=(1, 3), keepdim=True)
    var = (X - mean).square().mean(dim=(1, 3), keepdim=True)
    rstd = (var + eps) ** -0.5
    xhat = ((X - mean) * rstd).requires_grad_(dy is not None)
    w = (gamma.double() if gamma is not None else torch.ones(c, device=DEV, dtype=torch.float64)).view(groups, -1)
    b = (beta.double() if beta is not None else torch.zeros(c, device=DEV, dtype=torch.float64)).view(groups, -1)
    z = (xhat * w + b).detach().requires_grad_(dy is not None)
    y = _act(z, act)
    r = {"y": y.detach().view(n, p, c), "mean": mean.view(n, groups), "rstd": rstd.view(n, groups)}
    # a value's share of the statistics' errors: the group's largest value, scaled as the value itself is
    big = X.abs().amax(dim=(1, 3), keepdim=True)
    r["z_scale"] = (big * rstd * w.abs() + b.abs()).expand_as(X).reshape(n, p, c)
    r["big"], r["z"] = big.view(n, groups), z.detach().view(n, p, c)
    if dy is not None:
        xhat = xhat.detach()
        slope, = torch.autograd.grad(y.sum(), z)
        dz = dy.double().view_as(X) * slope
        g = dz * w
        s1, s2 = g.mean(dim=(1, 3), keepdim=True), (g * xhat).mean(dim=(1, 3), keepdim=True)
        r["dx"] = (rstd * (g - s1 - xhat * s2)).view(n, p, c)
        r["dgamma"], r["dbeta"] = (dz * xhat).sum(dim=(0, 1)).view(c), dz.sum(dim=(0, 1)).view(c)
        # errors of xhat (big * rstd) act on every term through the slope (whose own slope is 1.2 at most)
        xe = big * rstd + 1
        dye = dy.double().abs().view_as(X)
        ge = (dye * (w.abs() + 1) ** 2 * (1 + b.abs())).amax(dim=(1, 3), keepdim=True)
        r["dx_scale"] = (rstd * ge * xe * (2 + xhat.abs() + xhat.square())).view(n, p, c)
        par = dye * xe * (w.abs() + 1) * (1 + b.abs())
        r["dbeta_scale"] = par.sum(dim=(0, 1)).view(c)
        r["dgamma_scale"] = (par * (1 + xhat.abs())).sum(dim=(0, 1)).view(c)
    return r


def _norm_case(n, p, c, groups, dtype, act="none", params=True, seed=0, offset=0.0):
    gen = _gen(seed)
    x = (_randn(gen, n, p, c) + _randn(gen, c, scale=0.5) + offset).to(dtype)
    gamma = 1 + _randn(gen, c, scale=0.2) if params else None
    beta = _randn(gen, c, scale=0.2) if params else None
    dy = _randn(gen, n, p, c, dtype=dtype)
    if act == "relu":  # no value within rounding of the corner
        z = _norm_reference(x, groups, gamma, beta, 1e-5, "none")["z"]
        x = torch.where(z.abs() < 1e-3, x + 0.0625, x)
    return x, gamma, beta, dy


def _norm_check(x, groups, gamma, beta, dy, act, eps=1e-5, stream=None):
    code, u = B.BYZ_ACTS[act], _u(x.dtype)
    y, mean, rstd = B.byz_group_norm(x, groups, gamma, beta, eps, code, stream=stream)
    dx, dgamma, dbeta = B.byz_group_norm_backward(dy, x, groups, mean, rstd, gamma, beta, code, stream=stream)
    torch.cuda.synchronize()
    r = _norm_reference(x, groups, gamma, beta, eps, act, dy)
    _near(mean, r["mean"], 32 * E * r["big"], "mean")
    _near(rstd, r["rstd"], 32 * E * r["rstd"] * (1 + r["big"] ** 2 * r["rstd"] ** 2 * 2.0 ** -20), "rstd")
    _near(y, r["y"], u * r["y"].abs() + 64 * E * r["z_scale"], "y")
    _near(dx, r["dx"], u * r["dx"].abs() + 64 * E * r["dx_scale"], "dx")
    _near(dgamma, r["dgamma"], 64 * E * r["dgamma_scale"], "dgamma")
    _near(dbeta, r["dbeta"], 64 * E * r["dbeta_scale"], "dbeta")
    return y, mean, rstd, dx, dgamma, dbeta


NORM_SHAPES = [
    (1, 1, 1, 1), (1, 1, 8, 8), (2, 1, 32, 4), (3, 2, 2, 1), (30, 16, 512, 32), (2, 64, 48, 3), (5, 49, 120, 12), (3, 77, 30, 6),
    (2, 100, 15, 5), (4, 9, 7, 7), (2, 33, 1000, 8), (1, 65, 24, 1), (2, 31, 4096, 1), (1, 40, 6000, 2), (1, 7, 2051, 1),
    (2, 3000, 64, 32), (3, 4096, 32, 32), (2, 12544, 64, 32), (1, 20000, 12, 3), (1, 3001, 250, 10), (257, 4, 16, 2),
]


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
@pytest.mark.parametrize("shape", NORM_SHAPES, ids=str)
def test_group_norm_sizes(shape, dtype):
    x, gamma, beta, dy = _norm_case(*shape, dtype, "silu", seed=sum(shape))
    _norm_check(x, shape[3], gamma, beta, dy, "silu")


@pytest.mark.parametrize("params", [True, False])
@pytest.mark.parametrize("act", sorted(B.BYZ_ACTS))
@pytest.mark.parametrize("shape", [(4, 100, 64, 16), (2, 9000, 64, 16)], ids=str)
def test_group_norm_activations(shape, act, params):
    x, gamma, beta, dy = _norm_case(*shape, BF16, act, params, seed=3)
    _norm_check(x, shape[3], gamma, beta, dy, act)


@pytest.mark.parametrize("shape", [(2, 500, 32, 8), (2, 20000, 32, 8)], ids=str)
def test_group_norm_far_from_zero(shape):
    # a mean a thousand times the deviation: the distances are taken from the mean, not as a difference of squares
    x, gamma, beta, dy = _norm_case(*shape, F32, seed=5, offset=1000.0)
    _, _, rstd, _, _, _ = _norm_check(x, shape[3], gamma, beta, dy, "none")
    want = _norm_reference(x, shape[3], gamma, beta, 1e-5, "none")["rstd"]
    assert float((rstd.double() / want - 1).abs().max()) < 1e-5


@pytest.mark.parametrize("shape", [(2, 50, 32, 8), (1, 9000, 32, 8)], ids=str)
def test_group_norm_constant_groups(shape):
    # variance 0: y = act(beta), the gradient is rstd (dz - its mean)
    x, gamma, beta, dy = _norm_case(*shape, F32, seed=6)
    x[:] = 3.0
    y, mean, rstd, _, _, _ = _norm_check(x, shape[3], gamma, beta, dy, "silu")
    assert torch.equal(mean, torch.full_like(mean, 3.0))
    assert torch.allclose(rstd, torch.full_like(rstd, 1e-5 ** -0.5))


@pytest.mark.parametrize("shape", [(3, 50, 32, 8), (2, 9000, 32, 8)], ids=str)
@pytest.mark.parametrize("value", [math.inf, -math.inf, math.nan])
def test_group_norm_infinite_values_stay_in_their_group(shape, value):
    x, gamma, beta, dy = _norm_case(*shape, F32, seed=7)
    clean = B.byz_group_norm(x, shape[3], gamma, beta, act=B.BYZ_ACT_RELU)
    cx = B.byz_group_norm_backward(dy, x, shape[3], clean[1], clean[2], gamma, beta, B.BYZ_ACT_SILU)
    x = x.clone()
    x[1, shape[1] // 2, 5] = value  # sample 1, group 1
    y, mean, rstd = B.byz_group_norm(x, shape[3], gamma, beta, act=B.BYZ_ACT_RELU)
    dx, _, _ = B.byz_group_norm_backward(dy, x, shape[3], mean, rstd, gamma, beta, B.BYZ_ACT_SILU)
    hit = torch.zeros_like(x, dtype=torch.bool)
    hit[1, :, 4:8] = True
    assert bool(y[1, shape[1] // 2, 5].isnan()) and bool(dx[hit].isnan().all())
    assert torch.equal(y[~hit], clean[0][~hit]) and torch.equal(dx[~hit], cx[0][~hit])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("p", [49, 9000])
def test_group_norm_layouts(p, dtype):
    # a slice of wider pixels, off the 16-byte boundaries, samples apart, a 4-D channels_last tensor, in place:
    # the same values give the same results (bits too where the vector width is the same)
    x, gamma, beta, dy = _norm_case(3, p, 32, 8, dtype, "silu", seed=8)
    y, mean, rstd, dx, dgamma, dbeta = _norm_check(x, 8, gamma, beta, dy, "silu")
    wide = torch.full((3, p + 2, 80), float("nan"), dtype=dtype, device=DEV)
    for start in (16, 3):
        part, dpart = wide[:, 1:p + 1, start:start + 32], wide.clone()[:, 1:p + 1, start:start + 32]
        part.copy_(x)
        dpart.copy_(dy)
        got = _norm_check(part, 8, gamma, beta, dpart, "silu")
        if start == 16:
            for a, b in zip(got, (y, mean, rstd, dx, dgamma, dbeta)):
                assert torch.equal(a, b)
        keep = wide.clone()
        out, _, _ = B.byz_group_norm(part, 8, gamma, beta, act=B.BYZ_ACT_SILU, out=part)
        assert out.data_ptr() == part.data_ptr() and torch.equal(out, got[0])
        keep[:, 1:p + 1, start:start + 32] = out
        assert torch.equal(keep.nan_to_num(), wide.nan_to_num())  # nothing beside the slice was written
        part.copy_(x)
        dout, _, _ = B.byz_group_norm_backward(dpart, part, 8, mean, rstd, gamma, beta, B.BYZ_ACT_SILU, out=dpart)
        assert torch.equal(dout, got[3]) or start == 3
    h, w = (7, 7) if p == 49 else (90, 100)
    img = x.view(3, h, w, 32).permute(0, 3, 1, 2)
    y4, _, _ = B.byz_group_norm(img, 8, gamma, beta, act=B.BYZ_ACT_SILU)
    assert y4.shape == img.shape and y4.is_contiguous(memory_format=torch.channels_last)
    assert torch.equal(y4.permute(0, 2, 3, 1).reshape(3, p, 32), y)


def test_group_norm_images_one_wide():
    gen = _gen(9)
    for shape in ((2, 16, 1, 5), (2, 16, 5, 1), (2, 16, 1, 1), (1, 16, 3, 4), (2, 1, 4, 4)):
        x = _randn(gen, *shape).contiguous(memory_format=torch.channels_last)
        y, _, _ = B.byz_group_norm(x, min(4, shape[1]))
        n, c, h, w = shape
        r = _norm_reference(x.permute(0, 2, 3, 1).reshape(n, h * w, c), min(4, c), None, None, 1e-5, "none")
        _near(y.permute(0, 2, 3, 1).reshape(n, h * w, c), r["y"], E * r["y"].abs() + 64 * E * r["z_scale"], str(shape))


def test_group_norm_empty_and_parameters():
    gamma, beta = torch.ones(16, device=DEV), torch.zeros(16, device=DEV)
    x = torch.empty(0, 9, 16, device=DEV)
    y, mean, rstd = B.byz_group_norm(x, 4, gamma, beta)
    assert y.shape == x.shape and mean.shape == (0, 4)
    dx, dgamma, dbeta = B.byz_group_norm_backward(x, x, 4, mean, rstd, gamma, beta)
    assert dx.shape == x.shape and not bool(dgamma.any()) and not bool(dbeta.any())
    x = torch.empty(3, 0, 16, device=DEV)
    y, mean, rstd = B.byz_group_norm(x, 4, gamma, beta, eps=0.25)
    assert not bool(mean.any()) and torch.equal(rstd, torch.full((3, 4), 2.0, device=DEV))
    _, dgamma, dbeta = B.byz_group_norm_backward(x, x, 4, mean, rstd, gamma, beta)
    assert not bool(dgamma.any()) and not bool(dbeta.any())
    x, gamma, beta, dy = _norm_case(2, 30, 16, 4, F32)
    _, mean, rstd = B.byz_group_norm(x, 4, gamma, beta)
    full = B.byz_group_norm_backward(dy, x, 4, mean, rstd, gamma, beta)
    dx, a, b = B.byz_group_norm_backward(dy, x, 4, mean, rstd, gamma, beta, parameters=False)
    assert a is None and b is None and torch.equal(dx, full[0])


def test_group_norm_more_tiles_than_blocks():
    # over 2^20 samples of one position: the blocks take several each
    n = (1 << 20) + 4099
    x, gamma, beta, dy = _norm_case(n, 1, 8, 2, F32, seed=10)
    _norm_check(x, 2, gamma, beta, dy, "none")


def test_group_norm_offsets_past_32_bits():
    # two samples 2^31 + 64 elements apart
    base = torch.zeros((1 << 31) + 64 + 4 * 64, dtype=BF16, device=DEV)
    x = base.as_strided((2, 4, 64), ((1 << 31) + 64, 64, 1))
    gen = _gen(11)
    x.copy_(_randn(gen, 2, 4, 64))
    y, mean, rstd = B.byz_group_norm(x, 8, out=x.clone())
    got, _, _ = B.byz_group_norm(x, 8, out=x)  # in place: both strides are long
    assert torch.equal(got, y)


# ------------------------------------------------------------------ distillation


def _distill_reference(logits, teacher, index, tau, dloss):
    """(loss, lse, dlogits, scales) in 64 bits."""
    z = logits.double() / tau
    there = index >= 0
    t = torch.where(there, teacher.double() / tau, torch.full_like(teacher, -math.inf, dtype=torch.float64))
    top = t.max(dim=1, keepdim=True).values
    some = top > -math.inf
    e = torch.exp(t - torch.where(some, top, torch.zeros_like(top)))
    total = e.sum(dim=1, keepdim=True)
    p = torch.where(some, e / torch.where(some, total, torch.ones_like(total)), torch.zeros_like(e))
    lse = torch.logsumexp(z, dim=1, keepdim=True)
    at = index.clamp_min(0).long()
    lq = z.gather(1, at) - lse
    terms = torch.where(p > 0, p * (torch.log(p) - lq), torch.zeros_like(p))
    loss = tau * tau * terms.sum(dim=1)
    q = torch.exp(z - lse)
    dense = torch.zeros_like(z).scatter_add_(1, at, p)
    w = torch.where(some, tau * dloss.double()[:, None], torch.zeros_like(top))
    d = torch.where(some, w * (q - dense), torch.zeros_like(q))
    zmax = z.masked_fill(z == -math.inf, 0).abs().amax(dim=1)
    scale_loss = tau * tau * (1 + zmax + lse[:, 0].abs())
    scale_d = w.abs() * (q * (4 + zmax[:, None]) + dense)
    return loss, lse[:, 0], d, scale_loss, scale_d, some[:, 0]


def _distill_case(rows, vocab, k, dtype, seed, empty=True):
    gen = _gen(seed)
    logits = _randn(gen, rows, vocab, dtype=dtype, scale=3.0)
    teacher = _randn(gen, rows, k, scale=3.0)
    index = torch.randint(0, vocab, (rows, k), generator=gen, device=DEV, dtype=torch.int32)  # some places twice
    if empty and rows > 2:
        index[1] = -1
        index[2, k // 2:] = -7
        if k > 1:
            teacher[0, 0] = -math.inf
    dloss = _randn(gen, rows)
    return logits, teacher, index, dloss


def _distill_check(logits, teacher, index, dloss, tau, out=None):
    u = _u(logits.dtype)
    loss, lse = B.byz_distill_loss(logits, teacher, index, tau)
    d = B.byz_distill_loss_backward(dloss, logits, teacher, index, lse, tau)
    loss2, d2 = B.byz_distill_loss_step(logits, teacher, index, dloss, tau, out=out)
    torch.cuda.synchronize()
    want, wlse, wd, sl, sd, some = _distill_reference(logits, teacher, index, tau, dloss)
    tol = 2.0 ** -23 * want.abs() + 16 * E * sl
    _near(loss, want, tol, "loss")
    _near(loss2, want, tol, "loss of the step")
    _near(lse, wlse, 2.0 ** -23 * wlse.abs() + 16 * E * sl / tau ** 2, "lse")
    # and half a step of the type's smallest values: bf16's step there is 2^-133, fp16's 2^-24, fp32's 2^-149 (a whole
    # one allowed)
    tiny = {F32: 2.0 ** -149, BF16: 2.0 ** -134, F16: 2.0 ** -25}[logits.dtype]
    for got, what in ((d, "dlogits"), (d2, "dlogits of the step")):
        _near(got, wd, u * wd.abs() + 32 * E * sd + tiny, what)
    assert not bool(d[~some].any()) and not bool(loss[~some].any())
    return loss, lse, d, loss2, d2


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
@pytest.mark.parametrize("rows,vocab,k", [
    (1, 1, 1), (30, 10, 5), (5, 7, 3), (9, 8, 8), (17, 100, 1), (3, 1000, 1000), (64, 1000, 20), (4, 1024, 1024), (3, 2049, 7),
    (6, 4095, 64), (4, 8193, 300), (5, 16385, 64), (3, 50021, 100), (2, 131072, 64), (2, 131073, 64), (1, 262147, 1024),
    (300, 8200, 16)])
def test_distill_sizes(rows, vocab, k, dtype):
    case = _distill_case(rows, vocab, k, dtype, rows + vocab + k)
    _distill_check(*case, 2.0)


# rows enough for every compute unit and long enough for its registers: the kernel that holds them there
RESIDENT = [(130, 33000, 7), (129, 40001, 20), (257, 65533, 5), (140, 131072, 64), (300, 70001, 1024)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
@pytest.mark.parametrize("rows,vocab,k", RESIDENT)
def test_distill_rows_held_in_registers(rows, vocab, k, dtype):
    logits, teacher, index, dloss = _distill_case(rows, vocab, k, dtype, rows + k)
    _, _, d, _, d2 = _distill_check(logits, teacher, index, dloss, 2.0)
    _, d3 = B.byz_distill_loss_step(logits.clone(), teacher, index, dloss, 2.0)
    assert _same_bits(d2, d3)
    held = logits.clone()  # the gradient over the logits: the next row is loaded while this one is written
    loss, d4 = B.byz_distill_loss_step(held, teacher, index, dloss, 2.0, out=held)
    assert _same_bits(d4, d2)
    wide = torch.full((rows, vocab + 11), 1.0e4, dtype=dtype, device=DEV)  # other alignments, row by row
    part = wide[:, 3:vocab + 3]
    part.copy_(logits)
    out = torch.zeros((rows, vocab + 11), dtype=dtype, device=DEV)
    _, d5 = B.byz_distill_loss_step(part, teacher, index, dloss, 2.0, out=out[:, 3:vocab + 3])
    assert not bool(out[:, :3].any()) and not bool(out[:, vocab + 3:].any())
    _distill_check(part, teacher, index, dloss, 2.0, out=out[:, 3:vocab + 3])


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
def test_distill_rows_held_in_registers_special_values(dtype):
    rows, vocab, k = 140, 40000, 6
    logits, teacher, index, dloss = _distill_case(rows, vocab, k, dtype, 41)
    index = torch.where(index >= 0, index % 20000 + 15000, index)
    clean = B.byz_distill_loss_step(logits, teacher, index, dloss, 1.0)
    # values far above the first ones of every thread, and first values that are all banned
    logits[3, :10000] = -1000.0
    logits[4, :12000] = -math.inf
    logits[5, ::2] = -math.inf
    logits[5].scatter_(0, index[5].clamp_min(0).long(), 1.0)
    logits[6] = (logits[6] + 3.0e4 if dtype == F32 else logits[6] * 64).round()
    _distill_check(logits, teacher, index, dloss, 1.0)
    logits[7, 39999] = math.nan
    logits[8] = -math.inf
    logits[1] = math.nan  # a row without entries
    index[9, 0] = vocab
    logits[10, 17] = math.inf
    loss, d = B.byz_distill_loss_step(logits, teacher, index, dloss, 1.0)
    for row in (7, 8, 9, 10):
        assert bool(loss[row].isnan()) and bool(d[row].isnan().any())
    assert bool(d[[7, 8, 9]].isnan().all())
    assert float(loss[1]) == 0.0 and not bool(d[1].any())
    assert torch.equal(loss[11:], clean[0][11:]) and torch.equal(d[11:], clean[1][11:])
    logits[12, index[12, 0]] = -math.inf  # weight on a banned place
    loss, d = B.byz_distill_loss_step(logits, teacher, index, dloss, 1.0)
    assert float(loss[12]) == math.inf and bool(d[12].isfinite().all())


@pytest.mark.parametrize("tau", [0.1, 1.0, 3.0, 20.0])
@pytest.mark.parametrize("vocab", [10, 20011])
def test_distill_temperatures(vocab, tau):
    _distill_check(*_distill_case(5, vocab, 9, F32, 3), tau)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("vocab", [30, 900, 9001, 70001])
def test_distill_pitches_alignments_and_in_place(vocab, dtype):
    # rows at odd addresses, logits and gradients off the boundaries by different amounts, teacher rows apart
    logits, teacher, index, dloss = _distill_case(7, vocab, 5, dtype, 11)
    _distill_check(logits, teacher, index, dloss, 1.0)
    for off, out_off in ((0, 0), (1, 1), (3, 2), (0, 5)):
        wide = torch.full((7, vocab + 9), 1.0e4, dtype=dtype, device=DEV)
        part = wide[:, off:off + vocab]
        part.copy_(logits)
        wide_out = torch.zeros((7, vocab + 11), dtype=dtype, device=DEV)
        out = wide_out[:, out_off:out_off + vocab]
        tw = torch.zeros((7, 8), device=DEV)
        iw = torch.zeros((7, 8), dtype=torch.int32, device=DEV)
        tw[:, 2:7], iw[:, 2:7] = teacher, index
        got = _distill_check(part, tw[:, 2:7], iw[:, 2:7], dloss, 1.0, out=out)
        assert not bool(wide_out[:, :out_off].any()) and not bool(wide_out[:, out_off + vocab:].any())
        _, d = B.byz_distill_loss_step(part, teacher, index, dloss, 1.0, out=part)  # the gradient over the logits
        assert torch.equal(d, got[4]) and bool((wide[:, :off] == 1.0e4).all()) and bool((wide[:, off + vocab:] == 1.0e4).all())
        part.copy_(logits)
        d = B.byz_distill_loss_backward(dloss, part, teacher, index, got[1], 1.0, out=part)
        assert torch.equal(d, got[2])


@pytest.mark.parametrize("vocab", [40, 3000, 70000])
def test_distill_banned_entries(vocab):
    logits, teacher, index, dloss = _distill_case(6, vocab, 6, F32, 13)
    banned = torch.rand(6, vocab, generator=_gen(14), device=DEV) < 0.6
    banned[:, :20] = True  # whole vectors of nothing at a row's start, and at its end
    banned[:, -9:] = True
    banned.scatter_(1, index.clamp_min(0).long(), False)
    logits.masked_fill_(banned, -math.inf)
    loss, lse, d, _, _ = _distill_check(logits, teacher, index, dloss, 1.0)
    assert not bool(d[banned].any())
    # an entry without weight may be banned, one with weight costs infinitely much
    teacher[4, 2] = -math.inf
    keep = index[4, 2].item()
    if keep >= 0 and (index[4] == keep).sum() == 1:
        logits[4, keep] = -math.inf
        _distill_check(logits, teacher, index, dloss, 1.0)
    logits[5, index[5, 0]] = -math.inf
    loss, _ = B.byz_distill_loss(logits, teacher, index, 1.0)
    assert float(loss[5]) == math.inf and bool(loss[:5].isfinite().all())
    # every entry banned: no distribution is left
    logits[3] = -math.inf
    loss, _ = B.byz_distill_loss(logits, teacher, index, 1.0)
    assert bool(loss[3].isnan()) and bool(loss[:3].isfinite().all()) and bool(loss[4].isfinite())


@pytest.mark.parametrize("dtype", [F32, BF16], ids=str)
@pytest.mark.parametrize("vocab", [40, 3000, 70000])
def test_distill_nan_and_places_outside(vocab, dtype):
    logits, teacher, index, dloss = _distill_case(6, vocab, 6, dtype, 15)
    clean = B.byz_distill_loss_step(logits, teacher, index, dloss, 1.0)
    logits[1] = math.nan                     # a row without entries: whatever its logits are
    index[3, 2] = vocab                      # a place behind the vocabulary
    index[4, 1] = 2 ** 31 - 1
    logits[5, vocab // 2] = math.nan
    loss, d = B.byz_distill_loss_step(logits, teacher, index, dloss, 1.0)
    loss1, lse = B.byz_distill_loss(logits, teacher, index, 1.0)
    d1 = B.byz_distill_loss_backward(dloss, logits, teacher, index, lse, 1.0)
    for got, grad in ((loss, d), (loss1, d1)):
        assert float(got[1]) == 0.0 and not bool(grad[1].any())
        assert bool(got[3:].isnan().all()) and bool(grad[3:].isnan().all())
        assert torch.equal(got[[0, 2]], clean[0][[0, 2]])
    assert torch.equal(d[[0, 2]], clean[1][[0, 2]])


def test_distill_a_vector_of_nan_among_banned():
    # NaN where everything around it is -inf: a thread that sees nothing else must not lose it
    logits = torch.full((1, 4096), -math.inf, device=DEV)
    logits[0, 5] = 1.0
    logits[0, 2000:2004] = math.nan
    loss, lse = B.byz_distill_loss(logits, torch.zeros(1, 1, device=DEV), torch.full((1, 1), 5, dtype=torch.int32, device=DEV))
    assert bool(loss.isnan()) and bool(lse.isnan())


def test_distill_large_logits():
    # far from 0 on either side, and rows of one value
    for shift in (-3.0e4, 3.0e4):
        logits, teacher, index, dloss = _distill_case(4, 5000, 5, F32, 16)
        _distill_check((logits + shift).round(), teacher, index, dloss, 1.0)
    logits, teacher, index, dloss = _distill_case(4, 5000, 5, F32, 17)
    loss, lse, d, _, _ = _distill_check(torch.zeros_like(logits), teacher, index, dloss, 1.0)
    assert torch.allclose(lse, torch.full_like(lse, math.log(5000)))


def test_distill_gradient_against_differences():
    logits, teacher, index, _ = _distill_case(3, 50, 4, F32, 18, empty=False)
    one = torch.ones(3, device=DEV)
    _, d = B.byz_distill_loss_step(logits, teacher, index, one, 2.0)
    step = 2.0 ** -6
    for v in (0, 7, int(index[0, 1]), 49):
        hi, lo = logits.clone(), logits.clone()
        hi[:, v] += step
        lo[:, v] -= step
        diff = (B.byz_distill_loss(hi, teacher, index, 2.0)[0] - B.byz_distill_loss(lo, teacher, index, 2.0)[0]) / (2 * step)
        # third derivative (at most tau^-1) times step^2 / 6, and the losses' rounding over the step
        assert float((diff - d[:, v]).abs().max()) < step ** 2 / 6 + 16 * E * 40 / step


def test_distill_offsets_past_32_bits():
    rows, vocab, pitch = 20, 1000, 1 << 27
    base = torch.zeros((rows - 1) * pitch + vocab, dtype=BF16, device=DEV)
    logits, teacher, index, dloss = _distill_case(rows, vocab, 8, BF16, 19)
    far = base.as_strided((rows, vocab), (pitch, 1))
    far.copy_(logits)
    want = B.byz_distill_loss_step(logits, teacher, index, dloss, 1.0)
    got = B.byz_distill_loss_step(far, teacher, index, dloss, 1.0, out=far)
    assert _same_bits(got[0], want[0]) and _same_bits(got[1], want[1])


# ------------------------------------------------------------------ gated feed-forward


def _ffn_reference(x, wg, wu, act, dh=None):
    x, wg, wu = (t.double().requires_grad_(dh is not None) for t in (x, wg, wu))
    gate, up = x @ wg.t(), x @ wu.t()
    h = _act(gate, act) * up
    r = {"h": h.detach(), "gate": gate.detach(), "up": up.detach()}
    if dh is not None:
        r["dx"], r["dw_gate"], r["dw_up"] = torch.autograd.grad(h, (x, wg, wu), dh.double())
    return r


def _ffn_check(x, wg, wu, act, dh):
    code, u = B.BYZ_ACTS[act], _u(x.dtype)
    h, gate, up = B.byz_gated_ffn(x, wg, wu, code, save=True)
    h1 = B.byz_gated_ffn(x, wg, wu, code)
    dx, dwg, dwu = B.byz_gated_ffn_backward(dh, x, wg, wu, gate, up, code)
    torch.cuda.synchronize()
    assert torch.equal(h, h1)
    r = _ffn_reference(x, wg, wu, act, dh)
    m, k = x.shape
    n = wg.shape[0]
    tiny = 2.0 ** -25 if x.dtype == F16 else 0.0  # half a step of fp16's smallest
    # products: sums of k terms in fp32, in an order that is not this one's
    X, G, U = x.double().abs(), wg.double().abs(), wu.double().abs()
    eg, eu = (k + 8) * E * (X @ G.t()), (k + 8) * E * (X @ U.t())
    _near(gate, r["gate"], eg, "gate")
    _near(up, r["up"], eu, "up")
    a = _act(r["gate"], act).abs()
    # the activations' and their slopes' own slopes are 1.2 at most; exp and its like are good to some 2^-22
    eh = (1.2 * eg + 16 * E * (1 + r["gate"].abs())) * (r["up"].abs() + eu) + eu * (a + eg)
    _near(h, r["h"], u * r["h"].abs() + 1.01 * eh + tiny, "h")
    D = dh.double().abs()
    gate_g = r["gate"].clone().requires_grad_(True)
    slope, = torch.autograd.grad(_act(gate_g, act).sum(), gate_g)
    dg, du = D * r["up"].abs() * slope.abs(), D * a
    # dgate and dup: rounded to the type, off by what gate and up are
    edg = u * dg + D * ((1.2 * eg + 32 * E * (1 + r["gate"].abs())) * (r["up"].abs() + eu) + eu * (slope.abs() + 1)) * 1.01 + tiny
    edu = u * du + D * (1.2 * eg + 16 * E * (1 + r["gate"].abs())) * 1.01 + tiny
    bound = lambda err, val, other, terms: err @ other + (terms + 8) * E * ((val + err) @ other)  # noqa: E731
    _near(dx, r["dx"], u * r["dx"].abs() * 1.01 + 1.01 * (bound(edg, dg, G, 2 * n) + bound(edu, du, U, 2 * n)) + tiny, "dx")
    _near(dwg, r["dw_gate"], u * r["dw_gate"].abs() * 1.01 + 1.01 * bound(edg.t(), dg.t(), X, m) + tiny, "dw_gate")
    _near(dwu, r["dw_up"], u * r["dw_up"].abs() * 1.01 + 1.01 * bound(edu.t(), du.t(), X, m) + tiny, "dw_up")
    return h, gate, up, dx, dwg, dwu


def _ffn_case(m, k, n, dtype, seed):
    gen = _gen(seed)
    return (_randn(gen, m, k, dtype=dtype), _randn(gen, n, k, dtype=dtype, scale=max(k, 1) ** -0.5),
            _randn(gen, n, k, dtype=dtype, scale=max(k, 1) ** -0.5), _randn(gen, m, n, dtype=dtype))


FFN_SIZES = [(1, 1, 1), (1, 64, 16), (1, 2048, 100), (2, 7, 3), (5, 100, 33), (15, 65, 31), (16, 256, 129), (17, 64, 64), (31, 33, 65),
             (64, 128, 128), (65, 72, 130), (100, 1000, 77), (128, 8, 200), (129, 200, 256), (200, 520, 333), (257, 128, 1000),
             (1000, 96, 40), (333, 1000, 131), (24, 3001, 50)]


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("m,k,n", FFN_SIZES)
def test_gated_ffn_sizes(m, k, n, dtype):
    x, wg, wu, dh = _ffn_case(m, k, n, dtype, m + k + n)
    _ffn_check(x, wg, wu, "silu", dh)


@pytest.mark.parametrize("act", sorted(B.BYZ_ACTS))
@pytest.mark.parametrize("m", [3, 150])
def test_gated_ffn_activations(m, act):
    x, wg, wu, dh = _ffn_case(m, 192, 96, BF16, 21)
    if act == "relu":  # gates within rounding of the corner have no one gradient
        near = _ffn_reference(x, wg, wu, act)["gate"].abs() < 1e-5
        dh = dh.masked_fill(near, 0.0)
    _ffn_check(x, wg, wu, act, dh)


@pytest.mark.parametrize("m,k,n", [(2048, 1024, 1536), (2500, 640, 2000), (2049, 257, 3073)])
def test_gated_ffn_large_tiles(m, k, n):
    x, wg, wu, dh = _ffn_case(m, k, n, BF16, 22)
    got = _ffn_check(x, wg, wu, "silu", dh)
    # roundings alone: the result's own, and dgate's and dup's before the products (rms of a rounding is
    # 0.43 of the most it can be; two of them independent: 0.61)
    r = _ffn_reference(x, wg, wu, "silu", dh)
    for t, name in zip(got[3:], ("dx", "dw_gate", "dw_up")):
        assert float((t.double() - r[name]).norm() / r[name].norm()) < 0.7 * _u(BF16), name


@pytest.mark.parametrize("m,k,n", [(1, 40, 50), (9, 100, 33), (40, 65, 100), (300, 100, 260), (130, 129, 515)])
def test_gated_ffn_whole_numbers_exactly(m, k, n):
    # small whole numbers: every product and sum is one, so a value that went to a wrong place shows
    gen = _gen(23)
    x, wg, wu = (torch.randint(-1, 2, s, generator=gen, device=DEV).to(F16) for s in ((m, k), (n, k), (n, k)))
    dh = torch.randint(-1, 2, (m, n), generator=gen, device=DEV).to(F16)
    h, gate, up = B.byz_gated_ffn(x, wg, wu, B.BYZ_ACT_NONE, save=True)
    r = _ffn_reference(x, wg, wu, "none", dh)
    assert torch.equal(gate.double(), r["gate"]) and torch.equal(up.double(), r["up"])
    assert float(r["h"].abs().max()) <= 2048 and torch.equal(h.double(), r["h"])
    got = B.byz_gated_ffn_backward(dh, x, wg, wu, gate, up, B.BYZ_ACT_NONE)
    for t, name in zip(got, ("dx", "dw_gate", "dw_up")):
        fits = r[name].abs() <= 2048
        assert bool(fits.any()) and torch.equal(t.double()[fits], r[name][fits]), name


@pytest.mark.parametrize("m,k,n", [(3, 100, 40), (70, 100, 90), (300, 128, 200)])
def test_gated_ffn_pitches_and_alignments(m, k, n):
    x, wg, wu, dh = _ffn_case(m, k, n, BF16, 24)
    want = _ffn_check(x, wg, wu, "gelu", dh)

    def placed(t, off, more):
        wide = torch.full((t.shape[0], t.shape[1] + more), float("nan"), dtype=t.dtype, device=DEV)
        part = wide[:, off:off + t.shape[1]]
        part.copy_(t)
        return part

    for off, more in ((0, 8), (8, 16), (1, 3), (5, 13)):
        a = [placed(t, off, more) for t in (x, wg, wu, dh)]
        h, gate, up = B.byz_gated_ffn(*a[:3], B.BYZ_ACT_GELU, save=True)
        out = torch.zeros((m, n + 5), dtype=BF16, device=DEV)
        B.byz_gated_ffn(*a[:3], B.BYZ_ACT_GELU, out=out[:, 2:n + 2])
        assert torch.equal(h, want[0]) and torch.equal(out[:, 2:n + 2], h)
        assert not bool(out[:, :2].any()) and not bool(out[:, n + 2:].any())
        gate2, up2 = placed(gate, off, more), placed(up, off, more)
        for g, u in ((gate, up), (gate2, up2)):
            got = B.byz_gated_ffn_backward(a[3], *a[:3], g, u, B.BYZ_ACT_GELU)
            for t, w in zip(got, want[3:]):
                assert torch.equal(t, w)


def test_gated_ffn_empty():
    for m, k, n in ((0, 8, 8), (4, 0, 8), (4, 8, 0), (40, 0, 8), (0, 0, 0)):
        x, wg, wu, dh = _ffn_case(m, k, n, BF16, 25)
        h, gate, up = B.byz_gated_ffn(x, wg, wu, save=True)
        assert h.shape == (m, n) and not bool(h.any())
        dx, dwg, dwu = B.byz_gated_ffn_backward(dh, x, wg, wu, gate, up)
        assert dx.shape == (m, k) and dwg.shape == (n, k) and dwu.shape == (n, k)
        assert not bool(dx.any()) and not bool(dwg.any()) and not bool(dwu.any())


@pytest.mark.parametrize("m", [4, 100])
def test_gated_ffn_infinite_values_stay_in_their_rows(m):
    x, wg, wu, dh = _ffn_case(m, 72, 40, BF16, 26)
    clean = B.byz_gated_ffn(x, wg, wu)
    x2 = x.clone()
    x2[1, 70] = math.nan
    wg2 = wg.clone()
    wg2[39, 71] = math.inf
    h = B.byz_gated_ffn(x2, wg2, wu)
    hit = torch.zeros_like(h, dtype=torch.bool)
    hit[1], hit[:, 39] = True, True
    assert bool(h[1].isnan().all()) and torch.equal(h[~hit], clean[~hit]) and not bool(h[~hit].isnan().any())


@pytest.mark.parametrize("m", [3, 20])
def test_gated_ffn_offsets_past_32_bits(m):
    # rows 2^27 elements apart: the last start past 2^32 elements
    k, n, pitch = 64, 40, 1 << 27
    x, wg, wu, _ = _ffn_case(m, k, n, BF16, 27)
    base = torch.zeros((n - 1) * pitch + k, dtype=BF16, device=DEV)
    far = base.as_strided((n, k), (pitch, 1))
    far.copy_(wg)
    far_up = torch.zeros((n - 1) * pitch + k, dtype=BF16, device=DEV).as_strided((n, k), (pitch, 1))
    far_up.copy_(wu)
    assert torch.equal(B.byz_gated_ffn(x, far, far_up), B.byz_gated_ffn(x, wg, wu))


def test_gated_ffn_gradient_against_differences():
    gen = _gen(28)
    x, wg, wu = (_randn(gen, *s, dtype=F16, scale=0.5) for s in ((4, 8), (6, 8), (6, 8)))
    dh = torch.ones(4, 6, dtype=F16, device=DEV)
    _, gate, up = B.byz_gated_ffn(x, wg, wu, save=True)
    grads = B.byz_gated_ffn_backward(dh, x, wg, wu, gate, up)
    step = 2.0 ** -4

    def total(*a):  # from the fp32 sums, which the call keeps
        _, g, u = B.byz_gated_ffn(*a, save=True)
        return (g.double() * torch.sigmoid(g.double()) * u.double()).sum()

    for which in range(3):
        for at in ((0, 0), (3, 5), (2, 7)):
            lo, hi = [x, wg, wu], [x, wg, wu]
            lo[which], hi[which] = lo[which].clone(), hi[which].clone()
            lo[which][at] -= step
            hi[which][at] += step
            width = float(hi[which][at].double() - lo[which][at].double())
            diff = float(total(*hi) - total(*lo)) / width
            # third derivatives of the sum here are below 20; step^2 / 6 of it, and the gradient's roundings
            assert abs(diff - float(grads[which][at])) < 20 * step ** 2 / 6 + 4 * _u(F16) * 10


# ------------------------------------------------------------------ all three


def _all_three(x, gamma, beta, wg, wu, teacher, index, dloss, dy):
    """Every entry point once, chained -> all outputs."""
    y, mean, rstd = B.byz_group_norm(x, 8, gamma, beta, act=B.BYZ_ACT_SILU)
    rows = y.reshape(-1, y.shape[2])
    h, gate, up = B.byz_gated_ffn(rows, wg, wu, save=True)
    loss, dh = B.byz_distill_loss_step(h, teacher, index, dloss, 2.0)
    loss2, lse = B.byz_distill_loss(h, teacher, index, 2.0)
    dh2 = B.byz_distill_loss_backward(dloss, h, teacher, index, lse, 2.0)
    dr, dwg, dwu = B.byz_gated_ffn_backward(dh, rows, wg, wu, gate, up)
    dx, dgamma, dbeta = B.byz_group_norm_backward(dr.view_as(x) + dy, x, 8, mean, rstd, gamma, beta, B.BYZ_ACT_SILU)
    return [y, mean, rstd, h, gate, up, loss, dh, loss2, lse, dh2, dr, dwg, dwu, dx, dgamma, dbeta]


def _all_three_inputs(n, p, c, vocab, seed):
    gen = _gen(seed)
    m = n * p
    return [_randn(gen, n, p, c, dtype=BF16), 1 + _randn(gen, c, scale=0.1), _randn(gen, c, scale=0.1),
            _randn(gen, vocab, c, dtype=BF16, scale=c ** -0.5), _randn(gen, vocab, c, dtype=BF16, scale=c ** -0.5),
            _randn(gen, m, 6, scale=3.0), torch.randint(-1, vocab, (m, 6), generator=gen, device=DEV, dtype=torch.int32),
            torch.rand(m, generator=gen, device=DEV) / m, _randn(gen, n, p, c, dtype=BF16, scale=0.01)]


CHAINS = [(2, 4, 64, 200), (3, 100, 64, 1000), (1, 9000, 32, 520)]


@pytest.mark.parametrize("sizes", CHAINS, ids=str)
def test_the_same_bits_every_time_and_in_a_graph(sizes):
    inputs = [_all_three_inputs(*sizes, seed) for seed in (31, 32)]
    want = [_all_three(*i) for i in inputs]
    for i, w in zip(inputs, want):
        assert all(torch.equal(a, b) for a, b in zip(_all_three(*i), w))
    held = [t.clone() for t in inputs[0]]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _all_three(*held)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _all_three(*held)
    for which in (0, 1, 1, 0):
        for t, v in zip(held, inputs[which]):
            t.copy_(v)
        graph.replay()
        torch.cuda.synchronize()
        for j, (a, b) in enumerate(zip(got, want[which])):
            assert torch.equal(a, b), (which, j)
        eager = _all_three(*inputs[1 - which])  # eager work between the replays
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(eager, want[1 - which]))


def test_on_another_stream():
    inputs = _all_three_inputs(3, 100, 64, 1000, 33)
    x, gamma, beta, wg, wu, teacher, index, dloss, dy = inputs
    want = _all_three(*inputs)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    for stream in (side, side.cuda_stream):
        y, mean, rstd = B.byz_group_norm(x, 8, gamma, beta, act=B.BYZ_ACT_SILU, stream=stream)
        rows = y.reshape(-1, 64)
        h, gate, up = B.byz_gated_ffn(rows, wg, wu, save=True, stream=stream)
        loss, dh = B.byz_distill_loss_step(h, teacher, index, dloss, 2.0, stream=stream)
        loss2, lse = B.byz_distill_loss(h, teacher, index, 2.0, stream=stream)
        dh2 = B.byz_distill_loss_backward(dloss, h, teacher, index, lse, 2.0, stream=stream)
        dr, dwg, dwu = B.byz_gated_ffn_backward(dh, rows, wg, wu, gate, up, stream=stream)
        with torch.cuda.stream(side):
            dn = dr.view_as(x) + dy
        dx, dgamma, dbeta = B.byz_group_norm_backward(dn, x, 8, mean, rstd, gamma, beta, B.BYZ_ACT_SILU, stream=stream)
        torch.cuda.current_stream().wait_stream(side)
        got = [y, mean, rstd, h, gate, up, loss, dh, loss2, lse, dh2, dr, dwg, dwu, dx, dgamma, dbeta]
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        torch.cuda.synchronize()


def test_binding_refusals_on_the_gpu():
    x = torch.zeros(2, 9, 16, device=DEV)
    with pytest.raises(ValueError, match="gamma"):
        B.byz_group_norm(x, 4, torch.ones(15, device=DEV))
    with pytest.raises(ValueError, match="gamma"):
        B.byz_group_norm(x, 4, torch.ones(16, device=DEV).half())
    with pytest.raises(ValueError, match="gamma"):
        B.byz_group_norm(x, 4, torch.ones(32, device=DEV)[::2])
    with pytest.raises(ValueError, match="beta must be a CUDA"):
        B.byz_group_norm(x, 4, None, torch.ones(16))
    with pytest.raises(ValueError, match="dtype"):
        B.byz_group_norm(x.double(), 4)
    with pytest.raises(B.ByzError):
        B.byz_group_norm(x, 5)
    with pytest.raises(ValueError, match="out"):
        B.byz_group_norm(x, 4, out=x[:1])
    _, mean, rstd = B.byz_group_norm(x, 4)
    with pytest.raises(ValueError, match="mean"):
        B.byz_group_norm_backward(x, x, 4, mean[:1], rstd)
    with pytest.raises(ValueError, match="dy"):
        B.byz_group_norm_backward(x[:, :3], x, 4, mean, rstd)
    logits, t, i = torch.zeros(2, 8, device=DEV), torch.zeros(2, 3, device=DEV), torch.zeros(2, 3, dtype=torch.int32, device=DEV)
    with pytest.raises(ValueError, match="dloss"):
        B.byz_distill_loss_step(logits, t, i, torch.ones(3, device=DEV))
    with pytest.raises(ValueError, match="out"):
        B.byz_distill_loss_step(logits, t, i, torch.ones(2, device=DEV), out=logits.half())
    with pytest.raises(B.ByzError):
        B.byz_distill_loss(logits, t, i, temperature=0.0)
    w = torch.zeros(4, 8, device=DEV)
    with pytest.raises(B.ByzError) as e:
        B.byz_gated_ffn(w, w, w)
    assert e.value.code == -2
    w = w.bfloat16()
    _, gate, up = B.byz_gated_ffn(w, w, w, save=True)
    with pytest.raises(ValueError, match="dh"):
        B.byz_gated_ffn_backward(w, w, w, w, gate, up)
    with pytest.raises(ValueError, match="gate"):
        B.byz_gated_ffn_backward(torch.zeros(4, 4, device=DEV, dtype=BF16), w, w, w, gate.bfloat16(), up)
