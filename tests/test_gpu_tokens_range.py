"""The token operators at the ends of their values' range: dropped values that are no numbers, the statistics of rows whose largest
values lie anywhere, many small terms beside a large one, ratios next to the clipping's ends, banned tokens."""
import math

import pytest
import torch

import paper_2010_04902_amd as B
from test_gpu_tokens import DEV, F16, TYPES, _gen, _near, _randn, _residual_case, _residual_check, _residual_run, _residual_want, _same_bits, _u
from token_forms import E, kept, logp_terms

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows, cols, gate", [(8, 5, 1), (8, 64, 1), (40, 1000, 8), (8, 4104, 8), (24, 4104, 2), (9, 9000, 1), (9, 9000, 3),
                                              (6, 20000, 1)])
def test_dropped_values_reach_no_gradient(rows, cols, gate, dtype):
    """Without a norm of h, whatever lies where the mask drops gives the bits of any other value there, in every result."""
    for pre in ("none", "rms", "layer"):
        for bias in (False, True):
            c = _residual_case(rows, cols, dtype, "none", pre, gate, 0.5, bias=bias, seed=cols)
            want = _residual_run(c)
            mask = kept(rows, cols, 0.5, 99, cols).to(DEV)
            h = c["h"]
            for value in (math.inf, -math.inf, math.nan):
                c["h"] = torch.where(mask, h, value)
                got = _residual_run(c)
                assert got.keys() == want.keys() and "d_post_weight" in got
                for name in want:
                    assert _same_bits(got[name], want[name]), (pre, bias, value, name)


# ------------------------------------------------------------------ rows of losses

# one vocabulary at least for each way of holding a row of each type, and those beside it
HELD = [(1, 1), (3, 5), (5, 100), (6, 900), (9, 2047), (7, 4100), (5, 8192), (3, 9001), (6, 20011), (40, 32000), (4, 50021), (130, 33000),
        (130, 66001), (3, 140001)]


def _sum_tol(vocab, dtype):
    """A sum of exponentials, relative: a thread has vocab / (256 V) vectors of V values at most, each of whose sums is rounded once
    beside the thread's; 7 roundings within a vector, 3 at each of 10 joins of threads, 3 of a power, 8 of the logarithm."""
    return (vocab / (256 * 128 / torch.finfo(dtype).bits) + 48) * E


def _stats_check(stats, z, label, temperature):
    """The row's largest logit is one of its values, so exactly that."""
    d = z.double()
    top = d.amax(1)
    total = ((d - top[:, None]) / temperature).exp().sum(1).log()
    none = label < 0
    _near(stats[:, 0], torch.where(none, 0.0, top), torch.zeros_like(top), "largest logit")
    _near(stats[:, 1], torch.where(none, 0.0, total), _sum_tol(z.shape[1], z.dtype) + 2 * E * total, "log-sum")


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows, vocab", HELD)
def test_statistics_are_those_of_the_row(rows, vocab, dtype):
    z = _randn(_gen(vocab), rows, vocab, dtype=dtype, scale=3.0)
    label = torch.arange(rows, dtype=torch.int32, device=DEV) * 7 % vocab
    if rows > 2:
        label[1] = -1
    zeros = torch.zeros(rows, device=DEV)
    bounds = torch.tensor([0, rows // 2, rows], dtype=torch.int32, device=DEV)
    for temperature in (1.0, 0.7):
        _stats_check(B.byz_token_logp(z, label, temperature)[1], z, label, temperature)
        _stats_check(B.byz_policy_loss(z, label, zeros, zeros, temperature=temperature)[2], z, label, temperature)
        _stats_check(B.byz_preference_loss(z, label, bounds, temperature=temperature)[3], z, label, temperature)


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows, vocab", HELD)
def test_a_large_value_anywhere(rows, vocab, dtype):
    """A label far above the rest, wherever it lies: at 40 and more the rest does not reach the sum's last bit, so the sum is
    exactly 1, logp is off by one rounding of the sum at most, and the gradient by that and its exponents' rounding."""
    gen = _gen(vocab)
    rest = _randn(gen, rows, vocab, scale=0.5)
    places = torch.tensor([vocab - 1, vocab // 2, 0, vocab - 9, 3 * vocab // 4, vocab - 2, vocab // 3], device=DEV).clamp_min(0)
    at = places[torch.arange(rows, device=DEV) % len(places)]
    label = at.to(torch.int32)
    every = torch.arange(rows, device=DEV)
    d = _randn(gen, rows)
    for peak in (44.0, 60.0, 84.0, 120.0):
        z = rest.clone()
        z[every, at] = peak
        z = z.to(dtype)
        want, q, hot = logp_terms(z, label, 1.0)
        logp, stats = B.byz_token_logp(z, label)
        assert torch.equal(stats[:, 0], z[every, at].float())
        tol = torch.full_like(want, E)
        _near(logp, want, tol, "logp")
        w = d.double()
        full = w[:, None] * (hot - q)
        q_log = torch.where(q > 0, -q.clamp_min(1e-300).log(), 0.0)
        # of the rest: exponents of up to q_log log2(e), rounded three times, and the power's own error
        near = _u(dtype) * full.abs() + E * w.abs()[:, None] * torch.where(hot > 0, 4.0, q * (16 + 4 * q_log))
        near += torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
        _near(B.byz_token_logp_backward(d, z, label, stats), full, near, "dlogits")
        # the step at advantage -1 and old 0: its ratio is exp(logp), so 1
        zeros = torch.zeros(rows, device=DEV)
        loss, logp2, grad = B.byz_policy_loss_step(z, label, zeros, zeros - 1, d, clip_low=1.0)
        _near(logp2, want, tol, "logp of the step")
        _near(loss, want.exp(), 4 * tol, "loss of the step")
        _near(grad, full, near + 4 * E * full.abs(), "dlogits of the step")


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows, vocab", [(12, 40), (12, 700), (12, 3001), (12, 8192), (12, 20011), (12, 30000), (140, 33000), (140, 66001)])
def test_rows_with_what_is_no_number(rows, vocab, dtype):
    """NaN or +inf anywhere makes a row's log-probability and gradient NaN; banned entries anywhere weigh nothing; others stay."""
    gen = _gen(rows + vocab)
    z, label = _randn(gen, rows, vocab, dtype=dtype), torch.full((rows,), 17, dtype=torch.int32, device=DEV)
    clean = z.clone()
    for row, (place, value) in enumerate(((0, math.nan), (vocab - 1, math.nan), (vocab // 2, math.nan), (5, math.inf), (vocab - 3, math.inf))):
        z[row, place] = value
    z[5, :16] = z[5, 19:] = -math.inf
    z[6, 24:] = -math.inf  # whole threads and waves have nothing
    z[7, :17] = -math.inf
    z[8] = -math.inf
    z[9] = -math.nan
    ones, old = torch.ones(rows, device=DEV), torch.full((rows,), -9.0, device=DEV)
    logp, stats = B.byz_token_logp(z, label)
    loss, logp2, grad = B.byz_policy_loss_step(z, label, old, -ones, ones, clip_low=1.0)
    alone = B.byz_policy_loss_backward(ones, z, label, old, -ones, stats, clip_low=1.0)
    bad = [0, 1, 2, 3, 4, 9]
    for t in (logp, logp2, loss):
        assert bool(t[bad].isnan().all()) and not bool(t[[5, 6, 7, 8, 10, 11]].isnan().any())
    for t in (grad, alone):
        assert bool(t[bad].isnan().all()) and not bool(t[[5, 6, 7, 10, 11]].isnan().any())
        assert bool((t[8] == 0).all())  # a ratio of 0
        assert bool((t[5, :16] == 0).all() and (t[6, 24:] == 0).all() and (t[7, :17] == 0).all())
    assert logp[8] == -math.inf and logp2[8] == -math.inf
    want, _, _ = logp_terms(z[[5, 6, 7]], label[:3], 1.0)
    _near(logp[[5, 6, 7]], want, _sum_tol(vocab, dtype) + 2 * E * want.abs(), "logp")
    _near(logp2[[5, 6, 7]], want, _sum_tol(vocab, dtype) + 2 * E * want.abs(), "logp of the step")
    same, _ = B.byz_token_logp(clean, label)
    assert _same_bits(logp[10:], same[10:])


# ------------------------------------------------------------------ the policy loss at its ends


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows, vocab", [(140, 500), (140, 20011), (140, 50001), (140, 66001), (140, 140000)])
def test_ratios_next_to_the_clippings_ends(rows, vocab, dtype):
    """The step's gradient is clipped where the ratio is past the bound, also if it is so by 2e-5 and the log-probability some
    thousand: the sum's error of some 2^-20 at most is what may decide otherwise."""
    gen = _gen(vocab)
    z = _randn(gen, rows, vocab)
    label = torch.randint(0, vocab, (rows,), generator=gen, device=DEV).to(torch.int32)
    z[torch.arange(rows, device=DEV), label.long()] = -3008.0  # a number of every type
    z = z.to(dtype)
    logp, _, _ = logp_terms(z, label, 1.0)
    ones = torch.ones(rows, device=DEV)
    for sign, clip_low, clip_high in ((1.0, 0.2, 0.28), (-1.0, 0.2, 0.28)):
        low, high = (float(torch.tensor(1.0) + s * torch.tensor(c)) for s, c in ((-1, clip_low), (1, clip_high)))
        bound = high if sign > 0 else low
        old = (logp - math.log(bound)).float()
        away = ((logp - old.double()).exp() - bound) * sign  # more than 0: clipped
        clear = away.abs() > 2e-5
        assert int(clear.sum()) > rows // 2 and bool((away[clear] > 0).any()) and bool((away[clear] < 0).any())
        _, _, grad = B.byz_policy_loss_step(z, label, old, sign * ones, ones, clip_low=clip_low, clip_high=clip_high)
        clipped = (grad == 0).all(dim=1)
        assert torch.equal(clipped[clear], (away > 0)[clear])


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows, vocab", [(140, 30), (140, 9001), (140, 50001), (140, 66001), (130, 140001)])
def test_policy_loss_at_its_ends_of_long_rows(rows, vocab, dtype):
    """Ratios of exactly 0 and infinity, advantages of 0, banned labels, labels that are none, in every kernel."""
    z = torch.zeros(rows, vocab, dtype=dtype, device=DEV)
    label = torch.arange(rows, dtype=torch.int32, device=DEV) % 16
    z[3, 3] = -math.inf  # its token is banned
    z[4] = -math.inf  # nothing is left
    z[5] = math.nan
    label[5] = -1
    label[6] = vocab
    old = torch.full((rows,), -math.log(vocab), device=DEV)
    old[0] = math.inf  # ratio 0
    old[1] = -math.inf  # ratio infinite
    advantage = torch.ones(rows, device=DEV)
    advantage[2], advantage[7] = 0.0, -1.0
    dloss = torch.ones(rows, device=DEV)
    loss, logp, stats = B.byz_policy_loss(z, label, old, advantage)
    loss2, logp2, step = B.byz_policy_loss_step(z, label, old, advantage, dloss)
    alone = B.byz_policy_loss_backward(dloss, z, label, old, advantage, stats)
    want = torch.full((rows,), -1.0, dtype=torch.float64)
    want[:8] = torch.tensor([0.0, -1.2, 0.0, 0.0, 0.0, 0.0, math.nan, 1.0], dtype=torch.float64)
    # a sum of equal terms, its logarithm and old's rounding
    for got in (loss, loss2):
        _near(got, want, torch.full_like(want, (64 + 4 * math.log(vocab)) * E), "loss")
    for got in (logp, logp2):
        assert got[3] == -math.inf and got[4] == -math.inf and got[5] == 0 and bool(got[6].isnan())
    for grad in (step, alone):
        assert bool((grad[:6] == 0).all()) and bool(grad[6].isnan().all())
        each = grad[8:].double().cpu()
        hot = torch.zeros_like(each)
        hot[torch.arange(rows - 8), label[8:].long().cpu()] = 1
        full = 1 / vocab - hot
        _near(each, full, _u(dtype) * full.abs() + (256 + 8 * math.log(vocab)) * E * (hot + 1 / vocab) + 2.0 ** -24 * (dtype == F16), "dlogits")


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows, vocab", [(140, 30), (140, 9001), (140, 50001), (140, 66001), (130, 140001)])
def test_a_token_that_the_reference_bans(rows, vocab, dtype):
    """ref = -inf: an infinite loss whose gradient is kl (onehot - q), -kl (exp(g) - 1) being kl; and a banned token's loss is infinite."""
    gen = _gen(vocab)
    z = _randn(gen, rows, vocab, dtype=dtype)
    label = torch.randint(0, vocab, (rows,), generator=gen, device=DEV).to(torch.int32)
    z[0, label[0].long()] = -math.inf
    _, q, hot = logp_terms(z, label, 1.0)
    ref = torch.full((rows,), -math.inf, device=DEV)
    ref[0] = -1.0
    zeros, ones = torch.zeros(rows, device=DEV), torch.ones(rows, device=DEV)
    terms = {"ref": ref, "kl": 0.25}
    loss, _, stats = B.byz_policy_loss(z, label, zeros, zeros, **terms)
    loss2, _, step = B.byz_policy_loss_step(z, label, zeros, zeros, ones, **terms)
    assert bool((loss == math.inf).all()) and bool((loss2 == math.inf).all())
    alone = B.byz_policy_loss_backward(ones, z, label, zeros, zeros, stats, **terms)
    full = 0.25 * (hot - q)[1:]
    q_log = -q[1:].clamp_min(1e-300).log()
    tol = _u(dtype) * full.abs() + E * (128 * q[1:] + 4 * q[1:] * q_log + 8 * hot[1:]) + 2.0 ** -24 * (dtype == F16)
    for grad in (step, alone):
        _near(grad[1:], full, tol, "dlogits")


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows, vocab", [(130, 200003), (2, 200003), (130, 20011)])
def test_many_small_terms_next_to_a_large_one(rows, vocab, dtype):
    """256 vectors of 16 bytes start with a 1, all else terms that are each just under half of its last bit: they count."""
    V = 128 // torch.finfo(dtype).bits
    z = torch.full((rows, vocab), -16.75, dtype=dtype, device=DEV)
    z[:, :256 * V:V] = 0.0
    label = torch.arange(rows, dtype=torch.int32, device=DEV)
    want, _, _ = logp_terms(z, label, 1.0)
    _near(B.byz_token_logp(z, label)[0], want, _sum_tol(vocab, dtype) + 2 * E * want.abs(), "logp")
    _, lse = B.byz_distill_loss(z, torch.zeros(rows, 1, device=DEV), label[:, None].contiguous())
    want = z.double().logsumexp(1)
    _near(lse, want, _sum_tol(vocab, dtype) + 2 * E * want.abs(), "log-sum of distillation")


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows, vocab", [(6, 300), (5, 9001), (4, 50021), (130, 66001)])
def test_extreme_temperatures(rows, vocab, dtype):
    """The coldest leaves the largest logit alone, the hottest makes all alike that are not banned."""
    gen = _gen(vocab)
    z = _randn(gen, rows, vocab)
    z = z.masked_fill(torch.rand(rows, vocab, generator=gen, device=DEV) < 0.2, -math.inf)
    label = torch.randint(0, vocab, (rows,), generator=gen, device=DEV).to(torch.int32)
    z[torch.arange(rows, device=DEV), label.long()] = 20.0
    z = z.to(dtype)
    d = torch.rand(rows, generator=gen, device=DEV) + 0.5
    for temperature in (2.0 ** -64, 2.0 ** 64):
        want, q, hot = logp_terms(z, label, temperature)
        old = want.float()
        logp, stats = B.byz_token_logp(z, label, temperature)
        _, logp2, step = B.byz_policy_loss_step(z, label, old, -torch.ones(rows, device=DEV), d, clip_low=1.0, temperature=temperature)
        alone = B.byz_token_logp_backward(d, z, label, stats, temperature)
        for got in (logp, logp2):
            _near(got, want, (0.0 if temperature < 1 else _sum_tol(vocab, dtype)) + 2 * E * want.abs(), "logp")
        if temperature < 1:
            assert bool((alone == 0).all()) and bool((step == 0).all())
            continue
        w = d.double()[:, None] / temperature
        full = w * (hot - q)
        # q's exponents have some 20 units, of which 2^-20 is rounding; the step's ratio has that of logp and old
        tol = _u(dtype) * full.abs() + w * (q + hot) * 2.0 ** -17 + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
        _near(alone, full, tol, "dlogits")
        _near(step, full, tol, "dlogits of the step")


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows, cols, gate", [(1100, 8200, 550), (1030, 9001, 1)])
def test_wide_rows_in_turn_with_layer_norms(rows, cols, gate, dtype):
    """More rows than there are blocks, so that a block takes a second and a third one."""
    c = _residual_case(rows, cols, dtype, "layer", "layer", gate, 0.1, bias=True, seed=rows)
    want = _residual_want(c, "layer", "layer", 0.1)
    _residual_check(_residual_run(c), want, dtype)
