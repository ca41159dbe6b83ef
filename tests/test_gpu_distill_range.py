"""Distillation at the ends of the logits' range: sums next to the border of fp32, banned entries at any temperature, rows
far from 0, rows of the types' extreme values.

The reference is test_gpu_worker's, in 64 bits, on logits less their row's maximum (loss and gradient do not change by that).
Its tolerances go by the values' distances from the maximum then, not by their size, and by 200 temperatures of them at
most: what lies lower weighs nothing.
"""
import math

import pytest
import torch

import paper_2010_04902_amd as B
from test_gpu_worker import BF16, DEV, E, F16, F32, _distill_case, _distill_check, _distill_reference, _near, _same_bits, _u

pytestmark = pytest.mark.gpu

TINY = {F32: 2.0 ** -149, BF16: 2.0 ** -134, F16: 2.0 ** -25}


def _shifted_reference(logits, teacher, index, tau, dloss):
    z = logits.double()
    z = z - z.amax(dim=1, keepdim=True)
    loss, lse, d, _, _, some = _distill_reference(z, teacher, index, tau, dloss)
    near = _distill_reference(z.clamp_min(-200.0 * tau), teacher, index, tau, dloss)
    return loss, lse, d, near[3], near[4], some


def _check_gradient(got, ref, dtype, what, more=0.0):
    _, _, want, _, scale, _ = ref
    _near(got, want, _u(dtype) * want.abs() + (32 + more) * E * scale + TINY[dtype], what)


def _check_loss(got, ref, what):
    want, _, _, scale, _, _ = ref
    _near(got, want, 2.0 ** -23 * want.abs() + 16 * E * scale, what)


# ------------------------------------------------------------------ sums of rows held in registers


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
@pytest.mark.parametrize("vocab", [40000, 65536, 131072])
def test_rows_that_start_far_below_their_rest(vocab, dtype):
    # the first 16 KB of a row, every thread's first values, lie so far below the others that a thread's sum in fp32, or the
    # row's of 1024 such sums, reaches fp32's end
    if dtype == F32 and vocab > 65536:
        vocab = 61440
    gaps = [0.0, 60.0, 69.0, 70.0, 76.0, 77.0, 77.5, 78.0, 78.5, 79.0, 83.0, 88.0, 100.0]
    logits, teacher, index, dloss = _distill_case(130, vocab, 7, dtype, vocab)
    logits.zero_()
    first = 16384 // logits.element_size()
    for i, gap in enumerate(gaps):
        logits[i::len(gaps), first:] = gap
    loss, lse, _, loss2, d2 = _distill_check(logits, teacher, index, dloss, 1.0)
    assert bool(loss2.isfinite().all()) and bool(d2.isfinite().all())


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
@pytest.mark.parametrize("vocab", [40000, 65536, 131072])
def test_threads_whose_first_values_lie_far_apart(vocab, dtype):
    # all threads but one start at 0 and have 78 next: their sums of e^78 count beside the one that starts at 84 to 90, although
    # e^-87.4, what lies between their references, is 0 in fp32
    if dtype == F32 and vocab > 65536:
        vocab = 61440
    logits, teacher, index, dloss = _distill_case(130, vocab, 7, dtype, vocab)
    logits.zero_()
    first = 16384 // logits.element_size()
    logits[:, first:2 * first] = 78.0
    for i, high in enumerate((84.0, 86.0, 87.0, 87.5, 88.0, 90.0)):
        logits[i::6, first // 2] = high
    _distill_check(logits, teacher, index, dloss, 1.0)


# ------------------------------------------------------------------ banned entries


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
@pytest.mark.parametrize("tau", [0.1, 0.7, 1.0, 3.0, 10.0])
@pytest.mark.parametrize("rows,vocab", [(6, 40), (5, 3000), (4, 9000), (3, 70000), (1030, 20011), (130, 40000)])
def test_banned_entries_at_any_temperature(rows, vocab, tau, dtype):
    # log2(e) / temperature is rounded to fp32 upwards for some of these temperatures and downwards for others
    logits, teacher, index, dloss = _distill_case(rows, vocab, 6, dtype, vocab + rows)
    banned = torch.rand(rows, vocab, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV) < 0.4
    banned.scatter_(1, index.clamp_min(0).long(), False)
    logits.masked_fill_(banned, -math.inf)
    _, _, d, _, d2 = _distill_check(logits, teacher, index, dloss, tau)
    assert not bool(d[banned].any()) and not bool(d2[banned].any())


# ------------------------------------------------------------------ rows far from 0


def _far_case(rows, vocab, dtype, seed):
    """Rows around many values, those of 16 bits with the few different ones that the type has there."""
    logits, teacher, index, dloss = _distill_case(rows, vocab, 6, dtype, seed)
    most = 6.0e4 if dtype == F16 else 3.0e5
    shift = torch.tensor([0.0, 300.0, -300.0, 4.0e3, -4.0e3, 3.0e4, -3.0e4, most, -most], device=DEV)
    shift = shift[torch.arange(rows, device=DEV) % 9].unsqueeze(1)
    return (logits.float() + shift).to(dtype), teacher, index, dloss


FAR = [(9, 40), (9, 3000), (9, 9000), (9, 70000), (1030, 20011), (130, 40000), (130, 65536)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
@pytest.mark.parametrize("tau", [0.5, 1.0, 3.0])
@pytest.mark.parametrize("rows,vocab", FAR)
def test_rows_far_from_zero(rows, vocab, tau, dtype):
    logits, teacher, index, dloss = _far_case(rows, vocab, dtype, vocab)
    ref = _shifted_reference(logits, teacher, index, tau, dloss)
    loss, d = B.byz_distill_loss_step(logits, teacher, index, dloss, tau)
    _check_loss(loss, ref, "loss of the step")
    _check_gradient(d, ref, dtype, "dlogits of the step")
    loss, lse = B.byz_distill_loss(logits, teacher, index, tau)
    _check_loss(loss, ref, "loss")


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("base", [0.0, 2.0e4, -6.0e4])
def test_rows_held_in_registers_that_are_far_from_zero_and_start_below_their_rest(base, dtype):
    # sums taken again with a maximum, next to ones that were not, with rounded products of either
    logits, teacher, index, dloss = _distill_case(130, 40000, 6, dtype, 51)
    logits = (logits.float() + base).to(dtype)
    logits[:, :8192] -= 1024.0
    logits[5:20, ::3] = base
    ref = _shifted_reference(logits, teacher, index, 1.0, dloss)
    loss, d = B.byz_distill_loss_step(logits, teacher, index, dloss, 1.0)
    _check_loss(loss, ref, "loss")
    _check_gradient(d, ref, dtype, "dlogits")


# ------------------------------------------------------------------ rows of extreme values


def _extreme_case(rows, vocab, dtype):
    """Rows that a mask has filled with a value far below all others, or with the type's lowest, wholly or but for a few."""
    logits, teacher, index, dloss = _distill_case(rows, vocab, 6, dtype, 61)
    index = torch.where(index >= 0, index % vocab, index)
    info = torch.finfo(dtype)
    values = [info.min, info.max, info.min / 2] + ([-6.0e4] if dtype == F16 else [-1.0e9, -3.0e9, -1.0e30, 1.0e20, -1.0e38])
    at = 3
    for value in values:
        if at + 3 > rows:
            break
        logits[at] = value                      # nothing is left: all entries alike
        logits[at + 1, ::2] = value             # half of it
        logits[at + 2] = value                  # all but the teacher's places
        logits[at + 2].scatter_(0, index[at + 2].clamp_min(0).long(), 2.0)
        at += 3
    return logits, teacher, index, dloss


EXTREME = [(30, 40), (30, 3000), (30, 9000), (30, 70000), (1030, 20011), (130, 40000), (130, 65536)]


def _extreme_rows(logits, index):
    """Rows whose teacher's places are no further than 200 from the row's maximum, as far as the reference goes."""
    z = logits.double()
    near = z.gather(1, index.clamp_min(0).long()) >= z.amax(dim=1, keepdim=True) - 200.0
    return (near | (index < 0)).all(dim=1)


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
@pytest.mark.parametrize("rows,vocab", EXTREME)
def test_rows_of_extreme_values(rows, vocab, dtype):
    logits, teacher, index, dloss = _extreme_case(rows, vocab, dtype)
    keep = _extreme_rows(logits, index)
    assert int(keep.sum()) > 8
    for tau in (1.0, 2.0):
        ref = [r[keep] for r in _shifted_reference(logits, teacher, index, tau, dloss)]
        loss, lse = B.byz_distill_loss(logits, teacher, index, tau)
        _check_loss(loss[keep], ref, "loss")
        assert not bool(lse.isnan().any())
        loss, d = B.byz_distill_loss_step(logits, teacher, index, dloss, tau)
        _check_loss(loss[keep], ref, "loss of the step")
        _check_gradient(d[keep], ref, dtype, "dlogits of the step")
        assert bool(d.isfinite().all())  # of the others the gradient, too, is less than the weight
        held = logits.clone()
        loss3, d3 = B.byz_distill_loss_step(held, teacher, index, dloss, tau, out=held)
        assert _same_bits(loss3, loss) and _same_bits(d3, d)


# ------------------------------------------------------------------ the gradient by its own call

# It has the row's log-sum-exp in fp32: half a step of that is 2^-24 of 64 at most where it is used, 64 E of q.  Larger ones are
# not used.


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
@pytest.mark.parametrize("tau", [0.5, 1.0, 3.0])
@pytest.mark.parametrize("rows,vocab", FAR)
def test_gradient_of_rows_far_from_zero(rows, vocab, tau, dtype):
    logits, teacher, index, dloss = _far_case(rows, vocab, dtype, vocab)
    ref = _shifted_reference(logits, teacher, index, tau, dloss)
    _, lse = B.byz_distill_loss(logits, teacher, index, tau)
    d = B.byz_distill_loss_backward(dloss, logits, teacher, index, lse, tau)
    _check_gradient(d, ref, dtype, "dlogits", more=64)


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
@pytest.mark.parametrize("rows,vocab", EXTREME)
def test_gradient_of_rows_of_extreme_values(rows, vocab, dtype):
    logits, teacher, index, dloss = _extreme_case(rows, vocab, dtype)
    keep = _extreme_rows(logits, index)
    for tau in (0.5, 2.0):
        ref = [r[keep] for r in _shifted_reference(logits, teacher, index, tau, dloss)]
        _, lse = B.byz_distill_loss(logits, teacher, index, tau)
        d = B.byz_distill_loss_backward(dloss, logits, teacher, index, lse, tau)
        _check_gradient(d[keep], ref, dtype, "dlogits", more=64)
        assert bool(d.isfinite().all())
        held = logits.clone()
        assert _same_bits(B.byz_distill_loss_backward(dloss, held, teacher, index, lse, tau, out=held), d)
