"""Results do not depend on where their tensors lie: the same values at other addresses and pitches give the same bits, which
is what a vote over the copies of a file's gradient needs of workers that hold the file in other places."""
import pytest
import torch

import paper_2010_04902_amd as B
from test_gpu_worker import BF16, DEV, F16, F32, _distill_case, _norm_case, _same_bits

pytestmark = pytest.mark.gpu


def _placed(t, offset, more):
    """t's values, `offset` elements behind a 16-byte boundary, in rows `more` elements longer; what surrounds them is NaN."""
    wide = torch.full((t.shape[:-1].numel() * (t.shape[-1] + more) + offset + 64,), float("nan"), dtype=t.dtype, device=DEV)
    stride = [t.shape[-1] + more, 1]
    for n in reversed(t.shape[1:-1]):
        stride.insert(0, stride[0] * n)
    part = wide.as_strided(t.shape, stride, offset)
    part.copy_(t)
    return part, wide


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
@pytest.mark.parametrize("rows,vocab,k", [
    (5, 3, 2), (6, 10, 5), (7, 1001, 5), (5, 2049, 70), (4, 8191, 300), (9, 12345, 6), (3, 50021, 7), (1030, 20011, 6), (131, 40001, 6),
    (130, 65536, 6), (129, 100003, 20)])
def test_distillation(rows, vocab, k, dtype):
    logits, teacher, index, dloss = _distill_case(rows, vocab, k, dtype, rows + vocab)
    loss, lse = B.byz_distill_loss(logits, teacher, index, 2.0)
    d = B.byz_distill_loss_backward(dloss, logits, teacher, index, lse, 2.0)
    step = B.byz_distill_loss_step(logits, teacher, index, dloss, 2.0)
    for offset, more, out_offset, out_more in ((1, 0, 0, 0), (0, 1, 3, 2), (5, 11, 5, 11), (7, 3, 2, 8), (2, 6, 0, 1)):
        part, _ = _placed(logits, offset, more)
        out, wide = _placed(logits, out_offset, out_more)
        out.fill_(7.0)
        beside = wide.isnan()
        got = B.byz_distill_loss(part, teacher, index, 2.0)
        assert _same_bits(got[0], loss) and _same_bits(got[1], lse)
        assert _same_bits(B.byz_distill_loss_backward(dloss, part, teacher, index, lse, 2.0, out=out), d)
        assert torch.equal(wide.isnan(), beside)
        out.fill_(7.0)
        got = B.byz_distill_loss_step(part, teacher, index, dloss, 2.0, out=out)
        assert _same_bits(got[0], step[0]) and _same_bits(got[1], step[1])
        assert torch.equal(wide.isnan(), beside)
        got = B.byz_distill_loss_step(part, teacher, index, dloss, 2.0, out=part)
        assert _same_bits(got[0], step[0]) and _same_bits(got[1], step[1])


def test_distillation_of_a_file_in_a_batch():
    # rows of a file, sliced from a batch of logits and held alone: 30 rows of 1001 words start 12 bytes off a boundary
    logits, teacher, index, dloss = _distill_case(90, 1001, 5, BF16, 3)
    for at in (0, 30, 60):
        rows = slice(at, at + 30)
        a = B.byz_distill_loss_step(logits[rows], teacher[rows], index[rows], dloss[rows], 2.0)
        b = B.byz_distill_loss_step(logits[rows].clone(), teacher[rows].clone(), index[rows].clone(), dloss[rows].clone(), 2.0)
        assert _same_bits(a[0], b[0]) and _same_bits(a[1], b[1])


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
@pytest.mark.parametrize("shape", [
    (3, 1, 8, 2), (4, 49, 32, 8), (30, 16, 512, 32), (3, 77, 30, 6), (2, 100, 15, 5), (2, 31, 4096, 1), (1, 7, 2051, 1), (2, 9000, 32, 8),
    (2, 12544, 64, 32), (1, 3001, 250, 10)], ids=str)
def test_group_norm(shape, dtype):
    groups, act = shape[3], B.BYZ_ACT_SILU
    x, gamma, beta, dy = _norm_case(*shape, dtype, "silu", seed=sum(shape))
    y, mean, rstd = B.byz_group_norm(x, groups, gamma, beta, act=act)
    back = B.byz_group_norm_backward(dy, x, groups, mean, rstd, gamma, beta, act)
    for offset, more, other in ((1, 0, 0), (0, 1, 3), (5, 11, 2), (3, 8, 16), (2, 6, 1)):
        part, _ = _placed(x, offset, more)
        dpart, _ = _placed(dy, other, more + 3)
        out, wide = _placed(x, other, offset)
        out.fill_(7.0)
        beside = wide.isnan()
        got = B.byz_group_norm(part, groups, gamma, beta, act=act, out=out)
        assert all(_same_bits(a, b) for a, b in zip(got, (y, mean, rstd)))
        assert torch.equal(wide.isnan(), beside)
        out.fill_(7.0)
        got = B.byz_group_norm_backward(dpart, part, groups, mean, rstd, gamma, beta, act, out=out)
        assert all(_same_bits(a, b) for a, b in zip(got, back))
        assert torch.equal(wide.isnan(), beside)
        got = B.byz_group_norm_backward(dpart, part, groups, mean, rstd, gamma, beta, act, out=dpart)  # over dy
        assert all(_same_bits(a, b) for a, b in zip(got, back))
        got = B.byz_group_norm(part, groups, gamma, beta, act=act, out=part)  # in place
        assert all(_same_bits(a, b) for a, b in zip(got, (y, mean, rstd)))
