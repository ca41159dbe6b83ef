"""Distillation where the kernel changes with the row's length, the teacher's entries and the number of rows."""
import pytest

import paper_2010_04902_amd as B
from test_gpu_worker import BF16, F16, F32, _distill_case, _distill_check, _same_bits

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [F32, BF16, F16], ids=str)
@pytest.mark.parametrize("rows,vocab,k", [
    (7, 1023, 64), (7, 1025, 65), (5, 2048, 256), (5, 2049, 257), (9, 3000, 100), (6, 4096, 64), (6, 4097, 65), (3, 8191, 256), (3, 8192, 40),
    (2, 8193, 40), (1024, 8300, 7), (1023, 8300, 7), (1500, 17000, 70), (1025, 70001, 3)])
def test_distill_row_lengths(rows, vocab, k, dtype):
    logits, teacher, index, dloss = _distill_case(rows, vocab, k, dtype, rows + vocab + k)
    _, _, d, _, d2 = _distill_check(logits, teacher, index, dloss, 2.0)
    held = logits.clone()  # the gradient over the logits, in rows off the 16-byte boundaries
    _, d3 = B.byz_distill_loss_step(held, teacher, index, dloss, 2.0, out=held)
    assert _same_bits(d2, d3)


@pytest.mark.parametrize("vocab", [1000, 3001])
def test_distill_entries_at_one_place(vocab):
    logits, teacher, index, dloss = _distill_case(6, vocab, 200, BF16, 1)
    index[:, 100:] = index[:, :100]
    index[3] = 5
    _distill_check(logits, teacher, index, dloss, 1.0)
