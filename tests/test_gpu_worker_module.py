"""The worker operators without the native module of their common calls: the same bits by the Python path."""
import pytest
import torch

from paper_2010_04902_amd import worker
from test_gpu_worker import _all_three, _all_three_inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("sizes", [(2, 4, 64, 200), (1, 9000, 32, 520)], ids=str)
def test_every_operator_without_the_module(sizes, monkeypatch):
    inputs = _all_three_inputs(*sizes, 7)
    want = _all_three(*inputs)
    monkeypatch.setattr(worker, "_calls", worker._NoCalls())
    for a, b in zip(_all_three(*inputs), want):
        assert torch.equal(a, b)
