"""What csrc/worker_calls.cpp leaves to Python, without a GPU: everything, with no exception."""
import torch

from paper_2010_04902_amd import worker

worker._load()
CALLS = {"group_norm": 6, "group_norm_backward": 8, "distill_loss": 4, "distill_loss_step": 5, "gated_ffn": 5, "gated_ffn_backward": 7}


def test_names():
    assert sorted(n for n in dir(worker._calls) if not n.startswith("_")) == sorted(CALLS)


def test_arguments_that_are_no_common_call():
    class Own(torch.Tensor):
        pass

    things = [None, 1, 1.5, "x", (), object(), 1 << 80, torch.zeros(2, 3, 4), torch.zeros(2, 2).as_subclass(Own), torch.zeros(0),
              torch.zeros(2, 3, 4, device="meta"), torch.eye(2).to_sparse()]
    for name, count in CALLS.items():
        call = getattr(worker._calls, name)
        for thing in things:
            assert call(*[thing] * count) is None
            assert call(torch.zeros(2, 3, 4), *[thing] * (count - 1)) is None
        for wrong in (0, 1, count - 1, count + 1):
            assert call(*[torch.zeros(2, 2)] * wrong) is None
