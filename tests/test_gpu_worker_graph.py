"""Forward calls say where a tensor that requires a gradient leaves autograd's graph, on either way through the binding."""
import warnings

import pytest
import torch

import paper_2010_04902_amd as B
from test_gpu_worker import BF16, DEV, _distill_case, _ffn_case, _norm_case

pytestmark = pytest.mark.gpu


def _calls(stream):
    x, gamma, beta, dy = _norm_case(3, 20, 16, 4, torch.float32)
    logits, teacher, index, dloss = _distill_case(4, 50, 3, torch.float32, 1)
    t, wg, wu, dh = _ffn_case(5, 32, 24, BF16, 2)
    more = {"stream": torch.cuda.current_stream()} if stream else {}
    forward = [(lambda: B.byz_group_norm(x, 4, gamma, beta, **more), (x, gamma, beta)),
               (lambda: B.byz_distill_loss(logits, teacher, index, **more), (logits,)),
               (lambda: B.byz_gated_ffn(t, wg, wu, save=True, **more), (t, wg, wu))]
    _, mean, rstd = forward[0][0]()
    _, lse = forward[1][0]()
    _, gate, up = forward[2][0]()
    explicit = [(lambda: B.byz_group_norm_backward(dy, x, 4, mean, rstd, gamma, beta, **more), (x, gamma, beta)),
                (lambda: B.byz_distill_loss_backward(dloss, logits, teacher, index, lse, **more), (logits,)),
                (lambda: B.byz_distill_loss_step(logits, teacher, index, dloss, **more), (logits,)),
                (lambda: B.byz_gated_ffn_backward(dh, t, wg, wu, gate, up, **more), (t, wg, wu))]
    return forward, explicit


@pytest.mark.parametrize("stream", [False, True])
def test_a_forward_call_warns(stream):
    forward, explicit = _calls(stream)
    for call, tensors in forward:
        for t in tensors:
            with warnings.catch_warnings():
                warnings.simplefilter("error")
                want = call()
            t.requires_grad_()
            with pytest.warns(RuntimeWarning, match="autograd's graph.*backward call") as seen:
                got = call()
            assert len(seen) == 1 and seen[0].filename == __file__
            with warnings.catch_warnings():  # as an error it is one, and without a graph there is none
                warnings.simplefilter("error")
                with pytest.raises(RuntimeWarning, match="autograd's graph"):
                    call()
                with torch.no_grad():
                    call()
            t.requires_grad_(False)
            for a, b in zip(got, want):
                assert torch.equal(a, b) and not a.requires_grad


@pytest.mark.parametrize("stream", [False, True])
def test_calls_that_are_gradients_themselves_do_not(stream):
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        for call, tensors in _calls(stream)[1]:
            for t in tensors:
                t.requires_grad_()
            call()
            for t in tensors:
                t.requires_grad_(False)
