"""examples/token_step.py: the token operators together, and the server's vote over what they return."""
import importlib.util
import os

import pytest
import torch

import paper_2010_04902_amd as B
from token_forms import kept, kept_scale

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "token_step.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("token_step", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _gradient64(example, params, tokens, ref, step, file, kind):
    """Losses of a file and the gradient of their mean, by autograd in 64 bits on the bf16 weights."""
    leaves = {n: (p.bfloat16() if n in example.MATRICES else p).double().requires_grad_() for n, p in params.items()}
    inputs, label = example.split(tokens)

    def rms(v, weight):
        return v * (v.square().mean(1, keepdim=True) + 1e-5) ** -0.5 * weight

    x = leaves["embedding"][inputs]
    y = rms(x, leaves["norm"])
    h = torch.nn.functional.silu(torch.mm(y, leaves["w_gate"].t())) * torch.mm(y, leaves["w_up"].t())
    mask = kept(*x.shape, example.DROP, file, step).to(DEV).double() * kept_scale(example.DROP)
    last = rms(x + leaves["gate"] * mask * rms(h, leaves["post"]), leaves["last"])
    logp = torch.log_softmax(torch.mm(last, leaves["embedding"].t()), 1).gather(1, label.long()[:, None])[:, 0]
    ref = ref.double()
    if kind == "preference":
        gap = (logp - ref).view(-1, 2, example.LENGTH - 1).sum(2)
        loss = -torch.nn.functional.logsigmoid(example.BETA * (gap[:, 0] - gap[:, 1]))
    else:
        advantage = 2.0 * (label == (5 * inputs + 3) % example.VOCAB).double() - 1.0
        r = (logp - ref).exp()
        loss = -torch.minimum(r * advantage, r.clamp(0.8, 5.0) * advantage) + example.KL * ((ref - logp).exp() - 1 - (ref - logp))
    return loss.detach(), dict(zip(leaves, torch.autograd.grad(loss.mean(), list(leaves.values()))))


@pytest.mark.parametrize("kind", ["preference", "policy"])
def test_a_files_gradient(example, kind):
    # About ten values on the longest way are rounded to bf16 (norms, block, logits, and the gradients behind them), each off by
    # 2^-8 of itself at most; a gradient as a whole (norm of the difference to norm) may be off by the sum of them, and
    # twice that because a factor's error acts through its slope too.  The reference is that of other weights, so that
    # the log ratios, whose error is that of the logits, are not all of what there is.
    params, start = example.parameters(torch.device(DEV)), example.parameters(torch.device(DEV), 1)
    tokens = example.batch(torch.device(DEV), 3, 7)[2]
    inputs, label = example.split(tokens)
    ref = example.reference(start, tokens)
    if kind == "policy":  # ratios far from the clipping's ends, on either side of the lower one
        logp = B.byz_token_logp(example.forward(params, inputs, 5, 2)[0], label)[0]
        ref = logp + torch.where(torch.arange(len(label), device=DEV) % 3 == 0, 0.6, -0.4)
    out = torch.empty(example.SIZE, device=DEV)
    loss = example.file_gradient(params, tokens, ref, 5, 2, out, kind)
    loss64, grads64 = _gradient64(example, params, tokens, ref, 5, 2, kind)
    # a token's log-probability is off by three roundings of logits of some units
    assert bool(((loss.double() - loss64).abs() <= 0.1 * (1 + loss64.abs())).all())
    at = 0
    for name, shape in example.SHAPES.items():
        size = torch.Size(shape).numel()
        got, want = out[at:at + size].view(shape).double(), grads64[name]
        assert float((got - want).norm() / want.norm()) <= 20 * 2.0 ** -8, name
        at += size


@pytest.mark.parametrize("kind", ["preference", "policy"])
def test_honest_copies_are_the_same_bits_and_win_the_vote(example, kind):
    asg = B.byz_build_assignment(B.BYZ_SCHEME_MOLS, 5, 3)
    params, start = example.parameters(torch.device(DEV)), example.parameters(torch.device(DEV), 1)
    X = torch.zeros(asg.f * asg.r, (example.SIZE + 63) // 64 * 64, device=DEV)
    example.returns(asg, params, start, 0, set(), X, kind)
    honest = X.clone()
    table = asg.file_rows()
    for rows in table:
        for row in rows[1:]:
            assert torch.equal(honest[int(rows[0])].view(torch.int32), honest[int(row)].view(torch.int32))
    example.returns(asg, params, start, 0, {3}, X, kind)
    assert not torch.equal(X, honest)
    rows = torch.tensor(table.reshape(-1), dtype=torch.int32, device=DEV)
    got = B.byz_aggregate(X, example.SIZE, rows, asg.f, asg.r)[0]
    want = honest[torch.tensor(table[:, 0].astype("int64"), device=DEV), :example.SIZE].median(dim=0).values
    assert torch.equal(got, want)


@pytest.mark.parametrize("kind", ["preference", "policy"])
def test_training_runs(example, kind):
    history = example.train(3, 2, kind=kind)
    assert len(history) == 3 and all(v == v and abs(v) < 100 for v in history)
