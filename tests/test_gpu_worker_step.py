"""examples/worker_step.py: the operators together, and the server's vote over what they return."""
import importlib.util
import os

import pytest
import torch

import paper_2010_04902_amd as B

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "worker_step.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("worker_step", PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def _gradient64(example, params, x, teacher, index):
    """Losses of a file and its mean loss' gradient, by autograd in 64 bits on the bf16 weights."""
    leaves = {name: (p if name in ("gamma", "beta") else p.bfloat16()).double().requires_grad_()
              for name, p in params.items()}
    n, c = x.shape[:2]
    flat = x.double().reshape(n, example.GROUPS, -1)
    var, mean = torch.var_mean(flat, dim=2, correction=0, keepdim=True)
    z = ((flat - mean) / (var + 1e-5).sqrt()).view(x.shape) * leaves["gamma"][:, None, None] + leaves["beta"][:, None, None]
    tokens = torch.nn.functional.silu(z).permute(0, 2, 3, 1).reshape(-1, c)
    h = torch.nn.functional.silu(torch.mm(tokens, leaves["w_gate"].t())) * torch.mm(tokens, leaves["w_up"].t())
    pooled = h.view(n, -1, example.HIDDEN).mean(dim=1)
    logits = torch.sigmoid(torch.mm(pooled, leaves["r_gate"].t())) * torch.mm(pooled, leaves["r_up"].t())
    p = torch.softmax(teacher.double() / 2.0, dim=1)
    log_q = torch.log_softmax(logits / 2.0, dim=1).gather(1, index.long())
    loss = 4.0 * (p * (p.log() - log_q)).sum(dim=1)
    grads = torch.autograd.grad(loss.mean(), list(leaves.values()))
    return loss.detach(), dict(zip(leaves, grads))


def test_a_files_gradient(example):
    # About twelve values on the longest way are rounded to bf16, each off by 2^-8 of itself at most; each
    # gradient as a whole (norm of the difference to norm) may be off by the sum of them, and twice that because a
    # factor's error acts through its slope too.  The losses' logits are rounded three times on the way.
    params = example.parameters(torch.device(DEV))
    x, teacher, index = example.batch(torch.device(DEV), 30, 7)
    out = torch.empty(example.LENGTH, device=DEV)
    loss = example.file_gradient(params, x, teacher, index, out)
    loss64, grads64 = _gradient64(example, params, x, teacher, index)
    assert bool(((loss.double() - loss64).abs() <= 0.05 * (1 + loss64)).all())
    at = 0
    for name, shape in example.SHAPES.items():
        size = torch.Size(shape).numel()
        got, want = out[at:at + size].view(shape).double(), grads64[name]
        assert float((got - want).norm() / want.norm()) <= 24 * 2.0 ** -8, name
        at += size


def test_honest_copies_are_the_same_bits_and_win_the_vote(example):
    asg = B.byz_build_assignment(B.BYZ_SCHEME_MOLS, 5, 3)
    params = example.parameters(torch.device(DEV))
    X = torch.zeros(asg.f * asg.r, (example.LENGTH + 63) // 64 * 64, device=DEV)
    example.returns(asg, params, 750, 0, set(), X)
    honest = X.clone()
    table = asg.file_rows()
    for rows in table:
        for row in rows[1:]:
            assert torch.equal(honest[int(rows[0])].view(torch.int32), honest[int(row)].view(torch.int32))
    # one Byzantine worker has one copy of a file: it wins no vote
    example.returns(asg, params, 750, 0, {3}, X)
    assert not torch.equal(X, honest)
    rows = torch.tensor(table.reshape(-1), dtype=torch.int32, device=DEV)
    got = B.byz_aggregate(X, example.LENGTH, rows, asg.f, asg.r)[0]
    want = honest[torch.tensor(table[:, 0].astype("int64"), device=DEV), :example.LENGTH].median(dim=0).values
    assert torch.equal(got, want)


def test_training_with_the_vote_outlasts_byzantine_workers(example):
    history = example.train(12, 2)
    assert history[-1] < 0.7 * history[0], history
