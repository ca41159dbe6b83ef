"""A ByzShield training loop on one GPU: workers' steps with the library's operators, then the server's call.

Every worker of a MOLS cluster turns its files (images of a synthetic batch) into gradients with

    byz_group_norm       normalisation and activation of the channels-last features
    byz_gated_ffn        a gated block over the positions, and a gated readout of the pooled positions
    byz_distill_loss_step  the loss against a teacher's top logits, with its gradient

and their backward calls; Byzantine workers return reversed gradients.  Honest copies of a file's
gradient are the same bits, so byz_aggregate's vote finds them, and its median of the winners moves
the weights.  `--defence mean` averages all returned copies instead.

    python examples/worker_step.py [--steps 30] [--byzantine 2] [--defence vote|mean]
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2010_04902_amd as B  # noqa: E402

SIDE, CHANNELS, GROUPS, HIDDEN, CLASSES, TOP = 8, 64, 16, 128, 10, 5
SHAPES = {"gamma": (CHANNELS,), "beta": (CHANNELS,), "w_gate": (HIDDEN, CHANNELS), "w_up": (HIDDEN, CHANNELS),
          "r_gate": (CLASSES, HIDDEN), "r_up": (CLASSES, HIDDEN)}
LENGTH = sum(torch.Size(s).numel() for s in SHAPES.values())


def parameters(device, seed=0):
    """fp32 weights by name."""
    gen = torch.Generator(device=device)
    gen.manual_seed(seed)
    out = {}
    for name, shape in SHAPES.items():
        out[name] = torch.randn(*shape, generator=gen, device=device) * shape[-1] ** -0.5
    out["gamma"].fill_(1.0)
    out["beta"].fill_(0.0)
    return out


def batch(device, images, seed):
    """Images whose channels have means of their class, and a teacher's top logits that mostly know it: (x, teacher, index)."""
    gen = torch.Generator(device=device)
    gen.manual_seed(1)
    patterns = torch.randn(CLASSES, 1, 1, CHANNELS, generator=gen, device=device)
    gen.manual_seed(1000 + seed)
    label = torch.randint(0, CLASSES, (images,), generator=gen, device=device)
    x = patterns[label] + torch.randn(images, SIDE, SIDE, CHANNELS, generator=gen, device=device)
    index = (label[:, None] + torch.arange(TOP, device=device)) % CLASSES
    teacher = torch.randn(images, TOP, generator=gen, device=device).sort(dim=1, descending=True).values
    teacher[:, 0] += 5.0
    return x.bfloat16().permute(0, 3, 1, 2), teacher, index.to(torch.int32)


def file_gradient(params, x, teacher, index, out):
    """One file's losses; its gradient is written to the fp32 row `out`, parameter after parameter."""
    n, positions = x.shape[0], SIDE * SIDE
    half = {name: params[name].bfloat16() for name in ("w_gate", "w_up", "r_gate", "r_up")}
    y, mean, rstd = B.byz_group_norm(x, GROUPS, params["gamma"], params["beta"], act=B.BYZ_ACT_SILU)
    tokens = y.permute(0, 2, 3, 1).reshape(n * positions, CHANNELS)
    h, gate, up = B.byz_gated_ffn(tokens, half["w_gate"], half["w_up"], save=True)
    pooled = h.view(n, positions, HIDDEN).mean(dim=1, dtype=torch.float32).bfloat16()
    logits, r_gate, r_up = B.byz_gated_ffn(pooled, half["r_gate"], half["r_up"], B.BYZ_ACT_SIGMOID, save=True)

    weight = torch.full((n,), 1.0 / n, device=x.device)
    loss, dlogits = B.byz_distill_loss_step(logits, teacher, index, weight, temperature=2.0)

    dpooled, d_r_gate, d_r_up = B.byz_gated_ffn_backward(dlogits, pooled, half["r_gate"], half["r_up"], r_gate, r_up,
                                                         B.BYZ_ACT_SIGMOID)
    dh = (dpooled.float() / positions).bfloat16().repeat_interleave(positions, dim=0)
    dtokens, d_w_gate, d_w_up = B.byz_gated_ffn_backward(dh, tokens, half["w_gate"], half["w_up"], gate, up)
    dy = dtokens.view(n, SIDE, SIDE, CHANNELS).permute(0, 3, 1, 2)
    _, dgamma, dbeta = B.byz_group_norm_backward(dy, x, GROUPS, mean, rstd, params["gamma"], params["beta"],
                                                 B.BYZ_ACT_SILU)
    torch.cat([g.reshape(-1).float() for g in (dgamma, dbeta, d_w_gate, d_w_up, d_r_gate, d_r_up)], out=out)
    return loss


def returns(asg, params, images, step, byzantine, X):
    """All workers' returns in X, row after row as the assignment orders them, and the mean loss of the batch."""
    x, teacher, index = batch(X.device, images, step)
    per_file = images // asg.f
    losses = []
    for row, (worker, file) in enumerate((w, i) for w, files in enumerate(asg.worker_files()) for i in files):
        part = slice(int(file) * per_file, (int(file) + 1) * per_file)
        losses.append(file_gradient(params, x[part], teacher[part], index[part], X[row, :LENGTH]))
        if worker in byzantine:
            X[row, :LENGTH] *= -100.0
    return torch.stack(losses).mean()


def apply(params, gradient, rate, longest=1.0):
    gradient = gradient * (longest / gradient.norm().clamp_min(longest))
    at = 0
    for name, shape in SHAPES.items():
        size = torch.Size(shape).numel()
        params[name] -= rate * gradient[at:at + size].view(shape)
        at += size


def train(steps, byzantine, defence="vote", rate=1.0, images=750, device="cuda:0"):
    """Mean loss of the workers' files at each step."""
    asg = B.byz_build_assignment(B.BYZ_SCHEME_MOLS, 5, 3)
    bad = set(int(w) for w in B.byz_worst_case(asg, byzantine)[0]) if byzantine else set()
    rows = torch.tensor(asg.file_rows().reshape(-1), dtype=torch.int32, device=device)
    X = torch.zeros(asg.f * asg.r, (LENGTH + 63) // 64 * 64, device=device)
    params, history = parameters(device), []
    for step in range(steps):
        history.append(returns(asg, params, images, step, bad, X))
        if defence == "vote":
            gradient = B.byz_aggregate(X, LENGTH, rows, asg.f, asg.r)[0]
        else:
            gradient = X[:, :LENGTH].mean(dim=0)
        apply(params, gradient, rate)
    return [float(v) for v in history]


def main():
    parser = argparse.ArgumentParser(description=__doc__.splitlines()[0])
    parser.add_argument("--steps", type=int, default=30)
    parser.add_argument("--byzantine", type=int, default=2)
    parser.add_argument("--defence", choices=["vote", "mean"], default="vote")
    args = parser.parse_args()
    history = train(args.steps, args.byzantine, args.defence)
    for step, loss in enumerate(history):
        print("step %3d  loss %.4f" % (step, loss))


if __name__ == "__main__":
    main()
