"""The ways the token operators are called: captured and replayed, on other streams, without their native module, two at once, with
what they refuse."""
import math
import warnings

import pytest
import torch

import paper_2010_04902_amd as B
from paper_2010_04902_amd import worker, worker_tokens
from test_gpu_tokens import BF16, DEV, F16, F32, _gen, _pairs_case, _policy_case, _randn, _residual_case, _same_bits

pytestmark = pytest.mark.gpu


def _inputs(rows, cols, vocab, dtype, seed, gate=1):
    c = _residual_case(rows, cols, dtype, "layer", "rms", gate, 0.1, bias=True, seed=seed)
    given, dloss, terms, *_ = _policy_case(rows, vocab, dtype, 0.7, 0.05, seed)
    bounds = torch.tensor([0, rows // 3, rows // 2, rows // 2, rows], dtype=torch.int32, device=DEV)
    return c, given, dloss, terms, bounds


def _all(c, given, dloss, terms, bounds, stream=None):
    """Every operator and its gradients."""
    vectors = (c["w1"], c["b1"], c["gate"], c["w2"], c["b2"])
    more = {"stream": stream}
    x = B.byz_dropout(c["x"], 0.25, 5, 6, **more)
    out, y, stats = B.byz_residual_norm(x, c["h"], c["form"], *vectors, **more)
    dx, dh, grads = B.byz_residual_norm_backward(c["dout"], c["dy"], x, c["h"], stats, c["form"], *vectors, **more)
    alone = B.byz_residual_form(pre=B.BYZ_NORM_LAYER)
    _, last, stats2 = B.byz_residual_norm(out, None, alone, pre_weight=c["w2"], **more)
    dlast, _, _ = B.byz_residual_norm_backward(None, dx, out, None, stats2, alone, pre_weight=c["w2"], **more)
    z, label = given[:2]
    pairs = torch.ones(2, device=DEV) if stream is None else c["pairs"]
    logp, st = B.byz_token_logp(z, label, **more)
    results = [x, out, y, stats, dx, dh, *grads, last, stats2, dlast, logp, st, B.byz_token_logp_backward(dloss, z, label, st, **more)]
    results += B.byz_policy_loss(*given, **terms, **more)
    results.append(B.byz_policy_loss_backward(dloss, *given, results[-1], **terms, **more))
    results += B.byz_policy_loss_step(*given, dloss, **terms, **more)
    loss, sums, slope, st = B.byz_preference_loss(z, label, bounds, **more)
    results += [loss, sums, slope, st, B.byz_preference_loss_backward(pairs, z, label, bounds, slope, st, **more)]
    results += B.byz_preference_loss_step(z, label, bounds, pairs, **more)
    return results


SIZES = [(8, 40, 90, F32), (30, 520, 1000, BF16), (9, 1001, 2049, F16), (5, 2100, 20011, BF16), (3, 4104, 50021, F32), (7, 9000, 40000, BF16),
         (140, 8192, 70000, BF16), (2, 64, 300001, F32)]


@pytest.mark.parametrize("sizes", SIZES, ids=str)
def test_captured_and_replayed(sizes):
    """Two graphs of the same calls on other inputs, replayed in turn with eager calls between them."""
    first, second = _inputs(*sizes, 1), _inputs(*sizes, 2, gate=sizes[0])
    want = [_all(*i) for i in (first, second)]
    for i in (first, second):
        i[0]["pairs"] = torch.ones(2, device=DEV)
    graphs, results = [], []
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        for i in (first, second):
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=side):
                results.append(_all(*i, stream=side))
            graphs.append(graph)
    torch.cuda.current_stream().wait_stream(side)
    for turn in range(3):
        for which in (0, 1, 1, 0):
            for t in results[which]:
                if t is not None:
                    t.fill_(math.nan)
            graphs[which].replay()
            eager = _all(*(second if which == 0 else first))
            torch.cuda.synchronize()
            for a, b in zip(results[which], want[which]):
                assert (a is None and b is None) or _same_bits(a, b)
            for a, b in zip(eager, want[1 - which]):
                assert (a is None and b is None) or _same_bits(a, b)


def test_replays_take_their_offset_from_memory():
    x, h = _randn(_gen(0), 20, 300), _randn(_gen(1), 20, 300)
    at = torch.zeros(1, dtype=torch.int64, device=DEV)
    form = B.byz_residual_form(p=0.5, seed=3, offset=10, offset_at=at)
    B.byz_dropout(x, 0.5, 3, 10, offset_at=at)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side), torch.cuda.graph(graph, stream=side):
        y = B.byz_dropout(x, 0.5, 3, 10, offset_at=at, stream=side)
        out, _, stats = B.byz_residual_norm(x, h, form, stream=side)
        dx, dh, _ = B.byz_residual_norm_backward(x, x, x, h, stats, form, stream=side)
        at += 1
    torch.cuda.current_stream().wait_stream(side)
    at.fill_(0)
    for step in range(4):
        graph.replay()
        torch.cuda.synchronize()
        plain = B.byz_residual_form(p=0.5, seed=3, offset=10 + step)
        want, _, st = B.byz_residual_norm(x, h, plain)
        assert _same_bits(y, B.byz_dropout(x, 0.5, 3, 10 + step)) and _same_bits(out, want)
        assert _same_bits(dh, B.byz_residual_norm_backward(x, x, x, h, st, plain)[1])


@pytest.mark.parametrize("sizes", SIZES[:6], ids=str)
def test_on_other_streams_two_at_once(sizes):
    inputs = [_inputs(*sizes, seed) for seed in (3, 4)]
    want = [_all(*i) for i in inputs]
    for i in inputs:
        i[0]["pairs"] = torch.ones(2, device=DEV)
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    torch.cuda.synchronize()
    got = [_all(*i, stream=s if sizes[0] % 2 else s.cuda_stream) for i, s in zip(inputs, streams)]
    torch.cuda.synchronize()
    for results, wanted in zip(got, want):
        for a, b in zip(results, wanted):
            assert (a is None and b is None) or _same_bits(a, b)


@pytest.mark.parametrize("sizes", SIZES[:5], ids=str)
def test_without_the_native_module(sizes, monkeypatch):
    inputs = _inputs(*sizes, 7)
    want = _all(*inputs)
    monkeypatch.setattr(worker_tokens, "_calls", worker._NoCalls())
    for a, b in zip(_all(*inputs), want):
        assert (a is None and b is None) or _same_bits(a, b)


def test_native_module_is_there():
    worker_tokens._load()
    x = torch.ones(4, 64, device=DEV)
    assert worker_tokens._calls.dropout(x, 0.5, 1, 2, 0) is not None


def _cases():
    c, given, dloss, terms, bounds = _inputs(6, 40, 50, F32, 9)
    vectors = (c["w1"], c["b1"], c["gate"], c["w2"], c["b2"])
    z, label, old, advantage = given
    stats = torch.ones(6, 4, device=DEV)
    st, pairs = B.byz_token_logp(z, label)[1], torch.ones(2, device=DEV)
    return c, vectors, z, label, old, advantage, stats, st, dloss, bounds, pairs


@pytest.mark.parametrize("stream", [False, True])
def test_a_forward_call_warns(stream):
    c, vectors, z, label, old, advantage, stats, st, dloss, bounds, pairs = _cases()
    more = {"stream": torch.cuda.current_stream()} if stream else {}
    calls = [(lambda: B.byz_dropout(c["x"], 0.5, 1, **more), (c["x"],)),
             (lambda: B.byz_residual_norm(c["x"], c["h"], c["form"], *vectors, **more), (c["x"], c["h"], *vectors[:1])),
             (lambda: B.byz_token_logp(z, label, **more), (z,)), (lambda: B.byz_policy_loss(z, label, old, advantage, **more), (z, old)),
             (lambda: B.byz_preference_loss(z, label, bounds, **more), (z,))]
    for call, tensors in calls:
        for t in tensors:
            t.requires_grad_()
            with pytest.warns(RuntimeWarning, match="autograd's graph.*backward call") as seen:
                call()
            assert len(seen) == 1
            with warnings.catch_warnings():
                warnings.simplefilter("error")
                with pytest.raises(RuntimeWarning, match="autograd's graph"):
                    call()
                with torch.no_grad():
                    call()
            t.requires_grad_(False)


def test_refusals():
    c, vectors, z, label, old, advantage, stats, st, dloss, bounds, pairs = _cases()
    x, h, form = c["x"], c["h"], c["form"]
    none = B.byz_residual_form(pre=B.BYZ_NORM_NONE)
    wrong = [
        lambda: B.byz_dropout(x, 0.5, 1, out=x[:5]), lambda: B.byz_dropout(x, 0.5, 1, out=x.bfloat16()),
        lambda: B.byz_dropout(x.double(), 0.5, 1), lambda: B.byz_dropout(x, 0.5, 1, offset_at=torch.zeros(2, dtype=torch.int64, device=DEV)),
        lambda: B.byz_dropout(x, 0.5, 1, offset_at=torch.zeros(1, device=DEV)), lambda: B.byz_dropout(x, 0.5, 1, out=torch.zeros(6, 40)),
        lambda: B.byz_residual_norm(x, h[:5], form), lambda: B.byz_residual_norm(x, h.bfloat16(), form),
        lambda: B.byz_residual_norm(x, h, form, post_weight=vectors[0][:39]), lambda: B.byz_residual_norm(x, h, form, gate=torch.ones(4, 40, device=DEV)),
        lambda: B.byz_residual_norm(x, h, form, gate=torch.ones(0, 40, device=DEV)), lambda: B.byz_residual_norm(x, h, form, gate=torch.ones(6, 39, device=DEV)),
        lambda: B.byz_residual_norm(x, h, form, pre_bias=vectors[3].double()), lambda: B.byz_residual_norm(x, None, form, out=x),
        lambda: B.byz_residual_norm(x, h.t(), form), lambda: B.byz_residual_norm(x, h, form, out=x[:, :39]),
        lambda: B.byz_residual_norm_backward(x[:5], x, x, h, stats, form), lambda: B.byz_residual_norm_backward(x, x.half(), x, h, stats, form),
        lambda: B.byz_residual_norm_backward(x, x, x, h, stats[:, :2], form),
        lambda: B.byz_token_logp(z, label.long()), lambda: B.byz_token_logp(z, label[:5]), lambda: B.byz_token_logp(z.t(), label),
        lambda: B.byz_token_logp_backward(dloss[:5], z, label, st), lambda: B.byz_token_logp_backward(dloss, z, label, st[:5]),
        lambda: B.byz_token_logp_backward(dloss, z, label, st, out=z.half()),
        lambda: B.byz_policy_loss(z, label, old[:5], advantage), lambda: B.byz_policy_loss(z, label, old, advantage.double()),
        lambda: B.byz_policy_loss_step(z, label, old, advantage, dloss, out=z[:, :49]), lambda: B.byz_policy_loss(z, label[::2], old, advantage),
        lambda: B.byz_preference_loss(z, label, bounds[:4]), lambda: B.byz_preference_loss(z, label, bounds.long()),
        lambda: B.byz_preference_loss(z, label, bounds, ref=torch.ones(3, device=DEV)), lambda: B.byz_preference_loss(z, label, bounds[None]),
        lambda: B.byz_preference_loss_step(z, label, bounds, torch.ones(4, device=DEV)),
        lambda: B.byz_preference_loss_backward(pairs, z, label, bounds, pairs[:1], st), lambda: B.byz_token_logp(z, label.cpu()),
    ]
    for number, call in enumerate(wrong):
        with pytest.raises(ValueError):
            call()
            raise AssertionError(number)
    refused = [
        lambda: B.byz_dropout(x, 1.5, 1), lambda: B.byz_dropout(x, math.nan, 1), lambda: B.byz_dropout(x, 0.5, 1, first_row=2 ** 32 - 3),
        lambda: B.byz_dropout(x, 0.5, 1, first_row=-1), lambda: B.byz_residual_norm(x, h, none, pre_weight=vectors[3]),
        lambda: B.byz_residual_norm(x, None, form), lambda: B.byz_residual_norm_backward(x, x, x, h, stats, none),
        lambda: B.byz_residual_norm_backward(None, None, x, h, stats, form), lambda: B.byz_residual_norm(x, h, B.byz_residual_form(post=7)),
        lambda: B.byz_token_logp(z, label, 0.0), lambda: B.byz_policy_loss(z, label, old, advantage, kl=0.1),
        lambda: B.byz_policy_loss(z, label, old, advantage, clip_low=2.0), lambda: B.byz_preference_loss(z, label, bounds, smoothing=2.0),
        lambda: B.byz_preference_loss(z, label, bounds, beta=math.inf),
    ]
    for number, call in enumerate(refused):
        with pytest.raises(B.ByzError):
            call()
            raise AssertionError(number)


def test_without_gradients_of_the_vectors():
    c, vectors, *_ = _cases()
    _, _, stats = B.byz_residual_norm(c["x"], c["h"], c["form"], *vectors)
    want = B.byz_residual_norm_backward(c["dout"], c["dy"], c["x"], c["h"], stats, c["form"], *vectors)
    got = B.byz_residual_norm_backward(c["dout"], c["dy"], c["x"], c["h"], stats, c["form"], *vectors, parameters=False)
    assert _same_bits(got[0], want[0]) and _same_bits(got[1], want[1]) and got[2] == (None,) * 5


def test_forms_are_read_at_each_call():
    """A form's offset may be set anew for every step."""
    c = _residual_case(5, 64, F32, "rms", "rms", 0, 0.5)
    first = B.byz_residual_norm(c["x"], c["h"], c["form"])[0]
    c["form"].offset = 77
    other = B.byz_residual_norm(c["x"], c["h"], c["form"])[0]
    c["form"].offset = 0
    assert not torch.equal(first, other) and _same_bits(first, B.byz_residual_norm(c["x"], c["h"], c["form"])[0])


def test_preference_of_a_padded_batch():
    """Sequences of a padded batch, each with its padding behind it, are those without."""
    z, label, bounds, *_ = _pairs_case([5, 8, 3, 6], 0, 40, F32)
    long, edges = 9, bounds.tolist()
    wide, tokens = torch.full((4 * long, 40), math.nan, device=DEV), torch.full((4 * long,), -1, dtype=torch.int32, device=DEV)
    for s, (a, b) in enumerate(zip(edges, edges[1:])):
        wide[s * long:s * long + b - a], tokens[s * long:s * long + b - a] = z[a:b], label[a:b]
    ones = torch.ones(2, device=DEV)
    loss, sums, grad = B.byz_preference_loss_step(z, label, bounds.to(DEV), ones)
    at = torch.arange(0, 4 * long + 1, long, dtype=torch.int32, device=DEV)
    loss2, sums2, grad2 = B.byz_preference_loss_step(wide, tokens, at, ones)
    assert _same_bits(loss, loss2) and _same_bits(sums, sums2)
    for s, (a, b) in enumerate(zip(edges, edges[1:])):
        assert _same_bits(grad[a:b], grad2[s * long:s * long + b - a])
        assert bool((grad2[s * long + b - a:(s + 1) * long] == 0).all())


@pytest.mark.parametrize("rows, gate_rows", [(13, 5), (7, 7), (7, 100), (900, 7), (3001, 1000), (40, 39)])
@pytest.mark.parametrize("cols", [5, 40, 700, 1500, 4000, 8000, 9000])
def test_groups_of_gates_rows_that_end_early(cols, rows, gate_rows):
    """The C call takes groups that do not divide the rows: the last one is shorter."""
    L = worker_tokens._load()
    groups = -(-rows // gate_rows)
    c = _residual_case(rows, cols, BF16, "rms", "layer", 1, 0.1, seed=cols)
    gate = 1 + _randn(_gen(cols), groups, cols, scale=0.3)
    wide = gate.repeat_interleave(gate_rows, dim=0)[:rows].contiguous()

    def run(g, n):
        out, y, dx, dh = (torch.empty_like(c["x"]) for _ in range(4))
        stats, grads = torch.empty(rows, 4, device=DEV), [torch.full((cols,), math.nan, device=DEV) for _ in range(3)]
        d_gate = torch.full_like(g, math.nan)
        p = lambda t: t.data_ptr()  # noqa: E731
        assert L.byz_residual_norm(p(c["x"]), cols, p(c["h"]), cols, rows, cols, 1, c["form"], p(c["w1"]), None, p(g), n, p(c["w2"]),
                                   p(c["b2"]), p(out), cols, p(y), cols, p(stats), None) == 0
        need = L.byz_residual_norm_backward_workspace_bytes(rows, cols, 1, n)
        ws = torch.empty(need, dtype=torch.uint8, device=DEV)
        assert L.byz_residual_norm_backward(p(c["dout"]), cols, p(c["dy"]), cols, p(c["x"]), cols, p(c["h"]), cols, p(stats), rows, cols, 1,
                                            c["form"], p(c["w1"]), None, p(g), n, p(c["w2"]), p(dx), cols, p(dh), cols, p(grads[0]), None,
                                            p(d_gate), p(grads[1]), p(grads[2]), p(ws), need, None) == 0
        torch.cuda.synchronize()
        return out, y, stats, dx, dh, grads, d_gate

    got, want = run(gate, gate_rows), run(wide, 1)
    for a, b in zip(got[:3], want[:3]):
        assert _same_bits(a, b)
    # gate_rows is one of a call's sizes, which other kernels may take: both results are within half a step of bf16 (2^-8) of values
    # that some dozens of fp32 roundings of a row's largest ones, 64 at most, are apart
    for a, b in zip(got[3:5], want[3:5]):
        assert bool(((a.double() - b.double()).abs() <= 2 * 2.0 ** -8 * b.double().abs() + 64 * 2.0 ** -24 * 64).all())
    # sums over the rows in another order: some dozens of roundings of what they are made of, of which dx, dh and y are the scale
    for a, b in zip(got[5], want[5]):
        assert float((a - b).abs().max()) <= 64 * 2.0 ** -24 * rows * 16
    # a term is scale * v * dt: dt's own error, some dozens of roundings of a row's terms (10 at most), times scale * v (6 at most)
    each = want[6].double()
    for g in range(groups):
        part = each[g * gate_rows:(g + 1) * gate_rows]
        assert bool(((got[6][g].double() - part.sum(0)).abs() <= 64 * 2.0 ** -24 * (part.abs().sum(0) + 64 * len(part))).all())
