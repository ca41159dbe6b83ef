"""The feed-forward's input gradient where blocks share a tile's sum: few tokens, wide blocks."""
import pytest
import torch

import paper_2010_04902_amd as B
from test_gpu_worker import BF16, DEV, F16, _ffn_case, _ffn_check, _same_bits

pytestmark = pytest.mark.gpu

# sums of 16 steps of 64 and more; shares that end in, before and behind the gate half's last, partial step; odd widths of dx
SIZES = [(17, 64, 512), (20, 72, 545), (33, 130, 1000), (64, 128, 2752), (40, 257, 3001), (1, 40, 4100), (100, 515, 1344), (150, 64, 5504)]


@pytest.mark.parametrize("dtype", [BF16, F16], ids=str)
@pytest.mark.parametrize("m,k,n", SIZES)
def test_shared_sums(m, k, n, dtype):
    x, wg, wu, dh = _ffn_case(m, k, n, dtype, m + k + n)
    _, gate, up, dx, dwg, dwu = _ffn_check(x, wg, wu, "silu", dh)
    for again in range(2):
        got = B.byz_gated_ffn_backward(dh, x, wg, wu, gate, up)
        assert all(_same_bits(a, b) for a, b in zip(got, (dx, dwg, dwu)))


@pytest.mark.parametrize("m,k,n", [(17, 64, 512), (33, 131, 1000), (70, 200, 2050)])
def test_shared_sums_of_whole_numbers_exactly(m, k, n):
    # relu of gate with values of a few bits: every product and sum is a whole number below 2^24
    gen = torch.Generator(device=DEV).manual_seed(m)
    whole = lambda *s: torch.randint(-1, 2, s, generator=gen, device=DEV).to(BF16)  # noqa: E731
    x, wg, wu, dh = whole(m, k), whole(n, k), whole(n, k), whole(m, n)
    gate, up = (torch.randint(-3, 4, (m, (n + 3) // 4 * 4), generator=gen, device=DEV).float()[:, :n] for _ in range(2))
    dx, _, _ = B.byz_gated_ffn_backward(dh, x, wg, wu, gate, up, B.BYZ_ACT_RELU)
    dgate, dup = dh.double() * up.double() * (gate > 0), dh.double() * gate.double().clamp_min(0)
    want = dgate @ wg.double() + dup @ wu.double()
    assert _same_bits(dx, want.to(BF16))


def test_shared_sums_in_a_graph():
    x, wg, wu, dh = _ffn_case(40, 128, 2752, BF16, 3)
    _, gate, up = B.byz_gated_ffn(x, wg, wu, save=True)
    want = B.byz_gated_ffn_backward(dh, x, wg, wu, gate, up)
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        B.byz_gated_ffn_backward(dh, x, wg, wu, gate, up)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = B.byz_gated_ffn_backward(dh, x, wg, wu, gate, up)
    for _ in range(3):
        for t in got:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(_same_bits(a, b) for a, b in zip(got, want))
