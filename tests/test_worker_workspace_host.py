"""The feed-forward's backward workspace through the C-ABI, without a GPU: what aligned operands need, and who needs more."""
import pytest

from paper_2010_04902_amd import worker
from test_worker_host import ENOMEM, P, _ffn_backward

SIZES = [(40, 32, 8), (17, 64, 512), (300, 128, 264), (1, 8, 1)]


@pytest.mark.parametrize("m,k,n", SIZES)
def test_aligned_size_is_the_other_less_the_copies(m, k, n):
    lib = worker._load()
    need, full = (getattr(lib, "byz_gated_ffn_backward%s_workspace_bytes" % s)(m, k, n, 1) for s in ("_aligned", ""))
    assert need >= 4 * m * n and full - need == 2 * (m * k + 2 * n * k)
    sizes = dict(m=m, k=k, n=n, dh_ld=n, x_ld=k, w_ld=k, gate_ld=n, dx_ld=k, dw_ld=k)
    assert _ffn_backward(**sizes, nbytes=need - 1) == ENOMEM
    # rows that have to be copied: off the boundaries, and pitches of no whole 16 bytes
    for bad in (dict(x=P + 2), dict(wg=P + 8), dict(wu=P + 2), dict(x_ld=k + 1), dict(w_ld=k + 3)):
        assert _ffn_backward(**{**sizes, **bad}, nbytes=full - 1) == ENOMEM


def test_refused_sizes_need_none():
    for args in ((-1, 8, 8, 1), (8, 8, 8, 0), (8, 1 << 31, 8, 1)):
        assert worker._load().byz_gated_ffn_backward_aligned_workspace_bytes(*args) == 0
