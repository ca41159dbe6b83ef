"""The token operators at the ends of their values' range."""
import math

import pytest
import torch

from test_gpu_tokens import DEV, TYPES, _residual_case, _residual_run, _same_bits
from token_forms import kept

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES, ids=str)
@pytest.mark.parametrize("rows, cols, gate", [(8, 5, 1), (8, 64, 1), (40, 1000, 8), (8, 4104, 8), (24, 4104, 2), (9, 9000, 1), (9, 9000, 3),
                                              (6, 20000, 1)])
def test_dropped_values_reach_no_gradient(rows, cols, gate, dtype):
    """Without a norm of h, whatever lies where the mask drops gives the bits of any other value there, in every result."""
    for pre in ("none", "rms", "layer"):
        for bias in (False, True):
            c = _residual_case(rows, cols, dtype, "none", pre, gate, 0.5, bias=bias, seed=cols)
            want = _residual_run(c)
            mask = kept(rows, cols, 0.5, 99, cols).to(DEV)
            h = c["h"]
            for value in (math.inf, -math.inf, math.nan):
                c["h"] = torch.where(mask, h, value)
                got = _residual_run(c)
                assert got.keys() == want.keys() and "d_post_weight" in got
                for name in want:
                    assert _same_bits(got[name], want[name]), (pre, bias, value, name)
