"""ssa_attn_window_fp4 where many rows share a conversion: what depends on it, and what does not."""
import numpy as np
import pytest
import torch

from cache_util import Fp4Tokens, check_tokens
from paper_2404_09336_b200 import ssa

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [0, 8, 64])
@pytest.mark.parametrize("out_dtype", [BF16, F32])
def test_bits_do_not_depend_on_the_workspace(D, page, out_dtype):
    """Weights keep the bits of the calls of fewer rows, whether the call has room to convert once or converts in every block."""
    n = 70 if page else 200
    p = Fp4Tokens(2, 8, 2, 900, D, n, page=page, spread=2.0)
    for ctx, new, window, sinks in (([900, 641], None, 0, 0), ([877, 300], [n, n - 30], 150, 9)):
        got = [p.call(ctx, new, window, sinks, out_dtype, less=less) for less in (0, 1)]
        assert np.array_equal(got[0][0], got[1][0]) and np.array_equal(got[0][1], got[1][1]) and got[0][3] == got[1][3] == 0
        check_tokens(p, got[0], ctx, new, window, sinks, out_dtype, tiles=True)
