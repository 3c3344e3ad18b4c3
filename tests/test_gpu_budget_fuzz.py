"""Random calls of ssa_attn_window and ssa_attn_mass (shapes, groups, types, layouts, pages, lengths, windows, sinks) against fp64."""
import numpy as np
import pytest
import torch

from paper_2404_09336_b200 import ssa

from budget_util import DEV, Tokens, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("seed", range(48))
def test_random_call(seed):
    r = np.random.default_rng(seed)
    pick = lambda *x: x[int(r.integers(len(x)))]
    H_kv, group, D = pick(1, 2, 3), pick(1, 2, 3, 4, 5, 7, 8, 12), pick(64, 128)
    dtype, layout, page = pick("bf16", "f16", "fp8"), pick("bhtd", "bthd"), pick(0, 0, 1, 2, 4, 8, 16, 32, 64, 256)
    T, B = int(r.integers(1, 900)), int(r.integers(1, 4))
    n_q = min(T, int(pick(1, 2, 3, int(r.integers(4, 30)), int(r.integers(30, 300)))))
    p = Tokens(B, H_kv * group, H_kv, T, D, n_q, dtype, layout, page, seed=seed)
    out_dtype, many = pick(torch.float32, None), group * n_q > 24 and dtype != "fp8"
    for i in range(3):
        ctx = [int(r.integers(0, T + 1)) for _ in range(B)]
        new = [int(r.integers(0, n_q + 1)) for _ in range(B)]
        if i == 0:
            ctx[0], new[0] = T, n_q
        window, sinks = pick(0, 1, int(r.integers(1, T + 1)), int(r.integers(1, 200))), pick(0, 1, int(r.integers(0, T + 1)), int(r.integers(0, 64)))
        got = p.call(ctx, new, window, sinks, out_dtype)
        check(p, got, ctx, new, window, sinks, out_dtype or p.dt_q, many)
        assert got[3] == 0
        if H_kv * group * n_q <= ssa.MASS_MAX_ROWS and i < 2:
            old = torch.rand(B, T, generator=torch.Generator().manual_seed(seed)) * 2
            got = p.call(ctx, new, window, sinks, out_dtype, mass=True, mass_in=old.to(DEV), decay=0.5)
            check(p, got, ctx, new, window, sinks, out_dtype or p.dt_q, mass_in=old.double().numpy(), decay=0.5)
