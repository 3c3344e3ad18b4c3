"""ssa_mass_to_index where a block of 16384 positions keeps nearly all of them: more than its three digits' bins have room for."""
import numpy as np
import pytest
import torch

from oracle import budget_oracle as BO
from paper_2404_09336_b200 import ssa

from budget_util import DEV

pytestmark = pytest.mark.gpu


# (one block of 16384; clusters of two, four and eight, whose blocks keep most of their part, or all of it)
@pytest.mark.parametrize("T,budget,sinks,recent", [(16384, 12289, 4, 100), (16384, 16000, 0, 0), (16384, 16383, 64, 512), (15001, 14900, 3, 7),
                                                   (32768, 32767, 0, 0), (40000, 39000, 3, 1), (40000, 20000, 16384, 0), (131072, 131000, 5, 100),
                                                   (131072, 60000, 0, 50000)])
def test_keep_nearly_all(T, budget, sinks, recent):
    rng = np.random.default_rng(T + budget)
    mass = np.array([rng.standard_normal(T), np.round(rng.standard_normal(T)), np.zeros(T),
                     np.where(rng.random(T) < .3, np.nan, np.round(rng.standard_normal(T), 1))], np.float32)
    B = len(mass)
    d_mass = torch.from_numpy(mass).to(DEV)
    for ctx in ([T] * B, [T, T - 1, budget + 1, budget]):
        index = torch.full((B, budget + 2), -7, dtype=torch.int32, device=DEV)
        counts, status = torch.full((B,), -7, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        ssa.mass_to_index(d_mass, torch.tensor(ctx, dtype=torch.int32, device=DEV), budget, sinks, recent, index, counts, status)
        torch.cuda.synchronize()
        assert int(status) == 0
        for b in range(B):
            want = BO.kept(mass[b], ctx[b], budget, sinks, recent)
            c = int(counts[b])
            assert c == len(want) and np.array_equal(index[b, :c].cpu().numpy(), want), (b, ctx[b])
            assert (index[b, c:] == -7).all()
