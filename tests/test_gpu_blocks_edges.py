"""ssa_block_bounds and ssa_block_select at their edges: infinite bounds, blocks without rows, as many tokens as 32 bits hold."""
import numpy as np
import pytest
import torch

from cache_util import Cache
from oracle import budget_oracle as BO
from test_gpu_blocks_select import Choice, bounds_of

pytestmark = pytest.mark.gpu
INF = float("inf")


def scores(q, least, most):
    """sum_h sum_d max(q min, q max) for q[group, D], bounds [m, D]; zero times an infinity is zero."""
    def product(a, b):
        with np.errstate(invalid="ignore"):
            return np.where((a == 0) | (b == 0), 0.0, a * b)
    with np.errstate(invalid="ignore"):
        return np.maximum(product(q[:, None], least), product(q[:, None], most)).sum((0, 2))


def check(c, n, budget, sinks=0, recent=1):
    index, counts, got, status = c.call([n] * c.B, None, budget, sinks, recent)
    assert status == 0
    q, least, most, group = c.q.double().numpy(), *(c.bounds[:, :, :, i].double().numpy() for i in (0, 1)), c.H // c.H_kv
    m = (n - 1) // c.block + 1
    for b in range(c.B):
        for h in range(c.H_kv):
            lo, hi = least[b, h, :m], most[b, h, :m]
            want = scores(q[b, h * group: (h + 1) * group, 0], lo, hi)
            want[(lo == INF).any(1) & (hi == -INF).any(1)] = -INF            # (no rows)
            x = got[b, h, 0, :m]
            fine = np.isfinite(want)
            # 2 D exact products summed in 64 bits, in any order, and rounded to 32
            size = (np.abs(q[b, h * group: (h + 1) * group, 0]).sum(0) * np.where(np.isfinite(lo) & np.isfinite(hi), np.maximum(np.abs(lo), np.abs(hi)), 1e4)).sum(1)
            assert (np.abs(x[fine] - want[fine]) <= (2.0 ** -24 * np.abs(want) + 2.0 ** -40 * size)[fine]).all()
            assert np.array_equal(np.where(fine, 0, x), np.where(fine, 0, want), equal_nan=True)
            kept = BO.kept(want.astype(np.float32), m, budget, sinks, recent)
            assert counts[b, h, 0] == len(kept) and np.array_equal(index[b, h, 0, : len(kept)], kept)


def signed(c, sign):
    """Queries of one sign in a dimension, whatever the head."""
    c.q = (c.q.abs() * sign).to(c.dt)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,H_kv,T,block", [(2, 2, 1024, 32), (8, 2, 20000, 32)])
@pytest.mark.parametrize("sign", [1, -1, 0])
def test_infinite_bounds(dtype, D, H, H_kv, T, block, sign):
    c = Choice(2, H, H_kv, T, D, block, dtype=dtype)
    if sign:
        signed(c, sign)
    n = c.n
    c.bounds[:, :, n // 4: n // 2, 1, 5] = INF               # keys of +inf among others
    c.bounds[:, :, n // 3: n // 2 + 3, 0, 7] = -INF          # of -inf
    c.bounds[:, :, n // 2 + 5, :, 9] = INF                   # nothing else
    c.bounds[:, :, n // 2 + 6, :, 11] = -INF
    c.bounds[:, :, n // 2 + 7, 0, 12], c.bounds[:, :, n // 2 + 7, 1, 12] = -INF, INF
    for budget in (1, 6, n // 2, n - 1):
        check(c, T, budget)


@pytest.mark.parametrize("sign", [1, -1, 0])
def test_blocks_without_rows_rank_last(sign):
    c = Choice(1, 4, 2, 1024, 64, 32)
    if sign:
        signed(c, sign)
    for j in (3, 4, 17):
        c.bounds[:, :, j, 0], c.bounds[:, :, j, 1] = INF, -INF
    for budget in (2, 20, 29, 30):
        check(c, 1024, budget)
    index, counts, got, _ = c.call([1024], None, 29, 0, 1)
    assert np.isneginf(got[0, :, 0, [3, 4, 17]]).all() and not np.isin(index[0, :, 0, :29], [3, 4, 17]).any()


def test_a_zero_query_wants_nothing_of_an_infinity():
    c = Choice(1, 2, 1, 1024, 64, 32)
    c.q[:, :, :, 5] = 0
    c.bounds[:, :, 7, 1, 5] = INF
    c.bounds[:, :, 9, 0, 5] = -INF
    check(c, 1024, 6)
    c.q[:] = 0
    check(c, 1024, 6)


@pytest.mark.parametrize("n_q", [411, 2 ** 31 - 200, 2 ** 31 - 1])
def test_bounds_of_more_tokens_than_there_are(n_q):
    """As many as 32 bits hold: all blocks are made anew."""
    c = Cache(2, 2, 411, 64, "bf16")
    got, status = bounds_of(c, 2, [411, 100], None, n_q, 64)
    want, _ = bounds_of(c, 2, [411, 100], None, 411, 64)
    assert status == 0 and np.array_equal(got, want) and (got[0] != 5).any()


def test_an_infinite_key_in_a_cache():
    """Bounds made of a cache with an infinite key, and chosen by queries of the other sign: its block ranks by its other values."""
    cache = Cache(1, 1, 512, 64, "bf16")
    cache.parts["k"][0, 0, 70, 3] = INF
    got, status = bounds_of(cache, 1, [512], None, 512, 32)
    assert got[0, 0, 2, 1, 3] == np.inf and np.isfinite(got[0, 0, 2, 0]).all() and status == 0
    c = Choice(1, 1, 1, 512, 64, 32)
    c.bounds = torch.tensor(got).to(torch.bfloat16)
    signed(c, -1)
    for budget in (3, 8, 15):
        check(c, 512, budget)
