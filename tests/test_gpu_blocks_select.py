"""ssa_block_bounds and ssa_block_select against the oracle: bounds and lists exactly, scores to their rounding."""
import numpy as np
import pytest
import torch

from budget_util import DEV
from cache_util import DTYPES, Cache, far_apart, query_type
from oracle import budget_oracle as BO
from oracle import cache_oracle as CO
from paper_2404_09336_b200 import ssa

pytestmark = pytest.mark.gpu


def i32(x):
    return None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)


def bounds_of(c, H, ctx, new, n_q, block, table=None, fill=5.0):
    n = -(-c.T // block)
    got = torch.full((c.B, c.H_kv, n, 2, c.D), fill, dtype=query_type(c.dtype), device=DEV)
    q = torch.zeros(c.B, H, 1, c.D, dtype=got.dtype, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    d_ctx, d_new = i32(ctx), i32(new)
    k = ssa.make_blocks(n_q, block, 1, bounds=got, q_lens=d_new, paging=c.paging(table))
    ssa.block_bounds(c.desc(q, q), k, c.parts["k"], d_ctx, got, c.scales("k"), status)
    torch.cuda.synchronize()
    return got.cpu().double().numpy(), int(status)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("block", [32, 64, 128, 256])
@pytest.mark.parametrize("layout", ["bhtd", "bthd", "spaced", "paged"])
def test_bounds(dtype, D, block, layout):
    page = 16 if layout == "paged" else 0
    c = Cache(4, 3, 411, D, dtype, "bhtd" if page else layout, page, seed=block)
    ctx, K = [411, 256, 33, 0], c.values("k")
    for new, n_q in ((None, 411), ([411, 500, 33, 7], 411), (None, 1), ([70, 1, 0, 3], 70), ([1, 65, 33, 1], 65)):
        got, status = bounds_of(c, 3, ctx, new, n_q, block)
        for b in range(4):
            t = n_q if new is None else min(new[b], n_q)
            lo = max(0, ctx[b] - t) // block if t else 99
            for h in range(3):
                if ctx[b] and t:
                    least, most = CO.bounds(K[b, h], ctx[b], block)
                    assert np.array_equal(got[b, h, lo: len(least), 0], least[lo:]) and np.array_equal(got[b, h, lo: len(most), 1], most[lo:])
                    assert (got[b, h, :lo] == 5).all() and (got[b, h, len(least):] == 5).all()
                else:
                    assert (got[b, h] == 5).all()
        assert status == (ssa.DEV_BAD_COUNT if new and max(new) > n_q else 0)


@pytest.mark.parametrize("dtype", DTYPES)
def test_bounds_over_missing_pages_and_nan(dtype):
    c = Cache(2, 2, 128, 64, dtype, page=16)
    table = c.table.clone()
    table[0, 1], table[1, 2:4], table[1, 6] = -1, c.n_pages, 2 ** 31 - 1
    K = c.values("k")
    got, status = bounds_of(c, 2, [128, 128], None, 128, 32, table)
    assert status == ssa.DEV_BAD_INDEX
    for b, gone in ((0, [(16, 32)]), (1, [(32, 64), (96, 112)])):
        there = np.ones(128, bool)
        for lo, hi in gone:
            there[lo:hi] = False
        for j in range(4):
            rows = K[b, :, 32 * j: 32 * j + 32][:, there[32 * j: 32 * j + 32]]
            assert np.array_equal(got[b, :, j, 0], rows.min(1, initial=np.inf)) and np.array_equal(got[b, :, j, 1], rows.max(1, initial=-np.inf))
    if dtype in ("bf16", "f16"):
        c = Cache(1, 1, 64, 64, dtype)
        c.parts["k"][0, 0, 40, 7], c.parts["k"][0, 0, 5, 3] = float("nan"), float("inf")
        got, _ = bounds_of(c, 1, [64], None, 64, 32)
        assert np.isnan(got[0, 0, 1, :, 7]).all() and np.isfinite(got[0, 0, 1, :, :7]).all() and got[0, 0, 0, 1, 3] == np.inf
        assert np.isfinite(got[0, 0, 0, 0, 3])


class Choice:
    """Bounds and queries, and the calls on them."""

    def __init__(self, B, H, H_kv, T, D, block, n_q=1, dtype="bf16", seed=0, layout="bhtd"):
        g = torch.Generator().manual_seed(seed)
        self.__dict__.update(B=B, H=H, H_kv=H_kv, T=T, D=D, block=block, n_q=n_q, n=-(-T // block), dt=query_type(dtype))
        a, z = (torch.randn(B, H_kv, self.n, D, generator=g) for _ in range(2))
        self.bounds = torch.stack([torch.minimum(a, z), torch.maximum(a, z)], 3).to(self.dt)
        self.q = torch.randn(B, n_q, H, D, generator=g).to(self.dt).permute(0, 2, 1, 3)
        self.layout = layout

    def call(self, ctx, new, budget, sinks, recent, with_scores=True, stream=None):
        d_q, d_ctx, d_new = self.q.to(DEV), i32(ctx), i32(new)
        bounds = self.bounds.to(DEV)
        if self.layout == "spaced":                          # heads and requests apart
            room = torch.zeros(self.B, self.H_kv + 1, self.n + 3, 2, self.D, dtype=self.dt, device=DEV)[:, : self.H_kv, : self.n]
            bounds = room.copy_(bounds)
        index = torch.full((self.B, self.H_kv, self.n_q, budget), -7, dtype=torch.int32, device=DEV)
        counts = torch.full((self.B, self.H_kv, self.n_q), -7, dtype=torch.int32, device=DEV)
        scores = torch.full((self.B, self.H_kv, self.n_q, self.n), 777.0, device=DEV) if with_scores else None
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        k_dummy = d_q.new_zeros(1, 1, 1, self.D).expand(self.B, self.H_kv, self.T, self.D)
        desc = ssa.make_desc(d_q[:, :, 0], k_dummy, k_dummy, d_q[:, :, 0])
        k = ssa.make_blocks(self.n_q, self.block, budget, sinks, recent, q=d_q, bounds=bounds, q_lens=d_new)
        torch.cuda.synchronize()
        ssa.block_select(desc, k, d_q, bounds, d_ctx, index, counts, scores, status, stream)
        torch.cuda.synchronize()
        return index.cpu().numpy(), counts.cpu().numpy(), None if scores is None else scores.cpu().numpy(), int(status)

    def check(self, ctx, new=None, budget=8, sinks=1, recent=1, with_scores=True):
        index, counts, scores, status = self.call(ctx, new, budget, sinks, recent, with_scores)
        q, least, most = self.q.double().numpy(), *(self.bounds[:, :, :, i].double().numpy() for i in (0, 1))
        group = self.H // self.H_kv
        for b in range(self.B):
            t = self.n_q if new is None else min(new[b], self.n_q)
            for h in range(self.H_kv):
                for i in range(self.n_q):
                    pos = min(ctx[b], self.T) - t + i
                    if i >= t or pos < 0:
                        assert counts[b, h, i] == -7 and (index[b, h, i] == -7).all() and (scores is None or (scores[b, h, i] == 777).all())
                        continue
                    m = pos // self.block + 1
                    with np.errstate(invalid="ignore"):
                        s = CO.scores(q[b, h * group: (h + 1) * group, i], least[b, h, :m], most[b, h, :m])
                    if scores is not None:
                        # 2 D exact products summed in 64 bits, in any order, and rounded to 32
                        size = (np.abs(q[b, h * group: (h + 1) * group, i]).sum(0) * np.maximum(np.abs(least[b, h, :m]), np.abs(most[b, h, :m]))).sum(1)
                        with np.errstate(invalid="ignore"):
                            assert (np.abs(scores[b, h, i, :m] - s) <= 2.0 ** -24 * np.abs(s) + 2.0 ** -40 * size)[np.isfinite(s)].all()
                        assert np.array_equal(np.isnan(s), np.isnan(scores[b, h, i, :m])) and (scores[b, h, i, m:] == 777).all()
                    with np.errstate(over="ignore"):
                        kept = BO.kept(s.astype(np.float32), m, budget, sinks, recent)
                    assert counts[b, h, i] == len(kept) and np.array_equal(index[b, h, i, : len(kept)], kept)
                    assert (index[b, h, i, len(kept):] == -7).all()
        return status


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("H,H_kv", [(1, 1), (8, 8), (32, 8), (12, 1)])
def test_lists(dtype, D, H, H_kv):
    c = Choice(3, H, H_kv, 1000, D, 32, dtype=dtype)
    for budget, sinks, recent in ((8, 1, 1), (1, 0, 0), (5, 2, 3), (31, 0, 1), (32, 1, 1), (100, 3, 4), (6, 0, 0)):
        assert c.check([1000, 517, 1], None, budget, sinks, recent) == 0


@pytest.mark.parametrize("T,block", [(33, 32), (4096, 32), (9000, 64), (70000, 32), (70001, 128), (500000, 32), (524288, 32)])
def test_long_contexts(T, block):
    """One to eight thread blocks a token, up to the most blocks that there may be."""
    c = Choice(2, 4, 2, T, 64, block)
    n = -(-T // block)
    for budget in sorted({1, max(1, n // 3), n}):
        c.check([T, max(1, T // 2 + 1)], None, budget, min(2, budget // 2), budget - budget // 2 and 1)


def test_several_tokens_and_ragged_lengths():
    c = Choice(4, 8, 2, 700, 64, 32, n_q=7, layout="spaced")
    assert c.check([700, 95, 3, 0], [7, 4, 7, 5], 4, 1, 2) == 0
    assert c.check([700, 95, 3, 0], None, 30, 0, 0, with_scores=False) == 0
    assert c.check([701, 95, 64, 1], [9, 0, 1, 1], 2, 0, 0) == ssa.DEV_BAD_COUNT


def test_equal_scores_go_to_the_lowest_blocks():
    c = Choice(1, 2, 1, 2048, 64, 32)
    c.bounds[:, :, 3:60] = c.bounds[:, :, 3:4]
    for budget in (1, 5, 20, 40, 63):
        c.check([2048], None, budget, min(1, budget - 1), 0)
    c.bounds[:] = 0
    c.check([2048], None, 17, 1, 4)
    c.q[:] = 0
    c.check([1999], None, 17, 0, 0)


@pytest.mark.parametrize("dtype", ["bf16", "f16"])
@pytest.mark.parametrize("D", [64, 128])
def test_scores_that_fp32_sums_do_not_tell_apart(dtype, D):
    """Blocks that differ in one value, by less and less: down to ties after rounding, whatever the order of summation."""
    for seed, (T, block) in enumerate(((2048, 32), (20000, 64), (40000, 32))):
        c = Choice(2, 8, 2, T, D, block, dtype=dtype, seed=seed)
        n = c.n
        c.bounds[:, :, 2:] = c.bounds[:, :, 2:3]
        steps = 2.0 ** -(torch.arange(n - 2) % 23) * (1 + (torch.arange(n - 2) % 7) / 8)
        c.bounds[:, :, 2:, 1, 5] = steps.to(c.dt)
        c.bounds[:, :, 2:, 0, 5] = -1
        for budget in (1, 7, n // 3, n - 1):
            c.check([T, T - 700], None, budget, min(1, budget - 1), 0, with_scores=seed == 0)


def test_scores_beyond_fp32():
    c = Choice(1, 2, 1, 2048, 64, 32)
    c.bounds[:, :, 3:30] *= 2.0 ** 100
    c.q *= 2.0 ** 30                                         # sums of 2^130: infinite after rounding, of either sign
    c.check([2048], None, 20, 1, 1, with_scores=False)
    c.bounds[:], c.q[:] = c.bounds * 2.0 ** -60, c.q * 2.0 ** -130
    c.check([2048], None, 20, 1, 1, with_scores=False)


def test_nan_ranks_below_everything():
    c = Choice(1, 2, 1, 2048, 64, 32)
    c.bounds[0, 0, 5:55, 1, 9] = float("nan")
    c.check([2048], None, 20, 1, 1)
    c.q[0, 1, 0, 3] = float("nan")
    c.check([2048], None, 20, 1, 1)


def test_scores_need_not_be_asked_for():
    c = Choice(2, 8, 4, 3000, 128, 64)
    with_them, without = c.call([3000, 1234], None, 9, 1, 1), c.call([3000, 1234], None, 9, 1, 1, with_scores=False)
    assert np.array_equal(with_them[0], without[0]) and np.array_equal(with_them[1], without[1])


@pytest.mark.parametrize("dtype", DTYPES)
def test_keys_past_32_bits(dtype):
    c = far_apart(Cache(2, 2, 100, 128, dtype))
    got, status = bounds_of(c, 2, [100, 70], None, 100, 32)
    K = c.values("k")
    for b, n in ((0, 100), (1, 70)):
        for h in range(2):
            least, most = CO.bounds(K[b, h], n, 32)
            assert np.array_equal(got[b, h, : len(least), 0], least) and np.array_equal(got[b, h, : len(most), 1], most)
    assert status == 0
