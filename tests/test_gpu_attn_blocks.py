"""ssa_attn_blocks against attention over the listed positions in 64 bits."""
import numpy as np
import pytest
import torch

from budget_util import DEV, UNWRITTEN
from cache_util import DTYPES, Cache, check_rows, far_apart, query_type
from oracle import cache_oracle as CO
from paper_2404_09336_b200 import ssa

pytestmark = pytest.mark.gpu


class Lists:
    """Queries over a cache, and a list of blocks for every token and K/V head."""

    def __init__(self, B, H, H_kv, T, D, block, budget, n_q=1, dtype="bf16", layout="bhtd", page=0, seed=0):
        self.c = Cache(B, H_kv, T, D, dtype, layout, page, seed)
        self.__dict__.update(B=B, H=H, H_kv=H_kv, T=T, D=D, block=block, budget=budget, n_q=n_q, dtype=dtype, dt=query_type(dtype))
        g = torch.Generator().manual_seed(seed + 7)
        self.q = torch.randn(B, n_q, H, D, generator=g).to(self.dt).to(DEV).permute(0, 2, 1, 3)
        self.rng = np.random.default_rng(seed)

    def lists(self, ctx, new, count=None):
        """Random ascending blocks that each token sees."""
        index = np.full((self.B, self.H_kv, self.n_q, self.budget), -3, np.int32)
        counts = np.zeros((self.B, self.H_kv, self.n_q), np.int32)
        for b in range(self.B):
            t = self.n_q if new is None else min(new[b], self.n_q)
            for h in range(self.H_kv):
                for i in range(t):
                    m = (ctx[b] - t + i) // self.block + 1
                    n = min(m, self.budget if count is None else count)
                    index[b, h, i, :n] = np.sort(self.rng.choice(m, n, replace=False)) if m > 0 else 0
                    counts[b, h, i] = n
        return index, counts

    def call(self, ctx, new, index, counts, out_dtype=torch.float32, table=None, stream=None):
        c = self.c
        i32 = lambda x: None if x is None else torch.tensor(x, dtype=torch.int32, device=DEV)
        d_ctx, d_new, d_index, d_counts = i32(ctx), i32(new), i32(index), i32(counts)
        out = torch.full((self.B, self.n_q, self.H, self.D), UNWRITTEN, dtype=out_dtype or self.dt, device=DEV).permute(0, 2, 1, 3)
        lse = torch.full((self.B, self.H, self.n_q), UNWRITTEN, device=DEV)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        desc = c.desc(self.q, out)
        k = ssa.make_blocks(self.n_q, self.block, self.budget, q=self.q, out=out, q_lens=d_new, paging=c.paging(table))
        ws = torch.full((ssa.attn_blocks_workspace_bytes(desc, k),), 0xff, dtype=torch.uint8, device=DEV)
        torch.cuda.synchronize()
        ssa.attn_blocks(desc, k, self.q, c.parts["k"], c.parts["v"], d_ctx, d_index, d_counts, out, lse, c.scales("k"), c.scales("v"), ws, status,
                        stream)
        torch.cuda.synchronize()
        return out.double().cpu().numpy(), lse.double().cpu().numpy(), int(status)

    def check(self, ctx, new=None, out_dtype=torch.float32, index=None, counts=None):
        if index is None:
            index, counts = self.lists(ctx, new)
        out, lse, status = self.call(ctx, new, index, counts, out_dtype)
        q, K, V, group = self.q.cpu().double().numpy(), self.c.values("k"), self.c.values("v"), self.H // self.H_kv
        for b in range(self.B):
            t = self.n_q if new is None else min(new[b], self.n_q)
            assert (out[b, :, t:] == UNWRITTEN).all() and (lse[b, :, t:] == UNWRITTEN).all()
            for h in range(self.H_kv):
                heads = slice(h * group, (h + 1) * group)
                for i in range(t):
                    pos = ctx[b] - t + i
                    blocks = [j for j in index[b, h, i, : max(0, min(counts[b, h, i], self.budget))].tolist() if 0 <= j and j * self.block <= pos]
                    rows = np.array([x for j in blocks for x in range(j * self.block, min((j + 1) * self.block, pos + 1))], int)
                    want = CO.attention(q[b, heads, i], K[b, h], V[b, h], rows, self.D ** -0.5)
                    check_rows(out[b, heads, i], lse[b, heads, i], want, self.D, len(rows), self.dtype, out_dtype or self.dt, np.abs(V).max())
        return status


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout", ["bhtd", "bthd", "spaced", 4, 16, 64, 128])
@pytest.mark.parametrize("block", [32, 128])
def test_types_and_layouts(dtype, D, layout, block):
    page = layout if isinstance(layout, int) else 0
    p = Lists(3, 8, 2, 700, D, block, 4, dtype=dtype, layout="bhtd" if page else layout, page=page)
    assert p.check([700, 333, 1], out_dtype=None) == 0
    assert p.check([641, 96, 31]) == 0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("H,H_kv", [(1, 1), (4, 4), (8, 1), (9, 1), (24, 2), (34, 2), (80, 2)])
def test_heads(dtype, H, H_kv):
    assert Lists(2, H, H_kv, 300, 64, 64, 3, dtype=dtype).check([300, 170]) == 0
    assert Lists(2, H, H_kv, 300, 128, 64, 3, n_q=2, dtype=dtype).check([300, 170], [2, 1], out_dtype=None) == 0


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("block,budget", [(32, 1), (32, 70), (64, 45), (256, 11), (256, 12)])
def test_long_lists(dtype, block, budget):
    """Lists of more than the 32 blocks that a warp looks at together, in splits."""
    assert Lists(1, 4, 2, 2900, 128, block, budget, n_q=2, dtype=dtype).check([2900]) == 0
    assert Lists(2, 2, 2, 2900, 64, block, budget, dtype=dtype, page=64).check([2817, 2899]) == 0


def test_many_tokens_with_lists_of_their_own():
    p = Lists(3, 4, 2, 500, 64, 32, 5, n_q=40, layout="bthd")
    assert p.check([500, 20, 333], [40, 20, 7]) == 0


@pytest.mark.parametrize("dtype", ["bf16", "fp4"])
def test_lists_that_are_empty_wrong_or_repeated(dtype):
    p = Lists(1, 4, 2, 400, 64, 32, 6, n_q=3, dtype=dtype)
    index, counts = p.lists([400], None)
    counts[0, 0, 0], counts[0, 1, 2] = 0, -5                  # empty
    assert p.check([400], index=index, counts=counts) == 0
    index[0, 0, 1] = [12, 3, 3, 0, 12, 7]                    # out of order, twice
    counts[0, 0, 1] = 6
    assert p.check([400], index=index, counts=counts) == 0
    index[0, 1, 1, :4], counts[0, 1, 1] = [-1, 13, 2 ** 31 - 1, 5], 4        # no such blocks
    assert p.check([400], index=index, counts=counts) == ssa.DEV_BAD_INDEX
    index, counts = p.lists([400], None)
    counts[0, 0, 0] = 7
    assert p.check([400], index=index, counts=counts) == ssa.DEV_BAD_COUNT
    index[:], counts[:] = 99, 6
    out, lse, status = p.call([400], None, index, counts)
    assert not out.any() and np.isneginf(lse).all() and status == ssa.DEV_BAD_INDEX


@pytest.mark.parametrize("dtype", DTYPES)
def test_missing_pages(dtype):
    p = Lists(1, 4, 2, 256, 64, 64, 4, dtype=dtype, page=16)
    index, counts = p.lists([256], None)
    table = p.c.table.clone()
    table[0, 5], table[0, 9] = -1, p.c.n_pages
    out, lse, status = p.call([256], None, index, counts, table=table)
    assert status == ssa.DEV_BAD_INDEX
    there = [x for x in range(256) if x // 16 not in (5, 9)]
    for h in range(2):
        want = CO.attention(p.q.cpu().double().numpy()[0, 2 * h: 2 * h + 2, 0], p.c.values("k")[0, h], p.c.values("v")[0, h], np.array(there), 0.125)
        check_rows(out[0, 2 * h: 2 * h + 2, 0], lse[0, 2 * h: 2 * h + 2, 0], want, 64, len(there), dtype, torch.float32,
                   np.abs(p.c.values("v")).max())


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 128])
def test_infinities_and_nan_reach_the_tokens_that_see_them(dtype, D):
    p = Lists(1, 2, 1, 128, D, 32, 2, n_q=2, dtype=dtype)
    index, counts = np.array([[[[0, 3], [1, 3]]]], np.int32), np.full((1, 1, 2), 2, np.int32)
    want, want_lse, _ = p.call([127], None, index, counts)
    if dtype == "fp4":
        for name in "kv":
            for row in (40, 70, 127):                        # seen by token 1; on no list; behind both
                p.c.parts[name + "_scales"][0, 0, row, 1] = 0x7f
    else:
        for name in "kv":
            x = p.c.parts[name][0, 0].view(torch.uint8 if dtype == "fp8" else torch.int16)
            x[40, 17], x[70], x[127] = 0x7f, 0x7f if dtype == "fp8" else 0x7fff, 0x7f if dtype == "fp8" else 0x7fff
            if dtype != "fp8":
                x[40, 17] = 0x7fff
    out, lse, status = p.call([127], None, index, counts)
    assert status == 0
    assert np.array_equal(out[0, :, 0], want[0, :, 0]) and np.array_equal(lse[0, :, 0], want_lse[0, :, 0])
    assert np.isnan(out[0, :, 1]).all() and np.isnan(lse[0, :, 1]).all()           # a NaN key is one in every weight
    p.c.put("k", torch.zeros(1, 1, 128, D // 2, dtype=torch.uint8) if dtype == "fp4" else torch.zeros(1, 1, 128, D).to(p.c.parts["k"].dtype))
    if dtype == "fp4":
        p.c.put("k_scales", torch.zeros(1, 1, 128, D // 16, dtype=torch.uint8))
    out, lse, _ = p.call([127], None, index, counts)
    seen = np.zeros(D, bool)
    seen[16:32 if dtype == "fp4" else 17] = dtype == "fp4"
    seen[17] = True
    assert np.isfinite(out[0, :, 0]).all() and np.isfinite(lse).all()
    assert np.isnan(out[0, :, 1, seen]).all() and np.isfinite(out[0, :, 1, ~seen]).all()


@pytest.mark.parametrize("dtype", DTYPES)
def test_offsets_past_32_bits(dtype):
    p = Lists(2, 4, 2, 200, 128, 32, 3, dtype=dtype)
    far_apart(p.c)
    assert p.check([200, 150]) == 0
