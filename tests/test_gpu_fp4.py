"""ssa_attn_window_fp4 against 64 bits: the cases of ssa_attn_window over 4-bit values."""
import numpy as np
import pytest
import torch

from budget_util import half_step
from cache_util import Fp4Tokens, check_tokens, far_apart
from oracle import budget_oracle as BO
from paper_2404_09336_b200 import ssa

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def many(p):
    """Whether the tiles of 128 rows may serve the call."""
    return p.H // p.H_kv * p.n_q > 32


def shares(p):
    """Whether the seen part of the cache is converted once for all of the call's blocks, where there is room."""
    return p.H // p.H_kv * p.n_q > (256 if p.cache.page else 768)


def run(p, ctx, new=None, window=0, sinks=0, out_dtype=F32, **k):
    got = p.call(ctx, new, window, sinks, out_dtype, **k)
    check_tokens(p, got, ctx, new, window, sinks, out_dtype, many(p), shared=shares(p) and not k.get("less"), scale=k.get("scale") or None)
    return got


@pytest.mark.parametrize("D", [64, 128])
def test_every_code_and_scale_is_read_exactly(D):
    """One position: the output is its row of V, times a weight of 22 bits over the same weight of 24 (2^-22; the sum, 2^-24 of it, and
    the quotient's rounding make that 2^-21 at most)."""
    for seed in range(3):
        p = Fp4Tokens(4, 2, 2, 8, D, 1, seed=seed)
        scales = torch.randint(0, 256, (4, 2, 8, D // 16), generator=torch.Generator().manual_seed(seed)).to(torch.uint8)
        scales[(scales & 127) == 127] = 3
        p.cache.put("v_scales", scales)
        out, lse, _, status = p.call([8, 5, 2, 1], None, window=1)
        v = p.cache.values("v")
        for b, n in enumerate((8, 5, 2, 1)):
            assert (np.abs(out[b, :, 0] - v[b, :, n - 1]) <= 2.0 ** -21 * np.abs(v[b, :, n - 1])).all() and status == 0


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout", ["bhtd", "bthd", "spaced", 1, 4, 16, 64, 256])
def test_layouts(D, layout):
    page = layout if isinstance(layout, int) else 0
    for H, H_kv, n_q in ((4, 4, 1), (8, 2, 3), (4, 2, 30)):
        p = Fp4Tokens(3, H, H_kv, 300, D, n_q, layout="bhtd" if page else layout, page=page)
        run(p, [300, 177, 32], [n_q, max(1, n_q - 1), min(n_q, 2)])
        run(p, [300, 177, 32], None, window=50, sinks=3, out_dtype=BF16)


@pytest.mark.parametrize("n_q", [1, 2, 5, 16, 25, 33, 100, 129, 200])
@pytest.mark.parametrize("H,H_kv", [(1, 1), (8, 2), (12, 1)])
def test_tokens_and_heads(n_q, H, H_kv):
    p = Fp4Tokens(2, H, H_kv, 421, 128, n_q)
    run(p, [421, n_q], None)
    run(p, [400, 390], [n_q, (n_q + 1) // 2], window=130, sinks=17, out_dtype=BF16)
    run(p, [400, 390], [n_q, 0], window=1)


@pytest.mark.parametrize("window,sinks", [(0, 0), (1, 0), (1, 40), (31, 1), (32, 32), (64, 5), (127, 200), (128, 0), (1000, 1)])
@pytest.mark.parametrize("n_q", [3, 70])
def test_windows_and_sinks(window, sinks, n_q):
    run(Fp4Tokens(2, 4, 2, 500, 64, n_q, page=16), [500, 131], None, window, sinks)
    run(Fp4Tokens(2, 4, 2, 500, 128, n_q), [499, 129], [n_q, min(n_q, 9)], window, sinks, out_dtype=BF16)


@pytest.mark.parametrize("T", [1, 15, 16, 17, 31, 32, 33, 127, 128, 129, 1000, 5000])
def test_lengths(T):
    run(Fp4Tokens(2, 4, 2, T, 128, 1), [T, max(0, T // 2)])
    n_q = min(T, 40)
    run(Fp4Tokens(2, 4, 2, T, 64, n_q), [T, T], [n_q, 0])
    run(Fp4Tokens(2, 4, 2, T, 128, n_q), [T, T], [n_q, 1], out_dtype=BF16)


@pytest.mark.parametrize("n_q", [1, 4, 50])
def test_long_contexts_in_splits(n_q):
    run(Fp4Tokens(1, 8, 2, 16384, 128, n_q), [16384])
    run(Fp4Tokens(1, 2, 2, 9001, 64, n_q, page=64), [9001], out_dtype=BF16)


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout", ["spaced", 8, 16, 256])
@pytest.mark.parametrize("less", [0, 1])
def test_chunks_that_share_a_conversion(D, layout, less):
    """More than 256 rows a K/V head of a paged cache, 768 of another, with and without room for the seen part of it in bf16."""
    page = layout if isinstance(layout, int) else 0
    n = 60 if page else 160
    p = Fp4Tokens(3, 5, 1, 500, D, n, layout="bhtd" if page else layout, page=page)
    run(p, [500, 333, n], None, out_dtype=BF16 if less else F32, less=less)
    run(p, [477, 130, n - 10], [n, 5, 0], window=150, sinks=9, out_dtype=F32 if less else BF16, less=less)
    run(p, [499, 340, n], [n - 20, n, 1], window=128, sinks=200, less=less)
    run(p, [40, 0, n], [40, 0, n], window=5000, less=less)


@pytest.mark.parametrize("page", [0, 16])
@pytest.mark.parametrize("rows", [256, 257, 768, 769])
def test_rows_on_both_sides_of_a_shared_conversion(page, rows):
    p = Fp4Tokens(2, 1, 1, 900, 128, rows, page=page)
    run(p, [900, rows], [rows, rows - 1])
    run(p, [899, 700], [rows, 3], window=100, sinks=2, out_dtype=BF16)


def test_large_queries_and_scales():
    run(Fp4Tokens(2, 4, 2, 300, 128, 2, spread=30.0), [300, 200])
    run(Fp4Tokens(2, 4, 2, 300, 128, 40, spread=30.0), [300, 200], out_dtype=BF16)
    run(Fp4Tokens(2, 4, 2, 300, 128, 40, spread=1e-3), [300, 200], scale=0.7)


def test_tokens_of_negative_position_and_clamped_lengths():
    for n_q in (4, 60):
        p = Fp4Tokens(3, 4, 2, 90, 64, n_q)
        out, lse, _, status = p.call([2, 0, 95], [n_q, n_q, n_q + 5])
        assert status == ssa.DEV_BAD_COUNT
        assert not out[0, :, : n_q - 2].any() and np.isneginf(lse[0, :, : n_q - 2]).all() and np.isfinite(lse[0, :, n_q - 2:]).all()
        assert not out[1].any() and np.isneginf(lse[1]).all() and np.isfinite(lse[2]).all()


@pytest.mark.parametrize("n_q", [2, 40, 140])
def test_missing_pages(n_q):
    p = Fp4Tokens(2, 4, 2, 256, 128, n_q, page=16)
    table = p.cache.table.clone()
    table[0, 3], table[1, 0], table[1, 15] = -1, p.cache.n_pages, -9
    got = p.call([256, 230], [n_q, n_q], table=table)
    assert got[3] == ssa.DEV_BAD_INDEX
    gone = np.zeros((2, 256), bool)
    gone[0, 48:64] = gone[1, :16] = True
    check_tokens(p, got, [256, 230], [n_q, n_q], 0, 0, F32, tiles=many(p), skipped=gone)
    assert p.call([256, 230], [n_q, n_q], window=10, table=table)[3] == 0                # (no token sees them)


@pytest.mark.parametrize("n_q", [2, 40])
@pytest.mark.parametrize("out_dtype", [BF16, F32])
def test_nan_scales_reach_the_tokens_that_see_them(n_q, out_dtype):
    p = Fp4Tokens(1, 4, 2, 200, 128, n_q)
    want = p.call([150], None, window=60, out_dtype=out_dtype)
    for row in (20, 150, 199):                               # before every window; behind the context
        for name in ("k_scales", "v_scales"):
            p.cache.parts[name][0, :, row] = 0xff
    got = p.call([150], None, window=60, out_dtype=out_dtype)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
    p.cache.parts["v_scales"][0, 1, 150 - n_q - 60, 2] = 0x7f        # just in front of the first token's window; then in it
    got = p.call([150], None, window=60, out_dtype=out_dtype)
    assert np.array_equal(got[0], want[0])
    p.cache.parts["v_scales"][0, 1, 150 - n_q - 59, 2] = 0x7f
    out = p.call([150], None, window=60, out_dtype=out_dtype)[0]
    assert np.isnan(out[0, 2:, 0, 32:48]).all() and np.isfinite(out[0, 2:, 0, :32]).all() and np.isfinite(out[0, :2]).all()
    # the other tokens' rows of that head may be made once more, in fp32, by then
    p.cache.parts["v_scales"][0, 1, 150 - n_q - 59, 2] = 0
    assert np.array_equal(out[0, :2], want[0][0, :2])
    q, k, v = p.values()
    ref = BO.attention(q, k, v, [150], [n_q], 60, 0, 128 ** -0.5)[0]
    # weights off by 2^-11 and scores by D 2^-24 of theirs, below another 2^-11, in numerator and denominator; the output's rounding
    tol = 4 * 2.0 ** -11 * ref["spread"] + half_step(out_dtype) * np.abs(ref["out"])
    assert 130 * ref["score"] * 2.0 ** -24 < 2.0 ** -11 and (np.abs(out[0, 2:, 1:] - ref["out"][2:, 1:]) <= tol[2:, 1:]).all()


def test_nan_scales_in_a_chunk_that_shares_a_conversion():
    p = Fp4Tokens(1, 4, 2, 500, 64, 150)
    want = p.call([400], None, window=60, out_dtype=BF16)
    for row in (20, 400, 499):                               # before every window; behind the context
        for name in ("k_scales", "v_scales"):
            p.cache.parts[name][0, :, row] = 0xff
    got = p.call([400], None, window=60, out_dtype=BF16)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
    p.cache.parts["v_scales"][0, 1, 300, 3] = 0x7f           # tokens at 300 ... 359 see it
    out = p.call([400], None, window=60, out_dtype=BF16)[0]
    assert np.isnan(out[0, 2:, 50:110, 48:]).all() and np.isfinite(out[0, 2:, 50:110, :48]).all()
    assert np.isfinite(out[0, 2:, :50]).all() and np.isfinite(out[0, 2:, 110:]).all() and np.array_equal(out[0, :2], want[0][0, :2])


@pytest.mark.parametrize("n_q", [2, 40, 400])
def test_offsets_past_32_bits(n_q):
    """Codes of the second request lie beyond 2^32 values, scales beyond 2^28 bytes."""
    T = max(70, n_q)
    p = Fp4Tokens(2, 4, 2, T, 128, n_q)
    far_apart(p.cache)
    run(p, [T, T])
