"""ssa_attn_window_fp4 where many rows share a conversion: what depends on it, and what does not."""
import numpy as np
import pytest
import torch

from budget_util import DEV
from cache_util import Fp4Tokens, check_tokens
from paper_2404_09336_b200 import ssa

pytestmark = pytest.mark.gpu
BF16, F32 = torch.bfloat16, torch.float32


def least_room(p, *args):
    """Most bytes that the call may have less than it asks for (calls with less still are refused before anything is launched)."""
    desc, win = p.cache.desc(p.q, p.q), ssa.make_window(p.q, p.q, *args[2:4], None, p.cache.paging())
    taken, refused = 0, ssa.attn_window_fp4_workspace_bytes(desc, win)
    while refused - taken > 1:
        less = (taken + refused) // 2
        try:
            p.call(*args, less=less)
            taken = less
        except ssa.SsaError:
            refused = less
    return taken


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("page", [0, 8, 64])
@pytest.mark.parametrize("out_dtype", [BF16, F32])
def test_bits_do_not_depend_on_the_workspace(D, page, out_dtype):
    """Weights keep the bits of the calls of fewer rows, whether the call has room to convert once, in parts, or converts in every
    block."""
    n = 70 if page else 200
    p = Fp4Tokens(2, 8, 2, 900, D, n, page=page, spread=2.0)
    for ctx, new, window, sinks in (([900, 641], None, 0, 0), ([877, 300], [n, n - 30], 150, 9)):
        got, launches = [], []
        for less in (0, 1, least_room(p, ctx, new, window, sinks, out_dtype)):
            before = ssa.launch_count()
            got.append(p.call(ctx, new, window, sinks, out_dtype, less=less))
            launches.append(ssa.launch_count() - before)
        # conversion, tiles, a join perhaps; parts of a request, or of a head, each; no conversion
        assert launches[0] in (2, 3) and launches[1] >= 2 * launches[0] and launches[2] == launches[0] - 1, launches
        for x in got:
            assert np.array_equal(x[0], got[0][0]) and np.array_equal(x[1], got[0][1]) and x[3] == 0
        check_tokens(p, got[0], ctx, new, window, sinks, out_dtype, tiles=True)


@pytest.mark.parametrize("page,n_q", [(0, 400), (16, 150)])
@pytest.mark.parametrize("out_dtype", [BF16, F32])
def test_nan_scales_through_the_conversion(page, n_q, out_dtype):
    """More than 768 rows a K/V head, 256 in pages: a NaN scale reaches the tokens that see its row, nothing else."""
    T = n_q + 100
    p = Fp4Tokens(1, 4, 2, T, 64, n_q, page=page)
    ctx, first = T - 10, T - 10 - n_q                        # of positions first ... ctx - 1
    assert 2 * n_q > (256 if page else 768)
    row = (lambda j: (int(p.cache.table[0, j // page]), j % page)) if page else None

    def put(name, j, scale, h=slice(None), part=slice(None)):
        x = p.cache.parts[name]
        if page:
            x[row(j)[0], row(j)[1], h, part] = scale
        else:
            x[0, h, j, part] = scale

    want = p.call([ctx], None, window=60, out_dtype=out_dtype)
    for j in (first - 65, ctx, T - 1):                       # before every window; behind the context
        for name in ("k_scales", "v_scales"):
            put(name, j, 0xff)
    got = p.call([ctx], None, window=60, out_dtype=out_dtype)
    assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1])
    put("v_scales", first + 50, 0x7f, 1, 3)                  # tokens 50 ... 109 see it
    got = p.call([ctx], None, window=60, out_dtype=out_dtype)[0]
    assert np.isnan(got[0, 2:, 50:110, 48:]).all() and np.isfinite(got[0, 2:, 50:110, :48]).all()
    assert np.isfinite(got[0, 2:, :50]).all() and np.isfinite(got[0, 2:, 110:]).all() and np.array_equal(got[0, :2], want[0][0, :2])
    put("k_scales", first + 20, 0x7f, 0, 1)                  # scores of tokens 20 ... 79 of the other head
    got, lse = p.call([ctx], None, window=60, out_dtype=out_dtype)[:2]
    assert np.isnan(got[0, :2, 20:80]).all() and np.isnan(lse[0, :2, 20:80]).all()
    assert np.isfinite(got[0, :2, :20]).all() and np.isfinite(got[0, :2, 80:]).all() and np.isfinite(lse[0, :2, 80:]).all()


@pytest.mark.parametrize("page", [0, 16])
def test_scales_of_every_size_through_the_conversion(page):
    """One position a token sees: its row of V, every code and scale, times a weight of 22 bits over one of 24."""
    n_q = 400 if not page else 150
    p = Fp4Tokens(1, 2, 1, n_q, 64, n_q, page=page)
    scales = (torch.arange(n_q * 4) * 37 % 256).to(torch.uint8).view(1, 1, n_q, 4)
    scales[(scales & 127) == 127] = 3
    p.cache.put("v_scales", scales)
    out = p.call([n_q], None, window=1)[0]
    v = p.cache.values("v")
    assert (np.abs(out[0] - v[0]) <= 2.0 ** -21 * np.abs(v[0])).all()


def test_timing_events_bracket_the_conversion():
    """Many rows that are converted for few that attend to them, nothing to join: between the events lies all of the call."""
    B, T = 100, 2048
    p = Fp4Tokens(B, 264, 1, T, 128, 1, page=256)
    out, ctx = torch.zeros_like(p.q), torch.full((B,), T, dtype=torch.int32, device=DEV)
    c, share = p.cache, []
    desc, win = c.desc(p.q, out), ssa.make_window(p.q, out, paging=c.paging())
    ws = torch.empty(ssa.attn_window_fp4_workspace_bytes(desc, win), dtype=torch.uint8, device=DEV)
    for _ in range(20):
        a, b, y, z = (torch.cuda.Event(enable_timing=True) for _ in range(4))
        for e in (b, y):
            e.record()                                       # (made by then)
        torch.cuda.synchronize()
        ssa.set_kernel_events(b, y)
        before = ssa.launch_count()
        a.record()
        ssa.attn_window_fp4(desc, win, p.q, c.parts["k"], c.parts["v"], c.scales("k"), c.scales("v"), ctx, out, None, ws)
        z.record()
        torch.cuda.synchronize()
        assert ssa.launch_count() - before == 2              # conversion, tiles
        share.append(b.elapsed_time(y) / a.elapsed_time(z))
    assert max(share) > 0.85, share                          # (the tiles alone: 0.7)


def in_parts(p, T, ctx, new, window, sinks, out_dtype, less=0):
    """The call as one of a cache with room for T positions, of which there are as many as p has."""
    c, was, table = p.cache, p.cache.T, None
    if c.page:
        table = torch.full((p.B, T // c.page), -1, dtype=torch.int32)
        table[:, : c.table.shape[1]] = c.table
    c.T = T
    try:
        return p.call(ctx, new, window, sinks, out_dtype, table=table, less=less)
    finally:
        c.T = was


@pytest.mark.parametrize("B,T", [(5, 1 << 18), (2, 1 << 20), (3, 1 << 21), (2, 1 << 22)])
@pytest.mark.parametrize("page", [0, 16])
def test_requests_and_heads_in_turn(B, T, page):
    """Room for 512 MB of converted rows: 64, 256, 512 and 1024 MB a K/V head here, three heads.  Requests two at a time, and one left;
    heads two at a time; each by itself; none at all."""
    n_q = 150 if page else 400
    p = Fp4Tokens(B, 6, 3, n_q + 90, 64, n_q, page=page)
    ctx, new = [n_q + 90, n_q + 3, 40, 0, n_q][:B], [n_q, n_q - 1, 40, 0, 5][:B]
    for out_dtype, window, sinks in ((F32, 0, 0), (BF16, 0, 0)):
        want = p.call(ctx, new, window, sinks, out_dtype)
        check_tokens(p, want, ctx, new, window, sinks, out_dtype, tiles=True)
        before = ssa.launch_count()
        got = in_parts(p, T, ctx, new, window, sinks, out_dtype)
        launches = ssa.launch_count() - before
        assert launches >= {1 << 18: 2 * 3, 1 << 20: 2 * 2 * B, 1 << 21: 2 * 3 * B, 1 << 22: 1}[T]
        assert np.array_equal(got[0], want[0]) and np.array_equal(got[1], want[1]) and got[3] == want[3] == 0


@pytest.mark.parametrize("page", [0, 64])
def test_parts_that_are_split(page):
    """One K/V head at a time is few blocks for the GPU: long contexts are cut, and joined part by part."""
    n_q = 300 if page else 800
    p = Fp4Tokens(2, 2, 2, 6000, 64, n_q, page=page)
    for ctx, new, out_dtype in (([6000, 4100], None, F32), ([5999, 900], [n_q, 7], BF16)):
        got = in_parts(p, 1 << 21, ctx, new, 0, 0, out_dtype)
        check_tokens(p, got, ctx, new, 0, 0, out_dtype, tiles=True)
