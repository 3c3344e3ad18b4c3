"""ssa_attn_window against fp64: types, layouts, lengths from none to long, windows, sinks, rows that see nothing."""
import numpy as np
import pytest
import torch

from paper_2404_09336_b200 import ssa

from budget_util import DEV, Tokens, check

pytestmark = pytest.mark.gpu


def run(p, ctx, q_lens=None, window=0, sinks=0, out_dtype=torch.float32, many=False, **more):
    got = p.call(ctx, q_lens, window, sinks, out_dtype, **more)
    check(p, got, ctx, q_lens, window, sinks, out_dtype or p.dt_q, many)
    return got


@pytest.mark.parametrize("dtype", ["bf16", "f16", "fp8"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout", ["bhtd", "bthd", "paged"])
def test_one_token(dtype, D, layout):
    p = Tokens(3, 4, 4, 333, D, 1, dtype, layout, page=16 if layout == "paged" else 0)
    for ctx in ([333, 1, 17], [0, 200, 16]):
        for window, sinks in ((0, 0), (1, 0), (1, 1), (33, 5), (100, 300), (1000, 0), (16, 16)):
            run(p, ctx, None, window, sinks)
    run(p, [333, 1, 17], None, 40, 3, out_dtype=None)


@pytest.mark.parametrize("dtype,H,H_kv,n_q", [("bf16", 8, 2, 2), ("f16", 4, 4, 5), ("fp8", 8, 2, 3), ("bf16", 6, 2, 16),
                                              ("f16", 16, 1, 1), ("bf16", 24, 1, 1), ("fp8", 5, 1, 7), ("f16", 32, 1, 3),
                                              ("fp8", 4, 1, 8), ("fp8", 8, 1, 3), ("fp8", 10, 1, 13)])
@pytest.mark.parametrize("D", [64, 128])
def test_few_tokens_with_grouped_heads(dtype, H, H_kv, n_q, D):
    p = Tokens(3, H, H_kv, 290, D, n_q, dtype)
    ctx, new, many = [290, n_q, 61], [n_q, n_q, max(1, n_q - 1)], H // H_kv * n_q > 32
    for window, sinks in ((0, 0), (1, 0), (7, 2), (64, 30), (200, 0)):
        run(p, ctx, new, window, sinks, many=many)
    run(p, ctx, [0, 1, n_q], 9, 1, out_dtype=None, many=many)


def test_tokens_without_a_position_have_zero_rows():
    p = Tokens(3, 4, 2, 64, 128, 6)
    out, lse, _, status = run(p, [2, 0, 5], [6, 3, 6], 3, 1)
    assert (out[0, :, :4] == 0).all() and np.isneginf(lse[0, :, :4]).all() and np.isfinite(lse[0, :, 4:]).all()
    assert (out[1, :, :3] == 0).all() and (out[2, :, :1] == 0).all() and status == 0


@pytest.mark.parametrize("B,ctx", [(1, 9000), (2, 5000)])
@pytest.mark.parametrize("n_q", [1, 4])
def test_long_contexts_are_split(B, ctx, n_q):
    p = Tokens(B, 8, 2, ctx, 128, n_q)
    for window, sinks in ((0, 0), (2000, 64), (300, 0)):
        run(p, [ctx] + [ctx - 1234] * (B - 1), None, window, sinks)


def test_lengths_that_do_not_fit_are_clamped():
    p = Tokens(3, 2, 2, 100, 64, 2)
    got = p.call([150, 90, -3], [2, 5, 1], 20, 2)
    assert got[3] == ssa.DEV_BAD_COUNT
    check(p, got, [100, 90, 0], [2, 2, 1], 20, 2, torch.float32)
    got = p.call([50, 90, 10], [2, -1, 1], 20, 2)
    assert got[3] == 0
    check(p, got, [50, 90, 10], [2, 0, 1], 20, 2, torch.float32)


@pytest.mark.parametrize("page", [1, 4, 16, 64, 256])
def test_pages(page):
    p = Tokens(2, 4, 2, 300, 128, 3, page=page)
    run(p, [300, 131], [3, 2], 50, 20)
    run(p, [300, 131], [3, 2])


@pytest.mark.parametrize("page", [4, 32])
def test_pages_behind_the_window_may_be_gone(page):
    p = Tokens(1, 4, 2, 320, 128, 2, page=page)
    table = p.table.clone()
    window, sinks, ctx = 40, 5, 300
    j = torch.arange(p.table.shape[1]) * page
    gone = ((j >= sinks) & (j + page <= ctx - 2 - window + 1)) | (j >= ctx)
    table[0, gone] = -1
    assert gone.sum() > 3
    got = p.call([ctx], None, window, sinks, table=table)
    assert got[3] == 0
    check(p, got, [ctx], None, window, sinks, torch.float32)
    # without the window those positions are skipped, and said so
    got = p.call([ctx], None, 0, 0, table=table)
    assert got[3] == ssa.DEV_BAD_INDEX
    skipped = np.zeros((1, 320), bool)
    for x in np.flatnonzero(gone.numpy()):
        skipped[0, x * page:(x + 1) * page] = True
    check(p, got, [ctx], None, 0, 0, torch.float32, skipped=skipped)
    table[:] = p.n_pages                                     # no page at all
    out, lse, _, status = p.call([ctx], None, 0, 0, table=table)
    assert (out == 0).all() and np.isneginf(lse).all() and status == ssa.DEV_BAD_INDEX


@pytest.mark.parametrize("dtype", ["bf16", "f16", "fp8"])
@pytest.mark.parametrize("n_q", [1, 3, 70])
def test_what_is_not_seen_may_hold_anything(dtype, n_q):
    p = Tokens(1, 4, 2, 300, 128, n_q, dtype)
    window, sinks, ctx = 37, 3, 250
    clean = p.call([ctx], None, window, sinks)
    for bad in (float("nan"), float("inf"), -float("inf")):
        if dtype == "fp8" and bad == bad:
            continue                                         # the type has no infinities
        k, v = (x.clone() for x in p.host)
        for x in (k, v):
            x[:, :, ctx:] = bad
            x[:, :, sinks:ctx - n_q - window + 1] = bad
        kept = p.host
        p.put(k, v)
        got = p.call([ctx], None, window, sinks)
        assert np.array_equal(got[0], clean[0]) and np.array_equal(got[1], clean[1])
        p.put(*kept)


@pytest.mark.parametrize("dtype,bad", [("bf16", float("nan")), ("bf16", float("inf")), ("f16", -float("inf")), ("f16", float("nan")),
                                       ("fp8", float("nan"))])
@pytest.mark.parametrize("n_q", [1, 3, 40, 150])
def test_bad_values_reach_the_tokens_that_see_them_only(dtype, bad, n_q):
    p = Tokens(1, 4, 2, 300, 128, n_q, dtype)
    window, sinks, ctx = 30, 2, 290
    for name, at in (("k", ctx - 1), ("k", ctx - n_q - 20), ("v", ctx - 1), ("v", ctx - n_q - 20), ("v", ctx - n_q // 2 - 1), ("v", 1)):
        kept = p.host
        k, v = (x.clone() for x in p.host)
        clean = p.call([ctx], None, window, sinks)
        (k if name == "k" else v)[0, 1, at, 5] = bad
        p.put(k, v)
        got = p.call([ctx], None, window, sinks)
        if name == "v":
            check(p, got, [ctx], None, window, sinks, torch.float32, many=n_q > 16)
        else:                                                # rows that see the key are NaN; the rest are as without it
            pos = ctx - n_q + np.arange(n_q)
            sees = (at <= pos) & ((at > pos - window) | (at < sinks))
            if bad != bad:
                assert np.isnan(got[0][0, 2:][:, sees]).all() and np.isnan(got[1][0, 2:][:, sees]).all()
            assert np.array_equal(got[0][0, 2:][:, ~sees], clean[0][0, 2:][:, ~sees]) and np.array_equal(got[0][0, :2], clean[0][0, :2])
        p.put(*kept)


def test_a_scale_strides_and_a_batch_of_views():
    big = Tokens(2, 6, 3, 200, 64, 4)
    # views: every second head of a wider tensor, rows of a longer cache
    p = Tokens(2, 3, 3, 120, 64, 4)
    p.q = big.q[:, ::2]
    p.host = [x[:, :, 40:160] for x in big.host]
    p.stores = [x[:, :, 40:160] for x in big.stores]
    got = p.call([120, 77], [4, 3], 50, 10, torch.bfloat16, scale=0.3)
    check(p, got, [120, 77], [4, 3], 50, 10, torch.bfloat16, scale=0.3)


@pytest.mark.parametrize("n_q", [2, 100])
def test_large_scores_and_minus_infinity(n_q):
    p = Tokens(1, 2, 2, 190, 64, n_q, spread=200.0)          # softmax close to one position
    run(p, [190], None, 40, 4, many=n_q > 16)
    p = Tokens(1, 2, 2, 190, 64, n_q)
    k, v = (x.clone() for x in p.host)
    p.q[0, 0] = 1.0                                          # every score of head 0 is -inf: a zero row, as without positions
    k[0, 0] = -float("inf")
    p.put(k, v)
    out, lse, _, _ = p.call([190], None, 0, 0)
    assert (out[0, 0] == 0).all() and np.isneginf(lse[0, 0]).all() and np.isfinite(out[0, 1]).all()


@pytest.mark.parametrize("n_q,T", [(17, 100), (64, 64), (130, 130), (257, 700), (300, 1500)])
@pytest.mark.parametrize("dtype,H,H_kv,D", [("bf16", 4, 4, 128), ("f16", 4, 1, 64), ("bf16", 8, 2, 128), ("f16", 6, 2, 128), ("fp8", 4, 2, 128)])
def test_prompt_chunks(n_q, T, dtype, H, H_kv, D):
    p = Tokens(3, H, H_kv, T, D, n_q, dtype)
    ctx, new = [T, max(n_q, T - 33), n_q // 2], [n_q, n_q - 5, n_q // 2]
    for window, sinks in ((0, 0), (1, 0), (50, 7), (128, 130)):
        run(p, ctx, new, window, sinks, out_dtype=None, many=True)
    run(p, [T, 3, 0], [n_q, n_q, n_q], 64, 4, many=True)     # tokens before the first position


@pytest.mark.parametrize("page", [2, 8, 32, 128, 512])
def test_paged_prompt_chunks(page):
    p = Tokens(2, 8, 2, 600, 128, 150, "bf16", page=page)
    run(p, [600, 333], [150, 149], 100, 20, out_dtype=None, many=True)
    run(p, [600, 333], [150, 149], out_dtype=None, many=True)


def test_paged_chunk_whose_pages_are_gone():
    p = Tokens(1, 4, 2, 640, 128, 100, "f16", page=32)
    table = p.table.clone()
    table[0, 4:10], table[0, -2:] = -1, p.n_pages
    got = p.call([570], None, 200, 100, table=table)         # sinks 0..99, window from 271: pages 4..7 are not seen
    skipped = np.zeros((1, 640), bool)
    skipped[0, 128:320] = True
    assert got[3] == ssa.DEV_BAD_INDEX                       # pages 8 and 9 are
    check(p, got, [570], None, 200, 100, torch.float32, many=True, skipped=skipped)
    got = p.call([570], None, 150, 100, table=table)         # from 321: nothing that is gone is seen
    assert got[3] == 0
    check(p, got, [570], None, 150, 100, torch.float32, many=True)


@pytest.mark.parametrize("n_q", [1, 60])
def test_heads_and_requests_that_share_a_cache(n_q):
    """Strides of zero: one K/V head's rows for two heads, one request's for two."""
    p = Tokens(2, 4, 2, 200, 128, n_q)
    for heads, requests in ((True, False), (False, True), (True, True)):
        q = Tokens.__new__(Tokens)
        q.__dict__.update(p.__dict__)
        share = lambda x: (x[:, :1] if heads else x)[:1 if requests else 2].expand(2, 2, -1, -1)
        q.host, q.stores = [share(x) for x in p.host], [share(x) for x in p.stores]
        run(q, [200, 133], None, 70, 3, many=n_q > 16)


def test_a_chunk_is_its_tokens_one_by_one():
    """Chunks of any size and single tokens give the same rows, up to their bounds."""
    p = Tokens(1, 8, 2, 400, 128, 200, "bf16")
    whole = p.call([400], None, 60, 4)
    one = Tokens(1, 8, 2, 400, 128, 1, "bf16")
    one.stores, one.host = p.stores, p.host
    for t in (0, 1, 77, 128, 199):
        one.q = p.q[:, :, t:t + 1]
        got = one.call([200 + t + 1], None, 60, 4)
        check(one, got, [200 + t + 1], None, 60, 4, torch.float32)
        assert np.abs(got[0][:, :, 0] - whole[0][:, :, t]).max() < 0.02 and np.abs(got[1][:, :, 0] - whole[1][:, :, t]).max() < 1e-4


@pytest.mark.parametrize("n_q", [2, 40])
def test_offsets_beyond_32_bits(n_q):
    """The last request of a cache of more than 2^32 bytes and 2^31 elements."""
    B, T, D = 5, 1 << 19, 128
    k = torch.zeros(B, 8, T, D, dtype=torch.bfloat16, device=DEV)
    v = torch.zeros_like(k)
    ctx = T - 5
    p = Tokens(1, 8, 8, 400, D, n_q)
    for store, x in zip((k, v), p.host):
        store[-1, :, ctx - 400:ctx] = x[0].to(DEV)
    wide = Tokens.__new__(Tokens)
    wide.__dict__.update(p.__dict__, B=B, T=T, stores=[k, v], q=p.q.expand(B, -1, -1, -1).contiguous())
    out, lse, _, _ = wide.call([0, 0, 0, 0, ctx], None, 300, 0)
    check(p, (out[-1:], lse[-1:], None, 0), [400], None, 300, 0, torch.float32, many=n_q > 16)


@pytest.mark.parametrize("n_q", [1, 5, 200])
def test_captured_replayed_and_on_another_stream(n_q):
    p = Tokens(2, 8, 2, 1500, 128, n_q)
    k, v = p.stores
    ctx = torch.tensor([1500, 900], dtype=torch.int32, device=DEV)
    calls = []
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    for _ in range(2):
        out = torch.zeros(2, 8, n_q, 128, device=DEV)
        desc, win = ssa.make_desc(p.q[:, :, 0], k, v, out[:, :, 0]), ssa.make_window(p.q, out, 700, 4)
        calls.append((out, desc, win, torch.empty(ssa.attn_window_workspace_bytes(desc, win), dtype=torch.uint8, device=DEV)))
    side.wait_stream(torch.cuda.current_stream())
    out, desc, win, ws = calls[0]
    ssa.attn_window(desc, win, p.q, k, v, ctx, out, None, ws, None, side)
    out, desc, win, ws = calls[1]
    with torch.cuda.graph(graph):
        ssa.attn_window(desc, win, p.q, k, v, ctx, out, None, ws, None)
    side.synchronize()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(calls[0][0], out) and out.abs().sum() > 0
    first = out.clone()
    ctx.copy_(torch.tensor([700, 1400], dtype=torch.int32, device=DEV))      # lengths are read when the graph runs
    p.q.neg_()
    graph.replay()
    torch.cuda.synchronize()
    check(p, (out.double().cpu().numpy(), p.call([700, 1400], None, 700, 4)[1], None, 0), [700, 1400], None, 700, 4, torch.float32,
          many=n_q > 16)
    assert not torch.equal(first, out)
