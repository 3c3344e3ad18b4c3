"""DecodeStep.append among the calls of earlier tokens: eviction by sums, full contexts, refused calls, captured steps."""
import numpy as np
import pytest
import torch

from oracle import budget_oracle as BO
from oracle import cache_oracle as CO
from paper_2404_09336_b200 import inputs, ssa
from paper_2404_09336_b200.runner import DecodeStep

pytestmark = pytest.mark.gpu


def made(**kw):
    return DecodeStep(inputs.make_config(2, B=3, H=4), out_dtype=torch.float32, **kw)


def rows(ds, n, seed=3):
    g = torch.Generator(device=ds.device).manual_seed(seed)
    return torch.randn(n, ds.wl.B, ds.wl.H, ds.wl.D, generator=g, device=ds.device).to(ds.q.dtype)


@pytest.mark.parametrize("last", ["attend_mass", "attend_window"])
def test_tokens_appended_behind_a_compaction_have_sums_of_their_own(last):
    """Evict, append, evict: an appended token ranks by the weight that it got, not by that of the evicted one whose place it has."""
    ds = made()
    budget, sinks, recent = 40, 2, 3
    ds.attend_mass()
    ds.select_heaviest(60, sinks=2, recent=5)
    ds.compact()
    torch.cuda.synchronize()
    start, sums = ds.ctx_lens.tolist(), ds.mass.cpu().double().numpy()
    keys = rows(ds, 6)
    for x in keys:
        ds.append(x, x, x)
        ds.attend_window(20)
    if last == "attend_mass":
        ds.attend_mass()
    ds.select_heaviest(budget, sinks=sinks, recent=recent)
    torch.cuda.synchronize()
    assert int(ds.status) == 0
    got = ds.mass.cpu().double().numpy()
    for b, n in enumerate(ds.ctx_lens.tolist()):
        assert n == start[b] + 6
        want, tol = np.zeros(n), np.zeros(n)
        want[: start[b]] = sums[b, : start[b]]
        if last == "attend_mass":                            # the weights of the newest token's queries
            q, K = ds.q[b].double().cpu().numpy(), ds.k[b, :, :n].double().cpu().numpy()
            s = np.einsum("hd,hjd->hj", q, K) * ds.wl.D ** -0.5
            w = np.exp(s - s.max(1, keepdims=True))
            w = (w / w.sum(1, keepdims=True)).sum(0)
            # scores off by D + 2 roundings of fp32 of sum |q| |k|, a weight by twice that and its powers' and sums' own; one more sum
            S = (ds.wl.D ** -0.5 * np.einsum("hd,hjd->hj", np.abs(q), np.abs(K))).max()
            want, tol = want + w, 2 * (((ds.wl.D + 2) * S + 4) * 2.0 ** -24 + 2.0 ** -22 + (n + 64) * 2.0 ** -24) * w + 2.0 ** -23 * (want + w)
        assert (np.abs(got[b, :n] - want) <= tol).all()
        kept = BO.kept(got[b, :n].astype(np.float32), n, budget, sinks, recent)
        assert ds.counts[b] == len(kept) and np.array_equal(ds.index[b, : len(kept)].cpu().numpy(), kept)


@pytest.mark.parametrize("layout", ["bhtd", "bthd"])
def test_full_contexts_keep_their_rows(layout):
    ds = made(layout=layout, kv_copies=2)
    ds.enable_fp4()
    ds.enable_blocks(32, 4)
    T = ds.wl.max_ctx
    ds.attend_mass()
    ds.ctx_lens.copy_(torch.tensor([T, T - 1, 9], dtype=torch.int32))
    ds.refresh_bounds()
    torch.cuda.synchronize()
    kept = [x.clone() for x in (*ds.k_store, *ds.v_store, *ds.fp4, ds.bounds, ds.mass, ds.q)]
    x = rows(ds, 1)[0]
    ds.append(x, x, x)
    torch.cuda.synchronize()
    assert ds.ctx_lens.tolist() == [T, T, 10] and int(ds.status) == ssa.DEV_BAD_COUNT
    now = (*ds.k_store, *ds.v_store, *ds.fp4, ds.bounds, ds.mass, ds.q)
    assert all(torch.equal(a[0], b[0]) for a, b in zip(now, kept))
    for c in range(2):
        ds.select_copy(c)
        for b, n in ((1, T), (2, 10)):
            assert torch.equal(ds.k[b, :, n - 1], x[b]) and torch.equal(ds.v[b, :, n - 1], x[b]) and torch.equal(ds.q[b], x[b])
            was = kept[c][b] if layout == "bhtd" else kept[c][b].transpose(0, 1)
            assert torch.equal(ds.k[b, :, : n - 1], was[:, : n - 1])
    ds.append(x, x)
    torch.cuda.synchronize()
    assert ds.ctx_lens.tolist() == [T, T, 11]


def test_a_refused_token_changes_nothing():
    ds = made()
    ds.enable_fp4()
    x = rows(ds, 1)[0]
    torch.cuda.synchronize()
    ctx, k, q = ds.ctx_lens.clone(), ds.k_store[0].clone(), ds.q.clone()
    for R in (40, 160):                                      # no multiple of 32; more than a row has
        with pytest.raises(ssa.SsaError):
            ds.append(x, x, x, torch.zeros(ds.wl.max_ctx, R, device=ds.device))
    with pytest.raises(ValueError):
        ds.append(x.half(), x, x)
    torch.cuda.synchronize()
    assert torch.equal(ds.ctx_lens, ctx) and torch.equal(ds.k_store[0], k) and torch.equal(ds.q, q) and int(ds.status) == 0


def test_captured_appends_fill_a_cache_up():
    """A graph of one token, replayed past the end of the shortest room, gives what eager calls give."""
    eager, captured = made(), made()
    T = eager.wl.max_ctx
    for ds in (eager, captured):
        ds.enable_fp4()
        ds.enable_blocks(32, 5)
        ds.ctx_lens.copy_(torch.tensor([T - 2, T, 3], dtype=torch.int32))
        ds.refresh_bounds()
    xs = rows(eager, 4)
    k = xs[0].clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured.append(k, k, k)
    for x in xs:
        k.copy_(x)
        graph.replay()
        eager.append(x, x, x)
    torch.cuda.synchronize()
    assert eager.ctx_lens.tolist() == captured.ctx_lens.tolist() == [T, T, 7]
    for a, b in zip((*eager.k_store, *eager.v_store, *eager.fp4, eager.bounds, eager.q), (*captured.k_store, *captured.v_store, *captured.fp4, captured.bounds, captured.q)):
        assert torch.equal(a, b)
    assert int(eager.status) == int(captured.status) == ssa.DEV_BAD_COUNT


def over_4_bits(ds, b, h):
    n = int(ds.ctx_lens[b])
    K, V = (CO.fp4_values(ds.fp4[i][b, h, :n].cpu().numpy(), ds.fp4[2 + i][b, h, :n].cpu().numpy()) for i in (0, 1))
    return CO.attention(ds.q[b, h][None].double().cpu().numpy(), K, V, np.arange(n), ds.wl.D ** -0.5)[0][0]


def test_a_compacted_cache_is_attended_to_in_4_bits():
    ds = made()
    ds.enable_fp4()
    before = ds.ctx_lens.tolist()
    ds.attend_mass()
    ds.select_heaviest(70, sinks=2, recent=5)
    ds.compact()
    ds.attend_fp4()
    torch.cuda.synchronize()
    assert ds.ctx_lens.tolist() == [min(70, n) for n in before] and min(before) > 70
    for b in range(3):
        for h in range(4):
            assert np.abs(ds.out[b, h].cpu().numpy() - over_4_bits(ds, b, h)).max() < 1e-4


def test_captured_4_bit_steps():
    """Graphs of a token appended and attended to in 4 bits, and of other calls in the same workspace, replayed in turn: each output is
    what an eager runner gives, and the oracle."""
    eager, captured = made(), made()
    for ds in (eager, captured):
        ds.ctx_lens.sub_(30)
        ds.enable_fp4()
        ds.enable_blocks(32, 5)
        ds.attend_fp4()
        ds.attend_blocks()
    xs = rows(eager, 5)
    k = xs[0].clone()
    torch.cuda.synchronize()
    step, other = torch.cuda.CUDAGraph(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(step):
        captured.append(k, k, k)
        captured.attend_fp4()
        got = captured.out.clone()
    with torch.cuda.graph(other):
        captured.attend_window(9)
        captured.select_blocks()
        captured.attend_blocks()
    for x in xs:
        k.copy_(x)
        step.replay()
        other.replay()
        eager.append(x, x, x)
        eager.attend_fp4()
        torch.cuda.synchronize()
        assert torch.equal(got, eager.out) and not torch.equal(got, captured.out)
    for b in range(3):
        for h in range(4):
            assert np.abs(got[b, h].cpu().numpy() - over_4_bits(eager, b, h)).max() < 1e-4
    assert int(captured.status) == int(eager.status) == 0


def test_a_4_bit_copy_made_in_parts(monkeypatch):
    """As many query heads as make a call take fewer rows than the cache has: the copy is that of one call."""
    ds = DecodeStep(inputs.make_config(2, B=2, H=2), out_dtype=torch.float32, query_heads=1 << 14)
    ds.enable_fp4()
    whole = [x.clone() for x in ds.fp4]
    assert len(ds._filled) == 1
    few = DecodeStep(inputs.make_config(2, B=2, H=2), out_dtype=torch.float32, query_heads=3 << 13)      # 682 rows at a time
    few.enable_fp4()
    torch.cuda.synchronize()
    assert len(few._filled) == 2 and all(torch.equal(a, b) for a, b in zip(few.fp4, whole)) and int(few.status) == 0
    for b in range(2):
        want = CO.to_fp4(few.k[b].float().cpu().numpy())
        assert np.array_equal(few.fp4[0][b].cpu().numpy(), want[0]) and np.array_equal(few.fp4[2][b].cpu().numpy(), want[1])
