"""The operators together, as a decoding program calls them: append, bounds, selection, attention over blocks and over 4-bit values."""
import numpy as np
import pytest
import torch

from oracle import cache_oracle as CO
from paper_2404_09336_b200 import inputs, ssa
from paper_2404_09336_b200.runner import DecodeStep

pytestmark = pytest.mark.gpu


def made(**kw):
    wl = inputs.make_config(2, B=3, H=4)
    return DecodeStep(wl, out_dtype=torch.float32, **kw)


def shorter(ds, by):
    """Contexts with room for more tokens."""
    ds.ctx_lens.sub_(by).clamp_(min=1)
    torch.cuda.synchronize()


@pytest.mark.parametrize("layout", ["bhtd", "bthd"])
@pytest.mark.parametrize("heads", [4, 8])
def test_blocks_of_the_whole_context_are_full_attention(layout, heads):
    ds = made(layout=layout, query_heads=heads)
    n = -(-ds.wl.max_ctx // 64)
    ds.enable_blocks(64, n)
    ds.select_blocks()
    ds.attend_blocks()
    got, lse = ds.out.clone(), ds.lse.clone()
    ds.attend_dense()
    torch.cuda.synchronize()
    assert (got - ds.out).abs().max() < 2e-5 and (lse - ds.lse).abs().max() < 1e-5 and int(ds.status) == 0


def test_steps_of_a_generation():
    """Twenty tokens: contexts grow, the cache is what a cache filled at once is, bounds are those of the whole, lists hold the newest."""
    ds = made(kv_copies=2)
    shorter(ds, 40)
    ds.enable_fp4()
    ds.enable_blocks(32, 6, 1, 1)
    B, H, D, T = ds.wl.B, ds.wl.H, ds.wl.D, ds.wl.max_ctx
    angle = torch.arange(T, dtype=torch.float64)[:, None] * 10000.0 ** (-torch.arange(D // 2, dtype=torch.float64) * 2 / D)
    cos_sin = torch.cat([angle.cos(), angle.sin()], 1).float().to(ds.device)
    g = torch.Generator(device=ds.device).manual_seed(3)
    start, keys, values = ds.ctx_lens.clone(), [], []
    for step in range(20):
        k, v, q = (torch.randn(B, H, D, generator=g, device=ds.device).to(ds.q.dtype) for _ in range(3))
        keys.append(k), values.append(v)
        ds.append(k, v, q, cos_sin)
        ds.select_blocks()
        ds.attend_blocks()
        blocks = ds.out.clone()
        ds.attend_fp4()
    torch.cuda.synchronize()
    assert int(ds.status) == 0 and torch.equal(ds.ctx_lens, start + 20)
    index, counts = ds.block_lists
    for b, n in enumerate(ds.ctx_lens.tolist()):
        m = (n - 1) // 32 + 1
        assert (counts[b] == min(6, m)).all() and (index[b, :, 0, counts[b, 0, 0] - 1] == m - 1).all() and (index[b, :, 0, 0] == 0).all()
        at = np.arange(n - 20, n)
        want = CO.rotated(torch.stack([k[b] for k in keys], 1).float().cpu().numpy(), at, cos_sin.cpu().numpy(), False)
        for c in range(2):
            ds.select_copy(c)
            assert np.array_equal(ds.k[b, :, n - 20:n].float().cpu().numpy(), torch.from_numpy(want).to(ds.q.dtype).float().numpy())
            assert torch.equal(ds.v[b, :, n - 20:n], torch.stack([v[b] for v in values], 1))
        codes, scales = CO.to_fp4(want)
        assert np.array_equal(ds.fp4[0][b, :, n - 20:n].cpu().numpy(), codes) and np.array_equal(ds.fp4[2][b, :, n - 20:n].cpu().numpy(), scales)
        K = ds.k[b, :, :n].float().cpu().numpy()
        for h in range(H):
            least, most = CO.bounds(K[h], n, 32)
            assert np.array_equal(ds.bounds[b, h, :m, 0].float().cpu().numpy(), least) and np.array_equal(ds.bounds[b, h, :m, 1].float().cpu().numpy(), most)
            # the last step's outputs over its blocks, and over the whole 4-bit cache
            rows = np.concatenate([np.arange(32 * j, min(32 * j + 32, n)) for j in index[b, h, 0, : counts[b, h, 0]].tolist()])
            ref = CO.attention(ds.q[b, h][None].double().cpu().numpy(), K[h], ds.v[b, h, :n].float().cpu().numpy(), rows, D ** -0.5)
            assert np.abs(blocks[b, h].cpu().numpy() - ref[0][0]).max() < 1e-4
            K4, V4 = (CO.fp4_values(ds.fp4[i][b, h, :n].cpu().numpy(), ds.fp4[2 + i][b, h, :n].cpu().numpy()) for i in (0, 1))
            ref = CO.attention(ds.q[b, h][None].double().cpu().numpy(), K4, V4, np.arange(n), D ** -0.5)
            assert np.abs(ds.out[b, h].cpu().numpy() - ref[0][0]).max() < 1e-4


def test_a_compacted_cache_has_its_own_bounds_and_4_bit_values():
    ds = made()
    ds.enable_fp4()
    ds.enable_blocks(32, 4)
    ds.attend_mass()
    ds.select_heaviest(70, sinks=2, recent=5)
    ds.compact()
    ds.select_blocks()
    ds.attend_blocks()
    blocks = ds.out.clone()
    ds.attend_dense()
    dense = ds.out.clone()
    ds.attend_fp4()
    torch.cuda.synchronize()
    assert ds.ctx_lens.tolist() == [min(70, n) for n in ds.ctx_lens.tolist()] and (blocks - dense).abs().max() < 2e-5       # (4 blocks: all)
    for b, n in enumerate(ds.ctx_lens.tolist()):
        want = CO.to_fp4(ds.k[b, :, :n].float().cpu().numpy())
        assert np.array_equal(ds.fp4[0][b, :, :n].cpu().numpy(), want[0]) and np.array_equal(ds.fp4[2][b, :, :n].cpu().numpy(), want[1])
    assert (ds.out - dense).abs().max() < 0.5


def test_captured_steps_and_side_streams():
    """A step as a graph, replayed behind others that use the same workspace, gives what eager calls on another stream give."""
    def step(ds, k, v, q, stream=None):
        ds.append(k, v, q, stream=stream)
        ds.select_blocks(stream)
        ds.attend_blocks(stream)
        first = ds.out.clone() if stream is None else None
        ds.attend_fp4(stream=stream)
        return first

    wl = inputs.make_config(2, B=3, H=4)
    g = torch.Generator(device="cuda:0").manual_seed(5)
    rows = [torch.randn(3, 4, wl.D, generator=g, device="cuda:0").to(torch.bfloat16) for _ in range(3)]
    eager, captured = made(), made()
    for ds in (eager, captured):
        shorter(ds, 30)
        ds.enable_fp4()
        ds.enable_blocks(32, 5)
        ds.attend_fp4()
        ds.attend_blocks()
    k, v, q = (r.clone() for r in rows)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        first = step(captured, k, v, q)
    side = torch.cuda.Stream()
    for i in range(4):
        for a, r in zip((k, v, q), rows):
            a.copy_(r * (i + 1))
        graph.replay()
        captured.attend_window(9)                            # (the same workspace)
        with torch.cuda.stream(side):
            mine = [r * (i + 1) for r in rows]
        side.synchronize()
        eager.append(*mine, stream=side)
        eager.select_blocks(side)
        eager.attend_blocks(side)
        side.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(first, eager.out) and all(torch.equal(a, b) for a, b in zip(eager.block_lists, captured.block_lists))
        eager.attend_fp4(stream=side)
        graph_out = captured.out.clone()
        captured.attend_fp4()
        torch.cuda.synchronize()
        assert torch.equal(captured.out, eager.out) and torch.equal(captured.ctx_lens, eager.ctx_lens)
        assert graph_out.shape == eager.out.shape and int(captured.status) == int(eager.status) == 0


def test_calls_at_once_with_workspaces_of_their_own():
    """Two streams, split contexts, a workspace each."""
    from budget_util import DEV
    from cache_util import Fp4Tokens
    ps = [Fp4Tokens(1, 4, 2, 9000, 128, 2, seed=s) for s in (1, 2)]
    want = [p.call([9000]) for p in ps]
    streams, outs = [torch.cuda.Stream() for _ in ps], []
    ctx = torch.tensor([9000], dtype=torch.int32, device=DEV)
    for p, st in zip(ps, streams):
        c = p.cache
        out = torch.zeros(1, 2, 4, 128, device=DEV).permute(0, 2, 1, 3)
        lse = torch.zeros(1, 4, 2, device=DEV)
        desc, win = c.desc(p.q, out), ssa.make_window(p.q, out)
        ws = torch.empty(ssa.attn_window_fp4_workspace_bytes(desc, win), dtype=torch.uint8, device=DEV)
        outs.append((p, c, out, lse, desc, win, ws, st))
    torch.cuda.synchronize()
    for _ in range(20):
        for p, c, out, lse, desc, win, ws, st in outs:
            ssa.attn_window_fp4(desc, win, p.q, c.parts["k"], c.parts["v"], c.scales("k"), c.scales("v"), ctx, out, lse, ws, None, st)
    torch.cuda.synchronize()
    for (_, _, out, lse, *_), w in zip(outs, want):
        assert np.array_equal(out.double().cpu().numpy(), w[0]) and np.array_equal(lse.double().cpu().numpy(), w[1])
