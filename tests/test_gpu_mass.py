"""ssa_attn_mass, ssa_mass_to_index and ssa_cache_compact, alone and as a run of them."""
import numpy as np
import pytest
import torch

from oracle import budget_oracle as BO
from paper_2404_09336_b200 import ssa

from budget_util import DEV, Tokens, check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,H,H_kv,D,n_q,page", [("bf16", 4, 4, 128, 1, 0), ("f16", 8, 2, 64, 3, 0), ("fp8", 4, 1, 128, 2, 0),
                                                     ("bf16", 8, 2, 128, 17, 0), ("f16", 32, 8, 128, 1, 16), ("bf16", 4, 2, 128, 5, 2), ("fp8", 8, 2, 64, 6, 0), ("f16", 16, 1, 128, 2, 8)])
def test_mass(dtype, H, H_kv, D, n_q, page):
    p = Tokens(3, H, H_kv, 700, D, n_q, dtype, page=page)
    old = torch.rand(3, 700, generator=torch.Generator().manual_seed(1)) * 3
    ctx, new = [700, n_q, 259], [n_q, n_q, max(1, n_q - 1)]
    for window, sinks in ((0, 0), (100, 3)):
        for m in (None, old):
            got = p.call(ctx, new, window, sinks, mass=True, mass_in=None if m is None else m.to(DEV), decay=0.9)
            check(p, got, ctx, new, window, sinks, torch.float32, mass_in=None if m is None else m.double().numpy(), decay=float(np.float32(0.9)))


def test_mass_of_a_split_context_and_empty_requests():
    p = Tokens(2, 8, 2, 6000, 128, 1)
    for ctx in ([6000, 0], [1, 4321]):
        check(p, p.call(ctx, None, 0, 0, mass=True), ctx, None, 0, 0, torch.float32)
    p = Tokens(2, 4, 2, 40, 128, 4)                          # tokens without a position give no weight
    check(p, p.call([2, 30], [4, 0], 0, 0, mass=True), [2, 30], [4, 0], 0, 0, torch.float32)


def test_mass_in_place_repeats_to_the_bit_and_ignores_what_new_positions_hold():
    p = Tokens(2, 4, 2, 500, 128, 2)
    k, v = p.stores
    ctx = torch.tensor([500, 300], dtype=torch.int32, device=DEV)
    out, lse = torch.empty(2, 4, 2, 128, device=DEV), torch.empty(2, 4, 2, device=DEV)
    desc, win = ssa.make_desc(p.q[:, :, 0], k, v, out[:, :, 0]), ssa.make_window(p.q, out)
    ws = torch.empty(ssa.attn_mass_workspace_bytes(desc, win), dtype=torch.uint8, device=DEV)
    got = []
    for i in range(2):
        mass = torch.ones(2, 500, device=DEV)
        mass[0, 498:] = float("nan")
        mass[1, 298:300] = float("nan")
        ssa.attn_mass(desc, win, p.q, k, v, ctx, out, lse, mass, mass, 1.0, ws)
        got.append(mass)
    torch.cuda.synchronize()
    assert torch.equal(got[0], got[1]) and got[0].isfinite().all() and (got[0][1, 300:] == 1).all()
    assert abs(got[0][0].double().sum().item() - 498 - 8) < 1e-2      # every token and head hands out a weight of one


@pytest.mark.parametrize("T,budget,sinks,recent", [(1, 1, 0, 0), (40, 7, 2, 3), (700, 128, 4, 32), (1500, 1499, 0, 0), (5000, 700, 64, 100),
                                                   (5000, 100, 60, 40), (5000, 1, 0, 0), (16384, 3000, 0, 7), (40000, 9000, 3, 1), (140001, 20000, 5, 100)])
def test_keep(T, budget, sinks, recent):
    rng = np.random.default_rng(T + budget)
    kinds = [rng.standard_normal(T), np.round(rng.standard_normal(T)), np.zeros(T), rng.permutation(T) * 1e-42, np.where(rng.random(T) < .5, 0., -0.),
             np.where(rng.random(T) < .3, np.nan, np.round(rng.standard_normal(T), 1)), np.where(rng.random(T) < .5, np.inf, -np.inf),
             np.exp(rng.standard_normal(T) * 3), np.full(T, np.nan)]
    mass = np.array(kinds, np.float32)
    B = len(kinds)
    wide = torch.full((B, T + 3), 1e30, device=DEV)
    wide[:, :T] = torch.from_numpy(mass).to(DEV)
    for ctx in ([T] * B, [max(0, T - i * (T // B)) for i in range(B)], [min(budget + i, T) for i in range(B)]):
        index = torch.full((B, budget + 2), -7, dtype=torch.int32, device=DEV)
        counts, status = torch.full((B,), -7, dtype=torch.int32, device=DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
        ssa.mass_to_index(wide[:, :T], torch.tensor(ctx, dtype=torch.int32, device=DEV), budget, sinks, recent, index, counts, status)
        torch.cuda.synchronize()
        assert int(status) == 0
        for b in range(B):
            want = BO.kept(mass[b], ctx[b], budget, sinks, recent)
            c = int(counts[b])
            assert c == len(want) and index[b, :c].tolist() == want.tolist(), (b, ctx[b])
            assert (index[b, c:] == -7).all()


def test_keep_clamps_lengths():
    index, counts = torch.full((3, 4), -7, dtype=torch.int32, device=DEV), torch.zeros(3, dtype=torch.int32, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    mass = torch.arange(30, dtype=torch.float32, device=DEV).view(3, 10)
    ssa.mass_to_index(mass, torch.tensor([99, -5, 3], dtype=torch.int32, device=DEV), 4, 1, 1, index, counts, status)
    torch.cuda.synchronize()
    assert int(status) == ssa.DEV_BAD_COUNT and counts.tolist() == [4, 0, 3]
    assert index.tolist() == [[0, 7, 8, 9], [-7] * 4, [0, 1, 2, -7]]


@pytest.mark.parametrize("dtype,D,layout,page", [("bf16", 128, "bhtd", 0), ("f16", 64, "bthd", 0), ("fp8", 64, "bhtd", 0), ("fp8", 128, "bthd", 0),
                                                 ("bf16", 128, "", 16), ("f16", 64, "", 1)])
@pytest.mark.parametrize("T", [1, 50, 2000])
def test_compact(dtype, D, layout, page, T):
    B, rng = 4, np.random.default_rng(T)
    p = Tokens(B, 4, 2, T, D, 1, dtype, layout, page)
    ctx = [T, max(1, T // 2), T, 0]
    keep = [np.sort(rng.choice(ctx[0], (T + 2) // 3, replace=False)), np.arange(ctx[1]), np.arange(T - (T + 3) // 4, T), np.arange(0)]
    stride = max(len(x) for x in keep) + 1
    index = np.full((B, stride), 1 << 30, np.int32)
    for b, x in enumerate(keep):
        index[b, :len(x)] = x
    d_ctx, d_index, d_counts = (torch.tensor(x, dtype=torch.int32, device=DEV) for x in (ctx, index, [len(x) for x in keep]))
    mass = torch.rand(B, T + 1, generator=torch.Generator().manual_seed(2)).to(DEV)
    want, old = mass.clone(), mass.clone()
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    q = torch.empty(B, 4, D, dtype=p.dt_q, device=DEV)
    k, v = p.stores
    if page:
        desc, paging = ssa.make_desc_paged(q, k, v, q, T), ssa.make_paging(p.d_table, page, p.n_pages)
    else:
        desc, paging = ssa.make_desc(q, k, v, q), None
    ssa.cache_compact(desc, k, v, d_ctx, d_index, d_counts, stride, mass[:, :T], paging, status)
    torch.cuda.synchronize()
    assert int(status) == 0
    after = [x.clone() for x in p.host]
    for b, x in enumerate(keep):
        at = torch.from_numpy(x)
        for new, before in zip(after, p.host):
            new.view(torch.uint8)[b, :, :len(x)] = before.view(torch.uint8)[b][:, at]
        want[b, :len(x)] = old[b, at.to(DEV)]
    ref = Tokens.__new__(Tokens)                             # (rows of the pool that no request owns are zero in both)
    ref.__dict__.update(p.__dict__)
    ref.put(*after)
    raw = lambda x: x.cpu().contiguous().view(torch.uint8)
    assert all(torch.equal(raw(a), raw(b)) for a, b in zip(p.stores, ref.stores))
    assert torch.equal(mass, want)


def test_compact_skips_what_is_not_there():
    p = Tokens(2, 2, 2, 64, 64, 1, "bf16")
    k, v = p.stores
    before = [x.clone() for x in p.stores]
    index = torch.tensor([[0, 70, 5, -1, 9], [3, 4, 5, 6, 7]], dtype=torch.int32, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    desc = ssa.make_desc(p.q[:, :, 0], k, v, p.q[:, :, 0])
    as32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    ssa.cache_compact(desc, k, v, as32(64, 6), index, as32(5, 99), 5, dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == ssa.DEV_BAD_INDEX | ssa.DEV_BAD_COUNT
    for got, old in zip((k, v), before):
        old[0, :, 2], old[0, :, 4] = old[0, :, 5].clone(), old[0, :, 9].clone()
        old[1, :, :3] = old[1, :, 3:6].clone()
        assert torch.equal(got, old)


def test_compact_leaves_shared_pages_of_rows_that_stay():
    """Two requests share their first page; its rows stay, so both may be compacted."""
    page, T, H_kv, D = 8, 32, 2, 64
    pool = [torch.randn(8, page, H_kv, D, device=DEV).bfloat16() for _ in range(2)]
    before = [x.clone() for x in pool]
    table = torch.tensor([[0, 1, 2, 3], [0, 4, 5, -1]], dtype=torch.int32, device=DEV)
    index = torch.tensor([list(range(8)) + [10, 12, 31], list(range(8)) + [9, 20, 23]], dtype=torch.int32, device=DEV)
    as32 = lambda *x: torch.tensor(x, dtype=torch.int32, device=DEV)
    q, status = torch.empty(2, 4, D, dtype=torch.bfloat16, device=DEV), as32(0)
    ssa.cache_compact(ssa.make_desc_paged(q, *pool, q, T), *pool, as32(32, 24), index, as32(11, 11), 11,
                      paging=ssa.make_paging(table, page, 8), dev_status=status)
    torch.cuda.synchronize()
    assert int(status) == 0
    for got, old in zip(pool, before):
        assert torch.equal(got[[0, 2, 3, 5, 6, 7]], old[[0, 2, 3, 5, 6, 7]])
        assert torch.equal(got[1, :3], torch.stack([old[1, 2], old[1, 4], old[3, 7]])) and torch.equal(got[1, 3:], old[1, 3:])
        assert torch.equal(got[4, :3], torch.stack([old[4, 1], old[5, 4], old[5, 7]])) and torch.equal(got[4, 3:], old[4, 3:])


@pytest.mark.parametrize("page", [0, 16])
def test_a_run_of_steps_within_a_budget(page):
    """Prompt chunk, then steps that add up weight, then eviction through lists and through compaction: both attend to the same."""
    B, H, H_kv, T, D, budget, sinks, recent = 2, 8, 2, 400, 128, 96, 4, 32
    p = Tokens(B, H, H_kv, T, D, 20, "bf16", page=page)
    ctx, mass = [300, 180], None
    for step in range(3):
        q = Tokens(B, H, H_kv, T, D, 20 if step == 0 else 1, "bf16", seed=step + 1)
        q.__dict__.update(page=p.page, stores=p.stores, host=p.host, layout=p.layout)
        if page:
            q.__dict__.update(d_table=p.d_table, n_pages=p.n_pages, table=p.table)
        ctx = [c + (step > 0) for c in ctx]
        got = q.call(ctx, None, 0, 0, mass=True, mass_in=mass)
        check(q, got, ctx, None, 0, 0, torch.float32, mass_in=None if mass is None else mass.double().cpu().numpy())
        mass = torch.from_numpy(got[2]).float().to(DEV)
    d_ctx = torch.tensor(ctx, dtype=torch.int32, device=DEV)
    index, counts = torch.full((B, budget), -1, dtype=torch.int32, device=DEV), torch.zeros(B, dtype=torch.int32, device=DEV)
    ssa.mass_to_index(mass, d_ctx, budget, sinks, recent, index, counts)
    for b in range(B):
        assert index[b].tolist() == BO.kept(mass[b].double().cpu().numpy(), ctx[b], budget, sinks, recent).tolist()
    k, v = p.stores
    one = q.q[:, :, 0]
    out = torch.zeros(B, H, D, device=DEV)
    if page:
        desc, paging = ssa.make_desc_paged(one, k, v, out, T), ssa.make_paging(p.d_table, page, p.n_pages)
    else:
        desc, paging = ssa.make_desc(one, k, v, out), None
    ws = torch.empty(ssa.decode_workspace_bytes(desc, T), dtype=torch.uint8, device=DEV)
    attend = ssa.decode_attn_sparse_paged if page else ssa.decode_attn_sparse
    attend(desc, one, k, v, *([paging] if page else []), d_ctx, index, counts, budget, out, None, ws)
    by_list, old = out.clone(), mass.clone()
    ssa.cache_compact(desc, k, v, d_ctx, index, counts, budget, mass, paging)
    dense = ssa.decode_attn_dense_paged if page else ssa.decode_attn_dense
    dense(desc, one, k, v, *([paging] if page else []), counts, out, None, ws)
    torch.cuda.synchronize()
    assert (out - by_list).abs().max() < 1e-5 and torch.equal(mass[:, :budget], old.gather(1, index.long()))


def test_a_captured_step_replayed_on_new_lengths():
    """Sums, selection and attention through the lists in one graph; lengths, queries and sums are read when it runs."""
    B, H, H_kv, T, D, budget = 2, 8, 2, 700, 128, 64
    p = Tokens(B, H, H_kv, T, D, 1, "bf16")
    k, v = p.stores
    ctx = torch.tensor([700, 400], dtype=torch.int32, device=DEV)
    out, lse, mass = torch.zeros(B, H, 1, D, device=DEV), torch.zeros(B, H, 1, device=DEV), torch.zeros(B, T, device=DEV)
    by_list, index = torch.zeros(B, H, D, device=DEV), torch.zeros(B, budget, dtype=torch.int32, device=DEV)
    counts = torch.zeros(B, dtype=torch.int32, device=DEV)
    desc, win = ssa.make_desc(p.q[:, :, 0], k, v, out[:, :, 0]), ssa.make_window(p.q, out)
    ws = torch.empty(ssa.attn_mass_workspace_bytes(desc, win), dtype=torch.uint8, device=DEV)
    desc2 = ssa.make_desc(p.q[:, :, 0], k, v, by_list)
    ws2 = torch.empty(ssa.decode_workspace_bytes(desc2, budget), dtype=torch.uint8, device=DEV)

    def step():
        ssa.attn_mass(desc, win, p.q, k, v, ctx, out, lse, mass, mass, 0.5, ws)
        ssa.mass_to_index(mass, ctx, budget, 2, 16, index, counts)
        ssa.decode_attn_sparse(desc2, p.q[:, :, 0], k, v, ctx, index, counts, budget, by_list, None, ws2)

    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for lens in ([700, 400], [64, 1], [333, 699]):
        ctx.copy_(torch.tensor(lens, dtype=torch.int32, device=DEV))
        p.q.mul_(-0.5)
        mass.fill_(0.25)
        graph.replay()
        torch.cuda.synchronize()
        got = [x.clone() for x in (out, lse, mass, index, counts, by_list)]
        mass.fill_(0.25)
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (out, lse, mass, index, counts, by_list)))
        assert counts.tolist() == [min(n, budget) for n in lens]


def test_the_runner_keeps_a_workload_within_a_budget():
    """DecodeStep: weights of a step, selection, attention through the lists, then over the compacted cache: the same rows."""
    from paper_2404_09336_b200 import inputs
    from paper_2404_09336_b200.runner import DecodeStep
    ds = DecodeStep(inputs.make_config(2, B=3, H=4), out_dtype=torch.float32)
    budget = ds.index_stride + 40
    T = ds.wl.max_ctx
    ds.attend_window(T)
    whole = ds.out.clone()
    ds.attend_mass()
    assert torch.equal(ds.out, whole)
    ctx = ds.ctx_lens.tolist()
    assert all(abs(ds.mass[b].sum().item() - 4) < 1e-4 and (ds.mass[b, n:] == 0).all() for b, n in enumerate(ctx))
    ds.select_heaviest(budget, sinks=4, recent=32)
    ds.attend_sparse()
    by_list, counts = ds.out.clone(), ds.counts.tolist()
    assert counts == [min(n, budget) for n in ctx]
    ds.compact()
    assert ds.ctx_lens.tolist() == counts
    ds.attend_dense()
    torch.cuda.synchronize()
    assert (ds.out - by_list).abs().max() < 1e-5 and int(ds.status) == 0
    ds.attend_window(32, 4)
    torch.cuda.synchronize()
    assert int(ds.status) == 0 and ds.out.isfinite().all()
