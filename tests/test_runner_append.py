"""DecodeStep.append: what a token that is appended finds and leaves in the runner's own buffers (no GPU: the library's calls are
recorded)."""
import gc
import weakref

import pytest
import torch

from paper_2404_09336_b200 import ssa
from test_runner_blocks import made, small                   # noqa: F401  (made: a fixture)


def rows(ds, dtype=None):
    return [torch.zeros(ds.wl.B, ds.wl.H, ds.wl.D, dtype=dtype or ds.q.dtype) for _ in range(3)]


def test_an_appended_position_has_no_sum_yet(made):          # noqa: F811
    ds = small()
    ds.mass.fill_(7.0)
    ctx = ds.ctx_lens.clone()
    k, v, q = rows(ds)
    ds.append(k, v, q)
    ds.append(k, v)
    for b, n in enumerate(ctx.tolist()):
        assert not ds.mass[b, n:n + 2].any() and (ds.mass[b, :n] == 7).all() and (ds.mass[b, n + 2:] == 7).all()


def test_a_refused_token_changes_nothing(made, monkeypatch):             # noqa: F811
    ds = small()
    ds.enable_blocks(64, 8)
    ds.mass.fill_(7.0)
    ctx = ds.ctx_lens.clone()
    k, v, q = rows(ds)
    for bad in ((k.half(), v, q), (k, v.float(), q), (k[:2], v, q), (k, v, q.half()), (k, v, q, torch.zeros(9, 64).double())):
        with pytest.raises(ValueError):
            ds.append(*bad)

    def refuse(*a, **kw):
        raise ssa.SsaError("ssa_cache_append", 2)
    monkeypatch.setattr(ssa, "cache_append", refuse)
    with pytest.raises(ssa.SsaError):
        ds.append(k, v, q)
    assert torch.equal(ds.ctx_lens, ctx) and (ds.mass == 7).all()


def test_full_contexts_stay_as_they_are(made):               # noqa: F811
    """The library is told of their token (it flags it), but not to store one."""
    ds = small(kv_copies=2)
    T = ds.wl.max_ctx
    ds.ctx_lens.copy_(torch.tensor([T, T - 1, 5]))
    ds.mass.fill_(7.0)
    k, v, q = rows(ds)
    for want, stored in (([T, T, 6], [0, 1, 1]), ([T, T, 7], [0, 0, 1])):
        made.clear()
        before = ds.ctx_lens.clone()
        ds.append(k, v, q)
        calls = [a for n, a in made if n == "cache_append"]
        assert len(calls) == 2 and ds.ctx_lens.tolist() == want
        for a in calls:
            assert torch.equal(a["ctx_lens"], before + 1) and a["append"].q_lens == ds._new_lens.data_ptr()
        assert ds._new_lens.tolist() == stored
    assert (ds.mass[0] == 7).all() and ds.mass[1, T - 1] == 0 and (ds.mass[1, : T - 1] == 7).all()
    assert not ds.mass[2, 5:7].any() and (ds.mass[2, :5] == 7).all() and (ds.mass[2, 7:] == 7).all()


def test_a_4_bit_copy_of_more_rows_than_a_call_takes(made, monkeypatch):  # noqa: F811
    """H n_q <= 2^24 in a call: long contexts of many query heads are copied in parts."""
    ds = small(query_heads=4096)
    T = ds.wl.max_ctx                                        # 2^10: all at once
    ds.enable_fp4()
    assert [a["append"].n_q for _, a in made] == [T]
    ds.q, ds.out = (x.new_zeros(ds.wl.B, 1 << 16, ds.wl.D) for x in (ds.q, ds.out))      # as if there were 16 times as many heads
    made.clear()
    ds.enable_fp4()
    parts = [(int(a["ctx_lens"][0]) - a["append"].n_q, int(a["ctx_lens"][0])) for _, a in made]
    assert parts == [(t, t + 256) for t in range(0, T, 256)]
    for (t, z), (_, a) in zip(parts, made):
        assert a["append"].n_q * (1 << 16) <= 1 << 24 and torch.equal(a["k_new"], ds.k[:, :, t:z]) and a["k_new"].data_ptr() == ds.k[:, :, t:z].data_ptr()
        assert a["k_cache"] is ds.fp4[0] and a["v_scales"] is ds.fp4[3]


def test_blocks_that_are_refused_leave_none(made, monkeypatch):          # noqa: F811
    ds = small()

    def refuse(*a, **kw):
        raise ssa.SsaError("ssa_block_bounds", 9)
    with monkeypatch.context() as m:
        m.setattr(ssa, "block_bounds", refuse)
        with pytest.raises(ssa.SsaError):
            ds.enable_blocks(48, 8)
    made.clear()
    ds.append(*rows(ds))
    assert [n for n, _ in made] == ["cache_append"]
    ds.enable_blocks(64, 8)
    was = ds.bounds, ds.block_lists, ds.blocks
    with monkeypatch.context() as m:
        m.setattr(ssa, "block_bounds", refuse)
        with pytest.raises(ssa.SsaError):
            ds.enable_blocks(32, 2)
    assert ds.bounds is was[0] and ds.block_lists is was[1] and ds.blocks is was[2]


def test_what_graphs_were_captured_with_stays(made):         # noqa: F811
    """Blocks asked for once more have buffers of their own beside the first, a 4-bit copy is made anew in its place."""
    ds = small()
    ds.enable_blocks(64, 8)
    ds.enable_fp4()
    first = [weakref.ref(x) for x in (ds.bounds, *ds.block_lists, *ds.fp4, ds._filled[0][1])]
    places = [x.data_ptr() for x in ds.fp4]
    made.clear()
    ds.enable_blocks(32, 4)
    ds.enable_fp4()
    gc.collect()
    assert all(x() is not None for x in first) and [x.data_ptr() for x in ds.fp4] == places
    assert ds.bounds is not first[0]() and [n for n, _ in made] == ["block_bounds", "cache_append"]
