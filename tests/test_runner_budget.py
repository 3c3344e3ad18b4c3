"""DecodeStep's calls around a budget: what they hand to the library, and what they leave to the calls over span lists (no GPU: the
library's calls are recorded)."""
import inspect

import pytest
import torch

from paper_2404_09336_b200 import inputs, ssa
from paper_2404_09336_b200.runner import DecodeStep

CALLS = ("spans_to_index", "decode_attn_sparse", "decode_attn_spans", "decode_attn_dense", "attn_window", "attn_mass", "mass_to_index",
         "cache_compact", "decode_step", "make_step")


@pytest.fixture
def made(monkeypatch):
    """-> the calls made, as (name, arguments by name)."""
    calls = []

    def record(name):
        signature = inspect.signature(getattr(ssa, name))

        def call(*a, **k):
            bound = signature.bind(*a, **k)
            bound.apply_defaults()
            calls.append((name, bound.arguments))
            return 0
        return call

    for name in CALLS:
        monkeypatch.setattr(ssa, name, record(name))
    return calls


def small(**kw):
    return DecodeStep(inputs.make_config(2, B=3, H=4), device="cpu", **kw)


def budgets(ds):
    return [1, ds.max_selected // 2, ds.max_selected, ds.index_stride + 40, ds.wl.max_ctx, ds.wl.max_ctx + 100]


def test_a_budget_does_not_bound_the_span_lists(made):
    ds = small()
    spans = ds.max_selected, ds.index, ds.counts, ds.index_stride
    for budget in budgets(ds):
        ds.mass = torch.zeros(3, ds.wl.max_ctx)
        ds.select_heaviest(budget)
        ds.build_index()
        ds.attend_sparse()
        ds.select_heaviest(budget)
        ds.attend_spans()
        ds.step()
        ds.attend_sparse()
        ds.select_heaviest(budget)
        ds.attend_spans(want_lists=True)
        for name, a in made:
            if name in ("decode_attn_sparse", "decode_attn_spans", "make_step"):
                assert a["max_selected"] == spans[0], (name, budget)
                index = a.get("index", a.get("index_out"))
                assert index is None or (index is spans[1] and a.get("counts", a.get("counts_out")) is spans[2]), (name, budget)
        assert (ds.max_selected, ds.index, ds.counts, ds.index_stride) == spans
        made.clear()


def test_lists_of_a_budget_are_attended_to_and_compacted_with_its_bound(made):
    ds = small()
    ds.mass = torch.zeros(3, ds.wl.max_ctx)
    ds.build_index()
    for budget in budgets(ds):
        ds.select_heaviest(budget, sinks=1, recent=0)
        ds.attend_spans()                                    # writes no lists
        ds.attend_sparse()
        ds.compact()
        (_, kept), _, (_, sparse), (_, moved) = made[-4:]
        assert kept["budget"] == min(budget, ds.wl.max_ctx) == sparse["max_selected"] == moved["max_selected"]
        assert kept["sinks"] == (1 if budget <= ds.wl.max_ctx else 0) and kept["budget"] <= kept["index"].shape[1]
        assert kept["index"] is sparse["index"] is moved["index"] is ds.index
        assert kept["counts"] is sparse["counts"] is moved["counts"] is ds.counts
        assert sparse["workspace"].numel() >= ssa.decode_workspace_bytes(ds.desc, sparse["max_selected"])
    ds.step()
    ds.compact()
    assert made[-1][1]["max_selected"] == ds.max_selected and made[-1][1]["index"] is made[-3][1]["index"]


def test_refused_budgets_change_nothing():
    ds = small()
    ds.mass = torch.zeros(3, ds.wl.max_ctx)
    before = ds.index, ds.counts, ds.max_selected
    for bad in (dict(budget=0), dict(budget=-3), dict(budget=8, sinks=5, recent=4), dict(budget=8, sinks=-1), dict(budget=9999, recent=-1),
                dict(budget=9999, sinks=9000, recent=1000)):
        with pytest.raises(ssa.SsaError):
            ds.select_heaviest(**bad, stream=0)
        assert (ds.index, ds.counts, ds.max_selected) == before


def test_calls_around_a_budget_leave_the_other_calls_their_workspace_and_keep_their_own(made):
    import gc
    import weakref
    ds = small()
    ds.mass = torch.zeros(3, ds.wl.max_ctx)
    ds.step()
    steps, workspace = dict(ds._steps), ds.workspace
    refs, sizes = [], []
    for i, need in enumerate((1000, workspace.numel() + 1, 100, 2 * workspace.numel() + 7, 2 * workspace.numel() + 8)):
        with pytest.MonkeyPatch.context() as m:
            m.setattr(ssa, "attn_mass_workspace_bytes" if i % 2 else "attn_window_workspace_bytes", lambda *a: need)
            ds.attend_mass() if i % 2 else ds.attend_window(7)
        room = made.pop()[1]["workspace"]
        assert room.numel() >= need and room is not workspace
        refs.append(weakref.ref(room))
        sizes.append(room.numel())
        del room
    gc.collect()
    assert ds.workspace is workspace and ds._steps == steps
    assert all(r() is not None for r in refs)                # a captured graph may still hold their addresses
    assert sum(sorted(set(sizes))[:-1]) <= max(sizes)
    ds.select_heaviest(30)
    ds.attend_sparse()
    assert made[-1][1]["workspace"] is not workspace


def test_no_call_fills_a_buffer(made, monkeypatch):
    """A fill would go to torch's current stream and not to the call's, and into a graph that is being captured."""
    ds = small()
    assert ds.mass.shape == (3, ds.wl.max_ctx) and not ds.mass.any()

    def never(*a, **k):
        raise AssertionError("a buffer was filled")

    for name in ("zeros", "full", "ones", "zeros_like", "full_like", "tensor"):
        monkeypatch.setattr(torch, name, never)
    ds.select_heaviest(20)                                   # before any sums: nothing was looked at yet
    ds.attend_mass(0.5)
    ds.attend_window(30, 2)
    for budget in (50, ds.index_stride + 1, ds.wl.max_ctx):
        ds.select_heaviest(budget)
        ds.attend_sparse()
    assert all(a["mass"] is ds.mass for name, a in made if name == "mass_to_index")
    assert all(a["mass_in"] is a["mass_out"] is ds.mass for name, a in made if name == "attn_mass")


@pytest.mark.parametrize("layout", ["bhtd", "bthd"])
def test_every_copy_of_the_cache_is_compacted_the_sums_once(made, layout):
    ds = small(kv_copies=3, layout=layout)
    ds.counts.fill_(5)
    ds.select_copy(1)
    ds.compact()
    assert [a["k_cache"].data_ptr() for _, a in made] == [x.data_ptr() for x in ds.k_store]
    assert [a["v_cache"].data_ptr() for _, a in made] == [x.data_ptr() for x in ds.v_store]
    assert all(a["k_cache"].shape == a["v_cache"].shape == (3, 4, ds.wl.max_ctx, ds.wl.D) for _, a in made)
    assert [a["mass"] is ds.mass for _, a in made] == [True, False, False] and all(a["mass"] is None for _, a in made[1:])
    assert ds.ctx_lens.tolist() == [5, 5, 5] and ds.k.data_ptr() == ds.k_store[1].data_ptr()


def test_contexts_are_no_longer_than_what_was_moved(made):
    ds = small()
    bound = ds.max_selected
    ds.ctx_lens.copy_(torch.tensor([900, 100, 7]))
    ds.counts.copy_(torch.tensor([bound + 9, -7, 8]))        # clamped by the call: its bound, nothing, its context
    ds.compact()
    assert ds.ctx_lens.tolist() == [bound, 0, 7]


def test_a_workspace_that_block_lists_outgrow_stays_alive(made, monkeypatch):
    import gc
    import weakref
    ds = small()
    ds.attend_dense()
    ref = weakref.ref(made.pop()[1]["workspace"])
    monkeypatch.setattr(ssa, "decode_blockmask_workspace_bytes", lambda *a: ds.workspace.numel() + 1)
    ds.enable_blockmask()
    gc.collect()
    assert ref() is not None and ds.workspace is not ref()   # a captured graph may still hold its address
