"""DecodeStep's calls that fill the cache and read its blocks: what they hand to the library (no GPU: the library's calls are recorded)."""
import inspect

import pytest
import torch

from paper_2404_09336_b200 import inputs, ssa
from paper_2404_09336_b200.runner import DecodeStep

CALLS = ("cache_append", "block_bounds", "block_select", "attn_blocks", "attn_window_fp4", "cache_compact", "mass_to_index")


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


def test_a_token_goes_to_every_copy_and_to_the_4_bit_one(made):
    ds = small(kv_copies=2)
    ctx = ds.ctx_lens.clone()
    ds.enable_fp4()
    ds.enable_blocks(64, 8)
    made.clear()
    k, v, q = (torch.zeros(3, 4, ds.wl.D, dtype=ds.q.dtype) for _ in range(3))
    ds.append(k, v, q, torch.zeros(ds.wl.max_ctx, 64))
    assert torch.equal(ds.ctx_lens, ctx + 1)
    assert [n for n, _ in made] == ["cache_append"] * 3 + ["block_bounds"]
    caches = [a["k_cache"].data_ptr() for _, a in made[:3]]
    assert caches == [ds.k_store[0].data_ptr(), ds.k_store[1].data_ptr(), ds.fp4[0].data_ptr()]
    assert [a["q"] is q for _, a in made[:3]] == [True, False, False]            # queries are rotated once
    assert [a["desc"].kv_dtype for _, a in made[:3]] == [ssa.BF16, ssa.BF16, ssa.FP4_E2M1] and made[2][1]["k_scales"] is ds.fp4[2]
    assert all(a["append"].rotary_dims == 64 and a["append"].n_q == 1 for _, a in made[:3]) and made[3][1]["blocks"].n_q == 1


def test_a_compaction_renews_bounds_and_the_4_bit_copy(made):
    ds = small()
    ds.enable_fp4()
    ds.enable_blocks(32, 8)
    ds.select_heaviest(20)
    ds.counts.fill_(20)
    made.clear()
    ds.compact()
    assert [n for n, _ in made] == ["cache_compact", "block_bounds", "cache_append"]
    assert made[1][1]["blocks"].n_q == ds.wl.max_ctx and made[2][1]["append"].n_q == ds.wl.max_ctx
    assert made[2][1]["ctx_lens"].tolist() == [ds.wl.max_ctx] * 3


def test_lists_and_workspaces(made):
    ds = small()
    ds.enable_blocks(64, 8, 1, 2)
    ds.select_blocks()
    ds.attend_blocks()
    _, a = made[-1]
    assert a["index"].shape == (3, 4, 1, 8) and a["counts"].shape == (3, 4, 1) and a["workspace"].numel() >= ssa.attn_blocks_workspace_bytes(ds.desc, ds.blocks)
    assert made[-2][1]["index"] is a["index"] and (ds.blocks.sinks, ds.blocks.recent, ds.blocks.budget) == (1, 2, 8)
    assert made[0][0] == "block_bounds" and made[0][1]["blocks"].n_q == ds.wl.max_ctx


def test_4_bit_caches_go_with_bf16_queries():
    ds = small()
    ds.q = ds.q.to(torch.float16)
    with pytest.raises(ValueError, match="bf16"):
        ds.enable_fp4()
