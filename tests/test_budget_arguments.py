"""Tensors that the budget calls would read or write past, refused by the binding (no GPU)."""
import pytest
import torch

from paper_2404_09336_b200 import ssa


def test_lengths_of_new_tokens_are_one_per_request_side_by_side():
    q = torch.zeros(3, 8, 4, 128)
    lens = torch.arange(12, dtype=torch.int32).view(4, 3)
    for bad in (lens[:3, 0], lens[0, :2], lens.t()[:3], torch.zeros(0, dtype=torch.int32), lens[0].to("meta")):
        with pytest.raises(ValueError, match="one length per request"):
            ssa.make_window(q, q, q_lens=bad)
    for good in (lens[1], lens, lens[0, :3].view(3, 1)):
        assert ssa.make_window(q, q, q_lens=good).q_lens == good.data_ptr()
    assert ssa.make_window(q[:1], q[:1], q_lens=lens[2:3, 0]).q_lens == lens[2, 0].data_ptr()


def test_sums_have_a_row_for_every_request():
    d, w = ssa.AttnDesc(), ssa.Window()
    d.B, d.max_ctx = 3, 40
    i = torch.zeros(3, 40, dtype=torch.int32)
    few, enough = torch.zeros(2, 40), torch.zeros(3, 40)
    calls = {"attn_mass": lambda m: ssa.attn_mass(d, w, None, None, None, None, None, None, None, m, stream=0),
             "attn_mass in": lambda m: ssa.attn_mass(d, w, None, None, None, None, None, None, m, enough, stream=0),
             "mass_to_index": lambda m: ssa.mass_to_index(m, i[:, 0], 41, 0, 0, i, i[:, 0], stream=0),
             "cache_compact": lambda m: ssa.cache_compact(d, None, None, None, i, None, 5, mass=m, stream=0)}
    for name, call in calls.items():
        for bad in (few, enough[0], enough[None]):
            with pytest.raises(ValueError, match="3 rows of"):
                call(bad)
        with pytest.raises(ssa.SsaError):                    # (on to the library, which refuses the rest)
            call(enough)


def test_one_row_of_sums_has_no_row_stride():
    d, w = ssa.AttnDesc(), ssa.Window()
    d.B, d.max_ctx = 1, 40
    call = lambda a, b: ssa.attn_mass(d, w, None, None, None, None, None, None, a, b, stream=0)
    with pytest.raises(ssa.SsaError):                        # (on to the library, which refuses the rest)
        call(torch.zeros(1, 64), torch.zeros(1, 40))
    d.B = 2
    with pytest.raises(ValueError, match="row stride"):
        call(torch.zeros(2, 64), torch.zeros(2, 40))
