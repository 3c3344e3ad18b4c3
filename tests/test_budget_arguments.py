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
