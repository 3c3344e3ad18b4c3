"""DecodeStep.append: what a token that is appended finds and leaves in the runner's own buffers (no GPU: the library's calls are
recorded)."""
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
