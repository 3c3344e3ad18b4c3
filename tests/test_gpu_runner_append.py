"""DecodeStep.append among the calls of earlier tokens: eviction by sums, full contexts, refused calls, captured steps."""
import numpy as np
import pytest
import torch

from oracle import budget_oracle as BO
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
