"""The fp64 statement of the budget operators against hand-made cases and the framework's first oracle."""
import numpy as np
import pytest

from oracle import budget_oracle as BO
from oracle import ssa_oracle as O


def test_visible_by_hand():
    assert BO.visible(5, 2, 2, 1).tolist() == [[True, False, True, True, False], [True, False, False, True, True]]
    assert BO.visible(3, 3, 0, 0).tolist() == [[True, False, False], [True, True, False], [True, True, True]]
    assert BO.visible(1, 3, 4, 2).tolist() == [[False], [False], [True]]       # more tokens than positions: the first see nothing
    assert BO.visible(4, 1, 1, 0).tolist() == [[False, False, False, True]]
    assert BO.visible(0, 2, 0, 0).shape == (2, 0)


def test_one_token_is_the_attention_over_its_list():
    rng = np.random.default_rng(0)
    bits = lambda *s: (rng.standard_normal(s).astype(np.float16)).view(np.uint16)
    q, k, v = bits(2, 4, 64), bits(2, 4, 50, 64), bits(2, 4, 50, 64)
    ctx = np.array([50, 23], np.int32)
    index, counts = np.full((2, 50), -1, np.int32), []
    for b, n in enumerate(ctx):
        lst = [j for j in range(n) if j < 3 or j > n - 1 - 10]
        index[b, :len(lst)] = lst
        counts.append(len(lst))
    ref, ref_lse = O.decode_attn_sparse(q, k, v, ctx, index, np.array(counts), 0.125, "f16")
    f = lambda x: x.view(np.float16).astype(np.float64)
    got = BO.attention(f(q)[:, :, None], f(k), f(v), ctx, [1, 1], 10, 3, 0.125)
    for b in range(2):
        assert np.abs(got[b]["out"][:, 0] - ref[b]).max() < 1e-12
        assert np.abs(got[b]["lse"][:, 0] - ref_lse[b]).max() < 1e-12
        assert np.abs(got[b]["weights"].sum(-1) - 1).max() < 1e-12


def test_what_is_not_seen_does_not_matter_and_what_is_does():
    rng = np.random.default_rng(1)
    q, k, v = rng.standard_normal((1, 2, 3, 8)), rng.standard_normal((1, 1, 12, 8)), rng.standard_normal((1, 1, 12, 8))
    a = BO.attention(q, k, v, [10], [3], 4, 2, 1.0)[0]
    v2 = v.copy()
    v2[0, 0, 3] = np.nan                                     # before every window, behind the sinks
    assert np.array_equal(BO.attention(q, k, v2, [10], [3], 4, 2, 1.0)[0]["out"], a["out"])
    v2[0, 0, 4, 5] = np.inf                                  # seen by the first token only
    b = BO.attention(q, k, v2, [10], [3], 4, 2, 1.0)[0]["out"]
    assert np.isinf(b[:, 0, 5]).all() and np.abs(b[:, 1:] - a["out"][:, 1:]).max() < 1e-12


def test_kept_by_hand():
    m = np.array([9, 1, 5, np.nan, 5, 5, -np.inf, 0.0, -0.0, 7])
    assert BO.kept(m, 10, 10, 0, 0).tolist() == list(range(10))
    assert BO.kept(m, 10, 5, 1, 2).tolist() == [0, 2, 4, 8, 9]
    assert BO.kept(m, 10, 9, 0, 0).tolist() == [0, 1, 2, 4, 5, 6, 7, 8, 9]
    assert BO.kept(m, 10, 7, 0, 0).tolist() == [0, 1, 2, 4, 5, 7, 9]           # of the equal zeros the lower position
    assert BO.kept(m, 10, 3, 1, 2).tolist() == [0, 8, 9]
    assert BO.kept(m, 2, 3, 1, 2).tolist() == [0, 1]


@pytest.mark.parametrize("n,budget,sinks,recent", [(40, 17, 3, 5), (40, 1, 0, 0), (40, 39, 20, 19)])
def test_kept_is_sorted_and_of_the_right_size(n, budget, sinks, recent):
    m = np.random.default_rng(n).integers(0, 4, n).astype(float)
    got = BO.kept(m, n, budget, sinks, recent).tolist()
    assert len(got) == budget and got == sorted(set(got))
    assert set(range(sinks)) | set(range(n - recent, n)) <= set(got)
    out = sorted(set(range(n)) - set(got))
    mid = [j for j in got if sinks <= j < n - recent]
    assert all((m[j], -j) < (m[i], -i) for j in out for i in mid)
