"""The oracle of the cache's formats, of bounds and of selection, pinned on definitions and closed forms (no GPU)."""
import numpy as np
import torch

from oracle import budget_oracle as BO
from oracle import cache_oracle as CO


def test_e4m3_is_torchs():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    np.testing.assert_array_equal(CO.e4m3_values(), want)
    x = np.concatenate([want[np.isfinite(want)], np.linspace(-460, 460, 4001), np.geomspace(1e-5, 500, 4001), [17.0, 18.5, 2.0 ** -10, -0.0]])
    got = CO.to_e4m3(x.astype(np.float32))
    np.testing.assert_array_equal(got, torch.tensor(x, dtype=torch.float32).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_4_bit_values():
    codes = np.arange(16, dtype=np.uint8)
    row = (codes[::2] | codes[1::2] << 4).astype(np.uint8)
    one = CO.to_e4m3(np.array([1.0]))
    np.testing.assert_array_equal(CO.fp4_values(row, one), [0, .5, 1, 1.5, 2, 3, 4, 6, 0, -.5, -1, -1.5, -2, -3, -4, -6])
    x = CO.fp4_values(row, one).astype(np.float32)
    got = CO.to_fp4(x)
    np.testing.assert_array_equal(got[0], row)
    np.testing.assert_array_equal(got[1], one)


def test_4_bit_rounding_is_to_the_nearest_and_halfway_to_even():
    x = np.zeros(32, np.float32)
    x[0] = 6                                                   # scale 1
    x[1:16] = [.25, .75, 1.25, 1.75, 2.5, 3.5, 5, .26, .74, -.25, -.75, -5, 5.01, 2.49, 0]
    codes, scales = CO.to_fp4(x)
    np.testing.assert_array_equal(CO.fp4_values(codes, scales)[:16], [6, 0, 1, 1, 2, 2, 4, 4, .5, .5, 0, -1, -4, 6, 2, 0])
    assert scales[1] == 0 and not codes[8:].any()              # sixteen zeros: scale 0
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((200, 64)) * np.exp(rng.standard_normal((200, 1)) * 3)).astype(np.float32)
    codes, scales = CO.to_fp4(x)
    s = np.repeat(CO.e4m3_values()[scales], 16, -1)
    grid = np.concatenate([CO.E2M1, -CO.E2M1]) * s[..., None]
    np.testing.assert_allclose(np.abs(CO.fp4_values(codes, scales) - x), np.abs(grid - x[..., None]).min(-1), atol=1e-6 * np.abs(x).max())


def test_rotation_keeps_lengths_and_products_of_differences():
    rng = np.random.default_rng(1)
    x, y = rng.standard_normal((2, 1, 64))
    angle = np.arange(40)[:, None] * 100.0 ** (-np.arange(16) / 16)
    table = np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)
    for interleaved in (False, True):
        turn = lambda v, p: CO.rotated(v, np.array([p]), table, interleaved)[0].astype(np.float64)
        np.testing.assert_allclose(np.linalg.norm(turn(x, 33)), np.linalg.norm(x), rtol=1e-6)
        np.testing.assert_allclose(turn(x, 9) @ turn(y, 4), turn(x, 35) @ turn(y, 30), atol=1e-5)
        np.testing.assert_array_equal(turn(x, 7)[32:], x[0, 32:].astype(np.float32))
        np.testing.assert_array_equal(turn(x, 0), x[0].astype(np.float32))


def test_a_block_scores_at_least_as_its_best_keys():
    rng = np.random.default_rng(2)
    k, q = rng.standard_normal((150, 32)), rng.standard_normal((3, 32))
    least, most = CO.bounds(k, 141, 32)
    s = CO.scores(q, least, most)
    assert len(s) == 5
    for j in range(5):
        assert s[j] >= (q @ k[32 * j: min(141, 32 * j + 32)].T).max(1).sum() - 1e-12
    below, above = np.minimum(q, 0).sum(0), np.maximum(q, 0).sum(0)
    np.testing.assert_allclose(s, least @ below + most @ above)


def test_attention_over_all_positions_is_full_attention():
    rng = np.random.default_rng(3)
    q, k, v = rng.standard_normal((2, 16)), rng.standard_normal((40, 16)), rng.standard_normal((40, 16))
    got = CO.attention(q, k, v, np.arange(33), 0.25)
    want = BO.attention(q[None, :, None], k[None, None], v[None, None], [33], [1], 0, 0, 0.25)[0]
    np.testing.assert_allclose(got[0], want["out"][:, 0])
    np.testing.assert_allclose(got[1], want["lse"][:, 0])
    assert not CO.attention(q, k, v, np.arange(0), 0.25)[0].any()
