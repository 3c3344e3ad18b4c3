"""ssa_attn_window held to the bound of the kernel that serves the call: weights of two 16-bit parts wherever the tiles do not run."""
import pytest
import torch

from budget_util import Tokens, check

pytestmark = pytest.mark.gpu


def tiles_serve(p):
    """As the library chooses: more than 24 rows of a K/V head, a 16-bit cache, pages of eight rows at least, no strides of zero."""
    strides = [(s, n) for x in p.stores for s, n in zip(x.stride()[:3], x.shape[:3])]
    return (p.dt.itemsize == 2 and p.H // p.H_kv * p.n_q > 24 and (not p.page or p.page >= 8) and
            (p.page or all(s > 0 or n == 1 for s, n in strides)))


def run(p, ctx, new, window, sinks):
    assert not tiles_serve(p)
    got = p.call(ctx, new, window, sinks, torch.float32)
    check(p, got, ctx, new, window, sinks, torch.float32, many=False)


@pytest.mark.parametrize("dtype,H,H_kv,D,n_q,page", [
    ("fp8", 4, 2, 128, 64, 0), ("fp8", 8, 2, 64, 130, 0), ("fp8", 6, 1, 128, 40, 16), ("fp8", 4, 4, 128, 257, 0),    # chunks over an 8-bit cache
    ("bf16", 4, 4, 128, 17, 0), ("f16", 4, 4, 64, 24, 0), ("bf16", 8, 2, 128, 6, 0), ("f16", 24, 1, 128, 1, 0),       # 24 rows and fewer
    ("bf16", 8, 2, 128, 150, 2), ("f16", 4, 2, 64, 90, 4), ("bf16", 4, 4, 64, 33, 1)])                                # pages of fewer rows
def test_calls_that_the_tiles_do_not_serve(dtype, H, H_kv, D, n_q, page):
    T = 600
    p = Tokens(2, H, H_kv, T, D, n_q, dtype, page=page)
    for window, sinks in ((0, 0), (3, 1), (50, 7), (128, 130)):
        run(p, [T, max(n_q, 333)], [n_q, n_q - n_q // 3], window, sinks)


@pytest.mark.parametrize("n_q", [30, 60, 200])
@pytest.mark.parametrize("heads,requests", [(True, False), (False, True), (True, True)])
def test_strides_of_zero_are_left_to_the_kernel_for_few_rows(n_q, heads, requests):
    p = Tokens(2, 4, 2, 300, 128, n_q)
    share = lambda x: (x[:, :1] if heads else x)[:1 if requests else 2].expand(2, 2, -1, -1)
    p.host, p.stores = [share(x) for x in p.host], [share(x) for x in p.stores]
    for window, sinks in ((0, 0), (2, 1), (70, 3)):
        run(p, [300, 233], None, window, sinks)


@pytest.mark.parametrize("dtype,H,H_kv,D,n_q,page", [("bf16", 4, 4, 128, 130, 0), ("bf16", 8, 2, 64, 75, 0), ("f16", 4, 1, 64, 300, 0), ("f16", 6, 2, 128, 64, 0),
                                                     ("bf16", 8, 2, 128, 150, 8), ("f16", 4, 2, 128, 90, 32), ("bf16", 4, 2, 64, 257, 512)])
def test_fp32_outputs_of_the_tiles_have_weights_of_two_parts(dtype, H, H_kv, D, n_q, page):
    T = 700
    p = Tokens(3, H, H_kv, T, D, n_q, dtype, page=page)
    assert tiles_serve(p)
    ctx, new = [T, max(n_q, 333), 31], [n_q, n_q - n_q // 3, n_q]
    for window, sinks in ((0, 0), (3, 1), (50, 7), (128, 130)):
        got = p.call(ctx, new, window, sinks, torch.float32)
        check(p, got, ctx, new, window, sinks, torch.float32, many=False)


def test_fp32_outputs_of_a_chunk_over_a_split_context():
    p = Tokens(1, 4, 2, 5000, 128, 40)
    assert tiles_serve(p)
    for window, sinks in ((0, 0), (2500, 64)):
        got = p.call([5000], None, window, sinks, torch.float32)
        check(p, got, [5000], None, window, sinks, torch.float32, many=False)
