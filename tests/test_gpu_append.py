"""ssa_cache_append: what is stored, bit for bit, in every type and layout; what is left alone."""
import numpy as np
import pytest
import torch

from budget_util import DEV
from cache_util import DTYPES, Cache, query_type
from oracle import cache_oracle as CO
from paper_2404_09336_b200 import ssa

pytestmark = pytest.mark.gpu


def table_of(n, R):
    angle = np.arange(n)[:, None] * 10000.0 ** (-np.arange(R // 2) * 2 / R)
    return torch.tensor(np.concatenate([np.cos(angle), np.sin(angle)], 1), dtype=torch.float32)


def stored(x, dtype):
    """fp32 rows -> (bits, scales) as the cache has them."""
    x = np.ascontiguousarray(x, np.float32)
    if dtype == "fp4":
        return tuple(torch.from_numpy(np.ascontiguousarray(y)) for y in CO.to_fp4(x))
    if dtype == "fp8":
        return torch.from_numpy(CO.to_e4m3(x)), None
    return torch.from_numpy(x).to(query_type(dtype)), None


def raw(x):
    return x.view(torch.uint8) if x.element_size() == 1 else x.view(torch.int16)


def run(c, H, n_q, ctx, new, R=0, interleaved=False, positions=None, n_positions=None, table=None, with_q=True, spread=1.0, seed=5,
        factors=(1.0, 1.0), in_place=False, edit=None, stream=None):
    """Appends random rows and compares the whole cache, queries and status with the oracle's."""
    g = torch.Generator().manual_seed(seed)
    B, H_kv, D, dt = c.B, c.H_kv, c.D, query_type(c.dtype)
    k_new, v_new = ((torch.randn(B, n_q, H_kv, D, generator=g) * spread).to(dt).permute(0, 2, 1, 3) for _ in range(2))
    q = torch.randn(B, n_q, H, D, generator=g).to(dt).permute(0, 2, 1, 3)
    if edit:
        edit(k_new, v_new)
    cos_sin = table_of(n_positions or c.T, R) if R else None
    want = {n: c.get(n).clone() for n in c.parts}
    want_q = torch.full((B, H, n_q, D), 3.0, dtype=dt)
    if in_place:
        want_q = q.clone()
    pages = (c.table if table is None else table) if c.page else None
    bad = False
    for b in range(B):
        n, m = min(ctx[b], c.T), (n_q if new is None else min(new[b], n_q))
        for t in range(m):
            pos = n - m + t
            if pos < 0:
                continue
            at = pos if positions is None else int(positions[b][t])
            if R and not 0 <= at < len(cos_sin):
                bad = True
                continue
            turn = lambda x: CO.rotated(x[b, :, t].float().numpy(), np.full(x.shape[1], at), None if cos_sin is None else cos_sin.numpy(), interleaved)
            if with_q:
                want_q[b, :, t] = torch.from_numpy(turn(q)).to(dt)
            if c.page and not 0 <= int(pages[b, pos // c.page]) < c.n_pages:
                bad = True
                continue
            for name, x, f in (("k", turn(k_new), factors[0]), ("v", v_new[b, :, t].float().numpy(), factors[1])):
                bits, scales = stored(x * np.float32(f), c.dtype)
                raw(want[name])[b, :, pos] = raw(bits)
                if scales is not None:
                    want[name + "_scales"][b, :, pos] = scales
    d = lambda x: None if x is None else x.to(DEV)
    d_q, status = q.to(DEV), torch.zeros(1, dtype=torch.int32, device=DEV)
    d_out = d_q if in_place else torch.full((B, H, n_q, D), 3.0, dtype=dt, device=DEV)
    d_pos = None if positions is None else torch.tensor(positions, dtype=torch.int32, device=DEV)
    d_ctx, d_new, d_cs = torch.tensor(ctx, dtype=torch.int32, device=DEV), None if new is None else torch.tensor(new, dtype=torch.int32, device=DEV), d(cos_sin)
    d_k, d_v = d(k_new), d(v_new)
    a = ssa.make_append(d_k, d_v, d_q if with_q else None, d_out if with_q else None, d_cs, interleaved, d_pos, d_new, c.paging(table), *factors)
    desc = c.desc(d_q, d_q)
    torch.cuda.synchronize()
    ssa.cache_append(desc, a, d_k, d_v, d_ctx, c.parts["k"], c.parts["v"], d_q if with_q else None, d_out if with_q else None,
                     c.scales("k"), c.scales("v"), status, stream)
    torch.cuda.synchronize()
    for name in want:
        got, ref = raw(c.get(name)), raw(want[name])
        assert torch.equal(got, ref), f"{name}: {int((got != ref).sum())} of {got.numel()}"
    if with_q or in_place:
        assert torch.equal(raw(d_out.cpu().contiguous()), raw(want_q.contiguous()))
    clamped = any(x > c.T for x in ctx) or (new is not None and any(x > n_q for x in new))
    assert int(status) == (ssa.DEV_BAD_INDEX if bad else 0) | (ssa.DEV_BAD_COUNT if clamped else 0)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("layout", ["bhtd", "bthd", "spaced", "paged"])
def test_types_and_layouts(dtype, D, layout):
    page = 8 if layout == "paged" else 0
    c = Cache(3, 2, 60, D, dtype, "bhtd" if page else layout, page, seed=D)
    run(c, 6, 5, [60, 33, 5], [5, 3, 0], R=D, seed=1)
    run(c, 6, 1, [17, 1, 60], None, R=32, interleaved=True, seed=2)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("R", [0, 32, 64, 96, 128])
@pytest.mark.parametrize("interleaved", [False, True])
def test_rotations(dtype, R, interleaved):
    c = Cache(2, 3, 300, 128, dtype)
    run(c, 3, 70, [300, 290], [70, 64], R=R, interleaved=interleaved, spread=2.0)


@pytest.mark.parametrize("H,H_kv", [(1, 1), (8, 8), (32, 8), (40, 1), (33, 11)])
def test_heads(H, H_kv):
    for dtype in ("bf16", "fp4"):
        c = Cache(2, H_kv, 20, 64, dtype)
        run(c, H, 3, [20, 9], [3, 2], R=64)
        run(c, H, 3, [20, 9], [3, 2], R=64, with_q=False, seed=8)
        run(c, H, 3, [20, 9], [1, 2], R=64, in_place=True, seed=9)


@pytest.mark.parametrize("dtype", DTYPES)
def test_tokens_without_a_place(dtype):
    c = Cache(4, 2, 24, 128, dtype, page=8)
    table = c.table.clone()
    table[0, 1], table[1, 0] = -1, c.n_pages
    run(c, 4, 6, [14, 9, 3, 0], [6, 6, 6, 6], R=64, table=table)          # missing pages; positions below zero
    run(c, 4, 6, [30, 24, 1, 24], [6, 9, 1, 0], R=64, seed=7)              # more than the cache holds, or than there are rows


@pytest.mark.parametrize("dtype", ["f16", "fp4"])
def test_positions_of_their_own(dtype):
    c = Cache(2, 2, 24, 64, dtype)
    run(c, 2, 3, [10, 24], None, R=64, n_positions=50000, positions=[[40000, 0, 49999], [5, 5, 77]])
    run(c, 2, 3, [10, 24], [3, 1], R=64, n_positions=60, positions=[[60, 59, -1], [2 ** 31 - 1, -(2 ** 31), 3]], seed=6)
    run(c, 2, 3, [10, 24], None, R=64, n_positions=20, seed=7)             # the cache is longer than the table


@pytest.mark.parametrize("dtype", DTYPES)
def test_factors(dtype):
    run(Cache(2, 2, 24, 64, dtype), 2, 3, [10, 24], None, R=32, factors=(0.37, 5.5))


def test_8_bit_values_saturate():
    def edit(k, v):
        k[..., :5] = torch.tensor([448.0, 465, -1e30, 1e30, 3.0]).to(k.dtype)
        v[..., 0], v[..., 1], v[..., 2] = float("inf"), float("-inf"), float("nan")
    run(Cache(1, 2, 8, 64, "fp8"), 2, 2, [8], None, edit=edit)


def test_4_bit_blocks_of_zeros_tiny_and_huge_values():
    def edit(k, v):
        k[..., :16] = 0
        k[..., 16:32] *= 2.0 ** -12                          # below the smallest scale
        k[..., 32:48] *= 2.0 ** 14                           # beyond the largest: 448 * 6
        v[..., :16] *= 2.0 ** -9
        v[:, :, :, 20] = 100.0
    run(Cache(1, 2, 8, 64, "fp4"), 2, 2, [8], None, edit=edit)


def test_4_bit_infinities_and_nan():
    """A NaN makes its 16 values NaN; an infinity leaves the largest scale, and the others next to it what that holds of them."""
    c = Cache(1, 1, 4, 64, "fp4")
    x = torch.ones(1, 1, 1, 64, dtype=torch.bfloat16, device=DEV)
    x[..., 3], x[..., 20], x[..., 40] = float("nan"), float("inf"), float("-inf")
    ctx = torch.tensor([4], dtype=torch.int32, device=DEV)
    ssa.cache_append(c.desc(x, x), ssa.make_append(x, x), x, x, ctx, c.parts["k"], c.parts["v"], None, None, c.scales("k"), c.scales("v"))
    for name in "kv":
        got = c.values(name)[0, 0, 3]
        assert np.isnan(got[:16]).all() and np.array_equal(got[48:], CO.fp4_values(*CO.to_fp4(np.ones(16, np.float32))))
        assert got[20] == 2688 and got[40] == -2688 and not np.delete(got[16:48], [4, 24]).any()


def test_long_prompts_and_many_requests():
    run(Cache(1, 1, 4100, 64, "fp4"), 2, 4099, [4100], None, R=64)
    run(Cache(70, 2, 9, 64, "bf16", page=4), 4, 2, [int(x) for x in torch.randint(2, 10, (70,))], None, R=64)


def test_offsets_past_32_bits():
    """Two rows far apart: strides beyond 2^31 values."""
    T, far = 4, (1 << 31) + 64
    store = [torch.zeros(2 * far, dtype=torch.uint8, device=DEV) for _ in range(2)]
    k, v = (s.as_strided((2, 1, T, 64), (far, 64, 64, 1)).view(torch.float8_e4m3fn) for s in store)
    x = torch.randn(2, 1, T, 64, device=DEV).to(torch.bfloat16)
    ctx = torch.full((2,), T, dtype=torch.int32, device=DEV)
    ssa.cache_append(ssa.make_desc(x[:, :, 0], k, v, x[:, :, 0], T), ssa.make_append(x, x), x, x, ctx, k, v)
    want = x.float().clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    assert torch.equal(k.view(torch.uint8), want) and torch.equal(v.view(torch.uint8), want)
    assert int(store[0].count_nonzero()) == int(want.count_nonzero())
