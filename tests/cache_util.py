"""Inputs and calls of the tests of the operators that fill a cache and read the blocks of it that queries select."""
import numpy as np
import torch

from budget_util import DEV, DT, UNWRITTEN, Tokens, half_step
from oracle import budget_oracle as BO
from oracle import cache_oracle as CO
from paper_2404_09336_b200 import ssa

DTYPES = ("bf16", "f16", "fp8", "fp4")


def query_type(dtype):
    return torch.float16 if dtype == "f16" else torch.bfloat16


def random_fp4(shape, g, spread=1.0):
    """Codes of every kind and scales over a range of sizes."""
    codes = torch.randint(0, 256, (*shape[:-1], shape[-1] // 2), generator=g).to(torch.uint8)
    scales = (torch.rand(*shape[:-1], shape[-1] // 16, generator=g) * spread).to(torch.float8_e4m3fn).view(torch.uint8)
    return codes, scales


class Cache:
    """K and V of one type and layout on the device, [B,H_kv,T,D] logically; codes and scales where values have 4 bits.  layout: bhtd,
    bthd, or "spaced": rows, heads and requests apart."""

    def __init__(self, B, H_kv, T, D, dtype="bf16", layout="bhtd", page=0, seed=0, per=None):
        self.B, self.H_kv, self.T, self.D, self.dtype, self.layout, self.page = B, H_kv, T, D, dtype, layout, page
        self.g = torch.Generator().manual_seed(seed)
        if page:
            per = per or (T + page - 1) // page
            self.n_pages = B * per + 2
            self.table = torch.randperm(self.n_pages, generator=self.g)[: B * per].view(B, per).to(torch.int32)
        self.parts = {}                                      # name -> device tensor
        for name in "kv":
            if dtype == "fp4":
                codes, scales = random_fp4((B, H_kv, T, D), self.g)
                self.put(name, codes)
                self.put(name + "_scales", scales)
            else:
                self.put(name, torch.randn(B, H_kv, T, D, generator=self.g).to(DT[dtype]))

    def put(self, name, x):
        """x[B,H_kv,T,n] (host) in the layout on the device."""
        raw = x.view(torch.uint8) if x.element_size() == 1 else x.view(torch.int16)
        B, H, T, n = raw.shape
        if self.page:
            pool = torch.zeros(self.n_pages * self.page, H, n, dtype=raw.dtype)
            j = torch.arange(T)
            pool[self.table.long()[:, j // self.page] * self.page + j % self.page] = raw.permute(0, 2, 1, 3)
            y = pool.view(self.n_pages, self.page, H, n).to(DEV)
        elif self.layout == "bthd":
            y = raw.permute(0, 2, 1, 3).contiguous().to(DEV).permute(0, 2, 1, 3)
        elif self.layout == "spaced":                        # (rows two apart, heads three rows, requests five)
            store = torch.zeros(B, H * 2 * T * n + 3 * H * n + 5 * n, dtype=raw.dtype, device=DEV)
            y = store.as_strided((B, H, T, n), (store.stride(0), (2 * T + 3) * n, 2 * n, 1))
            y.copy_(raw)
        else:
            y = raw.to(DEV)
        self.parts[name] = y.view(x.dtype)

    def get(self, name):
        """The logical [B,H_kv,T,n] on the host."""
        x = self.parts[name]
        x = x.view(torch.uint8) if x.element_size() == 1 else x.view(torch.int16)
        if self.page:
            j = torch.arange(self.T)
            rows = (self.table.long().clamp(0, self.n_pages - 1)[:, j // self.page] * self.page + j % self.page).to(DEV)
            x = x.reshape(-1, *x.shape[2:])[rows].permute(0, 2, 1, 3)
        return x.cpu().contiguous().view(self.parts[name].dtype)

    def values(self, name):
        x = self.get(name)
        if self.dtype == "fp4":
            return CO.fp4_values(x.numpy(), self.get(name + "_scales").numpy())
        return x.double().numpy()

    def scales(self, name):
        return self.parts.get(name + "_scales")

    def paging(self, table=None):
        if not self.page:
            return None
        self.d_table = (self.table if table is None else table).to(DEV)
        return ssa.make_paging(self.d_table, self.page, self.n_pages)

    def desc(self, q, out, scale=0.0):
        """q, out [B,H,n_q,D]."""
        k, v, args = self.parts["k"], self.parts["v"], (out[:, :, 0], self.T)
        if self.dtype == "fp4":
            return ssa.make_desc_fp4(q[:, :, 0], k, v, self.scales("k"), self.scales("v"), *args, scale=scale, paged=bool(self.page))
        return (ssa.make_desc_paged if self.page else ssa.make_desc)(q[:, :, 0], k, v, *args, scale=scale)


def far_apart(c):
    """The cache's requests (two) more than 2^32 values apart."""
    for name, x in c.parts.items():
        B, H, T, n = x.shape
        far = ((1 << 32) + 128) // (c.D // n)
        y = torch.zeros(far + H * T * n, dtype=x.dtype, device=DEV).as_strided((B, H, T, n), (far, T * n, n, 1))
        y.copy_(x)
        c.parts[name] = y
    return c


class Fp4Tokens(Tokens):
    """budget_util.Tokens over a 4-bit cache (weights are fp16 pairs, as over an 8-bit one)."""

    def __init__(self, B, H, H_kv, T, D, n_q, layout="bhtd", page=0, seed=0, spread=1.0):
        super().__init__(B, H, H_kv, T, D, n_q, "fp8", "bhtd", 0, seed, spread)
        self.cache = Cache(B, H_kv, T, D, "fp4", layout, page, seed + 1)

    def values(self):
        return [self.q.cpu().double().numpy(), self.cache.values("k"), self.cache.values("v")]

    def call(self, ctx, q_lens=None, window=0, sinks=0, out_dtype=torch.float32, scale=0.0, stream=None, table=None, less=0):
        """less: bytes that the workspace lacks of what the library asks for."""
        c = self.cache
        d_ctx = torch.tensor(ctx, dtype=torch.int32, device=DEV)
        d_new = None if q_lens is None else torch.tensor(q_lens, dtype=torch.int32, device=DEV)
        out = torch.full((self.B, self.n_q, self.H, self.D), UNWRITTEN, dtype=out_dtype, device=DEV).permute(0, 2, 1, 3)
        lse = torch.full((self.B, self.H, self.n_q), UNWRITTEN, device=DEV)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        desc = c.desc(self.q, out, scale)
        win = ssa.make_window(self.q, out, window, sinks, d_new, c.paging(table))
        ws = torch.full((ssa.attn_window_fp4_workspace_bytes(desc, win) - less,), 0xff, dtype=torch.uint8, device=DEV)
        ssa.attn_window_fp4(desc, win, self.q, c.parts["k"], c.parts["v"], c.scales("k"), c.scales("v"), d_ctx, out, lse, ws, status, stream)
        torch.cuda.synchronize()
        f64 = lambda x: x.double().cpu().numpy()
        return f64(out), f64(lse), None, int(status.item())


# The smallest steps of fp16 are 2^-24, whatever a weight's size: a weight of two parts is off by half of one, 2^-25, besides its
# relative error.  The kernel for few rows scales weights so that the largest is 2^13 or more, the tiles 2^6: relative to the largest,
# and so to their sum, 2^-38 and 2^-31.  (bf16 has the range of fp32.)  Sums over rows of V get that for each row.
FLOOR_ROWS, FLOOR_TILES = 2.0 ** -38, 2.0 ** -31


def check_rows(got, lse, want, D, n, dt, out_dtype, v_most):
    """One token's rows of a K/V head against CO.attention's: the bounds of budget_util.check, and the floor of fp16 weights."""
    out, l, spread, score = want
    step = half_step(torch.float16 if dt in ("fp8", "fp4") else DT[dt])
    step = step if dt == "fp4" and out_dtype != torch.float32 else step * step
    score = (D * score + 2 * score + 4) * 2.0 ** -24
    tol = 2 * (score + 2.0 ** -22 + step + (n + 64) * 2.0 ** -24) * spread + 1e-30
    if dt != "bf16":
        tol = tol + 2 * FLOOR_ROWS * n * v_most
    if out_dtype != torch.float32:
        tol = tol + half_step(out_dtype) * (np.abs(out) + tol) + (2.0 ** -25 if out_dtype == torch.float16 else 0)
    assert (np.abs(got - out) <= tol).all(), float((np.abs(got - out) / tol).max())
    if n == 0:
        assert np.isneginf(lse).all()
        return
    assert (np.abs(lse - l) <= 2 * (score + 2.0 ** -22 + (n + 64) * 2.0 ** -24) + np.abs(l) * 2.0 ** -22).all()


def check_tokens(p, got, ctx, q_lens, window, sinks, out_dtype, tiles=False, shared=False, skipped=None, scale=None):
    """budget_util.check over a 4-bit cache, with the floor of fp16 weights: of one part for bf16 outputs, of two for fp32 ones.
    tiles: the call may go to the tiles; shared: to those of a bf16 cache, whose weights are bf16 of as many parts (and have no floor)."""
    out, lse, _, status = got
    assert not status & ssa.DEV_GAVE_UP
    q, k, v = p.values()
    q_lens = [p.n_q] * p.B if q_lens is None else q_lens
    ref = BO.attention(q, k, v, ctx, q_lens, window, sinks, p.D ** -0.5 if scale is None else scale, skipped)
    one = torch.bfloat16 if shared else torch.float16
    step = half_step(one) if out_dtype != torch.float32 else half_step(one) ** 2
    for b, r in enumerate(ref):
        n, t = ctx[b], q_lens[b]
        assert (out[b, :, t:] == UNWRITTEN).all() and (lse[b, :, t:] == UNWRITTEN).all(), "rows behind the last token were written"
        score = (p.D * r["score"] + 2 * r["score"] + 4) * 2.0 ** -24
        tol = 2 * (score + 2.0 ** -22 + step + (n + 64) * 2.0 ** -24) * r["spread"] + 1e-30
        tol = tol + 2 * (FLOOR_TILES if tiles else FLOOR_ROWS) * n * np.abs(v[b]).max(initial=0)
        if out_dtype != torch.float32:
            tol = tol + half_step(out_dtype) * (np.abs(r["out"]) + tol)
        err = np.abs(out[b, :, :t] - r["out"])
        assert (err <= tol).all(), f"request {b}: {(err / tol).max()} of the bound"
        x, y = lse[b, :, :t], r["lse"]
        fine = np.isfinite(y)
        assert np.array_equal(np.where(fine, 0, y), np.where(np.isfinite(x), 0, x)), f"request {b}: lse"
        bound = 2 * (score + 2.0 ** -22 + (n + 64) * 2.0 ** -24) + np.abs(y) * 2.0 ** -22
        assert (np.abs(x[fine] - y[fine]) <= bound[fine]).all(), f"request {b}: lse off by {np.abs(x[fine] - y[fine]).max()}"
