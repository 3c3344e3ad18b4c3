"""Inputs, calls and error bounds of the tests of the budget operators."""
import numpy as np
import torch

from oracle import budget_oracle as BO
from paper_2404_09336_b200 import ssa

DEV = "cuda:0"
DT = {"bf16": torch.bfloat16, "f16": torch.float16, "fp8": torch.float8_e4m3fn}
UNWRITTEN = 768.0                                            # a value of every type


def half_step(dtype):
    """Largest relative error of one rounding."""
    return torch.finfo(dtype).eps / 2


def _raw(x):
    return x.view(torch.uint8) if x.element_size() == 1 else x.view(torch.int16)


class Tokens:
    """q[B,H,n_q,D] over a cache [B,H_kv,T,D] (bhtd, bthd, or in pages), on the device; values on the host in fp64."""

    def __init__(self, B, H, H_kv, T, D, n_q, dtype="bf16", layout="bhtd", page=0, seed=0, spread=1.0):
        g = torch.Generator().manual_seed(seed)
        self.B, self.H, self.H_kv, self.T, self.D, self.n_q, self.page = B, H, H_kv, T, D, n_q, page
        self.dt, self.dt_q = DT[dtype], torch.bfloat16 if dtype == "fp8" else DT[dtype]
        self.q = (torch.randn(B, n_q, H, D, generator=g) * spread).to(self.dt_q).to(DEV).permute(0, 2, 1, 3)
        k, v = (torch.randn(B, H_kv, T, D, generator=g).to(self.dt) for _ in range(2))
        self.layout = layout
        if page:
            per = (T + page - 1) // page
            self.table = torch.randperm(B * per + 2, generator=g)[: B * per].view(B, per).to(torch.int32)
            self.n_pages = B * per + 2
        self.put(k, v)

    def put(self, k, v):
        """The logical caches (CPU tensors [B,H_kv,T,D]) in the layout."""
        self.host = [k, v]
        if self.page:
            self.d_table = self.table.to(DEV)
            self.stores = []
            for x in (k, v):
                pool = torch.zeros(self.n_pages * self.page, self.H_kv, self.D, dtype=self.dt)
                j = torch.arange(self.T)
                rows = self.table.long()[:, j // self.page] * self.page + j % self.page
                _raw(pool)[rows] = _raw(x).permute(0, 2, 1, 3)
                self.stores.append(pool.view(self.n_pages, self.page, self.H_kv, self.D).to(DEV))
        elif self.layout == "bthd":
            self.stores = [_raw(x).permute(0, 2, 1, 3).contiguous().view(self.dt).to(DEV).permute(0, 2, 1, 3) for x in (k, v)]
        else:
            self.stores = [x.to(DEV) for x in (k, v)]

    def values(self):
        return [x.float().double().numpy() for x in (self.q.cpu(), *self.host)]

    def call(self, ctx, q_lens=None, window=0, sinks=0, out_dtype=torch.float32, mass_in=None, mass=False, decay=1.0, scale=0.0,
             stream=None, table=None):
        """-> out[B,H,n_q,D], lse, mass_out or None (fp64, UNWRITTEN where nothing was written), status."""
        k, v = self.stores
        d_ctx = torch.tensor(ctx, dtype=torch.int32, device=DEV)
        d_new = None if q_lens is None else torch.tensor(q_lens, dtype=torch.int32, device=DEV)
        out = torch.full((self.B, self.n_q, self.H, self.D), UNWRITTEN, dtype=out_dtype or self.dt_q, device=DEV).permute(0, 2, 1, 3)
        lse = torch.full((self.B, self.H, self.n_q), UNWRITTEN, device=DEV)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        if self.page:
            d_table = self.d_table if table is None else table.to(DEV)
            desc = ssa.make_desc_paged(self.q[:, :, 0], k, v, out[:, :, 0], self.T, scale=scale)
            paging = ssa.make_paging(d_table, self.page, self.n_pages)
        else:
            desc, paging = ssa.make_desc(self.q[:, :, 0], k, v, out[:, :, 0], scale=scale), None
        win = ssa.make_window(self.q, out, window, sinks, d_new, paging)
        if mass:
            ws = torch.full((ssa.attn_mass_workspace_bytes(desc, win),), 0xff, dtype=torch.uint8, device=DEV)
            m_out = torch.full((self.B, self.T), UNWRITTEN, device=DEV)
            ssa.attn_mass(desc, win, self.q, k, v, d_ctx, out, lse, mass_in, m_out, decay, ws, status, stream)
        else:
            ws = torch.full((ssa.attn_window_workspace_bytes(desc, win),), 0xff, dtype=torch.uint8, device=DEV)
            m_out = None
            ssa.attn_window(desc, win, self.q, k, v, d_ctx, out, lse, ws, status, stream)
        torch.cuda.synchronize()
        f64 = lambda x: None if x is None else x.double().cpu().numpy()
        return f64(out), f64(lse), f64(m_out), int(status.item())


def weight_step(dtype, many):
    """Largest relative error of a softmax weight as the second contraction takes it: its 16-bit value and the 16-bit rest of it
    where few rows share a K/V head, the 16-bit value alone in prompt chunks (`many`)."""
    step = half_step(torch.float16 if dtype == torch.float8_e4m3fn else dtype)
    return step if many else step * step


def check(p, got, ctx, q_lens, window, sinks, out_dtype, many=False, mass_in=None, decay=1.0, skipped=None, scale=None):
    """Errors against fp64.  A score is a dot product of D terms in fp32: off by D 2^-24 of scale sum |q||k| at most, and so is,
    relatively, its exponential (and 2^-22 by exp2); the weight is rounded (weight_step); sums of n terms add n 2^-24.  Numerator
    and denominator both have it, each relative to sum weight |v|; the output is rounded once more."""
    out, lse, mass, status = got
    assert not status & ssa.DEV_GAVE_UP
    q, k, v = p.values()
    q_lens = [p.n_q] * p.B if q_lens is None else q_lens
    ref = BO.attention(q, k, v, ctx, q_lens, window, sinks, p.D ** -0.5 if scale is None else scale, skipped)
    for b, r in enumerate(ref):
        n, t = ctx[b], q_lens[b]
        assert (out[b, :, t:] == UNWRITTEN).all() and (lse[b, :, t:] == UNWRITTEN).all(), "rows behind the last token were written"
        score = (p.D * r["score"] + 2 * r["score"] + 4) * 2.0 ** -24
        weight = score + 2.0 ** -22 + weight_step(p.dt, many) + (n + 64) * 2.0 ** -24
        with np.errstate(invalid="ignore"):
            tol = 2 * weight * r["spread"] + 1e-30
            if out_dtype != torch.float32:
                tol = tol + half_step(out_dtype) * (np.abs(r["out"]) + tol) + (2.0 ** -25 if out_dtype == torch.float16 else 0)
            x, y = out[b, :, :t], r["out"]
            fine = np.isfinite(y)
            assert np.array_equal(np.where(fine, 0, y), np.where(np.isfinite(x), 0, x), equal_nan=True), f"request {b}: infinities"
            err = np.where(fine, np.abs(x - y), 0)
            assert (err[fine] <= tol[fine]).all(), f"request {b}: {(err / tol)[fine].max()} of the bound"
            x, y = lse[b, :, :t], r["lse"]
            fine = np.isfinite(y)
            assert np.array_equal(np.where(fine, 0, y), np.where(np.isfinite(x), 0, x), equal_nan=True), f"request {b}: lse"
            bound = 2 * (score + 2.0 ** -22 + (n + 64) * 2.0 ** -24) + np.abs(y) * 2.0 ** -22
            assert (np.abs(x - y)[fine] <= bound[fine]).all(), f"request {b}: lse off by {np.abs(x - y)[fine].max()}"
        if mass is not None:
            assert (mass[b, n:] == UNWRITTEN).all(), "sums behind the context were written"
            want = r["weights"].sum((0, 1))
            old = np.zeros(n) if mass_in is None else np.where(np.arange(n) < n - t, mass_in[b, :n] * decay, 0)
            # both the score and the normaliser are off by `score` and more; the sum has H t terms
            largest = np.abs(np.where(np.isfinite(r["lse"]), r["lse"], 0)).max(initial=0)
            tol = want * (2 * score + 2.0 ** -21 + (n + 64) * 2.0 ** -24 + (largest + 1) * 2.0 ** -21)
            tol += (want + np.abs(old)) * (p.H * t + 2) * 2.0 ** -24 + 1e-35
            assert (np.abs(mass[b, :n] - want - old) <= tol).all(), f"request {b}: mass {(np.abs(mass[b, :n] - want - old) / tol).max()}"
    return ref
