"""fp64 statements of the operators that keep a cache within a budget: attention of a request's newest tokens over their own
past (sliding window and sinks), the weight that each position was given, the positions a budget keeps, and their move.

Plain loops over requests and heads on numpy arrays of values (not storage bits); no code is shared with the GPU path.
"""
import numpy as np


def visible(ctx, n_new, window, sinks):
    """[n_new, ctx] truth values: what token t, at position ctx - n_new + t, sees."""
    pos = (ctx - n_new + np.arange(n_new))[:, None]
    j = np.arange(ctx)[None, :]
    seen = j <= pos
    if window:
        seen &= (pos - j < window) | (j < sinks)
    return seen


def attention(q, k, v, ctx_lens, q_lens, window, sinks, scale, skipped=None):
    """q[B,H,n_q,D], k/v[B,H_kv,T,D] -> per request out[H,t,D], lse[H,t], weights[H,t,ctx], and what error bounds are made of:
    the sums of weight * |v| and the largest scale * sum |q||k|.  skipped[b]: positions that do not count."""
    out = []
    H, H_kv = q.shape[1], k.shape[1]
    for b in range(q.shape[0]):
        n, t = int(ctx_lens[b]), int(q_lens[b])
        seen = visible(n, t, window, sinks)
        if skipped is not None:
            seen = seen & ~skipped[b][None, :n]
        o, l, w, a, s_abs = [], [], [], [], 0.0
        live = seen.any(0)                                 # rows that no token sees may hold anything
        for h in range(H):
            K, V = k[b, h * H_kv // H, :n].astype(np.float64), v[b, h * H_kv // H, :n].astype(np.float64)
            Q = q[b, h, :t].astype(np.float64)
            K, V = np.where(live[:, None], K, 0), np.where(live[:, None], V, 0)
            with np.errstate(all="ignore"):
                s = np.where(seen, scale * (Q @ K.T), -np.inf)
                top = s.max(1, initial=-np.inf)
                top = np.where(np.isneginf(top), 0.0, top)[:, None]
                p = np.where(seen, np.exp(s - top), 0.0)
                total = p.sum(1, keepdims=True)
                p = np.where(total == 0, 0.0, p / np.where(total == 0, 1, total))
                l.append(np.where(total[:, 0] == 0, -np.inf, top[:, 0] + np.log(total[:, 0])))
                finite = np.isfinite(V)
                row = p @ np.where(finite, V, 0)
                for j, d in np.argwhere(~finite):          # only the tokens that see the row
                    row[seen[:, j], d] += V[j, d]
            o.append(row)
            w.append(p)
            a.append(p @ np.abs(np.where(finite, V, 0)))
            if t and n and np.isfinite(Q).all() and np.isfinite(K).all():
                s_abs = max(s_abs, float((scale * (np.abs(Q) @ np.abs(K).T)).max()))
        out.append(dict(out=np.array(o), lse=np.array(l), weights=np.array(w), spread=np.array(a), score=s_abs))
    return out


def kept(mass, n, budget, sinks, recent):
    """The sorted positions of one request that stay."""
    if n <= budget:
        return np.arange(n)
    between = sorted(range(sinks, n - recent), key=lambda j: (np.isnan(mass[j]), 0.0 if np.isnan(mass[j]) else -mass[j], j))
    return np.array(sorted([*range(sinks), *between[: budget - sinks - recent], *range(n - recent, n)]), dtype=np.int64)
