"""Keeping a key-value cache within a budget: the operators' cases, plain forms and exact values.

  window   ssa_attn_window    attention of a step's tokens, each over its own past: a sliding window and the first tokens
  mass     ssa_attn_mass      the same, with the softmax weight that every cached position was given added up
  evict    ssa_mass_to_index  the positions that a budget keeps, by that sum: first ones, newest ones, heaviest ones
  compact  ssa_cache_compact  the kept rows of K and V, and their sums, moved to the front of the cache, in place

Sizes are those of the repository's workloads (batch 1 to 64, 8 or 32 heads of 64 or 128, contexts of 512 to 16384 tokens)
and of its variants: grouped query heads, several query tokens, 8-bit and paged caches.  Queries, keys and values are N(0, 1).
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "fp8": torch.float8_e4m3fn}
BYTES = {"bf16": 2, "f16": 2, "fp8": 1}
MAX_PAIRS = 2.2e9             # (head, token, position) triples of the largest listed attention, masked ones included ...
MAX_CACHE_BYTES = 2.2e9       # ... and K and V of the largest listed cache


def _case(name, op, B, T, *, H=32, H_kv=0, D=128, dtype="bf16", n_q=1, ctx_lo=0, window=0, sinks=0, page=0, budget=0,
          recent=0, decay=1.0):
    """Lengths are uniform in [ctx_lo, T] (0: all T); where n_q > 1 and lengths are ragged, requests bring 1..n_q tokens.
    window 0: no window.  page 0: one [T, D] plane per request and head, else rows per page of a [pages, rows, heads, D] pool."""
    c = {"op": op, "B": B, "T": T, "H": H, "H_kv": H_kv or H, "D": D, "dtype": dtype, "n_q": n_q, "ctx_lo": ctx_lo or T,
         "window": window, "sinks": sinks, "page": page, "budget": budget, "recent": recent, "decay": decay}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one token of one short request, few small heads: all latency
        _case("window_tiny", "window", 1, 512, H=8, D=64, dtype="f16", window=128, sinks=4),
        # one token each of a large batch of short ragged contexts, the instruction kept as sinks
        _case("window_decode", "window", 64, 1024, ctx_lo=256, window=256, sinks=64),
        # drafted tokens of a batch being checked over the full context, each seeing what came before it
        _case("window_drafts", "window", 16, 4096, H_kv=8, dtype="f16", n_q=5, ctx_lo=1001),
        # whole prompts of a summarization batch
        _case("window_prompt", "window", 4, 4096, n_q=4096, window=1024, sinks=64),
        # ragged chunks of long prompts over a paged cache, grouped query heads
        _case("window_chunks_paged", "window", 8, 16384, H_kv=8, n_q=509, ctx_lo=4100, window=4096, sinks=16, page=64),
        # the least work of a step that keeps the sums
        _case("mass_tiny", "mass", 1, 512, H=8, D=64, dtype="f16"),
        # long contexts with grouped query heads
        _case("mass_long", "mass", 8, 16384, H_kv=8, ctx_lo=9000),
        # an 8-bit cache, older weight fading
        _case("mass_fp8", "mass", 16, 4096, dtype="fp8", ctx_lo=1500, decay=0.98),
        # one short request over its budget
        _case("evict_tiny", "evict", 1, 512, sinks=4, budget=128, recent=32),
        # a batch of long contexts
        _case("evict_long", "evict", 32, 16384, ctx_lo=6001, sinks=64, budget=4096, recent=512),
        # a small paged cache of small heads
        _case("compact_paged", "compact", 4, 1024, H=8, D=64, dtype="f16", ctx_lo=700, sinks=4, budget=256, recent=64, page=16),
        # the long contexts of a batch cut to a quarter; the largest cache
        _case("compact_long", "compact", 8, 16384, ctx_lo=9000, sinks=64, budget=4096, recent=512),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["window", "window", "mass", "evict", "compact"])
    H, D = rng.choice([(8, 64), (32, 128), (32, 128)])
    H_kv = rng.choice([H, H // 4])
    dtype = rng.choice(["bf16", "bf16", "f16", "fp8"])
    B, T = _log_int(rng, 1, 64), _log_int(rng, 200, 16384)
    n_q = 1
    if op == "window":
        n_q = rng.choice([1, rng.randint(2, 16), _log_int(rng, 17, 4096)])
        if n_q > 16 and dtype == "fp8":
            dtype = "bf16"
        n_q = min(n_q, T)
    elif op == "mass":
        n_q = rng.choice([1, 1, rng.randint(2, 8)])
    if op != "evict":                                   # cut the batch, then the context, until it costs no more than the listed
        B = max(1, min(B, int(MAX_CACHE_BYTES / (2 * H_kv * T * D * BYTES[dtype])), int(MAX_PAIRS / (H * n_q * T))))
        T = max(n_q, min(T, int(MAX_PAIRS / (B * H * n_q))))
    sinks = rng.choice([0, 4, rng.randint(1, 64)])
    budget = max(8, _log_int(rng, max(8, T // 16), T)) if op in ("evict", "compact") else 0
    recent = rng.randint(0, budget // 4) if budget else 0
    window = rng.choice([0, _log_int(rng, 1, T)]) if op in ("window", "mass") else 0
    page = rng.choice([0, 0, 16, 64, 128]) if op != "evict" else 0
    return _case("", op, B, T, H=H, H_kv=H_kv, D=D, dtype=dtype, n_q=n_q, ctx_lo=max(n_q, rng.randint(1, T)), window=window,
                 sinks=min(sinks, budget // 4) if budget else sinks, page=page, budget=budget, recent=recent,
                 decay=rng.choice([1.0, 0.95]) if op == "mass" else 1.0)


def _lengths(c):
    """Context lengths and new tokens of every request: part of the case, the same for every seed."""
    rng = np.random.RandomState((c["B"] * 7919 + c["T"] * 31 + c["n_q"]) % (1 << 31))
    ctx = rng.randint(c["ctx_lo"], c["T"] + 1, c["B"])
    fixed = c["ctx_lo"] == c["T"] or c["n_q"] == 1
    return ctx, np.full(c["B"], c["n_q"]) if fixed else np.minimum(rng.randint(1, c["n_q"] + 1, c["B"]), ctx)


def work(c):
    ctx, new = _lengths(c)
    E, D, pairs, rows = BYTES[c["dtype"]], c["D"], 0, 0
    if c["op"] in ("window", "mass"):
        for n, t in zip(ctx.tolist(), new.tolist()):
            pos = np.arange(n - t, n)
            w = np.minimum(c["window"] or n, pos + 1)                         # positions inside the window ...
            first = np.minimum(c["sinks"], np.maximum(pos - w + 1, 0))        # ... and sinks in front of it
            pairs += int((w + first).sum())
            rows += min(n, n - int(max(0, pos[0] - w[0] + 1)) + int(first.max()))
        q_bytes = c["H"] * D * int(new.sum()) * 2
        moved = 2 * q_bytes + 4 * c["H"] * int(new.sum()) + 2 * rows * c["H_kv"] * D * E
        if c["op"] == "mass":
            moved += 4 * (2 * int(ctx.sum()) - int(new.sum()))
        return {"bytes": moved, "flops": 4 * D * c["H"] * pairs}
    kept = int(np.minimum(ctx, c["budget"]).sum())
    if c["op"] == "evict":
        return {"bytes": 4 * int(ctx.sum()) + 4 * kept, "flops": int(ctx.sum())}
    moving = int(np.where(ctx > c["budget"], c["budget"] - c["sinks"], 0).sum())
    return {"bytes": 2 * moving * (2 * c["H_kv"] * D * E + 4) + 4 * kept, "flops": 0}


def _kept(c, ctx, g):
    """Index lists for a compaction: the first ones, the newest ones, and a random choice between them, in order."""
    B, budget = len(ctx), c["budget"]
    j = torch.arange(c["T"], device="cuda")
    n = torch.as_tensor(ctx, device="cuda")[:, None]
    rank = torch.rand(B, c["T"], device="cuda", generator=g)
    rank = torch.where((j < c["sinks"]) | (j >= n - c["recent"]), 2.0, rank)
    rank = torch.where(j < n, rank, -1.0)
    kept = torch.where(n > budget, rank.argsort(dim=1, descending=True, stable=True)[:, :budget], c["T"])
    kept = torch.where(n <= budget, torch.where(j < n, j, c["T"])[:, :budget], kept).sort(1).values
    counts = torch.minimum(n[:, 0], torch.tensor(budget, device="cuda"))
    return torch.where(j[:budget] < counts[:, None], kept, -1).to(torch.int32).contiguous(), counts.to(torch.int32)


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    ctx, new = _lengths(c)
    B, T, H, H_kv, D = c["B"], c["T"], c["H"], c["H_kv"], c["D"]
    dt = DTYPES[c["dtype"]]
    dt_q = torch.bfloat16 if c["dtype"] == "fp8" else dt
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=g)  # noqa: E731
    s = {"case": c, "ctx": torch.as_tensor(ctx, device="cuda", dtype=torch.int32),
         "status": torch.zeros(1, dtype=torch.int32, device="cuda")}
    if c["op"] != "evict":
        if c["page"]:
            per = (T + c["page"] - 1) // c["page"]
            order = torch.randperm(B * per + 3, device="cuda", generator=g)[: B * per].view(B, per)
            used = torch.arange(per, device="cuda") * c["page"] < s["ctx"][:, None]
            s["table"] = torch.where(used, order, -1).to(torch.int32).contiguous()
            s["k"], s["v"] = (normal(B * per + 3, c["page"], H_kv, D).to(dt) for _ in range(2))
        else:
            s["k"], s["v"] = (normal(B, H_kv, T, D).to(dt) for _ in range(2))
    if c["op"] in ("window", "mass"):
        s["q"] = normal(B, c["n_q"], H, D).to(dt_q).permute(0, 2, 1, 3)       # token-major, as a projection leaves it
        s["q_lens"] = torch.as_tensor(new, device="cuda", dtype=torch.int32)
        s["out"] = torch.zeros(B, c["n_q"], H, D, device="cuda", dtype=dt_q).permute(0, 2, 1, 3)
        s["lse"] = torch.zeros(B, H, c["n_q"], device="cuda")
    if c["op"] == "mass":
        s["mass"] = torch.rand(B, T, device="cuda", generator=g) * 4
        s["mass_out"] = torch.zeros(B, T, device="cuda")
    if c["op"] == "evict":                                     # a few heavy positions, many light ones, some never looked at
        s["mass"] = torch.exp(2 * normal(B, T)) * (torch.rand(B, T, device="cuda", generator=g) > 0.1)
        s["mass"] = torch.where(s["mass"] < 0.1, torch.round(s["mass"] * 64) / 64, s["mass"]).contiguous()
        s["index"] = torch.full((B, c["budget"]), -1, dtype=torch.int32, device="cuda")
        s["counts"] = torch.zeros(B, dtype=torch.int32, device="cuda")
    if c["op"] == "compact":
        s["mass"] = torch.rand(B, T, device="cuda", generator=g)
        s["index"], s["counts"] = _kept(c, ctx, g)
    if own:
        _plan(s)
    return s


def _plan(s):
    """What a program keeps for its calls: descriptors and a workspace."""
    from paper_2404_09336_b200 import ssa
    c = s["case"]
    if c["op"] == "evict":
        return
    s["paging"] = ssa.make_paging(s["table"], c["page"], s["k"].shape[0]) if c["page"] else None
    if c["op"] == "compact":
        q = torch.empty(c["B"], c["H"], c["D"], device="cuda", dtype=torch.bfloat16 if c["dtype"] == "fp8" else s["k"].dtype)
    else:
        q = s["q"][:, :, 0]
    make = ssa.make_desc_paged if c["page"] else ssa.make_desc
    s["desc"] = make(q, s["k"], s["v"], q, c["T"])
    if c["op"] == "compact":
        return
    s["win"] = ssa.make_window(s["q"], s["out"], c["window"], c["sinks"], s["q_lens"], s["paging"])
    need = ssa.attn_mass_workspace_bytes if c["op"] == "mass" else ssa.attn_window_workspace_bytes
    s["workspace"] = torch.empty(need(s["desc"], s["win"]), dtype=torch.uint8, device="cuda")


def run(s):
    if own:
        return _own(s)
    return {"window": _plain_attention, "mass": _plain_attention, "evict": _plain_evict, "compact": _plain_compact}[s["case"]["op"]](s)


def _own(s):
    from paper_2404_09336_b200 import ssa
    c = s["case"]
    if c["op"] == "window":
        ssa.attn_window(s["desc"], s["win"], s["q"], s["k"], s["v"], s["ctx"], s["out"], s["lse"], s["workspace"], s["status"])
        return {"out": s["out"], "lse": s["lse"]}
    if c["op"] == "mass":
        ssa.attn_mass(s["desc"], s["win"], s["q"], s["k"], s["v"], s["ctx"], s["out"], s["lse"], s["mass"], s["mass_out"],
                      c["decay"], s["workspace"], s["status"])
        return {"out": s["out"], "lse": s["lse"], "mass": s["mass_out"]}
    if c["op"] == "evict":
        ssa.mass_to_index(s["mass"], s["ctx"], c["budget"], c["sinks"], c["recent"], s["index"], s["counts"], s["status"])
        return {"index": s["index"], "counts": s["counts"]}
    ssa.cache_compact(s["desc"], s["k"], s["v"], s["ctx"], s["index"], s["counts"], c["budget"], mass=s["mass"],
                      paging=s["paging"], dev_status=s["status"])
    return {"k": s["k"], "v": s["v"], "mass": s["mass"]}


def _rows(s):
    """Pool rows of the logical positions of every request, [B, T]."""
    page, j = s["case"]["page"], torch.arange(s["case"]["T"], device="cuda")
    return s["table"].long().clamp(min=0)[:, j // page] * page + j % page


def _logical(s, name):
    """A cache as [B, H_kv, T, D]."""
    x, c = s[name], s["case"]
    if not c["page"]:
        return x
    return x.reshape(-1, c["H_kv"], c["D"])[_rows(s)].permute(0, 2, 1, 3)


def _plain_attention(s):
    c = s["case"]
    B, H, H_kv, D, n_q, T = c["B"], c["H"], c["H_kv"], c["D"], c["n_q"], c["T"]
    ctx, new = s["ctx"].long()[:, None], s["q_lens"].long()[:, None]
    j, t = torch.arange(T, device="cuda"), torch.arange(n_q, device="cuda")
    pos = (ctx - new + t)[:, :, None]                                              # [B, n_q, 1]
    seen = (j <= pos) & (t < new)[:, :, None]
    if c["window"]:
        seen &= (j > pos - c["window"]) | (j < c["sinks"])
    q = s["q"].float().reshape(B, H_kv, -1, D)
    k, v = _logical(s, "k").float(), _logical(s, "v").float()
    x = (q @ k.transpose(-1, -2) * (1 / math.sqrt(D))).view(B, H, n_q, T)
    x = x.masked_fill_(~seen[:, None], -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    x = x.div_(total.masked_fill(total == 0, 1))
    rows = (t < new)[:, None, :, None]                                             # rows behind the last token stay as they were
    out = torch.where(rows, (x.view(B, H_kv, -1, T) @ v).view(B, H, n_q, D).to(s["out"].dtype), s["out"])
    lse = torch.where(rows[..., 0], (top + total.log())[..., 0], s["lse"])
    if c["op"] == "window":
        return {"out": out, "lse": lse}
    old = torch.where(j < ctx - new, s["mass"], 0) * c["decay"]
    return {"out": out, "lse": lse, "mass": torch.where(j < ctx, old + x.sum((1, 2)), s["mass_out"])}


def _plain_evict(s):
    c = s["case"]
    n, j, budget = s["ctx"].long()[:, None], torch.arange(c["T"], device="cuda"), c["budget"]
    rank = torch.where((j < c["sinks"]) | (j >= n - c["recent"]), math.inf, s["mass"])
    rank = torch.where(j < n, rank, -math.inf)
    kept = rank.sort(dim=1, descending=True, stable=True).indices[:, :budget]          # stable: ties go to the lowest position
    counts = n.clamp(max=budget)
    kept = torch.where(j[:budget] < counts, kept, c["T"]).sort(1).values
    index = torch.where(j[:budget] < counts, kept.to(torch.int32), s["index"])
    return {"index": index, "counts": counts[:, 0].to(torch.int32)}


def _plain_compact(s):
    c = s["case"]
    i = torch.arange(c["budget"], device="cuda")
    to = i < s["counts"][:, None]
    source = torch.where(to, s["index"].long(), i)                                 # rows behind the kept ones stay as they are
    s["mass"][:, : c["budget"]] = s["mass"].gather(1, source)
    if c["page"]:
        rows, (b, i) = _rows(s), to.nonzero(as_tuple=True)
        for name in ("k", "v"):
            pool = s[name].view(-1, c["H_kv"], c["D"])
            pool[rows[b, i]] = pool[rows[b, source[b, i]]]
    else:
        for name in ("k", "v"):
            s[name][:, :, : c["budget"]] = s[name].gather(2, source[:, None, :, None].expand(-1, c["H_kv"], -1, c["D"]))
    return {"k": s["k"], "v": s["v"], "mass": s["mass"]}


def exact(case, seed):
    """Request by request and head by head in 64 bits, the visible positions listed instead of masked."""
    c = case
    if c["op"] not in ("window", "mass"):
        return None                                            # selections and moves: nothing is rounded
    s = prepare(c, seed)
    ctx, new = s["ctx"].tolist(), s["q_lens"].tolist()
    out, lse = s["out"].double(), s["lse"].double()
    mass = s["mass_out"].double() if c["op"] == "mass" else None
    group = c["H"] // c["H_kv"]
    for b in range(c["B"]):
        n, t = ctx[b], new[b]
        if c["page"]:
            rows = torch.tensor([p * c["page"] + r for p in s["table"][b].tolist() if p >= 0 for r in range(c["page"])][:n], device="cuda")
        weight = torch.zeros(n, dtype=torch.float64, device="cuda")
        j = torch.arange(n, device="cuda")
        lo = torch.arange(n - t, n, device="cuda")[:, None]    # the token's own position
        hidden = j[None] > lo
        if c["window"]:
            hidden |= (lo - j[None] >= c["window"]) & (j[None] >= c["sinks"])
        for h in range(c["H"]):
            if h % group == 0:
                K, V = (x[:, :, h // group].reshape(-1, c["D"])[rows] if c["page"] else x[b, h // group, :n] for x in (s["k"], s["v"]))
                K, V = K.double(), V.double()
            x = torch.mm(s["q"][b, h, :t].double(), K.t()) / math.sqrt(c["D"])
            x[hidden] = -math.inf
            total = torch.logsumexp(x, 1)
            p = torch.exp(x - total[:, None])
            out[b, h, :t], lse[b, h, :t] = torch.mm(p, V), total
            weight += p.sum(0)
        if mass is not None:
            mass[b, :n] = weight
            mass[b, : n - t] += c["decay"] * s["mass"][b, : n - t].double()
    return {"out": out, "lse": lse} if mass is None else {"out": out, "lse": lse, "mass": mass}
