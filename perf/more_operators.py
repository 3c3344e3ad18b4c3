"""Filling a key-value cache and reading the part of it that the queries ask for: the operators' cases, plain forms and exact values.

  append  ssa_cache_append     a step's keys, values and queries: rotated by position; keys and values stored in the cache
  bounds  ssa_block_bounds     the least and the largest value of every dimension over the keys of a block of positions
  select  ssa_block_select     from a token's queries and the bounds: the blocks that it attends to
  blocks  ssa_attn_blocks      attention of every token over its own list of blocks
  fp4     ssa_attn_window_fp4  attention over a cache of 4-bit values (e2m1, with an e4m3 scale for each 16 of them)

Sizes are those of the repository's workloads (batch 1 to 64, 8 or 32 heads of 64 or 128, contexts of 512 to 16384 tokens)
and of its variants: grouped query heads, several query tokens, 8-bit and paged caches.  Queries, keys and values are N(0, 1).
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "fp8": torch.float8_e4m3fn}
BITS = {"bf16": 16, "f16": 16, "fp8": 8, "fp4": 4.5}         # of a cached value, its share of a scale included
MAX_PAIRS = 2.2e9             # (head, token, position) triples of the largest listed attention, masked ones included ...
MAX_VALUES = 1.1e9            # ... values of its cache, of K and V together, of the rows that its lists name ...
MAX_MOVED = 9e8               # ... and bytes of the largest listed step that is appended
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _case(name, op, B, T, *, H=32, H_kv=0, D=128, dtype="bf16", n_q=1, ctx_lo=0, window=0, sinks=0, page=0, block=64, budget=0,
          recent=0, rotary=0, interleaved=False):
    """Lengths are uniform in [ctx_lo, T] (0: all T); where n_q > 1 and lengths are ragged, requests bring 1..n_q tokens.
    page 0: one [T, D] plane per request and head, else rows per page of a [pages, rows, heads, D] pool.
    block: positions; budget, and for lists sinks and recent: blocks.  rotary: dimensions that are rotated."""
    c = {"op": op, "B": B, "T": T, "H": H, "H_kv": H_kv or H, "D": D, "dtype": dtype, "n_q": n_q, "ctx_lo": ctx_lo or T,
         "window": window, "sinks": sinks, "page": page, "block": block, "budget": budget, "recent": recent, "rotary": rotary,
         "interleaved": interleaved}
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one token of one request, few small heads: all latency
        _case("append_tiny", "append", 1, 512, H=8, D=64, dtype="f16", rotary=64),
        # one token each of a large batch into a 4-bit cache, grouped query heads
        _case("append_decode_fp4", "append", 64, 4096, H_kv=8, dtype="fp4", ctx_lo=1001, rotary=128),
        # whole prompts of a batch into a paged cache, half of the dimensions rotated, as pairs of neighbours
        _case("append_prompt", "append", 4, 4096, n_q=4096, page=16, rotary=64, interleaved=True),
        # the blocks of the newest token, an 8-bit cache
        _case("bounds_step", "bounds", 32, 4096, H_kv=8, dtype="fp8", ctx_lo=1500, page=64, block=64),
        # all blocks of long contexts: a cache that was filled or compacted
        _case("bounds_whole", "bounds", 8, 16384, H_kv=8, n_q=16384, ctx_lo=9000, block=64),
        # one short request
        _case("select_tiny", "select", 1, 512, H=8, D=64, dtype="f16", block=32, sinks=1, recent=1, budget=8),
        # long contexts of a batch in small blocks, an eighth of them kept
        _case("select_long", "select", 32, 16384, H_kv=8, ctx_lo=6001, block=32, sinks=1, recent=4, budget=64),
        # a batch of long contexts, 2048 positions of each
        _case("blocks_decode", "blocks", 32, 16384, H_kv=8, ctx_lo=6001, block=64, budget=32),
        # drafted tokens over a 4-bit cache in pages
        _case("blocks_drafts_fp4", "blocks", 8, 8192, H_kv=8, dtype="fp4", n_q=5, ctx_lo=3001, page=64, block=128, budget=8),
        # one short request over a 4-bit cache
        _case("fp4_tiny", "fp4", 1, 512, H=8, D=64, dtype="fp4"),
        # the full contexts of a batch, one token each
        _case("fp4_decode", "fp4", 32, 16384, H_kv=8, dtype="fp4", ctx_lo=9000),
        # ragged chunks of long prompts in pages, within a window
        _case("fp4_chunks_paged", "fp4", 8, 16384, H_kv=8, dtype="fp4", n_q=509, ctx_lo=4100, window=4096, sinks=16, page=64),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["append", "bounds", "select", "blocks", "fp4"])
    H, D = rng.choice([(8, 64), (32, 128), (32, 128)])
    H_kv = rng.choice([H, H // 4])
    dtype = "fp4" if op == "fp4" else rng.choice(["bf16", "f16", "fp8", "fp4"])
    B, T = _log_int(rng, 1, 64), _log_int(rng, 200, 16384)
    block = rng.choice([32, 64, 128, 256])
    n_q = rng.choice([1, rng.randint(2, 16), _log_int(rng, 17, 4096)])
    if op in ("select", "blocks"):
        n_q = rng.choice([1, 1, rng.randint(2, 16), _log_int(rng, 17, 512)])
    n_q = min(n_q, T)
    budget = _log_int(rng, 1, max(1, T // block)) if op in ("select", "blocks") else 0
    B = max(1, min(B, int(MAX_VALUES / (2 * H_kv * T * D))))
    if op == "append":
        n_q = max(1, min(n_q, int(MAX_MOVED / (4 * B * (H + 2 * H_kv) * D))))
    if op in ("fp4", "blocks"):                         # cut the tokens until it costs no more than the listed
        n_q = max(1, min(n_q, int(MAX_PAIRS / (B * H * T))))
    if op == "blocks":
        n_q = max(1, min(n_q, int(MAX_VALUES / (2 * B * H_kv * budget * block * D))))
    if op == "select":
        n_q = max(1, min(n_q, int(MAX_VALUES * block / (64 * B * H_kv * T * D))))
    sinks = rng.choice([0, 4, rng.randint(1, 64)])
    recent = 0
    if budget:
        sinks, recent = min(rng.randint(0, 2), budget // 2), min(rng.randint(0, 4), budget - budget // 2)
    return _case("", op, B, T, H=H, H_kv=H_kv, D=D, dtype=dtype, n_q=n_q, ctx_lo=max(n_q, rng.randint(1, T)),
                 window=rng.choice([0, _log_int(rng, 1, T)]) if op == "fp4" else 0, sinks=sinks,
                 page=rng.choice([0, 0, 16, 64, 128]) if op != "select" else 0, block=block, budget=budget, recent=recent,
                 rotary=rng.choice([0, D // 2, D, D]) if op == "append" else 0, interleaved=rng.random() < 0.3)


def _lengths(c):
    """Context lengths and new tokens of every request: part of the case, the same for every seed."""
    rng = np.random.RandomState((c["B"] * 7919 + c["T"] * 31 + c["n_q"]) % (1 << 31))
    ctx = rng.randint(c["ctx_lo"], c["T"] + 1, c["B"])
    if c["op"] == "bounds" and c["n_q"] == c["T"]:
        return ctx, ctx
    fixed = c["ctx_lo"] == c["T"] or c["n_q"] == 1
    return ctx, np.full(c["B"], c["n_q"]) if fixed else np.minimum(rng.randint(1, c["n_q"] + 1, c["B"]), ctx)


def work(c):
    ctx, new = _lengths(c)
    D, H, H_kv, block, tokens = c["D"], c["H"], c["H_kv"], c["block"], int(new.sum())
    row = D * BITS[c["dtype"]] / 8                                                 # bytes of a cached row
    if c["op"] == "append":
        moved = tokens * (4 * D * H + 2 * H_kv * (2 * D + row) + 4 * c["rotary"])
        return {"bytes": moved, "flops": 3 * tokens * (H + H_kv) * c["rotary"]}
    if c["op"] == "bounds":
        first = (ctx - new) // block * block
        return {"bytes": H_kv * (int((ctx - first).sum()) * row + 4 * D * int((-(-ctx // block) - first // block).sum())), "flops": 0}
    q_bytes = 2 * H * D * tokens
    if c["op"] == "select":
        pairs = sum(int((np.arange(n - t, n) // block + 1).sum()) for n, t in zip(ctx.tolist(), new.tolist()))
        kept = sum(int(np.minimum(np.arange(n - t, n) // block + 1, c["budget"]).sum()) for n, t in zip(ctx.tolist(), new.tolist()))
        return {"bytes": q_bytes + H_kv * (4 * D * int((-(-ctx // block)).sum()) + 4 * pairs + 4 * kept), "flops": 4 * D * H_kv * pairs}
    pairs = rows = 0
    if c["op"] == "blocks":                            # (a list's last block is seldom the newest: counted whole)
        for n, t in zip(ctx.tolist(), new.tolist()):
            pairs += int(np.minimum(np.arange(n - t, n) + 1, c["budget"] * block).sum())
            rows += min(n, int(np.minimum(np.arange(n - t, n) + 1, c["budget"] * block).sum()))
    else:
        for n, t in zip(ctx.tolist(), new.tolist()):
            pos = np.arange(n - t, n)
            w = np.minimum(c["window"] or n, pos + 1)                             # positions inside the window ...
            first = np.minimum(c["sinks"], np.maximum(pos - w + 1, 0))            # ... and sinks in front of it
            pairs += int((w + first).sum())
            rows += min(n, n - int(max(0, pos[0] - w[0] + 1)) + int(first.max()))
    return {"bytes": 2 * q_bytes + 4 * H * tokens + 2 * rows * H_kv * row, "flops": 4 * D * H * pairs}


def _split(x):
    """Values as the 4-bit cache holds them: codes (two a byte, the low half first) and the scales of each 16."""
    g = x.float().reshape(*x.shape[:-1], -1, 16)
    scale = (g.abs().amax(-1) / 6).clamp(max=448).to(torch.float8_e4m3fn)
    by = scale.float()[..., None]
    z = torch.where(by == 0, 0, g / by.masked_fill(by == 0, 1))
    a, code = z.abs(), torch.zeros_like(z)
    for edge, up in ((0.25, False), (0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (a >= edge) if up else (a > edge)      # a value half-way goes to the even code
    code = (code.to(torch.uint8) + 8 * z.signbit().to(torch.uint8)).reshape(x.shape)
    return code[..., ::2] | code[..., 1::2] << 4, scale.view(torch.uint8)


def _values(codes, scales):
    """What codes and scales stand for."""
    table = torch.tensor([[s * x for x in E2M1] for s in (1, -1)], device=codes.device).flatten()
    x = torch.stack([table[(codes & 15).int()], table[(codes >> 4).int()]], -1).reshape(*codes.shape[:-1], -1, 16)
    return (x * scales.view(torch.float8_e4m3fn).float()[..., None]).flatten(-2)


def _store(s, name, x):
    """A cache of these values."""
    if s["case"]["dtype"] == "fp4":
        s[name], s[name + "_scales"] = _split(x)
    else:
        s[name], s[name + "_scales"] = x.to(DTYPES[s["case"]["dtype"]]), None


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    ctx, new = _lengths(c)
    B, T, H, H_kv, D, n_q = c["B"], c["T"], c["H"], c["H_kv"], c["D"], c["n_q"]
    dt_q = DTYPES[c["dtype"]] if c["dtype"] in ("bf16", "f16") else torch.bfloat16
    normal = lambda *shape: torch.randn(*shape, device="cuda", generator=g)  # noqa: E731
    ints = lambda x: torch.as_tensor(x, device="cuda", dtype=torch.int32)  # noqa: E731
    s = {"case": c, "ctx": ints(ctx), "q_lens": ints(new), "status": torch.zeros(1, dtype=torch.int32, device="cuda")}
    if c["page"]:
        per = (T + c["page"] - 1) // c["page"]
        order = torch.randperm(B * per + 3, device="cuda", generator=g)[: B * per].view(B, per)
        used = torch.arange(per, device="cuda") * c["page"] < s["ctx"][:, None]
        s["table"] = torch.where(used, order, -1).to(torch.int32).contiguous()
    shape = (B * per + 3, c["page"], H_kv, D) if c["page"] else (B, H_kv, T, D)
    if c["op"] != "select":
        for name in ("k", "v")[: 1 if c["op"] == "bounds" else 2]:
            _store(s, name, normal(*shape))
    if c["op"] != "bounds":
        s["q"] = normal(B, n_q, H, D).to(dt_q).permute(0, 2, 1, 3)       # token-major, as a projection leaves it
    if c["op"] == "append":
        s["k_new"], s["v_new"] = (normal(B, n_q, H_kv, D).to(dt_q).permute(0, 2, 1, 3) for _ in range(2))
        s["q_out"] = torch.zeros(B, H, n_q, D, device="cuda", dtype=dt_q)
        s["cos_sin"] = None
        if c["rotary"]:
            angles = torch.arange(T, device="cuda").double()[:, None] * 10000.0 ** (-torch.arange(c["rotary"] // 2, device="cuda").double() * 2 / c["rotary"])
            s["cos_sin"] = torch.cat([angles.cos(), angles.sin()], 1).float()
        if c["dtype"] == "fp4":                                               # where the step's rows lie, to be read back
            t = torch.arange(n_q, device="cuda")
            b, t = (t < s["q_lens"][:, None]).nonzero(as_tuple=True)
            j = (s["ctx"] - s["q_lens"]).long()[b] + t
            h = torch.arange(H_kv, device="cuda")[:, None]
            s["written"] = (_rows(s)[b, j] * H_kv + h if c["page"] else (b * H_kv + h) * T + j).flatten()
    if c["op"] in ("bounds", "select"):
        n = -(-T // c["block"])
        s["bounds"] = torch.zeros(B, H_kv, n, 2, D, device="cuda", dtype=dt_q)
    if c["op"] == "select":                                                   # the bounds of N(0, 1) keys, heads of different spread
        lean = normal(B, H_kv, n, D)
        wide = math.sqrt(2 * math.log(c["block"])) * (1 + 0.2 * torch.rand(B, H_kv, n, D, device="cuda", generator=g))
        s["bounds"][:, :, :, 0], s["bounds"][:, :, :, 1] = lean - wide, lean + wide
        s["scores"] = torch.zeros(B, H_kv, n_q, n, device="cuda")
        s["index"] = torch.full((B, H_kv, n_q, c["budget"]), -1, dtype=torch.int32, device="cuda")
        s["counts"] = torch.zeros(B, H_kv, n_q, dtype=torch.int32, device="cuda")
    if c["op"] == "blocks":
        s["index"], s["counts"] = _lists(s, g)
    if c["op"] in ("fp4", "blocks"):
        s["out"] = torch.zeros(B, n_q, H, D, device="cuda", dtype=dt_q).permute(0, 2, 1, 3)
        s["lse"] = torch.zeros(B, H, n_q, device="cuda")
    if own:
        _plan(s)
    return s


def _lists(s, g):
    """Lists of blocks for every token and K/V head: the first one, the newest one, and a random choice between them, in order."""
    c = s["case"]
    n, budget = -(-c["T"] // c["block"]), c["budget"]
    j = torch.arange(n, device="cuda")
    seen = (_positions(s) // c["block"] + 1)[:, None, :, None]                     # [B, 1, n_q, 1] blocks that the token sees
    rank = torch.rand(c["B"], c["H_kv"], c["n_q"], n, device="cuda", generator=g)
    rank = torch.where((j == 0) | (j == seen - 1), 2.0, rank).masked_fill(j >= seen, -1.0)
    kept = rank.argsort(dim=-1, descending=True, stable=True)[..., :budget]
    counts = seen.clamp(0, budget).expand(-1, c["H_kv"], -1, -1)[..., 0]
    kept = torch.where(j[:budget] < counts[..., None], kept, n).sort(-1).values
    return torch.where(j[:budget] < counts[..., None], kept, -1).to(torch.int32).contiguous(), counts.to(torch.int32).contiguous()


def _positions(s):
    """[B, n_q] positions of the step's tokens; behind a request's last token -1."""
    t = torch.arange(s["case"]["n_q"], device="cuda")
    ctx, new = s["ctx"].long()[:, None], s["q_lens"].long()[:, None]
    return torch.where(t < new, ctx - new + t, -1)


def _plan(s):
    """What a program keeps for its calls: descriptors and a workspace."""
    from paper_2404_09336_b200 import ssa
    c = s["case"]
    s["paging"] = ssa.make_paging(s["table"], c["page"], s["table"].numel() + 3) if c["page"] else None
    B, T, H, H_kv, D = c["B"], c["T"], c["H"], c["H_kv"], c["D"]
    dt_q = DTYPES[c["dtype"]] if c["dtype"] in ("bf16", "f16") else torch.bfloat16
    q = s["q"][:, :, 0] if "q" in s else torch.empty(B, H, D, device="cuda", dtype=dt_q)
    out = s["out"][:, :, 0] if "out" in s else q
    k = s.get("k")
    if k is None:
        k = torch.empty(1, 1, 1, D, device="cuda", dtype=dt_q).expand(B, H_kv, T, D)
    v = s.get("v", k)
    if c["dtype"] == "fp4" and "k" in s:
        s["desc"] = ssa.make_desc_fp4(q, k, v, s["k_scales"], s.get("v_scales", s["k_scales"]), out, T, paged=bool(c["page"]))
    else:
        s["desc"] = (ssa.make_desc_paged if c["page"] else ssa.make_desc)(q, k, v, out, T)
    if c["op"] == "append":
        s["append"] = ssa.make_append(s["k_new"], s["v_new"], s["q"], s["q_out"], s["cos_sin"], interleaved=c["interleaved"],
                                      q_lens=s["q_lens"], paging=s["paging"])
    elif c["op"] == "fp4":
        s["win"] = ssa.make_window(s["q"], s["out"], c["window"], c["sinks"], s["q_lens"], s["paging"])
        need = ssa.attn_window_fp4_workspace_bytes(s["desc"], s["win"])
    else:
        s["blocks"] = ssa.make_blocks(c["n_q"], c["block"], c["budget"] or 1, c["sinks"] if c["op"] == "select" else 0, c["recent"],
                                      q=s.get("q"), out=s.get("out"), bounds=s.get("bounds"), q_lens=s["q_lens"], paging=s["paging"])
        need = ssa.attn_blocks_workspace_bytes(s["desc"], s["blocks"]) if c["op"] == "blocks" else 0
    if "out" in s:
        s["workspace"] = torch.empty(need, dtype=torch.uint8, device="cuda")


def run(s):
    if own:
        return _own(s)
    return {"append": _plain_append, "bounds": _plain_bounds, "select": _plain_select, "blocks": _plain_blocks, "fp4": _plain_fp4}[s["case"]["op"]](s)


def _own(s):
    from paper_2404_09336_b200 import ssa
    op = s["case"]["op"]
    if op == "append":
        ssa.cache_append(s["desc"], s["append"], s["k_new"], s["v_new"], s["ctx"], s["k"], s["v"], s["q"], s["q_out"], s["k_scales"],
                         s["v_scales"], s["status"])
        return _appended(s)
    if op == "bounds":
        ssa.block_bounds(s["desc"], s["blocks"], s["k"], s["ctx"], s["bounds"], s["k_scales"], s["status"])
        return {"bounds": s["bounds"]}
    if op == "select":
        ssa.block_select(s["desc"], s["blocks"], s["q"], s["bounds"], s["ctx"], s["index"], s["counts"], s["scores"], s["status"])
        return {"index": s["index"], "counts": s["counts"], "scores": s["scores"]}
    if op == "blocks":
        ssa.attn_blocks(s["desc"], s["blocks"], s["q"], s["k"], s["v"], s["ctx"], s["index"], s["counts"], s["out"], s["lse"],
                        s["k_scales"], s["v_scales"], s["workspace"], s["status"])
    else:
        ssa.attn_window_fp4(s["desc"], s["win"], s["q"], s["k"], s["v"], s["k_scales"], s["v_scales"], s["ctx"], s["out"], s["lse"],
                            s["workspace"], s["status"])
    return {"out": s["out"], "lse": s["lse"]}


def _appended(s):
    """The cache; of a 4-bit one the values of the step's rows (its other rows were not touched), in a type that holds them exactly."""
    D, got = s["case"]["D"], {"q": s["q_out"]}
    for name in ("k", "v"):
        got[name] = s[name]
        if s["case"]["dtype"] == "fp4":
            got[name] = _values(s[name].view(-1, D // 2)[s["written"]], s[name + "_scales"].view(-1, D // 16)[s["written"]]).to(torch.bfloat16)
    return got


def _rows(s):
    """Pool rows of the logical positions of every request, [B, T]."""
    page, j = s["case"]["page"], torch.arange(s["case"]["T"], device="cuda")
    return s["table"].long().clamp(min=0)[:, j // page] * page + j % page


def _logical(s, name):
    """A cache's values as [B, H_kv, T, D] in 32 bits."""
    x, c = s[name], s["case"]
    x = _values(x, s[name + "_scales"]) if c["dtype"] == "fp4" else x
    return (x.reshape(-1, c["H_kv"], c["D"])[_rows(s)].permute(0, 2, 1, 3) if c["page"] else x).float()


def _rotated(s, x):
    """x[B, heads, n_q, D], each token's rows rotated by its position; in 64 bits, rounded to 32 (8- and 4-bit values lie next to borders)."""
    c, R = s["case"], s["case"]["rotary"]
    if not R:
        return x.float()
    x = x.double()
    cos, sin = (y.double()[:, None] for y in s["cos_sin"][_positions(s).clamp(min=0)].chunk(2, -1))      # [B, 1, n_q, R / 2]
    a, z = (x[..., :R:2], x[..., 1:R:2]) if c["interleaved"] else (x[..., : R // 2], x[..., R // 2: R])
    pair = (a * cos - z * sin, z * cos + a * sin)
    turned = torch.stack(pair, -1).flatten(-2) if c["interleaved"] else torch.cat(pair, -1)
    return torch.cat([turned, x[..., R:]], -1).float()


def _plain_append(s):
    c = s["case"]
    D, n_q = c["D"], c["n_q"]
    pos = _positions(s)
    there = pos >= 0
    s["q_out"] = torch.where(there[:, None, :, None], _rotated(s, s["q"]).to(s["q_out"].dtype), s["q_out"])
    b, t = there.nonzero(as_tuple=True)
    j = pos[b, t]
    for name in ("k", "v"):
        x = _rotated(s, s["k_new"]) if name == "k" else s["v_new"].float()
        x = x.permute(0, 2, 1, 3)[b, t]                                             # [rows, H_kv, D]
        if c["dtype"] == "fp4":
            parts = list(zip((s[name], s[name + "_scales"]), _split(x)))
        elif c["dtype"] == "fp8":
            parts = [(s[name].view(torch.uint8), x.clamp(-448, 448).to(s[name].dtype).view(torch.uint8))]
        else:
            parts = [(s[name], x.to(s[name].dtype))]
        for cache, rows in parts:
            if c["page"]:
                cache.view(-1, c["H_kv"], cache.shape[-1])[_rows(s)[b, j]] = rows
            else:
                cache.permute(0, 2, 1, 3)[b, j] = rows
    return _appended(s)


def _plain_bounds(s):
    c = s["case"]
    B, H_kv, T, D, block = c["B"], c["H_kv"], c["T"], c["D"], c["block"]
    n = -(-T // block)
    x = _logical(s, "k")
    ctx, new = s["ctx"].long()[:, None], s["q_lens"].long()[:, None]
    there = (torch.arange(T, device="cuda") < ctx)[:, None, :, None]
    pad = (0, 0, 0, n * block - T)
    least = torch.nn.functional.pad(x.masked_fill(~there, math.inf), pad, value=math.inf).view(B, H_kv, n, block, D).amin(3)
    most = torch.nn.functional.pad(x.masked_fill(~there, -math.inf), pad, value=-math.inf).view(B, H_kv, n, block, D).amax(3)
    j = torch.arange(n, device="cuda")
    touched = ((j >= (ctx - new) // block) & (j * block < ctx))[:, None, :, None, None]
    return {"bounds": torch.where(touched, torch.stack([least, most], 3).to(s["bounds"].dtype), s["bounds"])}


def _plain_select(s):
    c = s["case"]
    B, H_kv, D, n_q, budget = c["B"], c["H_kv"], c["D"], c["n_q"], c["budget"]
    q = s["q"].double().reshape(B, H_kv, -1, n_q, D)
    least, most = s["bounds"].double().unbind(3)
    score = (q.clamp(min=0).sum(2) @ most.transpose(-1, -2) + q.clamp(max=0).sum(2) @ least.transpose(-1, -2)).float()
    n, j = score.shape[-1], torch.arange(score.shape[-1], device="cuda")
    seen = (_positions(s)[:, None, :, None] // c["block"] + 1)                    # 0: no token
    rank = torch.where((j < c["sinks"]) | (j >= seen - c["recent"]), math.inf, score).masked_fill(j >= seen, -math.inf)
    kept = rank.sort(dim=-1, descending=True, stable=True).indices[..., :budget]    # stable: ties go to the lowest block
    counts = seen.clamp(max=budget)
    kept = torch.where(j[:budget] < counts, kept, n).sort(-1).values
    return {"index": torch.where(j[:budget] < counts, kept.to(torch.int32), s["index"]),
            "counts": torch.where(seen > 0, counts, s["counts"][..., None]).to(torch.int32).expand(-1, H_kv, -1, -1)[..., 0],
            "scores": torch.where(j < seen, score, s["scores"])}


def _weighted(s, x, seen, v):
    """Softmax of the scores x over what is seen, its sums of v's rows, and the logarithm of its sum; in 32 bits."""
    x = x.masked_fill_(~seen, -math.inf)
    top = x.amax(-1, keepdim=True).clamp(min=torch.finfo(torch.float32).min)
    x = x.sub_(top).exp_()
    total = x.sum(-1, keepdim=True)
    x = x.div_(total.masked_fill(total == 0, 1))
    return (x.reshape(*v.shape[:-2], -1, v.shape[-2]) @ v), (top + total.log())[..., 0]


def _finished(s, out, lse):
    rows = (_positions(s) >= 0)[:, None]                                          # rows behind the last token stay as they were
    return {"out": torch.where(rows[..., None], out.to(s["out"].dtype), s["out"]), "lse": torch.where(rows, lse, s["lse"])}


def _plain_blocks(s):
    c = s["case"]
    B, H, H_kv, D, n_q, block = c["B"], c["H"], c["H_kv"], c["D"], c["n_q"], c["block"]
    pos = _positions(s)[:, None, :, None]
    j = (s["index"].long()[..., None] * block + torch.arange(block, device="cuda")).flatten(-2)      # [B, H_kv, n_q, listed]
    i = torch.arange(j.shape[-1], device="cuda") // block
    seen = (i < s["counts"][..., None]) & (j >= 0) & (j <= pos)
    j = j.clamp(0, c["T"] - 1)
    b, h = torch.arange(B, device="cuda")[:, None, None, None], torch.arange(H_kv, device="cuda")[:, None, None]
    place = _rows(s)[b, j] * H_kv + h if c["page"] else (b * H_kv + h) * c["T"] + j
    k, v = (_values(s[x].view(-1, D // 2)[place], s[x + "_scales"].view(-1, D // 16)[place]) if c["dtype"] == "fp4"
            else s[x].view(-1, D)[place].float() for x in ("k", "v"))              # [B, H_kv, n_q, listed, D]
    q = s["q"].float().reshape(B, H_kv, -1, n_q, D).transpose(2, 3)               # [B, H_kv, n_q, group, D]
    out, lse = _weighted(s, q @ k.transpose(-1, -2) * (1 / math.sqrt(D)), seen[:, :, :, None], v)
    return _finished(s, out.transpose(2, 3).reshape(B, H, n_q, D), lse.transpose(2, 3).reshape(B, H, n_q))


def _plain_fp4(s):
    c = s["case"]
    B, H, H_kv, D, n_q, T = c["B"], c["H"], c["H_kv"], c["D"], c["n_q"], c["T"]
    j, pos = torch.arange(T, device="cuda"), _positions(s)[:, :, None]
    seen = j <= pos
    if c["window"]:
        seen &= (j > pos - c["window"]) | (j < c["sinks"])
    k, v = _logical(s, "k"), _logical(s, "v")
    x = (s["q"].float().reshape(B, H_kv, -1, D) @ k.transpose(-1, -2) * (1 / math.sqrt(D))).view(B, H, n_q, T)
    out, lse = _weighted(s, x, seen[:, None], v)
    return _finished(s, out.view(B, H, n_q, D), lse)


def _held(codes, scales):
    """Values of a 4-bit cache in 64 bits, from the definition: sign, two bits of exponent (bias 1), one of fraction."""
    x = torch.stack([codes % 16, codes // 16], -1).flatten(-2).double()
    sign, e, f = 1 - 2 * (x // 8), x % 8 // 2, x % 2
    x = sign * torch.where(e == 0, f / 2, 2 ** (e - 1) * (1 + f / 2))
    return x * scales.view(torch.float8_e4m3fn).double().repeat_interleave(16, -1)


def _nearest(x):
    """x as a 4-bit cache holds it, in 64 bits: of the 16 values the nearest; half-way the one whose fraction is zero."""
    g = x.reshape(*x.shape[:-1], -1, 16)
    scale = (g.abs().amax(-1, keepdim=True) / 6).float().to(torch.float8_e4m3fn).double()
    z = g / scale.masked_fill(scale == 0, math.inf)
    step = torch.where(z.abs() < 2, 0.5, torch.where(z.abs() < 4, 1.0, 2.0))
    return ((z / step).round().mul(step).clamp(-6, 6) * scale).reshape(x.shape)   # (round: to the even multiple)


def exact(case, seed):
    """Request by request and head by head in 64 bits, the visible positions listed instead of masked."""
    c = case
    if c["op"] == "bounds":
        return None                                            # nothing is rounded
    s = prepare(c, seed)
    ctx, new = s["ctx"].tolist(), s["q_lens"].tolist()
    D, H_kv, group = c["D"], c["H_kv"], c["H"] // c["H_kv"]
    rows_of = lambda b: torch.tensor([p * c["page"] + r for p in s["table"][b].tolist() if p >= 0 for r in range(c["page"])][: ctx[b]], device="cuda")  # noqa: E731
    if c["op"] == "append":
        R = c["rotary"]
        turn = torch.zeros(c["T"], D, D, dtype=torch.float64, device="cuda") if D * D * c["T"] < 3e8 else None
        if turn is None:
            return None
        turn[:] = torch.eye(D, device="cuda")
        for i in range(R // 2):
            a, z = (2 * i, 2 * i + 1) if c["interleaved"] else (i, i + R // 2)
            cos, sin = s["cos_sin"][:, i].double(), s["cos_sin"][:, R // 2 + i].double()
            turn[:, a, a], turn[:, a, z], turn[:, z, a], turn[:, z, z] = cos, -sin, sin, cos
        q, k, v = s["q_out"].double(), s["k"], s["v"]
        flat = c["dtype"] == "fp4"
        k, v = (None, None) if flat else (k.double(), v.double())
        got = {"k": [], "v": []}
        for b in range(c["B"]):
            n, t = ctx[b], new[b]
            at = turn[n - t: n]
            q[b, :, :t] = torch.einsum("tij,htj->hti", at, s["q"][b, :, :t].double())
            kt, vt = torch.einsum("tij,htj->hti", at, s["k_new"][b, :, :t].double()), s["v_new"][b, :, :t].double()
            if flat:
                got["k"].append(_nearest(kt)), got["v"].append(_nearest(vt))
            elif c["page"]:
                k.view(-1, H_kv, D)[rows_of(b)[n - t:]], v.view(-1, H_kv, D)[rows_of(b)[n - t:]] = kt.transpose(0, 1), vt.transpose(0, 1)
            else:
                k[b, :, n - t: n], v[b, :, n - t: n] = kt, vt
        if flat:                                               # heads, then requests and tokens, as the rows are read back
            k, v = (torch.cat(got[x], 1).reshape(-1, D) for x in ("k", "v"))
        return {"q": q, "k": k, "v": v}
    if c["op"] == "select":
        scores = s["scores"].double()
        for b in range(c["B"]):
            for t in range(new[b]):
                n = (ctx[b] - new[b] + t) // c["block"] + 1
                for h in range(H_kv):
                    q = s["q"][b, h * group: (h + 1) * group, t].double()
                    scores[b, h, t, :n] = torch.maximum(q[:, None] * s["bounds"][b, h, :n, 0].double(), q[:, None] * s["bounds"][b, h, :n, 1].double()).sum((0, 2))
            if c["B"] * c["n_q"] * H_kv > 20000:
                return None
        return {"index": None, "counts": None, "scores": scores}
    out, lse = s["out"].double(), s["lse"].double()
    if c["op"] == "blocks" and sum(new) * H_kv > 12000:
        return None
    for b in range(c["B"]):
        n, t = ctx[b], new[b]
        for h in range(H_kv):
            K, V = ((_held(x.reshape(-1, D // 2), y.reshape(-1, D // 16)) if c["dtype"] == "fp4" else x.reshape(-1, D).double())
                    for x, y in ((z[:, :, h].reshape(-1, z.shape[-1])[rows_of(b)] if c["page"] else z[b, h, :n], w if w is None else
                                  w[:, :, h].reshape(-1, w.shape[-1])[rows_of(b)] if c["page"] else w[b, h, :n])
                                 for z, w in ((s["k"], s["k_scales"]), (s["v"], s["v_scales"]))))
            heads = range(h * group, (h + 1) * group)
            if c["op"] == "blocks":
                for i in range(t):
                    j = torch.cat([torch.arange(x * c["block"], min((x + 1) * c["block"], n - t + i + 1)) for x in s["index"][b, h, i, : s["counts"][b, h, i]].tolist()]).cuda()
                    x = s["q"][b, h * group: (h + 1) * group, i].double() @ K[j].t() / math.sqrt(D)
                    total = torch.logsumexp(x, 1)
                    out[b, heads, i], lse[b, heads, i] = torch.exp(x - total[:, None]) @ V[j], total
                continue
            j, lo = torch.arange(n, device="cuda"), torch.arange(n - t, n, device="cuda")[:, None]
            hidden = j[None] > lo
            if c["window"]:
                hidden |= (lo - j[None] >= c["window"]) & (j[None] >= c["sinks"])
            for head in heads:
                x = s["q"][b, head, :t].double() @ K.t() / math.sqrt(D)
                x[hidden] = -math.inf
                total = torch.logsumexp(x, 1)
                out[b, head, :t], lse[b, head, :t] = torch.exp(x - total[:, None]) @ V, total
    return {"out": out, "lse": lse}
