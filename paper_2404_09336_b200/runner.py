"""Device-side plumbing around the C-ABI calls: buffers for one workload and
the decode step (span lists -> index lists -> attention).

Only allocation, host<->device copies and calls of ``ssa.*`` happen here.
"""
from __future__ import annotations

import concurrent.futures as _cf
import contextlib
import os

import numpy as np
import torch

from . import ssa
from .inputs import Workload

_TORCH_DTYPE = {"bf16": torch.bfloat16, "f16": torch.float16}


def bits_to_tensor(bits: np.ndarray, dtype: str) -> torch.Tensor:
    """uint16 storage patterns -> CPU tensor of the storage type (no copy)."""
    return torch.from_numpy(bits.view(np.int16)).view(_TORCH_DTYPE[dtype])


def tensor_to_bits(t: torch.Tensor) -> np.ndarray:
    return t.detach().cpu().contiguous().view(torch.int16).numpy().view(np.uint16)


def _nbytes(shape, dt):
    return int(np.prod(shape)) * torch.empty((), dtype=dt).element_size()


def _views(buf, specs):
    """Tensors of the given (shape, dtype) laid back to back at 256-byte boundaries in the uint8 buffer."""
    views, o = [], 0
    for shape, dt in specs:
        n = _nbytes(shape, dt)
        views.append(buf[o:o + n].view(dt).view(shape))
        o += (n + 255) // 256 * 256
    return views


def _arena(device, specs):
    """One uint8 device buffer holding tensors of the given (shape, dtype)
    back to back at 256-byte boundaries; returns (buffer, views)."""
    total = sum((_nbytes(shape, dt) + 255) // 256 * 256 for shape, dt in specs)
    buf = torch.zeros(total, dtype=torch.uint8, device=device)
    return buf, _views(buf, specs)


class DecodeStep:
    """Buffers of one workload on one GPU.

    layout "bhtd": cache stored [B, H, T, D] (one contiguous plane per head);
    layout "bthd": cache stored [B, T, H, D] (token-major).  Either way
    ``self.k`` / ``self.v`` are the logical [B, H, T, D] views.
    ``kv_copies`` > 1 keeps several copies of the cache so that consecutive
    timed steps read different memory.  ``query_heads`` (a multiple of the
    workload's H) gives the query, output and lse that many heads over the
    workload's H cache heads (grouped query heads).
    """

    def __init__(self, wl: Workload, device="cuda:0", layout="bhtd", out_dtype=None, kv_copies=1,
                 index_stride=None, max_selected=None, gen_threads=None,
                 span_capacity=0, query_heads=None):
        self.wl, self.device, self.layout = wl, torch.device(device), layout
        dt = _TORCH_DTYPE[wl.dtype]
        dev = self.device
        B, H, D, T = wl.B, wl.H, wl.D, wl.max_ctx
        shape = (B, H, T, D) if layout == "bhtd" else (B, T, H, D)
        self.k_store = [torch.empty(shape, dtype=dt, device=dev) for _ in range(kv_copies)]
        self.v_store = [torch.empty(shape, dtype=dt, device=dev) for _ in range(kv_copies)]
        threads = gen_threads or max(1, min(B, (os.cpu_count() or 2) // 2, 8))
        with _cf.ThreadPoolExecutor(threads) as ex:          # draw on several cores, upload in order
            pending = []
            for i in range(B):
                pending.append(ex.submit(wl.kv_bits_seq, i))
                if len(pending) >= threads or i == B - 1:
                    first = i - len(pending) + 1
                    for j, fut in enumerate(pending):
                        kb, vb = fut.result()
                        kt, vt = bits_to_tensor(kb, wl.dtype), bits_to_tensor(vb, wl.dtype)
                        if layout == "bthd":
                            kt, vt = kt.permute(1, 0, 2), vt.permute(1, 0, 2)
                        self.k_store[0][first + j].copy_(kt)
                        self.v_store[0][first + j].copy_(vt)
                    pending = []
        for c in range(1, kv_copies):
            self.k_store[c].copy_(self.k_store[0])
            self.v_store[c].copy_(self.v_store[0])
        self.select_copy(0)
        spans = wl.spans if len(wl.spans) else np.zeros((1, 2), np.int32)
        self.max_selected = int(max_selected or max(wl.selected_upper_bound(), 1))
        self.index_stride = int(index_stride or (self.max_selected + 31) // 32 * 32)
        odt = out_dtype or dt
        QH = int(query_heads or H)
        if QH % H != 0:
            raise ValueError("query_heads must be a multiple of the workload's heads")
        # what changes every decode step lives in one input arena and one result
        # arena, so that a host-driven step is one copy in and one copy out
        self.in_arena, (self.q, self.ctx_lens, self.span_offsets, self.spans) = _arena(
            dev, [((B, QH, D), dt), ((B,), torch.int32), ((B + 1,), torch.int32), ((max(len(spans), span_capacity), 2), torch.int32)])
        self._out_specs = [((B, QH, D), odt), ((B, QH), torch.float32), ((B,), torch.int32), ((1,), torch.int32)]
        self.out_arena, (self.out, self.lse, self.counts, self.status) = _arena(dev, self._out_specs)
        self.q.copy_(bits_to_tensor(wl.q_bits(QH), wl.dtype))
        self.ctx_lens.copy_(torch.from_numpy(wl.ctx_lens.copy()))
        self.span_offsets.copy_(torch.from_numpy(wl.span_offsets.copy()))
        self.spans[: len(spans)].copy_(torch.from_numpy(np.ascontiguousarray(spans)))
        self.out.zero_()
        self.lse.zero_()
        self.counts.fill_(-7)
        self.status.zero_()
        self.index = torch.full((B, self.index_stride), -7, dtype=torch.int32, device=dev)
        self.mass = torch.zeros((B, T), dtype=torch.float32, device=dev)     # weight of every position so far (attend_mass)
        # what a budget keeps has lists of its own, with room for whole contexts: the span lists' bound and buffers stay theirs
        self.budget = 0
        self._budget_lists = (torch.full((B, (T + 31) // 32 * 32), -7, dtype=torch.int32, device=dev),
                              torch.full((B,), -7, dtype=torch.int32, device=dev))
        self._span_lists = None                              # (index, counts) while the budget's are in their place
        self.desc = ssa.make_desc(self.q, self.k, self.v, self.out, max_ctx=T)
        self.max_spans = int(max(1, np.diff(wl.span_offsets).max() if wl.B else 1))
        need = max(ssa.decode_workspace_bytes(self.desc, self.max_selected),
                   ssa.decode_workspace_bytes(self.desc, T),
                   ssa.decode_spans_workspace_bytes(self.desc, self.index_stride, ssa.MAX_SPANS_PER_SEQ))
        if need == 0:
            raise RuntimeError("ssa_decode_workspace_bytes rejected the descriptor")
        self.workspace = torch.empty(need, dtype=torch.uint8, device=dev)
        self._rooms, self._outgrown = [], []
        self._next_lens, self._new_lens = (torch.zeros_like(self.ctx_lens) for _ in range(2))    # of append
        self._steps = {}
        if dev.type == "cuda":                               # calls may come on any stream: what was filled above is there
            torch.cuda.current_stream(dev).synchronize()

    def _copy(self, c: int):
        ks, vs = self.k_store[c % len(self.k_store)], self.v_store[c % len(self.v_store)]
        return (ks, vs) if self.layout == "bhtd" else (ks.permute(0, 2, 1, 3), vs.permute(0, 2, 1, 3))

    def select_copy(self, c: int):
        self.k, self.v = self._copy(c)

    # ---- the calls ------------------------------------------------------------------
    # self.index, self.counts are the lists that were asked for last, from spans or by a budget; max_selected bounds the first,
    # budget the second.
    def _lists_of_spans(self):
        if self._span_lists is not None:
            (self.index, self.counts), self._span_lists = self._span_lists, None

    def build_index(self, stream=None):
        self._lists_of_spans()
        return ssa.spans_to_index(self.span_offsets, self.spans, self.ctx_lens, self.index, self.counts,
                                  self.status, stream)

    def attend_sparse(self, stream=None):
        if self._span_lists is not None:
            bound = self.budget
            workspace = self._room(ssa.decode_workspace_bytes(self.desc, bound), stream)
        else:
            bound, workspace = self.max_selected, self.workspace
        return ssa.decode_attn_sparse(self.desc, self.q, self.k, self.v, self.ctx_lens, self.index,
                                      self.counts, bound, self.out, self.lse, workspace,
                                      self.status, stream)

    def attend_spans(self, stream=None, want_lists=False):
        """Span lists -> attention output in one call (no index list unless want_lists)."""
        if want_lists:
            self._lists_of_spans()
        return ssa.decode_attn_spans(self.desc, self.q, self.k, self.v, self.ctx_lens, self.span_offsets, self.spans,
                                     self.max_spans, self.max_selected, self.out, self.lse,
                                     self.index if want_lists else None, self.counts if want_lists else None,
                                     self.workspace, self.status, stream)

    def attend_dense(self, stream=None):
        return ssa.decode_attn_dense(self.desc, self.q, self.k, self.v, self.ctx_lens, self.out, self.lse,
                                     self.workspace, self.status, stream)

    # ---- a cache kept within a budget ---------------------------------------------------
    def _on(self, stream):
        """The caller's stream as torch's current one."""
        if stream is None:
            return contextlib.nullcontext()
        return torch.cuda.stream(torch.cuda.ExternalStream(ssa._stream(stream), device=self.device))

    def _room(self, need, stream):
        """Workspace of these calls, apart from that of the calls over spans.  One that is too small stays as it is beside the
        next: graphs captured with it and calls still running on another stream go on using it."""
        most = self._rooms[-1].numel() if self._rooms else 0
        if need > most:
            with self._on(stream):
                self._rooms.append(torch.empty(max(need, 2 * most), dtype=torch.uint8, device=self.device))
        return self._rooms[-1]

    def _window(self, window, sinks, mass, stream):
        q, out = self.q.unsqueeze(2), self.out.unsqueeze(2)
        win = ssa.make_window(q, out, window, sinks)
        need = (ssa.attn_mass_workspace_bytes if mass else ssa.attn_window_workspace_bytes)(self.desc, win)
        return q, out, win, self._room(need, stream)

    def attend_window(self, window: int, sinks: int = 0, stream=None):
        """The step's token over the newest `window` positions and the first `sinks`."""
        q, out, win, room = self._window(window, sinks, False, stream)
        return ssa.attn_window(self.desc, win, q, self.k, self.v, self.ctx_lens, out, self.lse, room, self.status, stream)

    def attend_mass(self, decay: float = 1.0, window: int = 0, sinks: int = 0, stream=None):
        """The step's token over its context (or window), every position's weight added to self.mass [B, max_ctx]."""
        q, out, win, room = self._window(window, sinks, True, stream)
        return ssa.attn_mass(self.desc, win, q, self.k, self.v, self.ctx_lens, out, self.lse, self.mass, self.mass, decay,
                             room, self.status, stream)

    def select_heaviest(self, budget: int, sinks: int = 0, recent: int = 0, stream=None):
        """Index lists (self.index, self.counts, until the next ones from spans) of the positions that the budget keeps, by
        self.mass."""
        if budget > self._budget_lists[0].shape[1] and sinks >= 0 and recent >= 0 and sinks + recent <= budget:
            budget, sinks, recent = self.wl.max_ctx, 0, 0    # (room for every position: all stay)
        rc = ssa.mass_to_index(self.mass, self.ctx_lens, budget, sinks, recent, *self._budget_lists, self.status, stream)
        if self._span_lists is None:
            self._span_lists = self.index, self.counts
        self.index, self.counts = self._budget_lists
        self.budget = int(budget)
        return rc

    def compact(self, stream=None):
        """The listed rows of every copy of the cache, and their sums, to the front; contexts become the lists' lengths.  What names
        positions (lists, spans, lengths in host buffers) names those from before the move."""
        bound = self.max_selected if self._span_lists is None else self.budget
        for c in range(len(self.k_store)):                   # contexts and sums belong to all copies
            k, v = self._copy(c)
            ssa.cache_compact(self.desc, k, v, self.ctx_lens, self.index, self.counts, bound, None if c else self.mass, None,
                              self.status, stream)
        with self._on(stream):
            # (no longer than what was moved, where a count is above its bound or was never written)
            self.ctx_lens.copy_(torch.minimum(self.ctx_lens, self.counts.clamp(0, bound)))
        if hasattr(self, "bounds"):
            self.refresh_bounds(stream=stream)
        if hasattr(self, "fp4"):
            self._fill_fp4(self.fp4, stream)
        return ssa.OK

    # ---- filling the cache ----------------------------------------------------------------
    def append(self, k_new, v_new, q=None, cos_sin=None, interleaved=False, positions=None, stream=None):
        """A new token of every request that has room for one: contexts are one longer, its key k_new[B,H,D], rotated by position
        (cos_sin, positions as for make_append), and its value v_new are in every copy of the cache (the 4-bit one too), its query q,
        rotated, in self.q; the bounds of its block are made anew, its position's sum (attend_mass) starts from nothing.  A request
        whose context is max_ctx long already stays as it is, its row of self.q too (DEV_BAD_COUNT in self.status).  Refused arguments
        raise and change nothing.  What bounds lists on the host (max_selected, spans) stays."""
        k_new, v_new = k_new.unsqueeze(2), v_new.unsqueeze(2)
        q_new, q_out = (None, None) if q is None else (q.unsqueeze(2), self.q.unsqueeze(2))
        how = dict(cos_sin=cos_sin, interleaved=interleaved, positions=positions, q_lens=self._new_lens)
        first, others = ssa.make_append(k_new, v_new, q_new, q_out, **how), ssa.make_append(k_new, v_new, **how)
        desc = self.desc if q is None else ssa.make_desc(q, self.k, self.v, self.out, max_ctx=self.wl.max_ctx)
        caches = [(*self._copy(c), None, None) for c in range(len(self.k_store))]
        if hasattr(self, "fp4"):
            caches.append(self.fp4)
        with self._on(stream):
            torch.add(self.ctx_lens, 1, out=self._next_lens)
            self._new_lens.copy_(self.ctx_lens < self.wl.max_ctx)
        for i, (k, v, k_scales, v_scales) in enumerate(caches):          # (queries are rotated once)
            ssa.cache_append(desc if i == 0 else self.desc if k_scales is None else self.desc_fp4, others if i else first, k_new, v_new,
                             self._next_lens, k, v, None if i else q, None if i or q is None else self.q, k_scales, v_scales,
                             self.status, stream)
        with self._on(stream):
            # (the sum may be that of a position which was here before a compaction)
            at, new = self.ctx_lens.clamp(0, self.wl.max_ctx - 1).long().unsqueeze(1), self._new_lens.unsqueeze(1) > 0
            self.mass.scatter_(1, at, self.mass.gather(1, at).masked_fill(new, 0.0))
            self.ctx_lens.add_(self._new_lens)
        if hasattr(self, "bounds"):
            self.refresh_bounds(1, stream)
        return ssa.OK

    # ---- blocks that the queries select ------------------------------------------------------
    def enable_blocks(self, block_size: int = 64, budget: int = 32, sinks: int = 1, recent: int = 1, stream=None):
        """Bounds of every block of the cache, and room for the lists of attention over the `budget` blocks that score best.  (Asked for
        once more, e.g. with other blocks: graphs captured before go on using what they were captured with.)"""
        B, H, D, T, dev = self.wl.B, self.wl.H, self.wl.D, self.wl.max_ctx, self.device
        with self._on(stream):
            bounds = torch.zeros(B, H, -(-T // block_size), 2, D, dtype=self.q.dtype, device=dev)
            lists = (torch.full((B, H, 1, budget), -7, dtype=torch.int32, device=dev),
                     torch.zeros((B, H, 1), dtype=torch.int32, device=dev))
        blocks = ssa.make_blocks(1, block_size, budget, sinks, recent, self.q.unsqueeze(2), self.out.unsqueeze(2), bounds)
        self._refresh(blocks, bounds, None, stream)          # (refused: nothing has changed)
        if hasattr(self, "bounds"):
            self._outgrown += [self.bounds, self.block_lists]
        self.bounds, self.block_lists, self.blocks = bounds, lists, blocks
        return ssa.OK

    def _refresh(self, blocks, bounds, newest, stream):
        which = ssa.make_blocks(newest or self.wl.max_ctx, blocks.block_size, blocks.budget, bounds=bounds)
        return ssa.block_bounds(self.desc, which, self.k, self.ctx_lens, bounds, None, self.status, stream)

    def refresh_bounds(self, newest=None, stream=None):
        """Bounds of the blocks of the newest positions (None: of all)."""
        return self._refresh(self.blocks, self.bounds, newest, stream)

    def select_blocks(self, stream=None):
        """self.block_lists: for every K/V head the blocks that the step's queries rank first."""
        return ssa.block_select(self.desc, self.blocks, self.q, self.bounds, self.ctx_lens, *self.block_lists, None, self.status, stream)

    def attend_blocks(self, stream=None):
        """The step's token over the blocks on its lists."""
        room = self._room(ssa.attn_blocks_workspace_bytes(self.desc, self.blocks), stream)
        return ssa.attn_blocks(self.desc, self.blocks, self.q, self.k, self.v, self.ctx_lens, *self.block_lists, self.out, self.lse,
                               None, None, room, self.status, stream)

    # ---- the cache in 4 bits -------------------------------------------------------------------
    def enable_fp4(self, stream=None):
        """A copy of the cache in 4-bit values (codes and scales of K and of V).  Asked for once more, it is made anew in its place."""
        B, H, D, T, dev = self.wl.B, self.wl.H, self.wl.D, self.wl.max_ctx, self.device
        if self.q.dtype != torch.bfloat16:
            raise ValueError("queries over a 4-bit cache are bf16")
        fp4 = getattr(self, "fp4", None)
        with self._on(stream):
            if fp4 is None:
                fp4 = (*(torch.zeros(B, H, T, D // 2, dtype=torch.uint8, device=dev) for _ in range(2)),
                       *(torch.zeros(B, H, T, D // 16, dtype=torch.uint8, device=dev) for _ in range(2)))
            # rows at a time, as many as a call takes, and contexts of which they are the newest
            most = (1 << 24) // self.q.shape[1]
            filled = [(t, torch.full_like(self.ctx_lens, min(t + most, T))) for t in range(0, T, most)]
        self._outgrown.append(getattr(self, "_filled", None))
        self.desc_fp4, self._filled = ssa.make_desc_fp4(self.q, *fp4, self.out, T), filled
        rc = self._fill_fp4(fp4, stream)
        self.fp4 = fp4
        return rc

    def _fill_fp4(self, fp4, stream):
        k, v, k_scales, v_scales = fp4
        most = (1 << 24) // self.q.shape[1]
        for t, ends in self._filled:
            rows = self.k[:, :, t:t + most], self.v[:, :, t:t + most]
            ssa.cache_append(self.desc_fp4, ssa.make_append(*rows), *rows, ends, k, v, None, None, k_scales, v_scales, self.status, stream)
        return ssa.OK

    def attend_fp4(self, window: int = 0, sinks: int = 0, stream=None):
        """The step's token over its context (or window), read from the 4-bit cache."""
        q, out = self.q.unsqueeze(2), self.out.unsqueeze(2)
        win = ssa.make_window(q, out, window, sinks)
        room = self._room(ssa.attn_window_fp4_workspace_bytes(self.desc_fp4, win), stream)
        k, v, k_scales, v_scales = self.fp4
        return ssa.attn_window_fp4(self.desc_fp4, win, q, k, v, k_scales, v_scales, self.ctx_lens, out, self.lse, room, self.status,
                                   stream)

    # ---- the paper's blocked encoding as the metadata format ---------------------------
    def enable_blockmask(self, block_size: int = 256):
        """Buffers for the (block index, bitmask) lists of every request."""
        B, dev = self.wl.B, self.device
        self.block_size = block_size
        self.block_stride = (self.wl.max_ctx + block_size - 1) // block_size
        self._bound_blocks()
        self.block_idx = torch.full((B, self.block_stride), -7, dtype=torch.int32, device=dev)
        self.block_mask = torch.zeros((B, self.block_stride, block_size // 32), dtype=torch.int32, device=dev)
        self.block_counts = torch.zeros((B,), dtype=torch.int32, device=dev)
        need = ssa.decode_blockmask_workspace_bytes(self.desc, block_size, self.block_stride)
        if need > self.workspace.numel():
            self._outgrown.append(self.workspace)            # graphs captured with it go on using it
            self.workspace = torch.empty(need, dtype=torch.uint8, device=dev)
            self._steps = {}

    def _bound_blocks(self):
        """Host-side bound on the listed blocks of any request: no more than its context spans."""
        longest = int(self.wl.ctx_lens.max()) if len(self.wl.ctx_lens) else 1
        self.max_blocks = max(1, min(self.block_stride, (longest + self.block_size - 1) // self.block_size))

    def build_blockmask(self, stream=None):
        return ssa.spans_to_blockmask(self.span_offsets, self.spans, self.ctx_lens, self.block_size, self.block_idx,
                                      self.block_mask, self.block_counts, self.status, stream)

    def attend_blockmask(self, stream=None):
        return ssa.decode_attn_blockmask(self.desc, self.q, self.k, self.v, self.ctx_lens, self.block_idx,
                                         self.block_mask, self.block_counts, self.block_size, self.max_blocks,
                                         self.out, self.lse, self.workspace, self.status, stream)

    def step_blockmask(self, stream=None):
        self.build_blockmask(stream)
        self.attend_blockmask(stream)

    def step_two_calls(self, stream=None):
        """One decode step as two calls: span lists -> index lists -> attention."""
        self.build_index(stream)
        self.attend_sparse(stream)

    def step(self, stream=None, kernels="auto"):
        """One decode step of the method through ssa_decode_step with everything resident on the
        device: index lists, counts and the attention output are written.  kernels: "auto" (the
        library picks one kernel or index + attention launches), "one" or "two"."""
        self._lists_of_spans()
        key = ("resident", self.k.data_ptr(), self.max_selected, self.max_spans, kernels)
        st = self._steps.get(key)
        if st is None:
            st = ssa.make_step(self.span_offsets, self.spans, self.ctx_lens, self.index, self.counts, self.q, self.k,
                               self.v, self.max_selected, self.out, self.lse, self.workspace, self.status,
                               max_spans=self.max_spans, kernels=kernels)
            self._steps[key] = st
        return ssa.decode_step(self.desc, st, stream)

    # ---- host-buffer form (end-to-end timing) -----------------------------------------
    def make_host_buffers(self):
        """Pinned host copy of what changes every decode step (query rows,
        context lengths, span lists) and a pinned landing buffer for what the
        caller reads back (output rows, lse, counts, status word).
        Returns (host-to-device bytes, device-to-host bytes) per step."""
        self.h_in = self.in_arena.cpu().pin_memory()
        self.h_out = torch.empty(self.out_arena.shape, dtype=torch.uint8).pin_memory()
        self.h_out_rows, self.h_lse, self.h_counts, self.h_status = _views(self.h_out, self._out_specs)
        return self.h_in.numel(), self.h_out.numel()

    def step_from_host(self, stream=None, direct=False):
        """Decode step whose per-step inputs start in pinned host memory and
        whose result ends there (ssa_decode_step with both copies); the KV
        cache is the resident state.

        direct=False: one copy-engine transfer in, the kernels, one out.
        direct=True: the inputs are fetched by a kernel, the attention kernels
        store output rows and lse straight into the pinned landing buffer, and
        a kernel carries counts and the status word over
        (SSA_STEP_COPY_BY_KERNEL).  Same bytes, same result, less latency."""
        if not hasattr(self, "h_in"):
            raise RuntimeError("call make_host_buffers() before step_from_host()")
        self._lists_of_spans()
        key = ("host", self.k.data_ptr(), self.max_selected, self.max_spans, bool(direct))
        st = self._steps.get(key)
        if st is None:
            if direct:
                tail = self.counts.data_ptr() - self.out_arena.data_ptr()   # counts + status: kernels read them too
                st = ssa.make_step(self.span_offsets, self.spans, self.ctx_lens, self.index, self.counts, self.q,
                                   self.k, self.v, self.max_selected, self.h_out_rows, self.h_lse, self.workspace,
                                   self.status, host_in=self.h_in, dev_in=self.in_arena,
                                   host_out=self.h_out[tail:], dev_out=self.out_arena[tail:], copy_by_kernel=True,
                                   max_spans=self.max_spans)
            else:
                st = ssa.make_step(self.span_offsets, self.spans, self.ctx_lens, self.index, self.counts, self.q,
                                   self.k, self.v, self.max_selected, self.out, self.lse, self.workspace, self.status,
                                   host_in=self.h_in, dev_in=self.in_arena, host_out=self.h_out, dev_out=self.out_arena,
                                   max_spans=self.max_spans)
            self._steps[key] = st
        return ssa.decode_step(self.desc, st, stream)

    def set_spans(self, wl: Workload):
        """Replace the span lists (same geometry, same cache)."""
        assert (wl.B, wl.H, wl.D, wl.max_ctx) == (self.wl.B, self.wl.H, self.wl.D, self.wl.max_ctx)
        assert wl.spans.shape[0] <= self.spans.shape[0] and wl.selected_upper_bound() <= self.index_stride
        self.spans[: wl.spans.shape[0]].copy_(torch.from_numpy(np.ascontiguousarray(wl.spans)))
        self.span_offsets.copy_(torch.from_numpy(wl.span_offsets.copy()))
        self.ctx_lens.copy_(torch.from_numpy(wl.ctx_lens.copy()))
        self.max_selected = max(wl.selected_upper_bound(), 1)
        self.max_spans = int(max(1, np.diff(wl.span_offsets).max()))
        self.wl = wl
        if hasattr(self, "block_size"):
            self._bound_blocks()

    # ---- results ---------------------------------------------------------------------
    def out_f64(self) -> np.ndarray:
        return self.out.detach().to(torch.float64).cpu().numpy()

    def selected_bytes(self) -> int:
        return int(self.counts.clamp(min=0).sum().item()) * self.wl.kv_bytes_per_token()
