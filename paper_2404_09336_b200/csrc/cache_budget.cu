// Keeping a cache within a budget: which positions stay (ssa_mass_to_index) and moving their rows to the front
// (ssa_cache_compact).
#include <algorithm>

#include "ssa_common.cuh"

namespace ssa {

// ---- the positions that stay -----------------------------------------------------------------------------------------
// Of n positions the first `sinks` and the last `recent` stay, and of those between the `want` with the largest sums, ties to
// the lowest position.  Sums are compared as 32-bit keys of the same order (order_key); the key of the want-th largest is found
// in three digits from the top, each by a histogram of the keys that match the digits found.  Then every larger key stays and
// the first few equal ones, numbered by a prefix sum over (item, warp) counts.  Latency bounds it: a request is a few dozen KB.
constexpr int kBins = 2048;

__device__ __forceinline__ uint32_t order_key(float x) {
  if (x != x) return 0;                                    // NaN ranks below everything
  const uint32_t u = __float_as_uint(x == 0.f ? 0.f : x);  // -0 equals 0
  return (u & 0x80000000u) ? ~u : u | 0x80000000u;         // -inf is 0x007fffff: above NaN
}

struct KeepParams {
  const float* mass;
  const int32_t* ctx_lens;
  int32_t* index;
  int32_t* counts;
  uint32_t* status;
  int64_t mass_stride;
  int max_ctx, budget, sinks, recent, index_stride;
};

__device__ __forceinline__ int warp_inclusive(int x, int lane) {
#pragma unroll
  for (int o = 1; o < 32; o *= 2) {
    const int y = __shfl_up_sync(~0u, x, o);
    if (lane >= o) x += y;
  }
  return x;
}

__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %cluster_ctarank;" : "=r"(r));
  return r;
}
__device__ __forceinline__ void cluster_sync() {
  asm volatile("barrier.cluster.arrive.release.aligned;\nbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// A word of another block's shared memory.
__device__ __forceinline__ void store_to(const void* mine, uint32_t rank, uint32_t v) {
  uint32_t at = (uint32_t)__cvta_generic_to_shared(mine);
  asm volatile("mapa.shared::cluster.u32 %0, %0, %1;" : "+r"(at) : "r"(rank));
  asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(at), "r"(v) : "memory");
}
__device__ __forceinline__ uint32_t load_from(const void* mine, uint32_t rank) {
  uint32_t at = (uint32_t)__cvta_generic_to_shared(mine), v;
  asm volatile("mapa.shared::cluster.u32 %0, %0, %1;" : "+r"(at) : "r"(rank));
  asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(at) : "memory");
  return v;
}

// grid (blocks of a request, requests): kItems keys a thread, in registers: four neighbouring positions of each of the parts that a
// block has.  Several blocks of a request are a cluster; each adds up its share of all blocks' bins over distributed shared memory
// and hands the sums out.  kLong: more than a cluster's threads hold, keys are read anew each time.  Positions that are not
// ranked have key 0, the lowest, and are left out of the histograms; so are NaNs, and the lowest bin counts as one that never
// runs out.  What stays is put in order in shared memory and written from there.
template <int kThreads, int kItems, bool kLong>
__global__ void __launch_bounds__(kThreads)
mass_keep_kernel(const KeepParams p) {
  constexpr int kWarps = kThreads / 32, kOwn = kBins / kThreads, kParts = kItems / 4, kPart = 4 * kThreads;
  // One array: three digits' bins and, for clusters, all blocks' bins of the digit at hand; afterwards, over all of it, the
  // positions that stay, of which a block may have as many as it has items.
  __shared__ uint32_t s_mem[4 * kBins];
  uint32_t* const s_bins = s_mem;
  uint32_t* const s_all = s_mem + 3 * kBins;
  __shared__ uint32_t s_sum[kParts < 2 ? 2 : kParts][kWarps], s_total;
  static_assert(kLong || kItems * kThreads * sizeof(uint16_t) <= sizeof(s_mem), "");
  const int b = blockIdx.y, tid = threadIdx.x, lane = tid % 32, warp = tid / 32, blocks = gridDim.x;
  const int rank = blocks == 1 ? 0 : (int)cluster_rank();
  for (int i = tid; i < 3 * kBins; i += kThreads) s_bins[i] = 0;
  grid_dependency_wait();
  grid_launch_dependents();
  const float* mass = p.mass + (int64_t)b * p.mass_stride;
  const int block0 = rank * kItems * kThreads, j0 = block0 + tid * 4;
  auto place = [&](int i) { return j0 + i / 4 * kPart + i % 4; };
  uint32_t keys[kItems];                               // (asked for before it is known how long the context is)
  if constexpr (!kLong) {
    const bool wide = ((reinterpret_cast<uintptr_t>(mass) | (uintptr_t)p.max_ctx * 4) & 15) == 0;
#pragma unroll
    for (int i = 0; i < kItems; i += 4) {
      const int j = place(i);
      float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
      if (wide) {
        if (j < p.max_ctx) f = *reinterpret_cast<const float4*>(mass + j);
      } else {
        if (j < p.max_ctx) f.x = mass[j];
        if (j + 1 < p.max_ctx) f.y = mass[j + 1];
        if (j + 2 < p.max_ctx) f.z = mass[j + 2];
        if (j + 3 < p.max_ctx) f.w = mass[j + 3];
      }
      keys[i] = __float_as_uint(f.x); keys[i + 1] = __float_as_uint(f.y);
      keys[i + 2] = __float_as_uint(f.z); keys[i + 3] = __float_as_uint(f.w);
    }
  }
  int n = p.ctx_lens[b];
  if (n > p.max_ctx && tid == 0 && rank == 0 && p.status) atomicOr(p.status, SSA_DEV_BAD_COUNT);
  n = max(0, min(n, p.max_ctx));
  int32_t* index = p.index + (int64_t)b * p.index_stride;
  if (tid == 0 && rank == 0) p.counts[b] = min(n, p.budget);
  if (n <= p.budget) {
    for (int j = rank * kThreads + tid; j < n; j += blocks * kThreads) index[j] = j;
    return;
  }
  const int from = p.sinks, to = n - p.recent;             // those between are ranked
  int want = p.budget - p.sinks - p.recent;                // >= 0, and < to - from
  auto ranked = [&](int j) { return j >= from && j < to; };
  if constexpr (!kLong) {
#pragma unroll
    for (int i = 0; i < kItems; ++i) keys[i] = ranked(place(i)) ? order_key(__uint_as_float(keys[i])) : 0;
  }
  uint32_t key = 0, known = 0;                             // digits found so far, and their mask
  const bool none = want == 0;                             // the budget has no room for ranked positions
  if (blocks > 1) cluster_sync();                          // (every block has begun: its shared memory is there)
  else __syncthreads();
  if (!none) {
#pragma unroll 1
    for (int pass = 0; pass < 3; ++pass) {
      const int shift = pass == 0 ? 21 : pass == 1 ? 10 : 0;
      const uint32_t digits = pass == 2 ? 1023u : 2047u;
      uint32_t* const bins = s_bins + pass * kBins;
      // Sums are often all alike (nothing looked at yet): a warp whose first keys share the digit adds once for all that do.
      const uint32_t sample = kLong ? 0 : keys[0] >> shift & digits;
      const bool alike = kLong || __all_sync(~0u, sample == __shfl_sync(~0u, sample, 0));
      auto add = [&](uint32_t k) {
        const bool on = k != 0 && (k & known) == key;
        const uint32_t digit = k >> shift & digits;
        if (!alike) {
          if (on) atomicAdd(&bins[digit], 1u);
          return;
        }
        const unsigned votes = __ballot_sync(~0u, on);
        if (votes == 0) return;
        const uint32_t one = __shfl_sync(~0u, digit, __ffs(votes) - 1);
        if (__ballot_sync(~0u, on && digit == one) == votes) {
          if (lane == 0) atomicAdd(&bins[one], (uint32_t)__popc(votes));
        } else if (on) {
          atomicAdd(&bins[digit], 1u);
        }
      };
      if constexpr (kLong) {
        for (int j = from + tid; j - lane < to; j += kThreads) add(ranked(j) ? order_key(mass[j]) : 0);
      } else {
#pragma unroll
        for (int i = 0; i < kItems; ++i) add(keys[i]);
      }
      const uint32_t* all = bins;
      if (blocks == 1) {
        __syncthreads();
      } else {
        cluster_sync();
        const int share = kBins / blocks;
        for (int i = tid; i < share; i += kThreads) {
          uint32_t sum = 0;
#pragma unroll
          for (int r = 0; r < 8; ++r)
            if (r < blocks) sum += load_from(&bins[rank * share + i], r);
          for (int r = 0; r < blocks; ++r) store_to(&s_all[rank * share + i], r, sum);
        }
        cluster_sync();
        all = s_all;
      }
      // A warp sums its share of the bins, from the top; then every warp finds the share in which the count reaches `want`, and
      // the bin.
      uint32_t mine = 0;
#pragma unroll
      for (int i = 0; i < kOwn; ++i) mine += all[kBins - 1 - (i * 32 + warp * 32 * kOwn + lane)];
      const uint32_t sum = __reduce_add_sync(~0u, mine);
      if (lane == 0) s_sum[pass & 1][warp] = sum;
      __syncthreads();
      const int upto = warp_inclusive(lane < kWarps ? (int)s_sum[pass & 1][lane] : 0, lane);
      const unsigned reached = __ballot_sync(~0u, upto >= want) | 1u << (kWarps - 1);   // (the last bin never runs out)
      const int at = __ffs(reached) - 1;
      int above = at ? __shfl_sync(~0u, upto, at - 1) : 0;
      const int first = kBins - 1 - at * 32 * kOwn - lane * kOwn;      // bins first, first - 1, ... are this lane's
      int here = 0;
#pragma unroll
      for (int i = 0; i < kOwn; ++i) here += (int)all[first - i];
      const int end = above + warp_inclusive(here, lane);
      const int who = __ffs(__ballot_sync(~0u, end >= want) | 1u << 31) - 1;
      above = end - here;
      int digit = first, left = want - above;              // (of the lane in question: the last of its bins never runs out either)
      bool found = false;
#pragma unroll
      for (int i = 0; i < kOwn; ++i) {
        if (!found) { digit = first - i; left = want - above; }
        above += (int)all[first - i];
        found |= above >= want;
      }
      digit = __shfl_sync(~0u, digit, who);
      want = __shfl_sync(~0u, left, who);
      key |= (uint32_t)digit << shift;
      known |= digits << shift;
      if (key == 0) break;                                 // the rest are NaNs
    }
  }
  // `want` of the keys equal to `key` stay
  auto larger = [&](int j, uint32_t k) { return j < n && (!ranked(j) || (!none && k > key)); };
  auto equals = [&](int j, uint32_t k) { return ranked(j) && !none && k == key; };
  if constexpr (kLong) {
    int kept = 0, equal = 0;                               // before this step's positions
    __syncthreads();
    for (int at = 0; at < n; at += kThreads) {
      const int j = at + tid;
      const uint32_t k = ranked(j) ? order_key(mass[j]) : 0;
      const unsigned more = __ballot_sync(~0u, larger(j, k)), same = __ballot_sync(~0u, equals(j, k)), below = (1u << lane) - 1;
      if (lane == 0) s_sum[0][warp] = (uint32_t)__popc(more) | (uint32_t)__popc(same) << 16;
      __syncthreads();
      const uint32_t upto = (uint32_t)warp_inclusive((int)s_sum[0][lane], lane), before = warp ? __shfl_sync(~0u, upto, warp - 1) : 0;
      const uint32_t sums = __shfl_sync(~0u, upto, 31);
      const int more_before = kept + (int)(before & 0xffffu) + __popc(more & below);
      const int same_before = equal + (int)(before >> 16) + __popc(same & below);
      if (larger(j, k) || (equals(j, k) && same_before < want)) index[more_before + min(same_before, want)] = j;
      kept += (int)(sums & 0xffffu);
      equal += (int)(sums >> 16);
      __syncthreads();
    }
  } else {
    // larger keys, and equal ones from bit 16 on (a block has 2^14 positions at most), counted in order: part, thread, neighbour
    uint32_t more = 0, same = 0;                           // bits of this thread's items
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      more |= (uint32_t)larger(place(i), keys[i]) << i;
      same |= (uint32_t)equals(place(i), keys[i]) << i;
    }
    uint32_t before[kParts];
    __syncthreads();                                       // (the last digit's sums and bins have been read)
#pragma unroll
    for (int q = 0; q < kParts; ++q) {
      const uint32_t count = (uint32_t)__popc(more >> 4 * q & 15u) | (uint32_t)__popc(same >> 4 * q & 15u) << 16;
      const uint32_t upto = (uint32_t)warp_inclusive((int)count, lane);
      before[q] = upto - count;
      if (lane == 31) s_sum[q][warp] = upto;
    }
    __syncthreads();
    uint32_t total = 0;
#pragma unroll
    for (int q = 0; q < kParts; ++q) {
      const uint32_t upto = (uint32_t)warp_inclusive(lane < kWarps ? (int)s_sum[q][lane] : 0, lane);
      before[q] += total + (warp ? __shfl_sync(~0u, upto, warp - 1) : 0);
      total += __shfl_sync(~0u, upto, kWarps - 1);
    }
    int kept = 0, equal = 0;                               // in the blocks before this one
    if (blocks > 1) {
      if (tid == 0) s_total = total;
      cluster_sync();
#pragma unroll
      for (int r = 0; r < 8; ++r)
        if (r < rank) {
          const uint32_t theirs = load_from(&s_total, r);
          kept += (int)(theirs & 0xffffu);
          equal += (int)(theirs >> 16);
        }
      cluster_sync();                                      // (totals are read by the others until here)
    }
    const int room = max(0, want - equal);                 // equal keys of this block that stay
    uint16_t* const list = reinterpret_cast<uint16_t*>(s_mem);       // positions within the block
#pragma unroll
    for (int i = 0; i < kItems; ++i) {
      uint32_t& at = before[i / 4];                          // counts so far
      const int equals_before = (int)(at >> 16);
      const bool is_more = more >> i & 1, is_same = same >> i & 1;
      if (is_more || (is_same && equals_before < room)) list[(int)(at & 0xffffu) + min(equals_before, room)] = (uint16_t)(place(i) - block0);
      at += is_more ? 1u : is_same ? 1u << 16 : 0u;
    }
    __syncthreads();
    const int stay = (int)(total & 0xffffu) + min((int)(total >> 16), room), first = kept + min(equal, want);
    for (int i = tid; i < stay; i += kThreads) index[first + i] = block0 + list[i];
  }
}

// A request's blocks as one cluster.
template <typename... KArgs, typename... Args>
static cudaError_t launch_cluster(void (*kernel)(KArgs...), dim3 grid, dim3 block, cudaStream_t stream, Args... args) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = block;
  cfg.stream = stream;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = grid.x;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 2;
  return cudaLaunchKernelEx(&cfg, kernel, args...);
}

// Few positions take few threads, whose barriers are short (512 positions: 256 threads of 4 items 4.6 us, of 16 items 7.5); a block
// has up to 1024 x 16, a cluster eight times that.
static cudaError_t launch_keep(const KeepParams& p, int B, cudaStream_t st) {
  constexpr int kBlock = 1024 * 16, kMost = 8;             // blocks of a cluster that every GPU takes
  if (p.max_ctx <= 256 * 4) return launch_pdl(mass_keep_kernel<256, 4, false>, dim3(1, (unsigned)B), dim3(256), st, p);
  if (p.max_ctx <= 1024 * 4) return launch_pdl(mass_keep_kernel<1024, 4, false>, dim3(1, (unsigned)B), dim3(1024), st, p);
  if (p.max_ctx <= kBlock) return launch_pdl(mass_keep_kernel<1024, 16, false>, dim3(1, (unsigned)B), dim3(1024), st, p);
  if (p.max_ctx > kMost * kBlock) return launch_pdl(mass_keep_kernel<1024, 16, true>, dim3(1, (unsigned)B), dim3(1024), st, p);
  const unsigned blocks = p.max_ctx <= 2 * kBlock ? 2 : p.max_ctx <= 4 * kBlock ? 4 : 8;
  return launch_cluster(mass_keep_kernel<1024, 16, false>, dim3(blocks, (unsigned)B), dim3(1024), st, p);
}

// ---- moving their rows ----------------------------------------------------------------------------------------------
// Row index[i] of a request goes to row i.  Lists ascend, so index[i] >= i: a row's place is at or before where it comes from,
// and what a block writes in its step was read in this step or an earlier one.  A block owns a column of bytes of one head of K
// or V and goes through the list in order: loads of a step, barrier, stores.  Columns never meet, so blocks need not wait for
// one another.
constexpr int kMoveThreads = 256;
constexpr int kMoveSteps = 2;          // rows of a step, per thread (4: 85 registers, 250 us instead of 175 for the 8 requests below)

struct MoveParams {
  char *k, *v;
  float* mass;
  const int32_t *ctx_lens, *index, *counts, *page_table;
  uint32_t* status;
  int64_t k_sb, k_sh, k_st, v_sb, v_sh, v_st, mass_stride;     // bytes (mass: elements)
  int H_kv, row_bytes, max_ctx, index_stride, max_selected, page_table_stride, page_shift, n_pages, paged;
};

__device__ __forceinline__ int64_t move_row(const MoveParams& p, const int32_t* table, int j) {
  if (!p.paged) return j;
  const int page = table[j >> p.page_shift];
  if ((unsigned)page >= (unsigned)p.n_pages) return -1;
  return ((int64_t)page << p.page_shift) + (j & ((1 << p.page_shift) - 1));
}

__global__ void __launch_bounds__(kMoveThreads)
cache_move_kernel(const MoveParams p, const int column_bytes) {
  grid_dependency_wait();
  grid_launch_dependents();
  const int b = blockIdx.z, tid = threadIdx.x;
  const int parts = p.row_bytes / column_bytes;
  const bool sums = blockIdx.y == 2;                       // the sums: one block
  if (sums && (blockIdx.x != 0 || !p.mass)) return;
  const int h = blockIdx.x / parts, part = blockIdx.x % parts;
  int ctx = p.ctx_lens[b], n = p.counts[b];
  uint32_t flags = 0;
  if (ctx > p.max_ctx || n > p.max_selected || n > ctx) flags |= SSA_DEV_BAD_COUNT;
  ctx = max(0, min(ctx, p.max_ctx));
  n = max(0, min(n, min(p.max_selected, ctx)));            // (no more rows than there are: every place is inside the cache)
  const int32_t* index = p.index + (int64_t)b * p.index_stride;
  const int32_t* table = p.paged ? p.page_table + (int64_t)b * p.page_table_stride : nullptr;
  if (sums) {
    float* mass = p.mass + (int64_t)b * p.mass_stride;
    for (int i0 = 0; i0 < n; i0 += kMoveThreads) {
      const int i = i0 + tid, j = i < n ? index[i] : -1;
      const bool ok = i < n && j >= 0 && j < ctx;
      const float x = ok ? mass[j] : 0.f;
      __syncthreads();
      if (ok) mass[i] = x;
    }
    return;
  }
  const bool is_v = blockIdx.y == 1;
  char* base = (is_v ? p.v : p.k) + (is_v ? p.v_sh : p.k_sh) * h + (p.paged ? 0 : (is_v ? p.v_sb : p.k_sb) * b) + part * column_bytes;
  const int64_t st = is_v ? p.v_st : p.k_st;
  const int lanes = column_bytes / 16, rows = kMoveThreads / lanes;   // threads of a row, rows of a pass
  const int lane = tid % lanes, r = tid / lanes;
  uint4 x[2][kMoveSteps];
  int list[kMoveSteps];                                    // the next step's entries; -1: none
  auto ask = [&](int i0) {
#pragma unroll
    for (int s = 0; s < kMoveSteps; ++s) {
      const int i = i0 + s * rows + r;
      list[s] = i < n ? index[i] : -1;
      if (i < n && (list[s] < 0 || list[s] >= ctx)) { flags |= SSA_DEV_BAD_INDEX; list[s] = -1; }
    }
  };
  int to[2][kMoveSteps];                                   // rows; -1: nothing to move
  auto load = [&](int i0, uint4 (&x)[kMoveSteps], int (&to)[kMoveSteps]) {
#pragma unroll
    for (int s = 0; s < kMoveSteps; ++s) {
      const int i = i0 + s * rows + r;
      to[s] = -1;
      if (list[s] < 0 || list[s] == i) continue;
      const int64_t from = move_row(p, table, list[s]), at = move_row(p, table, i);
      if (from < 0 || at < 0) { flags |= SSA_DEV_BAD_INDEX; continue; }
      x[s] = *reinterpret_cast<const uint4*>(base + from * st + lane * 16);
      to[s] = (int)at;
    }
  };
  // A step's loads are asked for while the step before it is stored: what they read lies behind everything stored so far and in
  // that step, for a list that ascends.
  const int step = rows * kMoveSteps;
  auto turn = [&](int i0, uint4 (&now)[kMoveSteps], int (&now_to)[kMoveSteps], uint4 (&next)[kMoveSteps], int (&next_to)[kMoveSteps]) {
    load(i0 + step, next, next_to);
    ask(i0 + 2 * step);
    __syncthreads();                                       // every thread has this step's rows
#pragma unroll
    for (int s = 0; s < kMoveSteps; ++s)
      if (now_to[s] >= 0) *reinterpret_cast<uint4*>(base + now_to[s] * st + lane * 16) = now[s];
  };
  ask(0);
  load(0, x[0], to[0]);
  ask(step);
  for (int i0 = 0; i0 < n; i0 += 2 * step) {
    turn(i0, x[0], to[0], x[1], to[1]);
    turn(i0 + step, x[1], to[1], x[0], to[0]);
  }
  if (flags && p.status) atomicOr(p.status, flags);
}

}  // namespace ssa

extern "C" {

int32_t ssa_mass_to_index(const float* mass, int64_t mass_stride, const int32_t* ctx_lens, int32_t B, int32_t max_ctx,
                          int32_t budget, int32_t sinks, int32_t recent, int32_t* index, int32_t index_stride,
                          int32_t* counts, uint32_t* dev_status, void* stream) {
  if (!mass || !ctx_lens || !index || !counts) return SSA_ERR_NULL;
  if (B <= 0 || B > 65535 || max_ctx <= 0 || max_ctx > ssa::kMostContext || index_stride <= 0 || mass_stride < max_ctx) return SSA_ERR_SHAPE;
  if (budget <= 0 || sinks < 0 || recent < 0 || (int64_t)sinks + recent > budget || budget > index_stride) return SSA_ERR_CAPACITY;
  const ssa::KeepParams p = {mass, ctx_lens, index, counts, dev_status, mass_stride, max_ctx, budget, sinks, recent, index_stride};
  if (ssa::launch_keep(p, B, (cudaStream_t)stream) != cudaSuccess) return SSA_ERR_CUDA;
  ssa::note_launches(1);
  return SSA_OK;
}

int32_t ssa_cache_compact(const ssa_attn_desc* desc, const ssa_paging* paging, void* k_cache, void* v_cache,
                          const int32_t* ctx_lens, const int32_t* index, int32_t index_stride, const int32_t* counts,
                          int32_t max_selected, float* mass, int64_t mass_stride, uint32_t* dev_status, void* stream) {
  if (!desc || !k_cache || !v_cache || !ctx_lens || !index || !counts) return SSA_ERR_NULL;
  int32_t rc = ssa::check_desc(desc);
  if (rc == SSA_OK && paging) rc = ssa::check_paging(paging, desc->max_ctx);
  if (rc != SSA_OK) return rc;
  if (desc->max_ctx > ssa::kMostContext || (mass && mass_stride < desc->max_ctx)) return SSA_ERR_SHAPE;
  // rows that several heads or requests share, or that K and V do, would be moved more than once
  if (k_cache == v_cache || desc->k_stride_t == 0 || desc->v_stride_t == 0 ||
      (desc->H_kv > 1 && (desc->k_stride_h == 0 || desc->v_stride_h == 0)) ||
      (desc->B > 1 && !paging && (desc->k_stride_b == 0 || desc->v_stride_b == 0)))
    return SSA_ERR_UNSUPPORTED;
  if (index_stride <= 0 || max_selected <= 0 || max_selected > index_stride) return SSA_ERR_CAPACITY;
  if (!ssa::aligned16(k_cache) || !ssa::aligned16(v_cache)) return SSA_ERR_ALIGN;
  const int E = desc->kv_dtype == SSA_FP8_E4M3 ? 1 : 2;
  ssa::MoveParams p = {};
  p.k = static_cast<char*>(k_cache);
  p.v = static_cast<char*>(v_cache);
  p.mass = mass;
  p.ctx_lens = ctx_lens; p.index = index; p.counts = counts;
  p.page_table = paging ? paging->page_table : nullptr;
  p.status = dev_status;
  p.k_sb = desc->k_stride_b * E; p.k_sh = desc->k_stride_h * E; p.k_st = desc->k_stride_t * E;
  p.v_sb = desc->v_stride_b * E; p.v_sh = desc->v_stride_h * E; p.v_st = desc->v_stride_t * E;
  p.mass_stride = mass_stride;
  p.H_kv = desc->H_kv;
  p.row_bytes = desc->D * E;
  p.max_ctx = desc->max_ctx;
  p.index_stride = index_stride;
  p.max_selected = max_selected;
  p.page_table_stride = paging ? paging->page_table_stride : 0;
  p.n_pages = paging ? paging->n_pages : 0;
  while (paging && (1 << p.page_shift) < paging->page_size) ++p.page_shift;
  p.paged = paging != nullptr;
  // Whole rows where the heads of all requests make enough blocks, else narrower columns, down to a sector: 8 requests, 32 heads,
  // 256-byte rows 175 us whole, 181 in columns of 64 bytes; 2 requests, 8 heads 64 and 23 us.
  int column = p.row_bytes;
  while (column > 32 && 2ll * desc->B * desc->H_kv * (p.row_bytes / column) < 3ll * ssa::sm_count()) column /= 2;
  const dim3 grid((unsigned)(desc->H_kv * (p.row_bytes / column)), 3, (unsigned)desc->B);
  if (ssa::launch_pdl(ssa::cache_move_kernel, grid, dim3(ssa::kMoveThreads), (cudaStream_t)stream, p, column) != cudaSuccess)
    return SSA_ERR_CUDA;
  ssa::note_launches(1);
  return SSA_OK;
}

}  // extern "C"
