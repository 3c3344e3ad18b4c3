// Keeping a cache within a budget: which positions stay (ssa_mass_to_index) and moving their rows to the front
// (ssa_cache_compact).
#include <algorithm>

#include "ssa_common.cuh"

namespace ssa {

// ---- the positions that stay -----------------------------------------------------------------------------------------
// Of n positions the first `sinks` and the last `recent` stay, and of those between the `want` with the largest sums, ties to
// the lowest position.  Sums are compared as 32-bit keys of the same order (order_key); the key of the want-th largest is
// found digit by digit from the top (a histogram per digit of those that match the digits found), then one pass numbers what
// stays: every larger key, and the first few equal ones.
constexpr int kKeepThreads = 1024;
constexpr int kKeepWarps = kKeepThreads / 32;

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

__global__ void __launch_bounds__(kKeepThreads)
mass_keep_kernel(const KeepParams p) {
  __shared__ uint32_t s_count[256];
  __shared__ int s_warp[2][kKeepWarps], s_digit, s_left;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
  grid_dependency_wait();
  grid_launch_dependents();
  int n = p.ctx_lens[b];
  if (n > p.max_ctx && tid == 0 && p.status) atomicOr(p.status, SSA_DEV_BAD_COUNT);
  n = max(0, min(n, p.max_ctx));
  const float* mass = p.mass + (int64_t)b * p.mass_stride;
  int32_t* index = p.index + (int64_t)b * p.index_stride;
  const int keep = min(n, p.budget);
  if (tid == 0) p.counts[b] = keep;
  if (n <= p.budget) {
    for (int j = tid; j < n; j += kKeepThreads) index[j] = j;
    return;
  }
  const int from = p.sinks, to = n - p.recent;             // those between are ranked
  int want = p.budget - p.sinks - p.recent;                // >= 0, and < to - from
  uint32_t key = 0, known = 0;                             // digits found so far, and their mask
  for (int shift = 24; shift >= 0; shift -= 8) {
    for (int i = tid; i < 256; i += kKeepThreads) s_count[i] = 0;
    __syncthreads();
    for (int j = from + tid; j < to; j += kKeepThreads) {
      const uint32_t k = order_key(mass[j]);
      if ((k & known) == key) atomicAdd(&s_count[(k >> shift) & 255], 1u);
    }
    __syncthreads();
    if (warp == 0) {                                       // the digit at which the count from the top reaches `want`
      int mine[8], sum = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) sum += mine[i] = (int)s_count[255 - (lane * 8 + i)];
      int above = warp_inclusive(sum, lane) - sum;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (above < want && above + mine[i] >= want) { s_digit = 255 - (lane * 8 + i); s_left = want - above; }
        above += mine[i];
      }
      if (want == 0 && lane == 0) { s_digit = 255; s_left = 0; }
    }
    __syncthreads();
    key |= (uint32_t)s_digit << shift;
    known |= 255u << shift;
    want = s_left;
    __syncthreads();
  }
  // `want` of the keys equal to `key` stay (none where the budget has no room for ranked positions: key is all ones then)
  int kept = 0, equal = 0;                                 // before this step's positions
  for (int j0 = 0; j0 < n; j0 += kKeepThreads) {
    const int j = j0 + tid;
    const bool ranked = j >= from && j < to;
    const uint32_t k = ranked ? order_key(mass[j]) : 0;
    const bool same = ranked && k == key;
    const unsigned votes = __ballot_sync(~0u, same);
    if (lane == 0) s_warp[0][warp] = __popc(votes);
    __syncthreads();
    const int eq_before = warp_inclusive(s_warp[0][lane], lane) - s_warp[0][lane];
    const int eq_total = __shfl_sync(~0u, eq_before + s_warp[0][lane], 31);
    const int rank = equal + __shfl_sync(~0u, eq_before, warp) + __popc(votes & ((1u << lane) - 1));
    const bool stays = j < n && (!ranked || k > key || (same && rank < want));
    const unsigned staying = __ballot_sync(~0u, stays);
    if (lane == 0) s_warp[1][warp] = __popc(staying);
    __syncthreads();
    const int st_before = warp_inclusive(s_warp[1][lane], lane) - s_warp[1][lane];
    const int st_total = __shfl_sync(~0u, st_before + s_warp[1][lane], 31);
    const int at = kept + __shfl_sync(~0u, st_before, warp) + __popc(staying & ((1u << lane) - 1));
    if (stays) index[at] = j;
    kept += st_total;
    equal += eq_total;
  }
}

// ---- moving their rows ----------------------------------------------------------------------------------------------
// Row index[i] of a request goes to row i.  Lists ascend, so index[i] >= i: a row's place is at or before where it comes from,
// and what a block writes in its step was read in this step or an earlier one.  A block owns one 64-byte-wide column group of
// one head of K or V and goes through the list in order: loads of a step, barrier, stores.  Columns never meet, so blocks need
// not wait for one another.
constexpr int kMoveThreads = 256;
constexpr int kMoveSteps = 4;          // rows that a thread has in flight

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
  for (int i0 = 0; i0 < n; i0 += rows * kMoveSteps) {
    uint4 x[kMoveSteps];
    char* to[kMoveSteps];
#pragma unroll
    for (int s = 0; s < kMoveSteps; ++s) {
      const int i = i0 + s * rows + r;
      to[s] = nullptr;
      if (i >= n) continue;
      const int j = index[i];
      if (j < 0 || j >= ctx) { flags |= SSA_DEV_BAD_INDEX; continue; }
      if (j == i) continue;
      const int64_t from = move_row(p, table, j), at = move_row(p, table, i);
      if (from < 0 || at < 0) { flags |= SSA_DEV_BAD_INDEX; continue; }
      x[s] = *reinterpret_cast<const uint4*>(base + from * st + lane * 16);
      to[s] = base + at * st + lane * 16;
    }
    __syncthreads();
#pragma unroll
    for (int s = 0; s < kMoveSteps; ++s)
      if (to[s]) *reinterpret_cast<uint4*>(to[s]) = x[s];
  }
  if (flags && p.status) atomicOr(p.status, flags);
}

}  // namespace ssa

extern "C" {

int32_t ssa_mass_to_index(const float* mass, int64_t mass_stride, const int32_t* ctx_lens, int32_t B, int32_t max_ctx,
                          int32_t budget, int32_t sinks, int32_t recent, int32_t* index, int32_t index_stride,
                          int32_t* counts, uint32_t* dev_status, void* stream) {
  if (!mass || !ctx_lens || !index || !counts) return SSA_ERR_NULL;
  if (B <= 0 || B > 65535 || max_ctx <= 0 || index_stride <= 0 || mass_stride < max_ctx) return SSA_ERR_SHAPE;
  if (budget <= 0 || sinks < 0 || recent < 0 || (int64_t)sinks + recent > budget || budget > index_stride) return SSA_ERR_CAPACITY;
  const ssa::KeepParams p = {mass, ctx_lens, index, counts, dev_status, mass_stride, max_ctx, budget, sinks, recent, index_stride};
  if (ssa::launch_pdl(ssa::mass_keep_kernel, dim3((unsigned)B), dim3(ssa::kKeepThreads), (cudaStream_t)stream, p) != cudaSuccess)
    return SSA_ERR_CUDA;
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
  if (mass && mass_stride < desc->max_ctx) return SSA_ERR_SHAPE;
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
  const int column = 64;
  const dim3 grid((unsigned)(desc->H_kv * (p.row_bytes / column)), 3, (unsigned)desc->B);
  if (ssa::launch_pdl(ssa::cache_move_kernel, grid, dim3(ssa::kMoveThreads), (cudaStream_t)stream, p, column) != cudaSuccess)
    return SSA_ERR_CUDA;
  ssa::note_launches(1);
  return SSA_OK;
}

}  // extern "C"
