// Blocks of positions that a token's own queries select: what is kept of the keys of a block (ssa_block_bounds) and the blocks
// that it ranks first (ssa_block_select).
//
//   min_j, max_j   per dimension, over the keys of block j
//   score_j = sum_h sum_d max(q_hd min_jd, q_hd max_jd) = sum_d N_d min_jd + P_d max_jd,  N_d = sum_h min(q_hd, 0), P_d likewise
// so that the heads of a group cost no more than one.  (With infinite bounds too, as long as nothing times an infinity is nothing.)
#include <algorithm>
#include <type_traits>

#include "ranking.cuh"
#include "window.cuh"

namespace ssa {

// ---- bounds -----------------------------------------------------------------------------------------------------------
constexpr int kBoundThreads = 128;

struct BoundsParams {
  const char* k;
  const uint8_t* k_scales;
  const int32_t *ctx_lens, *q_lens, *page_table;
  void* bounds;
  uint32_t* status;
  int64_t k_sb, k_sh, k_st, bounds_sb, bounds_sh;            // values, elements
  int n_q, max_ctx, block_shift, page_table_stride, page_shift, n_pages;
};

// Pairs of 16-bit values, NaN where one of them is.
__device__ __forceinline__ __half2 least(__half2 a, __half2 b) { return __hmin2_nan(a, b); }
__device__ __forceinline__ __half2 most(__half2 a, __half2 b) { return __hmax2_nan(a, b); }
__device__ __forceinline__ __nv_bfloat162 least(__nv_bfloat162 a, __nv_bfloat162 b) { return __hmin2_nan(a, b); }
__device__ __forceinline__ __nv_bfloat162 most(__nv_bfloat162 a, __nv_bfloat162 b) { return __hmax2_nan(a, b); }
template <typename P> __device__ __forceinline__ P from_bits(uint32_t w) { return *reinterpret_cast<const P*>(&w); }
template <typename P> __device__ __forceinline__ uint32_t to_bits(P x) { return *reinterpret_cast<const uint32_t*>(&x); }

// grid (blocks of positions, H_kv, B).  Lanes take 16-byte pieces of rows, the thread block's rows at a time, keep the least and the
// largest of their piece, and meet at the end.  8- and 4-bit values become fp16 on the way, which holds them exactly.  Bound by HBM
// over whole contexts (8 requests of 9000 to 16384 positions, 8 heads: 33 to 34 us, 5.7 to 5.9 TB/s), over 8- and 4-bit ones, 27 and 36 us, by the conversions and comparisons; one round trip for a
// step's newest blocks.
template <typename T, int D, bool kPaged>
__global__ void __launch_bounds__(kBoundThreads)
block_bounds_kernel(const BoundsParams p) {
  using TQ = typename Storage<T>::Query;
  using Pair = std::conditional_t<std::is_same<T, __nv_bfloat16>::value, __nv_bfloat162, __half2>;
  constexpr int kBits = kIsFp4<T> ? 4 : kIsFp8<T> ? 8 : 16, kN = 128 / kBits;        // values of a piece
  constexpr int kLanes = D / kN, kRows = kBoundThreads / kLanes, kWarps = kBoundThreads / 32;
  __shared__ uint32_t s_part[kWarps][2][D / 2];
  grid_dependency_wait();
  grid_launch_dependents();
  const int b = blockIdx.z, hkv = blockIdx.y, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int piece = threadIdx.x % kLanes, slot = threadIdx.x / kLanes;
  uint32_t flags = 0;
  int ctx, n_new;
  window_sizes(p, b, ctx, n_new, flags);
  const int j = (max(0, ctx - n_new) >> p.block_shift) + (int)blockIdx.x;
  if (flags && p.status && blockIdx.x == 0 && hkv == 0 && threadIdx.x == 0) atomicOr(p.status, flags);
  const int j0 = j << p.block_shift, jz = min(ctx, j0 + (1 << p.block_shift));
  if (n_new == 0 || j0 >= ctx) return;
  const int32_t* table = kPaged ? p.page_table + (int64_t)b * p.page_table_stride : nullptr;
  const int64_t o0 = (kPaged ? 0 : (int64_t)b * p.k_sb) + (int64_t)hkv * p.k_sh + piece * kN;
  const Pair none_least = from_bits<Pair>(std::is_same<Pair, __half2>::value ? 0x7c007c00u : 0x7f807f80u);
  const Pair none_most = from_bits<Pair>(std::is_same<Pair, __half2>::value ? 0xfc00fc00u : 0xff80ff80u);
  Pair lo[kN / 2], hi[kN / 2];
#pragma unroll
  for (int i = 0; i < kN / 2; ++i) { lo[i] = none_least; hi[i] = none_most; }
#pragma unroll 4
  for (int at = j0 + slot; at < jz; at += kRows) {
    const int64_t row = row_of<kPaged>(p, table, at);
    if (row < 0) { flags |= SSA_DEV_BAD_INDEX; continue; }
    const int64_t o = o0 + row * p.k_st;
    const uint4 w4 = ld_stream_16B(p.k + (kIsFp4<T> ? o / 2 : o * (kBits / 8)));
    const uint32_t w[4] = {w4.x, w4.y, w4.z, w4.w};
    uint32_t x[kN / 2];
    if constexpr (kIsFp4<T>) {
      const uint32_t pair = e4m3x2_to_half2(*reinterpret_cast<const uint16_t*>(p.k_scales + o / kScaleDims));
      const uint32_t by[2] = {__byte_perm(pair, 0, 0x1010), __byte_perm(pair, 0, 0x3232)};
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        uint32_t h[4];
        e2m1x8_to_half2(w[i], h);
#pragma unroll
        for (int e = 0; e < 4; ++e) x[4 * i + e] = half2_mul(h[e], by[i / 2]);
      }
    } else if constexpr (kIsFp8<T>) {
#pragma unroll
      for (int i = 0; i < 8; ++i) x[i] = e4m3x2_to_half2(w[i / 2] >> i % 2 * 16 & 0xffffu);
    } else {
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = w[i];
    }
#pragma unroll
    for (int i = 0; i < kN / 2; ++i) { lo[i] = least(lo[i], from_bits<Pair>(x[i])); hi[i] = most(hi[i], from_bits<Pair>(x[i])); }
  }
#pragma unroll
  for (int i = 0; i < kN / 2; ++i) {
#pragma unroll
    for (int o = kLanes; o < 32; o *= 2) {
      lo[i] = least(lo[i], from_bits<Pair>(__shfl_xor_sync(~0u, to_bits(lo[i]), o)));
      hi[i] = most(hi[i], from_bits<Pair>(__shfl_xor_sync(~0u, to_bits(hi[i]), o)));
    }
    if (lane < kLanes) {
      s_part[warp][0][piece * (kN / 2) + i] = to_bits(lo[i]);
      s_part[warp][1][piece * (kN / 2) + i] = to_bits(hi[i]);
    }
  }
  if (kPaged && p.status && (flags & SSA_DEV_BAD_INDEX)) atomicOr(p.status, SSA_DEV_BAD_INDEX);
  __syncthreads();
  if (threadIdx.x >= D) return;                              // D / 2 pairs of the least, D / 2 of the largest
  const int is_most = threadIdx.x / (D / 2), i = threadIdx.x % (D / 2);
  Pair x = from_bits<Pair>(s_part[0][is_most][i]);
#pragma unroll
  for (int y = 1; y < kWarps; ++y) {
    const Pair z = from_bits<Pair>(s_part[y][is_most][i]);
    x = is_most ? most(x, z) : least(x, z);
  }
  uint32_t bits = to_bits(x);
  if constexpr (kIsNarrow<T>) {
    const float2 f = unpack2<__half>(bits);
    bits = to_bits(__floats2bfloat162_rn(f.x, f.y));         // (exact: four significant bits, or six)
  }
  TQ* to = static_cast<TQ*>(p.bounds) + (int64_t)b * p.bounds_sb + (int64_t)hkv * p.bounds_sh + (int64_t)j * 2 * D;
  reinterpret_cast<uint32_t*>(to)[threadIdx.x] = bits;
}

// ---- selection ----------------------------------------------------------------------------------------------------------
constexpr int kSelectThreads = 256, kSelectWarps = kSelectThreads / 32;
constexpr int kDeep = 8;               // 16-byte pieces that a lane asks for at a time, of as many blocks of positions

struct SelectParams {
  const void *q, *bounds;
  const int32_t *ctx_lens, *q_lens;
  int32_t *index, *counts;
  float* scores;
  uint32_t* status;
  int64_t q_sb, q_sh, q_st, bounds_sb, bounds_sh;
  int H_kv, group, n_q, max_ctx, block_shift, n_blocks, budget, sinks, recent;
};

// Sums of v[i] over the kLanes lanes of a block's bounds, eight blocks together: each exchange halves what a lane has left.  The lane
// ends up with the sum of block `which`, or (the last lanes' bits) one that another has too.
template <int kLanes>
__device__ __forceinline__ double sums_of(double (&v)[kDeep], int lane, int& which) {
  which = 0;
  int o = kLanes / 2;
#pragma unroll
  for (int left = kDeep / 2; left >= 1; left /= 2, o /= 2) {
    const bool high = lane & o;
    which = 2 * which + high;
#pragma unroll
    for (int i = 0; i < left; ++i) {
      const double mine = high ? v[i + left] : v[i], theirs = high ? v[i] : v[i + left];
      v[i] = mine + __shfl_xor_sync(~0u, theirs, o);
    }
  }
#pragma unroll
  for (; o >= 1; o /= 2) v[0] += __shfl_xor_sync(~0u, v[0], o);
  return v[0];
}

// grid (ranks x tokens, H_kv, B).  Thread blocks share a token's blocks of positions out; the first of them gets all scores, over
// distributed shared memory where they are a cluster, and ranks them: the key of the last one that stays is found in digits of eight
// bits from the top, each by a histogram of the keys that match the digits found, and what stays is numbered by a prefix sum.
// Products of 16-bit values are summed in fp64, so that lists depend on no order; HBM bounds the scores (the bounds' bytes) all the
// same, as long as eight pieces a lane are under way while the eight before them are converted and summed.  32 requests of 6001 to
// 16384 positions, 8 K/V heads, blocks of 32: 18.8 us (four pieces 25, blocks of 128 threads 24); conversions to fp64 take a quarter.
template <typename TQ, int D>
__global__ void __launch_bounds__(kSelectThreads, 2)
block_select_kernel(const SelectParams p, const int ranks) {
  constexpr int kLanes = 2 * D / 8, kSide = 32 / kLanes;     // lanes of a block's bounds; blocks side by side in a warp
  constexpr int kStep = kSelectWarps * kSide * kDeep;        // blocks that a thread block scores at a time
  extern __shared__ uint32_t s_key[];                        // [n_blocks], of the first thread block
  __shared__ double s_weight[2 * D];
  __shared__ uint32_t s_bins[4][256], s_sum[kSelectWarps];
  __shared__ uint2 s_range[kSelectWarps];
  const int t = (int)blockIdx.x / ranks, rank = (int)blockIdx.x - t * ranks, hkv = blockIdx.y, b = blockIdx.z;
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32;
  grid_dependency_wait();
  grid_launch_dependents();
  // the first pieces are asked for before it is known how many blocks the token sees: there is room for n_blocks
  const uint4* bounds = reinterpret_cast<const uint4*>(static_cast<const TQ*>(p.bounds) + (int64_t)b * p.bounds_sb + (int64_t)hkv * p.bounds_sh) +
                        lane % kLanes;
  auto place = [&](int j0, int i) { return j0 + (warp * kDeep + i) * kSide + lane / kLanes; };
  uint4 w[2][kDeep];
  auto ask = [&](int j0, int upto, uint4 (&x)[kDeep]) {
#pragma unroll
    for (int i = 0; i < kDeep; ++i) {
      const int j = place(j0, i);
      x[i] = j < upto ? ld_stream_16B(bounds + (int64_t)j * kLanes) : make_uint4(0, 0, 0, 0);
    }
  };
  ask(rank * kStep, p.n_blocks, w[0]);
  uint32_t flags = 0;
  int ctx, n_new;
  window_sizes(p, b, ctx, n_new, flags);
  if (flags && p.status && blockIdx.x == 0 && hkv == 0 && tid == 0) atomicOr(p.status, flags);
  const int pos = ctx - n_new + t;
  if (t >= n_new || pos < 0) return;
  const int m = (pos >> p.block_shift) + 1;                  // blocks that the token sees
  const int64_t r = ((int64_t)b * p.H_kv + hkv) * p.n_q + t;
  int32_t* index = p.index + r * p.budget;
  if (rank == 0 && tid == 0) p.counts[r] = min(m, p.budget);
  if (m <= p.budget) {
    for (int i = rank * kSelectThreads + tid; i < m; i += ranks * kSelectThreads) index[i] = i;
    if (!p.scores) return;
  }
  if (ranks > 1) cluster_sync();                             // (every block has begun: its shared memory is there)
  if (tid < D) {
    const TQ* q = static_cast<const TQ*>(p.q) + (int64_t)b * p.q_sb + (int64_t)hkv * p.group * p.q_sh + (int64_t)t * p.q_st + tid;
    double below = 0, above = 0;
#pragma unroll 4
    for (int h = 0; h < p.group; ++h) {
      const double x = (double)to_float(q[h * p.q_sh]);
      below += fmin(x, 0.0);
      above += fmax(x, 0.0);
      if (x != x) below = above = x;
    }
    s_weight[tid] = below;
    s_weight[D + tid] = above;
  }
  for (int i = tid; i < 4 * 256; i += kSelectThreads) s_bins[i / 256][i % 256] = 0;
  __syncthreads();
  double weight[8];
#pragma unroll
  for (int e = 0; e < 8; ++e) weight[e] = s_weight[lane % kLanes * 8 + e];
  // Infinite bounds of which the queries, all of the other sign, want nothing become zero.
  auto drop = [&](uint32_t& w, double lo, double hi) {
    constexpr uint32_t kInf = std::is_same<TQ, __half>::value ? 0x7c00u : 0x7f80u;
    if (lo == 0 && (w & 0x7fffu) == kInf) w &= 0xffff0000u;
    if (hi == 0 && (w & 0x7fff0000u) == kInf << 16) w &= 0xffffu;
  };
  bool careful = false, odd = false;
  auto score = [&](int j0, uint4 (&x)[kDeep]) {
    if (careful) {
#pragma unroll
      for (int i = 0; i < kDeep; ++i) {
        drop(x[i].x, weight[0], weight[1]);
        drop(x[i].y, weight[2], weight[3]);
        drop(x[i].z, weight[4], weight[5]);
        drop(x[i].w, weight[6], weight[7]);
      }
    }
    double sum[kDeep];
#pragma unroll
    for (int i = 0; i < kDeep; ++i) {
      float f[8];
      unpack8<TQ>(x[i], f);
      double a = (double)f[0] * weight[0], z = (double)f[1] * weight[1];
#pragma unroll
      for (int e = 2; e < 8; e += 2) { a = fma((double)f[e], weight[e], a); z = fma((double)f[e + 1], weight[e + 1], z); }
      sum[i] = a + z;
    }
    int which;
    const float total = (float)sums_of<kLanes>(sum, lane, which);
    const int j = place(j0, which);
    if (j < m && lane % (kLanes / kDeep) == 0) {
      odd |= total != total;
      if (p.scores) p.scores[r * p.n_blocks + j] = total;
      if (rank == 0) s_key[j] = order_key(total);
      else store_to(&s_key[j], 0, order_key(total));
    }
  };
again:
#pragma unroll 1
  for (int j0 = rank * kStep; j0 < m; j0 += 2 * ranks * kStep) {
    ask(j0 + ranks * kStep, m, w[1]);
    score(j0, w[0]);
    ask(j0 + 2 * ranks * kStep, m, w[0]);
    if (j0 + ranks * kStep < m) score(j0 + ranks * kStep, w[1]);
  }
  if (!careful && __any_sync(~0u, odd)) {                    // a warp that met a NaN scores its blocks once more
    careful = true;
    ask(rank * kStep, m, w[0]);
    goto again;
  }
  if (ranks > 1) cluster_sync();
  else __syncthreads();
  if (rank != 0 || m <= p.budget) return;

  const int from = p.sinks, to = m - p.recent;               // those between are ranked
  int want = p.budget - p.sinks - p.recent;                  // >= 0, and < to - from
  const bool none = want == 0;
  uint32_t key = 0, known = 0;                               // bits found so far, and their mask
  if (!none) {
    // Scores are alike: digits start at the first bit in which the keys differ, which also keeps them off one bin.
    uint32_t low = ~0u, high = 0;
    for (int j = from + tid; j < to; j += kSelectThreads) { low = min(low, s_key[j]); high = max(high, s_key[j]); }
    low = __reduce_min_sync(~0u, low);
    high = __reduce_max_sync(~0u, high);
    if (lane == 0) s_range[warp] = make_uint2(low, high);
    __syncthreads();
#pragma unroll
    for (int w = 0; w < kSelectWarps; ++w) { low = min(low, s_range[w].x); high = max(high, s_range[w].y); }
    int bits = 32 - __clz(low ^ high);                       // still to be found
    known = bits == 32 ? 0u : ~0u << bits;
    key = low & known;
#pragma unroll 1
    for (int digit = 0; bits > 0; ++digit) {
      const int shift = max(0, bits - 8);
      const uint32_t mask = (1u << (bits - shift)) - 1;
      for (int j = from + tid; j < to; j += kSelectThreads) {
        const uint32_t k = s_key[j];
        if ((k & known) == key) atomicAdd(&s_bins[digit][k >> shift & mask], 1u);
      }
      __syncthreads();
      // every warp looks for the bin in which the count from the top reaches `want`: eight bins to a lane
      uint32_t mine[8];
      int sum = 0;
#pragma unroll
      for (int i = 0; i < 8; ++i) { mine[i] = s_bins[digit][255 - (lane * 8 + i)]; sum += (int)mine[i]; }
      const int end = warp_inclusive(sum, lane);
      const int who = __ffs(__ballot_sync(~0u, end >= want)) - 1;            // (all of them together reach `want`)
      int above = end - sum, at = 0, left = 0, here = 0;
      bool found = false;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        if (!found && above + (int)mine[i] >= want) { at = 255 - (lane * 8 + i); left = want - above; here = (int)mine[i]; found = true; }
        above += (int)mine[i];
      }
      key |= (uint32_t)__shfl_sync(~0u, at, who) << shift;
      known |= mask << shift;
      want = __shfl_sync(~0u, left, who);
      if (__shfl_sync(~0u, here, who) == want) break;        // all that share these bits stay
      bits = shift;
    }
  }
  // what stays, in order: a thread has `each` neighbouring blocks; `want` of the keys that share the bits of `key` stay
  const int each = (m + kSelectThreads - 1) / kSelectThreads, first = tid * each, end = min(m, first + each);
  auto stays = [&](int j) { return j < from || j >= to || (!none && (s_key[j] & known) > key); };
  auto equals = [&](int j) { return j >= from && j < to && !none && (s_key[j] & known) == key; };
  uint32_t count = 0;                                        // (at most SSA_MAX_BLOCKS of either)
  for (int j = first; j < end; ++j) count += (uint32_t)stays(j) | (uint32_t)equals(j) << 16;
  const uint32_t upto = (uint32_t)warp_inclusive((int)count, lane);
  if (lane == 31) s_sum[warp] = upto;
  __syncthreads();
  uint32_t before = upto - count;
  for (int w = 0; w < warp; ++w) before += s_sum[w];
  int more = (int)(before & 0xffffu), same = (int)(before >> 16);
  for (int j = first; j < end; ++j) {
    const bool is_more = stays(j), is_same = equals(j);
    if (is_more || (is_same && same < want)) index[more + min(same, want)] = j;
    more += is_more;
    same += is_same;
  }
}

// ---- host -----------------------------------------------------------------------------------------------------------------
int32_t check_cache(const ssa_attn_desc* d) {
  if (d->kv_dtype != SSA_FP4_E2M1) return check_desc(d);
  ssa_attn_desc c = *d;
  c.kv_dtype = SSA_BF16;                                     // (whose queries and outputs are the same)
  const int32_t rc = check_desc(&c);
  if (rc != SSA_OK) return rc;
  for (int64_t s : {d->k_stride_b, d->k_stride_t, d->k_stride_h, d->v_stride_b, d->v_stride_t, d->v_stride_h})
    if (s % d->D != 0) return SSA_ERR_ALIGN;
  return SSA_OK;
}

int32_t check_block_sizes(const ssa_attn_desc* d, const ssa_blocks* k) {
  if (k->block_size != 32 && k->block_size != 64 && k->block_size != 128 && k->block_size != 256) return SSA_ERR_UNSUPPORTED;
  if (k->n_q <= 0 || d->max_ctx > kMostContext || (d->max_ctx + k->block_size - 1) / k->block_size > SSA_MAX_BLOCKS) return SSA_ERR_SHAPE;
  return SSA_OK;
}

static int32_t check_bounds(const ssa_attn_desc* d, const ssa_blocks* k, const void* bounds) {
  int32_t rc = check_cache(d);
  if (rc == SSA_OK) rc = check_block_sizes(d, k);
  if (rc != SSA_OK) return rc;
  if (k->bounds_stride_b < 0 || k->bounds_stride_h < 0) return SSA_ERR_SHAPE;
  return k->bounds_stride_b % 8 != 0 || k->bounds_stride_h % 8 != 0 || !aligned16(bounds) ? SSA_ERR_ALIGN : SSA_OK;
}

static int shift_of(int power) {
  int s = 0;
  while ((1 << s) < power) ++s;
  return s;
}

template <typename T, int D>
static cudaError_t launch_bounds(const BoundsParams& p, dim3 grid, cudaStream_t st) {
  return p.page_table ? launch_pdl(block_bounds_kernel<T, D, true>, grid, dim3(kBoundThreads), st, p)
                      : launch_pdl(block_bounds_kernel<T, D, false>, grid, dim3(kBoundThreads), st, p);
}

template <typename TQ, int D>
static cudaError_t launch_select(const SelectParams& p, int B, cudaStream_t st) {
  // Thread blocks of a token, as long as there are too few for the GPU and each has a step's blocks of positions to score
  constexpr int kStep = kSelectWarps * (32 / (2 * D / 8)) * kDeep;
  unsigned ranks = 1;
  while (ranks < 8 && 2ll * ranks * p.n_q * p.H_kv * B <= 2 * sm_count() && p.n_blocks / (2 * (int)ranks) >= kStep) ranks *= 2;
  const size_t smem = (size_t)p.n_blocks * sizeof(uint32_t);
  auto kernel = block_select_kernel<TQ, D>;
  const cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, SSA_MAX_BLOCKS * (int)sizeof(uint32_t));
  if (err != cudaSuccess) return err;
  const dim3 grid(ranks * (unsigned)p.n_q, (unsigned)p.H_kv, (unsigned)B);
  if (ranks == 1) return launch_pdl_smem(kernel, grid, dim3(kSelectThreads), smem, st, p, 1);
  return launch_cluster(kernel, ranks, grid, dim3(kSelectThreads), smem, st, p, (int)ranks);
}

}  // namespace ssa

extern "C" {

int32_t ssa_block_bounds(const ssa_attn_desc* desc, const ssa_blocks* blocks, const void* k_cache, const void* k_scales,
                         const int32_t* ctx_lens, void* bounds, uint32_t* dev_status, void* stream) {
  using namespace ssa;
  if (!desc || !blocks || !k_cache || !ctx_lens || !bounds) return SSA_ERR_NULL;
  const bool fp4 = desc->kv_dtype == SSA_FP4_E2M1;
  if (fp4 && !k_scales) return SSA_ERR_NULL;
  int32_t rc = check_bounds(desc, blocks, bounds);
  if (rc == SSA_OK && blocks->paging) rc = check_paging(blocks->paging, desc->max_ctx);
  if (rc != SSA_OK) return rc;
  if (!aligned16(k_cache) || (fp4 && !aligned16(k_scales))) return SSA_ERR_ALIGN;
  if ((desc->B > 1 && blocks->bounds_stride_b == 0) || (desc->H_kv > 1 && blocks->bounds_stride_h == 0)) return SSA_ERR_UNSUPPORTED;
  const ssa_paging* pg = blocks->paging;
  BoundsParams p = {};
  p.k = static_cast<const char*>(k_cache);
  p.k_scales = static_cast<const uint8_t*>(k_scales);
  p.ctx_lens = ctx_lens; p.q_lens = blocks->q_lens; p.page_table = pg ? pg->page_table : nullptr;
  p.bounds = bounds; p.status = dev_status;
  p.k_sb = desc->k_stride_b; p.k_sh = desc->k_stride_h; p.k_st = desc->k_stride_t;
  p.bounds_sb = blocks->bounds_stride_b; p.bounds_sh = blocks->bounds_stride_h;
  p.n_q = blocks->n_q; p.max_ctx = desc->max_ctx; p.block_shift = shift_of(blocks->block_size);
  p.page_table_stride = pg ? pg->page_table_stride : 0; p.n_pages = pg ? pg->n_pages : 0; p.page_shift = pg ? shift_of(pg->page_size) : 0;
  // the newest n_q positions lie in that many blocks
  const long long n = (desc->max_ctx + blocks->block_size - 1ll) / blocks->block_size;
  const long long touched = std::min(n, (blocks->n_q - 2ll + blocks->block_size) / blocks->block_size + 1);
  const dim3 grid((unsigned)touched, (unsigned)desc->H_kv, (unsigned)desc->B);
  cudaStream_t st = (cudaStream_t)stream;
  const bool wide = desc->D == 128;
  cudaError_t err;
  switch (desc->kv_dtype) {
    case SSA_FP4_E2M1: err = wide ? launch_bounds<Fp4E2M1, 128>(p, grid, st) : launch_bounds<Fp4E2M1, 64>(p, grid, st); break;
    case SSA_FP8_E4M3: err = wide ? launch_bounds<Fp8E4M3, 128>(p, grid, st) : launch_bounds<Fp8E4M3, 64>(p, grid, st); break;
    case SSA_BF16: err = wide ? launch_bounds<__nv_bfloat16, 128>(p, grid, st) : launch_bounds<__nv_bfloat16, 64>(p, grid, st); break;
    default: err = wide ? launch_bounds<__half, 128>(p, grid, st) : launch_bounds<__half, 64>(p, grid, st);
  }
  if (err != cudaSuccess) return SSA_ERR_CUDA;
  note_launches(1);
  return SSA_OK;
}

int32_t ssa_block_select(const ssa_attn_desc* desc, const ssa_blocks* blocks, const void* q, const void* bounds,
                         const int32_t* ctx_lens, int32_t* index, int32_t* counts, float* scores,
                         uint32_t* dev_status, void* stream) {
  using namespace ssa;
  if (!desc || !blocks || !q || !bounds || !ctx_lens || !index || !counts) return SSA_ERR_NULL;
  const int32_t rc = check_bounds(desc, blocks, bounds);
  if (rc != SSA_OK) return rc;
  if (blocks->q_stride_t < 0 || (long long)desc->H * blocks->n_q > 1ll << 24) return SSA_ERR_SHAPE;
  if (blocks->q_stride_t % 8 != 0 || !aligned16(q)) return SSA_ERR_ALIGN;
  if (blocks->budget <= 0 || blocks->sinks < 0 || blocks->recent < 0 || (int64_t)blocks->sinks + blocks->recent > blocks->budget)
    return SSA_ERR_CAPACITY;
  SelectParams p = {};
  p.q = q; p.bounds = bounds; p.ctx_lens = ctx_lens; p.q_lens = blocks->q_lens;
  p.index = index; p.counts = counts; p.scores = scores; p.status = dev_status;
  p.q_sb = desc->q_stride_b; p.q_sh = desc->q_stride_h; p.q_st = blocks->q_stride_t;
  p.bounds_sb = blocks->bounds_stride_b; p.bounds_sh = blocks->bounds_stride_h;
  p.H_kv = desc->H_kv; p.group = desc->H / desc->H_kv; p.n_q = blocks->n_q; p.max_ctx = desc->max_ctx;
  p.block_shift = shift_of(blocks->block_size);
  p.n_blocks = (desc->max_ctx + blocks->block_size - 1) / blocks->block_size;
  p.budget = blocks->budget; p.sinks = blocks->sinks; p.recent = blocks->recent;
  cudaStream_t st = (cudaStream_t)stream;
  const bool wide = desc->D == 128, half = desc->kv_dtype == SSA_F16;
  const cudaError_t err = half ? (wide ? launch_select<__half, 128>(p, desc->B, st) : launch_select<__half, 64>(p, desc->B, st))
                               : (wide ? launch_select<__nv_bfloat16, 128>(p, desc->B, st) : launch_select<__nv_bfloat16, 64>(p, desc->B, st));
  if (err != cudaSuccess) return SSA_ERR_CUDA;
  note_launches(1);
  return SSA_OK;
}

}  // extern "C"
