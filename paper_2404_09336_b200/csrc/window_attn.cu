// Attention of the newest tokens of every request, each over its own past: causal, within a sliding window, with the first
// positions (sinks) visible to all; and the same with the softmax weight of every position added up.
//
//   token t of n at position pos = ctx - n + t sees V(t) = { j <= pos : j > pos - window or j < sinks }
//   s_j = scale <q_t, K_j>,  out = sum_{V(t)} softmax(s)_j V_j,  lse = log sum_{V(t)} exp(s_j)
//   mass_out[j] = decay mass_in[j] + sum over heads and tokens of exp(s_j - lse)
//
// window_rows_kernel serves few query rows per K/V head (decode steps, drafted tokens): all of a K/V head's query heads and
// tokens are rows of warp-level m16n8k16 tiles, so a cached row is read once for up to 32 of them.  HBM bounds it.
// window_tile_kernel (window_tile.cuh) serves many: prompt chunks.  The tensor cores bound it.
#include <algorithm>
#include <type_traits>

#include "mma.cuh"
#include "window_tile.cuh"

namespace ssa {

constexpr int kGroup = 8;              // query rows of a matrix tile: (token, head of the group) pairs
constexpr int kWarps = 4;              // of a block
constexpr int kSplitKeys = 256;        // fewest positions worth a split of their own
constexpr int kMostGroups = 4;         // of kGroup rows, of a warp
constexpr float kLazyRows = 2.f;       // log2 of how far weights may exceed 1 before sums are rescaled (fp16: 2^13 times that)
// Rows of a K/V head up to which this kernel is the faster one (16 requests of up to 4096, 8 K/V heads: 41 us for 16 rows, 55 for
// 24, 82 for 32; the tiles 54 to 58 for 32 and more, up to 128).  25 rows with 1 to 16 requests, 1 to 8 K/V heads and 512 to 65536
// positions take 15 to 97 us here, and with the tiles 0.54 to 0.89 of that, in each of 31 shapes; 16 rows over one K/V head take
// 9.6 us (512 positions) to 29 (65536) here, 25 rows with the tiles 11.6 to 27.
constexpr int kFewRows = 24;

// The weights enter the second contraction as a 16-bit value plus the 16-bit rest, so that the sums keep 16 bits (bf16) or 22
// (fp16) of each.  fp16 has little range below 1: its weights are scaled by 2^13, which the sum divides out again.
template <typename T> struct Weight { using Type = __half; static constexpr float kShift = 13.f; };
template <> struct Weight<__nv_bfloat16> { using Type = __nv_bfloat16; static constexpr float kShift = 0.f; };

// How the kernel cuts cache rows.  16-bit rows come out of shared memory by ldmatrix.  8-bit rows have to be converted on the
// way; the order of the dimensions within a contraction is free as long as both sides agree, so lanes take whole 16-byte pieces
// of them (8 bytes of V's 64-byte rows).
template <typename T, int D, int kGroups = 1>
struct RowShape {
  static constexpr int kBytes = kIsFp8<T> ? 1 : 2, kRow = D * kBytes, kChunks = kRow / 16;
  static constexpr int kNK = D / 64, kV = D / 8;                       // 8-bit: pieces of K per lane; elements of V's piece
  static constexpr int kHalves = kRow == 256 ? 1 : 2;                  // tiles of 16 positions, or of 32 where rows are short
  static constexpr int kKeys = 16 * kHalves, kTile = 2 * kKeys * kRow; // bytes: of K and V of a tile
  // blocks that fit an SM by their registers, and tiles of a warp's ring: 64 KB a block, or 96
  static constexpr int kBlocks = kGroups <= 2 ? 3 : 2, kRingBytes = kBlocks == 3 ? 16384 : 24576;
  static constexpr int kRingTiles = kRingBytes / kTile < 4 ? kRingBytes / kTile : 4;
  static constexpr int kSmem = kWarps * kRingTiles * kTile;
};

// Where 16-byte piece `chunk` of row `key` lies in a tile.  16-bit rows: the eight rows of an ldmatrix hit eight different bank
// groups.  8-bit rows: so do reads of K (lanes 4g+c: rows g, pieces c) and of V (rows 2c, pieces g) by eight lanes at a time.
template <typename T, int kChunks>
__device__ __forceinline__ int turned(int key, int chunk) {
  const int x = kIsFp8<T> ? ((key >> 1 & 3) << 1) ^ ((key & 1) << 2) : key & 7;
  return chunk ^ (x & (kChunks - 1));
}
template <typename T, int kChunks>
__device__ __forceinline__ int chunk_at(int key, int chunk) { return key * kChunks + turned<T, kChunks>(key, chunk); }

template <bool kTrans>
__device__ __forceinline__ void ldmatrix(uint32_t (&w)[4], uint32_t at) {
  if constexpr (kTrans)
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at));
  else
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];" : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3]) : "r"(at));
}
__device__ __forceinline__ uint32_t transposed(uint32_t w) {
  uint32_t t;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(t) : "r"(w));
  return t;
}

__device__ __forceinline__ void copy_16B(uint32_t to, const void* from, bool there) {     // zeros where it is not
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(there ? 16 : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory"); }

// Two e4m3 values -> two fp16 values (exact).
__device__ __forceinline__ uint32_t e4m3x2_to_half2(uint32_t pair) {
  uint32_t h2;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"((unsigned short)pair));
  return h2;
}

// A row of bf16 queries over an 8-bit cache as fp16 values times a power of two that brings its largest to 2^14: what the others
// lose is below 2^-39 of that.  w: the row's part of this lane, the rest in the three neighbouring lanes.  Returns the power's
// inverse.
template <int N>
__device__ __forceinline__ float rows_to_half(uint32_t (&w)[N]) {
  uint32_t most = 0;                                         // bits of the largest finite magnitude
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t a = w[i] & 0x7fffu, z = w[i] >> 16 & 0x7fffu;
    most = max(most, max(a < 0x7f80u ? a : 0u, z < 0x7f80u ? z : 0u));
  }
  most = max(most, __shfl_xor_sync(~0u, most, 1));
  most = max(most, __shfl_xor_sync(~0u, most, 2));
  const int up = min(141 - (int)(most >> 7), 126);           // 2^up: the exponent 127 + 14 - that of the largest
  const float by = __int_as_float((127 + up) << 23), back = __int_as_float((127 - up) << 23);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const float2 f = unpack2<__nv_bfloat16>(w[i]);
    w[i] = pack2<__half>(f.x * by, f.y * by);
  }
  return back;
}

// Whether one of two 16-bit values is infinite or NaN.
template <typename T> __device__ __forceinline__ bool pair_not_finite(uint32_t w);
template <> __device__ __forceinline__ bool pair_not_finite<__nv_bfloat16>(uint32_t w) {
  return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}
template <> __device__ __forceinline__ bool pair_not_finite<__half>(uint32_t w) {
  return (w & 0x7c00u) == 0x7c00u || (w & 0x7c000000u) == 0x7c000000u;
}

// grid (splits x row blocks, H_kv, B).  A team of kTeam warps, kGroups times eight query rows each, shares the tiles that it copies
// into a ring of its own (16 bytes a lane, asynchronously; no block barrier inside the loop); the block's teams take tiles in turn.  Cached
// rows and dimensions are the long side of the matrix instructions, m16n8k16, query rows the short one:
//   S^T[16 keys, 8 rows] += K . Q^T   and   O^T[16 dims, 8 rows] += V^T . P^T   (P transposed by movmatrix)
// Lane 4g+c holds, of S^T, keys g and g + 8 of rows 2c and 2c + 1 of each group of eight.  Bound by HBM where lists are long; by the instructions of a
// tile (some 230) and a block's start and end where they are short.
template <typename T, int D, bool kPaged, bool kMass, int kTeam, int kGroups>
__global__ void __launch_bounds__(kWarps * 32, (RowShape<T, D, kGroups>::kBlocks))
window_rows_kernel(const WindowParams p) {
  using TQ = typename Storage<T>::Query;
  using TP = typename Weight<T>::Type;                       // of the second contraction; of the first: TS
  using TS = std::conditional_t<kIsFp8<T>, __half, TQ>;
  using RS = RowShape<T, D, kGroups>;
  constexpr int kKeys = RS::kKeys, kHalves = RS::kHalves;
  constexpr float kShift = Weight<T>::kShift;
  constexpr int kRows = kGroups * kGroup;                    // of a warp
  constexpr int kTeams = kWarps / kTeam, kRing = RS::kRingTiles * kTeam, kChunks = RS::kChunks;
  extern __shared__ __align__(128) uint8_t smem[];
  __shared__ float2 s_ml[kWarps][kRows];
  __shared__ uint32_t s_have[kTeams][kRing];                 // which rows of a tile there are: seen, and on a page that exists

  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, c = lane % 4;
  const int team = warp / kTeam, member = warp % kTeam;
  const int block = p.n_splits == 1 ? blockIdx.x : blockIdx.x / p.n_splits, split = blockIdx.x - block * p.n_splits;
  const int hkv = blockIdx.y, b = blockIdx.z, row0 = block * kTeam * kRows;
  grid_dependency_wait();
  grid_launch_dependents();
  uint32_t flags = 0;
  int ctx, n_new;
  window_sizes(p, b, ctx, n_new, flags);
  if (flags && p.status && split == 0 && row0 == 0 && hkv == 0 && threadIdx.x == 0) atomicOr(p.status, flags);
  const int rows = min(kTeam * kRows, n_new * p.group - row0);         // rows of tokens that exist
  if (rows <= 0) return;
  const int first = ctx - n_new, t_lo = token_of(p, row0), t_hi = token_of(p, row0 + rows - 1);
  const Seen seen(p, kKeys, first, t_lo, t_hi);
  const int n_splits = splits_used(p, seen.tiles);
  if (split >= n_splits) return;
  const int2 range = split_tiles(seen.tiles, split, n_splits);
  const int lo = first + t_lo, hi = first + t_hi, from = p.window == 0 ? 0 : max(0, lo - p.window + 1);

  const int32_t* table = kPaged ? p.page_table + (int64_t)b * p.page_table_stride : nullptr;
  uint8_t* const ring = smem + team * (kRing * RS::kTile);
  const uint32_t ring_at = (uint32_t)__cvta_generic_to_shared(ring);
  const int n_tiles = (range.y - range.x - team + kTeams - 1) / kTeams;     // of this team
  // a lane copies piece my_chunk of rows my_key, my_key + kPass, ... of K and of V
  constexpr int kAll = kKeys * kChunks, kLanes = 32 * kTeam, kPass = kLanes / kChunks, kPasses = kAll < kLanes ? 1 : kAll / kLanes;
  const int my = member * 32 + lane, my_key = my / kChunks, my_chunk = my % kChunks;
  const bool copies = kAll >= kLanes || my < kAll;
  const char* const kb = reinterpret_cast<const char*>(p.k) + my_chunk * 16 +
                         ((kPaged ? 0 : (int64_t)b * p.k_sb) + (int64_t)hkv * p.k_sh) * RS::kBytes;
  const char* const vb = reinterpret_cast<const char*>(p.v) + my_chunk * 16 +
                         ((kPaged ? 0 : (int64_t)b * p.v_sb) + (int64_t)hkv * p.v_sh) * RS::kBytes;
  const int64_t k_step = (int64_t)p.k_st * RS::kBytes, v_step = (int64_t)p.v_st * RS::kBytes;
  auto load = [&](int n) {
    if (n < n_tiles) {
      const int stage = n % kRing, j0 = seen.position(range.x + team + n * kTeams);
      const uint32_t to = ring_at + stage * RS::kTile;
      // tiles that are seen as a whole and lie on one page have rows in a row
      int64_t at = -1;
      if (j0 + kKeys - 1 <= hi && (j0 >= from || j0 + kKeys <= p.sinks) && (!kPaged || kKeys >> p.page_shift <= 1)) at = row_of<kPaged>(p, table, j0);
      unsigned have = ~0u;
      if (at >= 0) {
        if (copies) {
          const char *k = kb + (at + my_key) * k_step, *v = vb + (at + my_key) * v_step;
#pragma unroll
          for (int i = 0; i < kPasses; ++i) {
            const int key = i * kPass;
            const uint32_t x = to + (my_key + key) * kChunks * 16 +
                               (turned<T, kChunks>(my_key, my_chunk) ^ turned<T, kChunks>(key, 0)) * 16;
            copy_16B(x, k, true);
            copy_16B(x + kKeys * RS::kRow, v, true);
            k += kPass * k_step;
            v += kPass * v_step;
          }
        }
      } else {
        // what no row sees is not read: it may hold anything, or have no page
        const int j = j0 + lane % kKeys;
        const bool any = j <= hi && (j >= from || j < p.sinks);
        const int row = any ? (int)row_of<kPaged>(p, table, j) : -1;
        if (kPaged && any && row < 0) flags |= SSA_DEV_BAD_INDEX;
        have = __ballot_sync(~0u, row >= 0);
#pragma unroll 1
        for (int i = 0; i < kPasses; ++i) {
          const int key = (my_key + i * kPass) % kKeys;
          const int64_t r = __shfl_sync(~0u, row, key);
          if (copies) {
            const uint32_t x = to + chunk_at<T, kChunks>(key, my_chunk) * 16;
            copy_16B(x, kb + (r < 0 ? 0 : r * k_step), r >= 0);
            copy_16B(x + kKeys * RS::kRow, vb + (r < 0 ? 0 : r * v_step), r >= 0);
          }
        }
      }
      if (lane == 0 && member == 0) s_have[team][stage] = have;
    }
    copies_commit();
  };
#pragma unroll 1
  for (int n = 0; n < kRing - 1; ++n) load(n);

  // the queries: row g of each group, as the short side of the first contraction; a lane's scores are of rows 2c, 2c + 1
  const int wrow0 = row0 + member * kRows, wrows = min(kRows, rows - member * kRows);
  constexpr int kSteps = D / 16;
  uint32_t qb[kGroups][2 * kSteps];
  float unit[kGroups][2];
  int pos[kGroups][2];                                       // (a row that does not exist sees nothing)
#pragma unroll
  for (int y = 0; y < kGroups; ++y) {
    const int row = wrow0 + y * kGroup + g, t = token_of(p, row), h = hkv * p.group + row - t * p.group;
    const bool there = y * kGroup + g < wrows;
    const TQ* q = reinterpret_cast<const TQ*>(p.q) + (int64_t)b * p.q_sb + (int64_t)h * p.q_sh + (int64_t)t * p.q_st;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      if constexpr (kIsFp8<T>) {                             // step 4 u + i takes elements 4 i ... of the lane's piece 4 u + c
        uint2 x = make_uint2(0, 0);
        if (there) x = *reinterpret_cast<const uint2*>(q + (i / 4 * 4 + c) * 16 + i % 4 * 4);
        qb[y][2 * i] = x.x;
        qb[y][2 * i + 1] = x.y;
      } else {
        qb[y][2 * i] = there ? *reinterpret_cast<const uint32_t*>(q + 16 * i + 2 * c) : 0;
        qb[y][2 * i + 1] = there ? *reinterpret_cast<const uint32_t*>(q + 16 * i + 2 * c + 8) : 0;
      }
    }
    float back = 1.f;
    if constexpr (kIsFp8<T>) back = rows_to_half(qb[y]);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      unit[y][r] = kIsFp8<T> ? p.scale_log2 * __shfl_sync(~0u, back, (2 * c + r) * 4) : p.scale_log2;
      const int mine = y * kGroup + 2 * c + r;
      pos[y][r] = mine < wrows ? first + token_of(p, wrow0 + mine) : -1;
    }
  }
  // every row of the warp sees all of [all_lo, all_hi]; the sinks as well
  const int all_hi = first + token_of(p, wrow0);
  const int all_lo = p.window == 0 ? 0 : first + token_of(p, wrow0 + max(wrows, 1) - 1) - p.window + 1;
  // ldmatrix addresses: lane i of matrix y = i / 8 gives row i % 8 of it.  K: keys 8 (y % 2) ..., pieces 2 s + y / 2;
  // V: keys 8 (y / 2) ..., pieces 2 i + y % 2
  const int k_key = lane % 16, v_key = lane % 8 + lane / 16 * 8;       // (of each sixteen positions)

  // An infinite or NaN element of V must not reach rows that do not see it (0 * inf), and has to stay infinite for those that do
  // (its product with a weight's two parts may be inf - inf).  Sums that come out finite met none; else the block goes through
  // its tiles once more and takes such elements out of the contraction, to add them to the rows that see them.
  constexpr int kTiles = D / 16;
  float acc[kGroups][kTiles][4], m[kGroups][2], l[kGroups][2];   // dimensions (16-bit: 16 i + g, + 8; 8-bit: g kV + 2 i, + 1), rows
  bool careful = false;
again:
#pragma unroll
  for (int y = 0; y < kGroups; ++y) {
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[y][i][e] = 0.f;
    m[y][0] = m[y][1] = neg_inf();
    l[y][0] = l[y][1] = 0.f;
  }
#pragma unroll 1
  for (int n = 0; n < n_tiles; ++n) {
    copies_wait<kRing - 2>();
    if constexpr (kTeam == 1) __syncwarp();                  // the tile is there, and every warp of the team has left the last one
    else asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "n"(kTeam * 32) : "memory");
    const int j0 = seen.position(range.x + team + n * kTeams), stage = n % kRing;
    load(n + kRing - 1);
    if (kTeam > 1 && wrows <= 0) continue;
    const uint32_t k_at = ring_at + stage * RS::kTile, v_at = k_at + kKeys * RS::kRow;
    const uint8_t* const kt = ring + stage * RS::kTile;
    const uint8_t* const vt = kt + kKeys * RS::kRow;
    const unsigned have = s_have[team][stage];
    float s[kHalves][kGroups][4];
#pragma unroll
    for (int x = 0; x < kHalves; ++x) {
      float s2[kGroups][4];                                  // (two chains of half the steps each)
#pragma unroll
      for (int y = 0; y < kGroups; ++y)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[x][y][e] = s2[y][e] = 0.f;
      if constexpr (kIsFp8<T>) {
#pragma unroll
        for (int u = 0; u < RS::kNK; ++u) {
          const uint4 a4 = *reinterpret_cast<const uint4*>(kt + chunk_at<T, kChunks>(16 * x + g, u * 4 + c) * 16);
          const uint4 z4 = *reinterpret_cast<const uint4*>(kt + chunk_at<T, kChunks>(16 * x + g + 8, u * 4 + c) * 16);
          const uint32_t a[4] = {a4.x, a4.y, a4.z, a4.w}, z[4] = {z4.x, z4.y, z4.z, z4.w};
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const uint32_t a0 = e4m3x2_to_half2(a[i] & 0xffffu), a1 = e4m3x2_to_half2(z[i] & 0xffffu), a2 = e4m3x2_to_half2(a[i] >> 16),
                           a3 = e4m3x2_to_half2(z[i] >> 16);
#pragma unroll
            for (int y = 0; y < kGroups; ++y)
              mma_16816<TS>(i % 2 ? s2[y] : s[x][y], a0, a1, a2, a3, qb[y][2 * (u * 4 + i)], qb[y][2 * (u * 4 + i) + 1], i % 2 ? s2[y] : s[x][y]);
          }
        }
      } else {
#pragma unroll
        for (int i = 0; i < kSteps; ++i) {
          uint32_t a[4];
          ldmatrix<false>(a, k_at + chunk_at<T, kChunks>(16 * x + k_key, 2 * i + lane / 16) * 16);
#pragma unroll
          for (int y = 0; y < kGroups; ++y)
            mma_16816<TS>(i % 2 ? s2[y] : s[x][y], a[0], a[1], a[2], a[3], qb[y][2 * i], qb[y][2 * i + 1], i % 2 ? s2[y] : s[x][y]);
        }
      }
#pragma unroll
      for (int y = 0; y < kGroups; ++y)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[x][y][e] = (s[x][y][e] + s2[y][e]) * unit[y][e % 2];
    }

    // scores in log2 units; what a row does not see is -inf
    if (!(have == ~0u && j0 + kKeys - 1 <= all_hi && (j0 >= all_lo || j0 + kKeys <= p.sinks))) {
#pragma unroll
      for (int x = 0; x < kHalves; ++x)
#pragma unroll
        for (int y = 0; y < kGroups; ++y)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int key = 16 * x + g + e / 2 * 8;
            if (!(have >> key & 1) || !sees(p, pos[y][e % 2], j0 + key)) s[x][y][e] = neg_inf();
          }
    }
    float top[kGroups][2];
#pragma unroll
    for (int y = 0; y < kGroups; ++y) {
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        top[y][r] = m[y][r];
#pragma unroll
        for (int x = 0; x < kHalves; ++x) top[y][r] = fmaxf(top[y][r], fmaxf(s[x][y][r], s[x][y][r + 2]));
      }
      if constexpr (kMass) {
#pragma unroll
        for (int r = 0; r < 2; ++r)
          if (y * kGroup + 2 * c + r < wrows) {
            const int row = wrow0 + y * kGroup + 2 * c + r, t = token_of(p, row), h = hkv * p.group + row - t * p.group;
            float* to = p.ws_s + (((int64_t)b * p.H + h) * p.n_q + t) * p.s_pitch + j0 + g;
#pragma unroll
            for (int x = 0; x < kHalves; ++x) {
              to[16 * x] = s[x][y][r];
              to[16 * x + 8] = s[x][y][r + 2];
            }
          }
      }
    }
#pragma unroll
    for (int o = 4; o < 32; o *= 2)
#pragma unroll
      for (int y = 0; y < kGroups; ++y) {
        top[y][0] = fmaxf(top[y][0], __shfl_xor_sync(~0u, top[y][0], o));
        top[y][1] = fmaxf(top[y][1], __shfl_xor_sync(~0u, top[y][1], o));
      }
    bool higher = false;
#pragma unroll
    for (int y = 0; y < kGroups; ++y) higher |= top[y][0] > m[y][0] + kLazyRows || top[y][1] > m[y][1] + kLazyRows;   // (m = -inf: anything)
    if (__any_sync(~0u, higher)) {
#pragma unroll
      for (int y = 0; y < kGroups; ++y)
#pragma unroll
        for (int r = 0; r < 2; ++r) {
          const float alpha = top[y][r] == m[y][r] ? 1.f : fast_exp2(m[y][r] - top[y][r]);
#pragma unroll
          for (int i = 0; i < kTiles; ++i) { acc[y][i][r] *= alpha; acc[y][i][r + 2] *= alpha; }
          l[y][r] *= alpha;
          m[y][r] = top[y][r];
        }
    }
    uint32_t ph[kHalves][kGroups][2], pl[kHalves][kGroups][2];         // the weights, keys 0-7 and 8-15, and what their rounding left
#pragma unroll
    for (int y = 0; y < kGroups; ++y) {
      float shift[2];
#pragma unroll
      for (int r = 0; r < 2; ++r) shift[r] = (m[y][r] == neg_inf() ? 0.f : m[y][r]) - kShift;
#pragma unroll
      for (int x = 0; x < kHalves; ++x)
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          const float w0 = fast_exp2(s[x][y][2 * z] - shift[0]), w1 = fast_exp2(s[x][y][2 * z + 1] - shift[1]);
          l[y][0] += w0;
          l[y][1] += w1;
          const uint32_t w = pack2<TP>(w0, w1);
          const float2 back = unpack2<TP>(w);
          ph[x][y][z] = transposed(w);
          pl[x][y][z] = transposed(pack2<TP>(w0 - back.x, w1 - back.y));
        }
    }
    bool odd = false;
#pragma unroll
    for (int x = 0; x < kHalves; ++x) {
      uint32_t vw[4][kIsFp8<T> ? RS::kV / 4 : 1];            // 8-bit rows: the pieces of keys 2c, 2c + 1, 2c + 8, 2c + 9
      if constexpr (kIsFp8<T>) {
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          const int key = 16 * x + 2 * c + (y & 1) + 4 * (y & 2);
          if constexpr (D == 128) {
            const uint4 w = *reinterpret_cast<const uint4*>(vt + chunk_at<T, kChunks>(key, g) * 16);
            vw[y][0] = w.x; vw[y][1] = w.y; vw[y][2] = w.z; vw[y][3] = w.w;
          } else {
            const uint2 w = *reinterpret_cast<const uint2*>(vt + chunk_at<T, kChunks>(key, g / 2) * 16 + g % 2 * 8);
            vw[y][0] = w.x; vw[y][1] = w.y;
          }
        }
      }
#pragma unroll
      for (int i = 0; i < kTiles; ++i) {
        uint32_t a[4];
        if constexpr (kIsFp8<T>) {
          // bytes 2 i, 2 i + 1 of two keys' pieces: two keys' values of one dimension, then of the next
          const uint32_t lo2 = __byte_perm(vw[0][i / 2], vw[1][i / 2], i % 2 ? 0x7362 : 0x5140);
          const uint32_t hi2 = __byte_perm(vw[2][i / 2], vw[3][i / 2], i % 2 ? 0x7362 : 0x5140);
          a[0] = e4m3x2_to_half2(lo2 & 0xffffu);
          a[1] = e4m3x2_to_half2(lo2 >> 16);
          a[2] = e4m3x2_to_half2(hi2 & 0xffffu);
          a[3] = e4m3x2_to_half2(hi2 >> 16);
        } else {
          ldmatrix<true>(a, v_at + chunk_at<T, kChunks>(16 * x + v_key, 2 * i + lane / 8 % 2) * 16);
        }
        if (careful) {
#pragma unroll
          for (int y = 0; y < 4; ++y)
            if (pair_not_finite<TP>(a[y])) {
              odd = true;
              if (pair_not_finite<TP>(a[y] & 0xffffu)) a[y] &= 0xffff0000u;
              if (pair_not_finite<TP>(a[y] & 0xffff0000u)) a[y] &= 0xffffu;
            }
        }
#pragma unroll
        for (int y = 0; y < kGroups; ++y) mma_16816<TP>(acc[y][i], a[0], a[1], a[2], a[3], ph[x][y][0], ph[x][y][1], acc[y][i]);
#pragma unroll
        for (int y = 0; y < kGroups; ++y) mma_16816<TP>(acc[y][i], a[0], a[1], a[2], a[3], pl[x][y][0], pl[x][y][1], acc[y][i]);
      }
    }
    if (careful && __any_sync(~0u, odd)) {                   // add what was taken out, element by element
#pragma unroll 1
      for (int key = 0; key < kKeys; ++key)
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            const int at = (kIsFp8<T> ? g * RS::kV + 2 * i + z : 16 * i + g + 8 * z) * RS::kBytes;
            const uint8_t* v = vt + chunk_at<T, kChunks>(key, at / 16) * 16 + at % 16;
            float f;
            if constexpr (kIsFp8<T>) f = e4m3x2_to_float2(*v).x;
            else f = to_float(*reinterpret_cast<const TQ*>(v));
            if (!isfinite(f)) {
#pragma unroll
              for (int y = 0; y < kGroups; ++y)
#pragma unroll
                for (int r = 0; r < 2; ++r)
                  if (sees(p, pos[y][r], j0 + key)) acc[y][i][2 * z + r] += f;
            }
          }
    }
  }
  copies_wait<0>();
  float test = 0.f;                                          // (0 times an infinity or a NaN is NaN)
#pragma unroll
  for (int y = 0; y < kGroups; ++y)
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) test = fmaf(acc[y][i][e], 0.f, test);
  const bool finite = test == 0.f;
  if (__syncthreads_or(!finite) && !careful) {               // (the barrier: the rings' place is free from here on)
    careful = true;
#pragma unroll 1
    for (int n = 0; n < kRing - 1; ++n) load(n);
    goto again;
  }

  // the teams' results, joined by the block
  float (*s_acc)[kRows][D + 4] = reinterpret_cast<float (*)[kRows][D + 4]>(smem);
#pragma unroll
  for (int y = 0; y < kGroups; ++y)
#pragma unroll
    for (int r = 0; r < 2; ++r) {
#pragma unroll
      for (int o = 4; o < 32; o *= 2) l[y][r] += __shfl_xor_sync(~0u, l[y][r], o);
      const int mine = y * kGroup + 2 * c + r;
      if (g == 0) s_ml[warp][mine] = make_float2(m[y][r] - kShift, l[y][r]);   // what acc and l are relative to
#pragma unroll
      for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int z = 0; z < 2; ++z) s_acc[warp][mine][kIsFp8<T> ? g * RS::kV + 2 * i + z : 16 * i + g + 8 * z] = acc[y][i][2 * z + r];
    }
  if (kPaged && p.status && (flags & SSA_DEV_BAD_INDEX)) atomicOr(p.status, SSA_DEV_BAD_INDEX);
  __syncthreads();
  for (int i = warp; i < rows; i += kWarps) {
    const int of = i / kRows, y = i % kRows;                 // member of every team, its row
    float M = neg_inf(), L = 0.f, w[kTeams];
#pragma unroll
    for (int x = 0; x < kTeams; ++x) M = fmaxf(M, s_ml[x * kTeam + of][y].x);
#pragma unroll
    for (int x = 0; x < kTeams; ++x) {
      const float2 ml = s_ml[x * kTeam + of][y];
      w[x] = ml.y == 0.f ? 0.f : fast_exp2(ml.x - M);
      L += ml.y * w[x];
    }
    const int row = row0 + i, t = token_of(p, row), h = hkv * p.group + row - t * p.group;
    const int64_t at = ((int64_t)b * p.H + h) * p.n_q + t, slot = at * p.n_splits + split;
    for (int d = lane; d < D; d += 32) {
      float A = 0.f;
#pragma unroll
      for (int x = 0; x < kTeams; ++x) A += s_acc[x * kTeam + of][y][d] * w[x];
      if (n_splits == 1) store_window_value<TQ>(p, b, h, t, d, L == 0.f ? 0.f : A / L);
      else p.ws_acc[slot * D + d] = A;
    }
    if (lane == 0) {
      if (n_splits == 1 && p.lse) p.lse[at] = L == 0.f ? neg_inf() : (M + log2f(L)) * kLn2;
      if (n_splits > 1 || kMass) p.ws_ml[slot] = make_float2(M, L);
    }
  }
}

// Splits that query row (h, t) of a request was served by.
__device__ __forceinline__ int row_splits(const WindowParams& p, int h, int t, int ctx, int n_new) {
  const int row0 = (t * p.group + h % p.group) / p.block_rows * p.block_rows, rows = min(p.block_rows, n_new * p.group - row0);
  return splits_used(p, Seen(p, p.tile_keys, ctx - n_new, token_of(p, row0), token_of(p, row0 + rows - 1)).tiles);
}

// Joins the splits of query row `row` (of H n_q) of a request: a warp, whose lanes have D / 32 dimensions each.  The first few
// splits are asked for before it is known how many there are: they have their place, and what nothing was written to is not
// used.  Rows with one split are finished already.
template <typename TQ, int D>
__device__ __forceinline__ void join_rows(const WindowParams& p, int b, int row) {
  constexpr int kN = D / 32, kAhead = 4;
  if (row >= p.H * p.n_q) return;
  const int lane = threadIdx.x % 32, h = p.n_q == 1 ? row : row / p.n_q, t = row - h * p.n_q;
  const int64_t at = (int64_t)b * p.H * p.n_q + row, slot = at * p.n_splits;
  float2 ml[kAhead];
  float a[kAhead][kN];
  auto ask = [&](int i, int x) {
    if (i >= p.n_splits) return;
    ml[x] = p.ws_ml[slot + i];
    const float* from = p.ws_acc + (slot + i) * D + lane * kN;
    if constexpr (kN == 4) {
      const float4 f = *reinterpret_cast<const float4*>(from);
      a[x][0] = f.x; a[x][1] = f.y; a[x][2] = f.z; a[x][3] = f.w;
    } else {
      const float2 f = *reinterpret_cast<const float2*>(from);
      a[x][0] = f.x; a[x][1] = f.y;
    }
  };
#pragma unroll
  for (int x = 0; x < kAhead; ++x) ask(x, x);
  uint32_t flags = 0;
  int ctx, n_new;
  window_sizes(p, b, ctx, n_new, flags);
  if (t >= n_new) return;
  const int n = row_splits(p, h, t, ctx, n_new);
  if (n == 1) return;
  float M = neg_inf(), L = 0.f, A[kN];
#pragma unroll
  for (int y = 0; y < kN; ++y) A[y] = 0.f;
  for (int i0 = 0; i0 < n; i0 += kAhead) {
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {
      if (i0 + x < n && ml[x].y != 0.f) {                    // (a split without a weight adds nothing)
        const float top = fmaxf(M, ml[x].x), base = top == neg_inf() ? 0.f : top, w = fast_exp2(ml[x].x - base), old = fast_exp2(M - base);
        L = fmaf(L, old, ml[x].y * w);
#pragma unroll
        for (int y = 0; y < kN; ++y) A[y] = fmaf(A[y], old, a[x][y] * w);
        M = top;
      }
      ask(i0 + kAhead + x, x);
    }
  }
#pragma unroll
  for (int y = 0; y < kN; ++y) store_window_value<TQ>(p, b, h, t, lane * kN + y, L == 0.f ? 0.f : A[y] / L);
  if (lane == 0 && p.lse) p.lse[at] = L == 0.f ? neg_inf() : (M + log2f(L)) * kLn2;
}

constexpr int kJoinWarps = 4;

template <typename TQ, int D>
__global__ void __launch_bounds__(kJoinWarps * 32)
window_join_kernel(const WindowParams p) {
  grid_dependency_wait();
  grid_launch_dependents();
  join_rows<TQ, D>(p, blockIdx.y, blockIdx.x * kJoinWarps + threadIdx.x / 32);
}

constexpr int kMassThreads = 256;
constexpr int kMassKeys = 128;         // positions of a block: four to a lane, every warp of the block has them all
constexpr int kMassWarps = kMassThreads / 32;
constexpr int kMassAhead = 4;          // query rows that a warp has in flight

// Blocks x < mass_blocks of a request: the weights of kMassKeys positions.  Warp w sums the query rows w, w + 8, ..., the block
// then the warps, always in that order.  The scores are asked for before the rows' normalisers are made from their splits.  The
// other blocks join the splits of query rows.
template <typename TQ, int D>
__global__ void __launch_bounds__(kMassThreads)
window_mass_kernel(const WindowParams p, const int mass_blocks) {
  __shared__ float s_lse[SSA_MASS_MAX_ROWS];
  __shared__ float s_sum[kMassWarps][kMassKeys];
  const int b = blockIdx.y, warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  grid_dependency_wait();
  grid_launch_dependents();
  if ((int)blockIdx.x >= mass_blocks) {
    join_rows<TQ, D>(p, b, (blockIdx.x - mass_blocks) * kMassWarps + warp);
    return;
  }
  uint32_t flags = 0;
  int ctx, n_new;
  window_sizes(p, b, ctx, n_new, flags);
  const int j = blockIdx.x * kMassKeys + lane * 4;
  if ((int)blockIdx.x * kMassKeys >= ctx) return;
  const int n_rows = p.H * p.n_q, first = ctx - n_new;
  const float* scores = p.ws_s + (int64_t)b * n_rows * p.s_pitch + j;
  // (a row of scores is a multiple of 32 long: four of them are there, or none; what a token does not see is not used)
  auto ask = [&](int i) {
    return i < n_rows && j < p.s_pitch ? *reinterpret_cast<const float4*>(scores + (int64_t)i * p.s_pitch) : make_float4(0.f, 0.f, 0.f, 0.f);
  };
  float4 s[kMassAhead];
#pragma unroll
  for (int x = 0; x < kMassAhead; ++x) s[x] = ask(warp + x * kMassWarps);
  for (int i = threadIdx.x; i < n_rows; i += kMassThreads) {
    const int h = p.n_q == 1 ? i : i / p.n_q, t = i - h * p.n_q;
    float lse = __int_as_float(0x7f800000);                  // +inf: nothing seen, weights of zero
    if (t < n_new) {
      const int n = row_splits(p, h, t, ctx, n_new);
      const float2* ml = p.ws_ml + ((int64_t)b * n_rows + i) * p.n_splits;
      float M = neg_inf(), L = 0.f;
#pragma unroll 4
      for (int x = 0; x < n; ++x) M = fmaxf(M, ml[x].x);
#pragma unroll 4
      for (int x = 0; x < n; ++x) L += ml[x].y == 0.f ? 0.f : ml[x].y * fast_exp2(ml[x].x - M);
      if (L != 0.f) lse = M + log2f(L);
    }
    s_lse[i] = lse;
  }
  __syncthreads();
  float sum[4] = {0.f, 0.f, 0.f, 0.f};
  for (int i0 = warp; i0 < n_rows; i0 += kMassAhead * kMassWarps) {
#pragma unroll
    for (int x = 0; x < kMassAhead; ++x) {
      const int i = i0 + x * kMassWarps;
      if (i < n_rows) {
        const int t = p.n_q == 1 ? 0 : i % p.n_q, pos = t < n_new ? first + t : -1;
        const float lse = s_lse[i];
        const float v[4] = {s[x].x, s[x].y, s[x].z, s[x].w};
#pragma unroll
        for (int y = 0; y < 4; ++y)
          if (sees(p, pos, j + y)) sum[y] += fast_exp2(v[y] - lse);
      }
      s[x] = ask(i + kMassAhead * kMassWarps);
    }
  }
  *reinterpret_cast<float4*>(&s_sum[warp][lane * 4]) = make_float4(sum[0], sum[1], sum[2], sum[3]);
  __syncthreads();
  const int key = blockIdx.x * kMassKeys + threadIdx.x;
  if (threadIdx.x >= kMassKeys || key >= ctx) return;
  float total = 0.f;
#pragma unroll
  for (int x = 0; x < kMassWarps; ++x) total += s_sum[x][threadIdx.x];
  if (p.mass_in && key < first) total = fmaf(p.decay, p.mass_in[(int64_t)b * p.mass_stride + key], total);
  p.mass_out[(int64_t)b * p.mass_stride + key] = total;
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
struct WindowPlan { bool tiles; int block_rows, keys, fewest, n_splits, s_pitch; size_t ml_bytes, acc_bytes, s_bytes, total_bytes; };

int32_t check_paging(const ssa_paging* pg, int32_t max_ctx) {
  if (!pg->page_table) return SSA_ERR_NULL;
  if (pg->page_size <= 0 || (pg->page_size & (pg->page_size - 1)) != 0 || pg->n_pages <= 0 || pg->page_table_stride <= 0 ||
      (long long)pg->n_pages * pg->page_size > 0x7fffffffll || (long long)pg->page_table_stride * pg->page_size < max_ctx)
    return SSA_ERR_SHAPE;
  return SSA_OK;
}

static int32_t check_window(const ssa_attn_desc* d, const ssa_window* w, bool mass) {
  const int32_t rc = check_desc(d);
  if (rc != SSA_OK) return rc;
  if (d->max_ctx > kMostContext || w->n_q <= 0 || w->window < 0 || w->sinks < 0 || w->q_stride_t < 0 || w->o_stride_t < 0) return SSA_ERR_SHAPE;
  if (w->q_stride_t % 8 != 0 || w->o_stride_t % 8 != 0) return SSA_ERR_ALIGN;
  if ((long long)d->H * w->n_q > (mass ? (long long)SSA_MASS_MAX_ROWS : 1ll << 24)) return SSA_ERR_SHAPE;
  return w->paging ? check_paging(w->paging, d->max_ctx) : SSA_OK;
}

static size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// Whether the tiles of 128 rows serve a call.
static bool tiles_pay(const ssa_attn_desc* d, const ssa_window* w, bool mass) {
  return !mass && d->kv_dtype != SSA_FP8_E4M3 && (long long)(d->H / d->H_kv) * w->n_q > kFewRows &&
         (!w->paging || w->paging->page_size >= 8);          // (a box of a copy is eight rows at least)
}

static bool plan_window(const ssa_attn_desc* d, const ssa_window* w, bool mass, bool tiles, WindowPlan* pl) {
  pl->tiles = tiles;
  const long long per_head = (long long)(d->H / d->H_kv) * w->n_q;
  const int keys = tiles ? kTileKeys : d->D * (d->kv_dtype == SSA_FP8_E4M3 ? 1 : 2) == 256 ? 16 : 32, fewest = tiles ? kTileSplit : kSplitKeys / keys;
  // rows of a block: a warp's groups of eight, or four groups of two warps each
  const int groups = (int)std::min<long long>((per_head + kGroup - 1) / kGroup, 8);
  const int rows = tiles ? kTileRows : kGroup * (groups <= kMostGroups ? groups : 8);
  const long long group = d->H / d->H_kv, row_tiles = (per_head + rows - 1) / rows;
  const long long blocks = row_tiles * d->H_kv * d->B, tokens = (rows - 1) / group + 2;
  const long long most = w->window == 0 ? d->max_ctx : std::min<long long>(d->max_ctx, (long long)w->window + w->sinks + tokens);
  const long long n_tiles = (most + keys - 1) / keys + 2;
  pl->keys = keys;
  pl->fewest = fewest;
  const long long most_splits = std::max(1ll, std::min(n_tiles / fewest, 64ll));
  long long splits = std::min(most_splits, std::max(1ll, 2ll * sm_count() / blocks));   // tiles: two blocks to an SM
  if (!tiles) {
    // The kernel for few rows: what n splits cost in units of one tile's time.  The work of all blocks, each with a start and an
    // end, over the places that there are (two or three blocks to an SM), but no less than one block's; half a block's until the
    // last is done (lengths differ: three quarters of the longest are taken for the mean); joining.
    const int teams = rows <= kMostGroups * kGroup ? kWarps : kWarps / 2;
    const double steps = (double)n_tiles / teams, places = (rows <= 2 * kGroup ? 3.0 : 2.0) * sm_count(), ends = 5, join = 6;
    double least = 0;
    for (long long n = 1; n <= most_splits; ++n) {
      const double one = steps / n + ends, all = blocks * n * (0.75 * steps / n + ends) / places;
      const double cost = std::max(one, all) + 0.5 * one + (n > 1 ? join : 0);
      if (n == 1 || cost < least) { least = cost; splits = n; }
    }
  }
  pl->n_splits = (int)splits;
  pl->block_rows = rows;
  const size_t slots = (size_t)d->B * d->H * w->n_q * pl->n_splits;
  pl->ml_bytes = up256(slots * sizeof(float2));
  pl->acc_bytes = pl->n_splits > 1 ? up256(slots * d->D * sizeof(float)) : 0;
  pl->s_pitch = mass ? (int)(((long long)d->max_ctx + 31) / 32 * 32) : 0;
  pl->s_bytes = up256((size_t)d->B * d->H * w->n_q * pl->s_pitch * sizeof(float));
  pl->total_bytes = pl->ml_bytes + pl->acc_bytes + pl->s_bytes;
  return row_tiles * pl->n_splits <= 0x7fffffffll;
}

// Room for either kernel: which one runs may depend on the cache's strides.
static size_t window_bytes(const ssa_attn_desc* d, const ssa_window* w, bool mass) {
  WindowPlan pl;
  if (!d || !w || check_window(d, w, mass) != SSA_OK || !plan_window(d, w, mass, false, &pl)) return 0;
  const size_t few = pl.total_bytes;
  if (!tiles_pay(d, w, mass) || !plan_window(d, w, mass, true, &pl)) return few;
  return std::max(few, pl.total_bytes);
}

template <typename T, int D>
static cudaError_t launch_tiles(const WindowParams& p, const CUtensorMap& k_map, const CUtensorMap& v_map, int box_rows, cudaStream_t st) {
  const dim3 grid((unsigned)((p.group * p.n_q + kTileRows - 1) / kTileRows * p.n_splits), (unsigned)p.H_kv, (unsigned)p.B);
  auto kernel = p.page_table ? (p.out_f32 ? window_tile_kernel<T, D, true, true> : window_tile_kernel<T, D, true, false>)
                             : (p.out_f32 ? window_tile_kernel<T, D, false, true> : window_tile_kernel<T, D, false, false>);
  constexpr int kSmem = TileShape<D>::kSmem;
  const cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
  if (err != cudaSuccess) return err;
  return launch_pdl_smem(kernel, grid, dim3(kTileThreads), kSmem, st, p, k_map, v_map, box_rows);
}

template <typename T, int D, bool kPaged, bool kMass>
static cudaError_t launch_rows(const WindowParams& p, cudaStream_t st) {
  const dim3 grid((unsigned)((p.group * p.n_q + p.block_rows - 1) / p.block_rows * p.n_splits), (unsigned)p.H_kv, (unsigned)p.B);
  auto launch = [&](auto kernel, int bytes, int warp_rows) {
    const int smem = std::max(bytes, kWarps * warp_rows * (D + 4) * (int)sizeof(float));     // (the join's place)
    const cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
    return err != cudaSuccess ? err : launch_pdl_smem(kernel, grid, dim3(kWarps * 32), smem, st, p);
  };
  switch (p.block_rows / kGroup) {
    case 1: return launch(window_rows_kernel<T, D, kPaged, kMass, 1, 1>, RowShape<T, D, 1>::kSmem, kGroup);
    case 2: return launch(window_rows_kernel<T, D, kPaged, kMass, 1, 2>, RowShape<T, D, 2>::kSmem, 2 * kGroup);
    case 3: return launch(window_rows_kernel<T, D, kPaged, kMass, 1, 3>, RowShape<T, D, 3>::kSmem, 3 * kGroup);
    case 4: return launch(window_rows_kernel<T, D, kPaged, kMass, 1, 4>, RowShape<T, D, 4>::kSmem, 4 * kGroup);
    default: return launch(window_rows_kernel<T, D, kPaged, kMass, 2, 4>, RowShape<T, D, 4>::kSmem, 4 * kGroup);
  }
}

template <typename T, int D>
static int32_t launch_window(const WindowParams& p, bool mass, const CUtensorMap* maps, int box_rows, cudaStream_t st) {
  using TQ = typename Storage<T>::Query;
  cudaEvent_t begin, end;
  take_kernel_events(&begin, &end);
  if (begin) cudaEventRecord(begin, st);
  cudaError_t err = cudaErrorInvalidValue;
  if (maps) {
    if constexpr (!kIsFp8<T>) err = launch_tiles<T, D>(p, maps[0], maps[1], box_rows, st);
  } else {
    err = p.page_table ? (mass ? launch_rows<T, D, true, true>(p, st) : launch_rows<T, D, true, false>(p, st))
                       : (mass ? launch_rows<T, D, false, true>(p, st) : launch_rows<T, D, false, false>(p, st));
  }
  if (err != cudaSuccess) return SSA_ERR_CUDA;
  if (end) cudaEventRecord(end, st);
  note_launches(1);
  if (mass) {
    const int mass_blocks = (p.max_ctx + kMassKeys - 1) / kMassKeys, joins = p.n_splits > 1 ? (p.H * p.n_q + kMassWarps - 1) / kMassWarps : 0;
    err = launch_pdl(window_mass_kernel<TQ, D>, dim3((unsigned)(mass_blocks + joins), (unsigned)p.B), dim3(kMassThreads), st, p, mass_blocks);
  } else if (p.n_splits > 1) {
    err = launch_pdl(window_join_kernel<TQ, D>, dim3((unsigned)((p.H * p.n_q + kJoinWarps - 1) / kJoinWarps), (unsigned)p.B),
                     dim3(kJoinWarps * 32), st, p);
  } else {
    return SSA_OK;
  }
  if (err != cudaSuccess) return SSA_ERR_CUDA;
  note_launches(1);
  return SSA_OK;
}

static int32_t run_window(const ssa_attn_desc* d, const ssa_window* w, const void* q, const void* k, const void* v,
                          const int32_t* ctx_lens, void* out, float* lse, bool mass, const float* mass_in, float* mass_out,
                          int64_t mass_stride, float decay, void* ws, size_t ws_bytes, uint32_t* status, void* stream) {
  if (!d || !w || !q || !k || !v || !ctx_lens || !out || (mass && !mass_out)) return SSA_ERR_NULL;
  const int32_t rc = check_window(d, w, mass);
  if (rc != SSA_OK) return rc;
  if (mass && mass_stride < d->max_ctx) return SSA_ERR_SHAPE;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(ws)) return SSA_ERR_ALIGN;
  if (!ws || ws_bytes < window_bytes(d, w, mass)) return SSA_ERR_WORKSPACE;
  const ssa_paging* pg = w->paging;
  CUtensorMap maps[2];
  const int box_rows = pg ? std::min(pg->page_size, kTileKeys) : kTileKeys;
  const int64_t pool_rows = pg ? (int64_t)pg->n_pages * pg->page_size : d->max_ctx;
  WindowPlan pl;
  const bool tiles = tiles_pay(d, w, mass) && plan_window(d, w, mass, true, &pl) &&
                     tile_map(&maps[0], k, d->kv_dtype, d->D, pool_rows, d->k_stride_t, d->H_kv, d->k_stride_h, pg ? 1 : d->B,
                              d->k_stride_b, box_rows) &&
                     tile_map(&maps[1], v, d->kv_dtype, d->D, pool_rows, d->v_stride_t, d->H_kv, d->v_stride_h, pg ? 1 : d->B,
                              d->v_stride_b, box_rows);
  if (!tiles && !plan_window(d, w, mass, false, &pl)) return SSA_ERR_SHAPE;
  WindowParams p;
  p.block_rows = pl.block_rows;
  p.tile_keys = pl.keys;
  p.split_tiles = pl.fewest;
  p.q = q; p.k = k; p.v = v; p.out = out; p.lse = lse;
  p.ctx_lens = ctx_lens; p.q_lens = w->q_lens; p.page_table = pg ? pg->page_table : nullptr;
  char* at = static_cast<char*>(ws);
  p.ws_ml = reinterpret_cast<float2*>(at);
  p.ws_acc = reinterpret_cast<float*>(at + pl.ml_bytes);
  p.ws_s = reinterpret_cast<float*>(at + pl.ml_bytes + pl.acc_bytes);
  p.mass_in = mass_in; p.mass_out = mass_out; p.status = status;
  p.q_sb = d->q_stride_b; p.q_sh = d->q_stride_h; p.q_st = w->q_stride_t;
  p.o_sb = d->o_stride_b; p.o_sh = d->o_stride_h; p.o_st = w->o_stride_t;
  p.k_sb = d->k_stride_b; p.k_sh = d->k_stride_h; p.k_st = (int)d->k_stride_t;
  p.v_sb = d->v_stride_b; p.v_sh = d->v_stride_h; p.v_st = (int)d->v_stride_t;
  p.mass_stride = mass_stride;
  p.B = d->B; p.H = d->H; p.H_kv = d->H_kv; p.group = d->H / d->H_kv; p.n_q = w->n_q; p.max_ctx = d->max_ctx;
  p.window = w->window >= d->max_ctx ? 0 : w->window;                  // (no window at all; and no overflow in sums with it)
  p.sinks = std::min(w->sinks, d->max_ctx);
  p.n_splits = pl.n_splits; p.s_pitch = pl.s_pitch;
  p.page_table_stride = pg ? pg->page_table_stride : 0;
  p.n_pages = pg ? pg->n_pages : 0;
  p.page_shift = 0;
  while (pg && (1 << p.page_shift) < pg->page_size) ++p.page_shift;
  p.group_shift = -1;
  for (int i = 0; i < 16; ++i)
    if (p.group == 1 << i) p.group_shift = i;
  p.out_f32 = d->out_dtype == SSA_F32;
  p.scale_log2 = (d->scale > 0.f ? d->scale : 1.0f / sqrtf((float)d->D)) * kLog2e;
  p.decay = decay;
  cudaStream_t st = (cudaStream_t)stream;
  const CUtensorMap* m = tiles ? maps : nullptr;
  if (d->kv_dtype == SSA_FP8_E4M3)
    return d->D == 128 ? launch_window<Fp8E4M3, 128>(p, mass, m, box_rows, st) : launch_window<Fp8E4M3, 64>(p, mass, m, box_rows, st);
  if (d->kv_dtype == SSA_BF16)
    return d->D == 128 ? launch_window<__nv_bfloat16, 128>(p, mass, m, box_rows, st)
                       : launch_window<__nv_bfloat16, 64>(p, mass, m, box_rows, st);
  return d->D == 128 ? launch_window<__half, 128>(p, mass, m, box_rows, st) : launch_window<__half, 64>(p, mass, m, box_rows, st);
}

}  // namespace ssa

extern "C" {

size_t ssa_attn_window_workspace_bytes(const ssa_attn_desc* desc, const ssa_window* window) {
  return ssa::window_bytes(desc, window, false);
}

size_t ssa_attn_mass_workspace_bytes(const ssa_attn_desc* desc, const ssa_window* window) {
  return ssa::window_bytes(desc, window, true);
}

int32_t ssa_attn_window(const ssa_attn_desc* desc, const ssa_window* window, const void* q, const void* k_cache,
                        const void* v_cache, const int32_t* ctx_lens, void* out, float* lse, void* workspace,
                        size_t workspace_bytes, uint32_t* dev_status, void* stream) {
  return ssa::run_window(desc, window, q, k_cache, v_cache, ctx_lens, out, lse, false, nullptr, nullptr, 0, 0.f, workspace,
                         workspace_bytes, dev_status, stream);
}

int32_t ssa_attn_mass(const ssa_attn_desc* desc, const ssa_window* window, const void* q, const void* k_cache,
                      const void* v_cache, const int32_t* ctx_lens, void* out, float* lse, const float* mass_in,
                      float* mass_out, int64_t mass_stride, float decay, void* workspace, size_t workspace_bytes,
                      uint32_t* dev_status, void* stream) {
  return ssa::run_window(desc, window, q, k_cache, v_cache, ctx_lens, out, lse, true, mass_in, mass_out, mass_stride, decay,
                         workspace, workspace_bytes, dev_status, stream);
}

}  // extern "C"
