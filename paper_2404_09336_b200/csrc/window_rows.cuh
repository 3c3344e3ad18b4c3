// The kernel for few query rows per K/V head (decode steps, drafted tokens) and what joins its splits: window attention over
// 16-bit, 8-bit and 4-bit caches, and attention over lists of blocks.  Included by the files of those calls.
#pragma once
#include <algorithm>
#include <type_traits>

#include "mma.cuh"
#include "window.cuh"

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
// of them (8 bytes of V's 64-byte rows).  So are 4-bit rows, a quarter of K's row and an eighth of V's to a lane; a tile has the
// scales of its rows behind the codes.
template <typename T, int D, int kGroups = 1>
struct RowShape {
  static constexpr int kBytes = kIsNarrow<T> ? 1 : 2;                  // of a value; of two values of 4 bits
  static constexpr int kRow = kIsFp4<T> ? D / 2 : D * kBytes, kChunks = kRow / 16, kScaleRow = kIsFp4<T> ? D / kScaleDims : 0;
  static constexpr int kNK = D / 64, kV = D / 8;                       // 8-bit: pieces of K per lane; elements of V's piece
  static constexpr int kHalves = kRow == 256 ? 1 : 2;                  // tiles of 16 positions, or of 32 where rows are short
  static constexpr int kKeys = 16 * kHalves;
  static constexpr int kCodes = 2 * kKeys * kRow, kTile = 2 * kKeys * (kRow + kScaleRow);   // bytes: of K and V of a tile
  // blocks that fit an SM by their registers, and bytes of a warp's ring: 64 KB a block (4-bit: 54 or 72), or 96
  static constexpr int kBlocks = kIsFp4<T> && kGroups == 1 ? 4 : kGroups <= 2 ? 3 : 2;
  static constexpr int kRingBytes = kBlocks == 4 ? 13824 : kBlocks == 3 ? (kIsFp4<T> ? 18432 : 16384) : 24576;
  __host__ __device__ static constexpr int64_t bytes(int64_t values) { return kIsFp4<T> ? values / 2 : values * kBytes; }
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
// 4-bit rows, two or four to 128 bytes: so do reads of K by eight lanes and of V (rows 2c, eighths g) by sixteen, or all.
template <typename T, int kChunks>
__device__ __forceinline__ int chunk_at(int key, int chunk) {
  if constexpr (kIsFp4<T>) return (key * kChunks + chunk) ^ (kChunks == 4 ? (key >> 1 & 3) << 1 : (key >> 2 & 1) << 1);
  return key * kChunks + turned<T, kChunks>(key, chunk);
}

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
template <int kSize>
__device__ __forceinline__ void copy_few(uint32_t to, const void* from, bool there) {     // 4 or 8 bytes
  asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;" ::"r"(to), "l"(from), "n"(kSize), "r"(there ? kSize : 0) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int kLeft>
__device__ __forceinline__ void copies_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(kLeft) : "memory"); }

// A row of bf16 queries over an 8-bit cache as fp16 values times a power of two that brings its largest to 2^14: what the others
// lose is below 2^-39 of that.  w: the row's part of this lane, the rest in the kLanes - 1 neighbouring lanes.  Returns the power's
// inverse.
template <int N, int kLanes = 4>
__device__ __forceinline__ float rows_to_half(uint32_t (&w)[N]) {
  uint32_t most = 0;                                         // bits of the largest finite magnitude
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const uint32_t a = w[i] & 0x7fffu, z = w[i] >> 16 & 0x7fffu;
    most = max(most, max(a < 0x7f80u ? a : 0u, z < 0x7f80u ? z : 0u));
  }
#pragma unroll
  for (int o = 1; o < kLanes; o *= 2) most = max(most, __shfl_xor_sync(~0u, most, o));
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
// kListed parameters: the rows are the query heads of one token, grid.x (splits x parts of them x tokens), the tiles those of the
// blocks on its list.
// kBoth: weights as a 16-bit value and the 16-bit rest.  Without (4-bit values, 16-bit outputs): rounded to fp16 once, 2^-11, less
// than the output is.  32 requests of up to 16384 positions, 32 heads over 8, 4-bit values: 119 us instead of 132, before splits were
// planned for four blocks to an SM (115 to 120 by the GPU since).
template <typename T, int D, bool kPaged, bool kMass, int kTeam, int kGroups, bool kBoth, typename Params>
__global__ void __launch_bounds__(kWarps * 32, (RowShape<T, D, kGroups>::kBlocks))
window_rows_kernel(const Params p) {
  constexpr bool kListed = Params::kListed;
  using TQ = typename Storage<T>::Query;
  using TP = typename Weight<T>::Type;                       // of the second contraction; of the first: TS
  using TS = std::conditional_t<kIsNarrow<T>, __half, TQ>;
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
  __shared__ int s_j0[kListed ? kTeams : 1][kListed ? kRing : 1];      // where a tile starts
  const int block = p.n_splits == 1 ? blockIdx.x : blockIdx.x / p.n_splits, split = blockIdx.x - block * p.n_splits;
  const int hkv = blockIdx.y, b = blockIdx.z;
  int row0 = block * kTeam * kRows, row_end = 0;
  if constexpr (kListed) {
    const int t = block / p.parts;
    row0 = t * p.group + (block - t * p.parts) * kTeam * kRows;
    row_end = (t + 1) * p.group;
  }
  grid_dependency_wait();
  grid_launch_dependents();
  uint32_t flags = 0;
  int ctx, n_new;
  window_sizes(p, b, ctx, n_new, flags);
  if (flags && p.status && split == 0 && row0 == 0 && hkv == 0 && threadIdx.x == 0) atomicOr(p.status, flags);
  const int rows = min(kTeam * kRows, (kListed ? min(row_end, n_new * p.group) : n_new * p.group) - row0);   // rows of tokens that exist
  if (rows <= 0) return;
  const int first = ctx - n_new, t_lo = token_of(p, row0), t_hi = token_of(p, row0 + rows - 1);
  auto seen = [&] {
    if constexpr (kListed) return Listed(p, kKeys, b, hkv, t_lo, first + t_lo, flags);
    else return Seen(p, kKeys, first, t_lo, t_hi);
  }();
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
                         RS::bytes((kPaged ? 0 : (int64_t)b * p.k_sb) + (int64_t)hkv * p.k_sh);
  const char* const vb = reinterpret_cast<const char*>(p.v) + my_chunk * 16 +
                         RS::bytes((kPaged ? 0 : (int64_t)b * p.v_sb) + (int64_t)hkv * p.v_sh);
  const int64_t k_step = RS::bytes(p.k_st), v_step = RS::bytes(p.v_st);
  // 4-bit: lanes my and my + kLanes copy the scales of row my % kKeys, of K (below kKeys), of V
  const int scale_key = my % kKeys, scale_copies = 2 * kKeys / kLanes;
  const uint8_t* scales[2] = {nullptr, nullptr};
  int64_t scale_step[2] = {0, 0};
  if constexpr (kIsFp4<T>) {
#pragma unroll
    for (int x = 0; x < scale_copies; ++x) {
      const bool of_v = my + x * kLanes >= kKeys;
      scales[x] = (of_v ? p.v_scales : p.k_scales) + ((kPaged ? 0 : (int64_t)b * (of_v ? p.v_sb : p.k_sb)) + (int64_t)hkv * (of_v ? p.v_sh : p.k_sh)) / kScaleDims;
      scale_step[x] = (of_v ? p.v_st : p.k_st) / kScaleDims;
    }
  }
  auto load_scales = [&](uint32_t to, int64_t row) {         // row < 0: there is none
    if constexpr (kIsFp4<T>) {
#pragma unroll
      for (int x = 0; x < scale_copies; ++x)
        copy_few<RS::kScaleRow>(to + RS::kCodes + (my + x * kLanes) * RS::kScaleRow, scales[x] + (row < 0 ? 0 : row * scale_step[x]), row >= 0);
    }
  };
  auto load = [&](int n) {
    if (n < n_tiles) {
      const int stage = n % kRing;
      int j0;
      if constexpr (kListed) j0 = seen.position(range.x + team + n * kTeams, flags);
      else j0 = seen.position(range.x + team + n * kTeams);
      const uint32_t to = ring_at + stage * RS::kTile;
      // tiles that are seen as a whole and lie on one page have rows in a row
      int64_t at = -1;
      if (j0 + kKeys - 1 <= hi && (j0 >= from || j0 + kKeys <= p.sinks) && (!kPaged || kKeys >> p.page_shift <= 1)) at = row_of<kPaged>(p, table, j0);
      unsigned have = ~0u;
      if (at >= 0) {
        if (copies) {
          const char *k = kb + (at + my_key) * k_step, *v = vb + (at + my_key) * v_step;
          if (kIsFp4<T> && k_step == RS::kRow && v_step == RS::kRow) {   // (rows side by side: fixed offsets)
            const uint32_t x = to + chunk_at<T, kChunks>(my_key, my_chunk) * 16;
#pragma unroll
            for (int i = 0; i < kPasses; ++i) {
              copy_16B(x + i * kPass * RS::kRow, k + i * kPass * RS::kRow, true);
              copy_16B(x + (i * kPass + kKeys) * RS::kRow, v + i * kPass * RS::kRow, true);
            }
          } else {
#pragma unroll
            for (int i = 0; i < kPasses; ++i) {
              const int key = i * kPass;
              const uint32_t x = kIsFp4<T> ? to + (chunk_at<T, kChunks>(my_key, my_chunk) + key * kChunks) * 16   // (key: a multiple of 8)
                                           : to + (my_key + key) * kChunks * 16 +
                                                 (turned<T, kChunks>(my_key, my_chunk) ^ turned<T, kChunks>(key, 0)) * 16;
              copy_16B(x, k, true);
              copy_16B(x + kKeys * RS::kRow, v, true);
              k += kPass * k_step;
              v += kPass * v_step;
            }
          }
        }
        load_scales(to, at + scale_key);
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
        load_scales(to, row);                                // (kKeys = 32: the lane's own row)
      }
      if (lane == 0 && member == 0) {
        s_have[team][stage] = have;
        if constexpr (kListed) s_j0[team][stage] = j0;
      }
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
      if constexpr (kIsNarrow<T>) {                          // step 4 u + i takes elements 4 i ... of the lane's piece 4 u + c;
        uint2 x = make_uint2(0, 0);                          // 4-bit: step i takes elements 4 i ... of the lane's quarter c
        if (there) x = *reinterpret_cast<const uint2*>(q + (kIsFp4<T> ? c * (D / 4) + i * 4 : (i / 4 * 4 + c) * 16 + i % 4 * 4));
        qb[y][2 * i] = x.x;
        qb[y][2 * i + 1] = x.y;
      } else {
        qb[y][2 * i] = there ? *reinterpret_cast<const uint32_t*>(q + 16 * i + 2 * c) : 0;
        qb[y][2 * i + 1] = there ? *reinterpret_cast<const uint32_t*>(q + 16 * i + 2 * c + 8) : 0;
      }
    }
    float back = 1.f;
    if constexpr (kIsNarrow<T>) back = rows_to_half(qb[y]);
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      unit[y][r] = kIsNarrow<T> ? p.scale_log2 * __shfl_sync(~0u, back, (2 * c + r) * 4) : p.scale_log2;
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

  // 4-bit: where the lane's part of K's row g is, of V's rows 2c and 2c + 1; rows 8 and 16 further on lie as many rows behind
  const int k_off = D == 128 ? chunk_at<T, kChunks>(g, c) * 16 : chunk_at<T, kChunks>(g, c / 2) * 16 + c % 2 * 8;
  const int v_off[2] = {chunk_at<T, kChunks>(2 * c, g * RS::kV / 32) * 16 + g * RS::kV / 2 % 16,
                        chunk_at<T, kChunks>(2 * c + 1, g * RS::kV / 32) * 16 + g * RS::kV / 2 % 16};

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
    const int stage = n % kRing;
    int j0;
    if constexpr (kListed) j0 = s_j0[team][stage];
    else j0 = seen.position(range.x + team + n * kTeams);
    load(n + kRing - 1);
    if (kTeam > 1 && wrows <= 0) continue;
    const uint32_t k_at = ring_at + stage * RS::kTile, v_at = k_at + kKeys * RS::kRow;
    const uint8_t* const kt = ring + stage * RS::kTile;
    const uint8_t* const vt = kt + kKeys * RS::kRow;
    const unsigned have = s_have[team][stage];
    float s[kHalves][kGroups][4];
#pragma unroll
    for (int x = 0; x < kHalves; ++x) {
      float s2[kGroups][4];                                  // (two chains of half the steps each; 4-bit: of the two halves)
#pragma unroll
      for (int y = 0; y < kGroups; ++y)
#pragma unroll
        for (int e = 0; e < 4; ++e) s[x][y][e] = s2[y][e] = 0.f;
      if constexpr (kIsFp4<T>) {
        // the lane's quarter of rows g and g + 8, as fp16 values: pairs 2 i and 2 i + 1 are step i's
        constexpr int kWords = D / 32;
        uint32_t codes[2][kWords], by[2][2];
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          const int rows_on = 16 * x + 8 * z;
          const uint8_t* scales = kt + RS::kCodes + (g + rows_on) * RS::kScaleRow;
          uint32_t pair;
          if constexpr (D == 128) {
            const uint4 w = *reinterpret_cast<const uint4*>(kt + k_off + rows_on * RS::kRow);
            codes[z][0] = w.x; codes[z][1] = w.y; codes[z][2] = w.z; codes[z][3] = w.w;
            pair = e4m3x2_to_half2(*reinterpret_cast<const uint16_t*>(scales + 2 * c));
          } else {
            const uint2 w = *reinterpret_cast<const uint2*>(kt + k_off + rows_on * RS::kRow);
            codes[z][0] = w.x; codes[z][1] = w.y;
            pair = e4m3x2_to_half2(scales[c]);
          }
          by[z][0] = __byte_perm(pair, 0, 0x1010);
          by[z][1] = __byte_perm(pair, 0, 0x3232);
        }
#pragma unroll
        for (int w = 0; w < kWords; ++w) {
          uint32_t a[4], z[4];
          e2m1x8_to_half2(codes[0][w], a);
          e2m1x8_to_half2(codes[1][w], z);
#pragma unroll
          for (int e = 0; e < 4; ++e) { a[e] = half2_mul(a[e], by[0][w / 2]); z[e] = half2_mul(z[e], by[1][w / 2]); }
#pragma unroll
          for (int i = 0; i < 2; ++i)
#pragma unroll
            for (int y = 0; y < kGroups; ++y)
              mma_16816<TS>(s[x][y], a[2 * i], z[2 * i], a[2 * i + 1], z[2 * i + 1], qb[y][2 * (2 * w + i)], qb[y][2 * (2 * w + i) + 1], s[x][y]);
        }
      } else if constexpr (kIsFp8<T>) {
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
        for (int e = 0; e < 4; ++e) s[x][y][e] = (kIsFp4<T> ? s[x][y][e] : s[x][y][e] + s2[y][e]) * unit[y][e % 2];
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
    bool higher = false;
#pragma unroll
    for (int y = 0; y < kGroups; ++y) higher |= top[y][0] > m[y][0] + kLazyRows || top[y][1] > m[y][1] + kLazyRows;   // (m = -inf: anything)
    if (__any_sync(~0u, higher)) {                           // (the lanes' maxima meet only then)
#pragma unroll
      for (int o = 4; o < 32; o *= 2)
#pragma unroll
        for (int y = 0; y < kGroups; ++y) {
          top[y][0] = fmaxf(top[y][0], __shfl_xor_sync(~0u, top[y][0], o));
          top[y][1] = fmaxf(top[y][1], __shfl_xor_sync(~0u, top[y][1], o));
        }
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
          ph[x][y][z] = transposed(w);
          if constexpr (kBoth) {
            const float2 back = unpack2<TP>(w);
            pl[x][y][z] = transposed(pack2<TP>(w0 - back.x, w1 - back.y));
          }
        }
    }
    bool odd = false;
#pragma unroll
    for (int x = 0; x < kHalves; ++x) {
      uint32_t vw[4][kIsFp8<T> ? RS::kV / 4 : 1];            // 8-bit rows: the pieces of keys 2c, 2c + 1, 2c + 8, 2c + 9
      // 4-bit rows: two keys' codes of a dimension in a byte, of the even and the odd dimensions of the lane's eighth, for keys 2c
      // and 2c + 1 and for 2c + 8 and 2c + 9; and the two keys' scales
      constexpr int kVWords = kIsFp4<T> ? RS::kV / 8 : 1;
      uint32_t both[2][2][kVWords], by[2];
      if constexpr (kIsFp4<T>) {
#pragma unroll
        for (int z = 0; z < 2; ++z) {
          uint32_t w[2][kVWords], scale[2];
#pragma unroll
          for (int y = 0; y < 2; ++y) {
            const uint8_t* row = vt + v_off[y] + (16 * x + 8 * z) * RS::kRow;
            if constexpr (D == 128) {
              const uint2 u = *reinterpret_cast<const uint2*>(row);
              w[y][0] = u.x; w[y][1] = u.y;
            } else {
              w[y][0] = *reinterpret_cast<const uint32_t*>(row);
            }
            scale[y] = kt[RS::kCodes + (kKeys + 2 * c + y + 16 * x + 8 * z) * RS::kScaleRow + g * RS::kV / kScaleDims];
          }
          by[z] = e4m3x2_to_half2(scale[0] | scale[1] << 8);
          if (careful && pair_not_finite<TP>(by[z])) {       // (values are finite but for their scale)
            odd = true;
            if (pair_not_finite<TP>(by[z] & 0xffffu)) by[z] &= 0xffff0000u;
            if (pair_not_finite<TP>(by[z] & 0xffff0000u)) by[z] &= 0xffffu;
          }
#pragma unroll
          for (int i = 0; i < kVWords; ++i) {
            both[z][0][i] = (w[0][i] & 0x0f0f0f0fu) | (w[1][i] << 4 & 0xf0f0f0f0u);
            both[z][1][i] = (w[0][i] >> 4 & 0x0f0f0f0fu) | (w[1][i] & 0xf0f0f0f0u);
          }
        }
      }
      uint32_t vh[2][2][4];                                  // four bytes of each, as fp16 values
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
        if constexpr (kIsFp4<T>) {
          if (i % 4 == 0) {
#pragma unroll
            for (int z = 0; z < 2; ++z)
#pragma unroll
              for (int o = 0; o < 2; ++o) e2m1x8_to_half2(both[z][o][i / 4], vh[z][o]);
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) a[e] = half2_mul(vh[e / 2][e % 2][i % 4], by[e / 2]);
        } else if constexpr (kIsFp8<T>) {
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
        if (!kIsFp4<T> && careful) {
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
        if constexpr (kBoth) {
#pragma unroll
          for (int y = 0; y < kGroups; ++y) mma_16816<TP>(acc[y][i], a[0], a[1], a[2], a[3], pl[x][y][0], pl[x][y][1], acc[y][i]);
        }
      }
    }
    if (careful && __any_sync(~0u, odd)) {                   // add what was taken out, element by element
#pragma unroll 1
      for (int key = 0; key < kKeys; ++key)
#pragma unroll
        for (int i = 0; i < kTiles; ++i)
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            const int d = kIsNarrow<T> ? g * RS::kV + 2 * i + z : 16 * i + g + 8 * z, at = (int)RS::bytes(d);
            const uint8_t* v = vt + chunk_at<T, kChunks>(key, at / 16) * 16 + at % 16;
            float f;
            if constexpr (kIsFp4<T>) {                       // (finite but for its scale)
              const float2 pair = e2m1x2_to_float2(*v);
              f = (z ? pair.y : pair.x) * e4m3x2_to_float2(kt[RS::kCodes + (kKeys + key) * RS::kScaleRow + d / kScaleDims]).x;
            } else if constexpr (kIsFp8<T>) f = e4m3x2_to_float2(*v).x;
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
        for (int z = 0; z < 2; ++z) s_acc[warp][mine][kIsNarrow<T> ? g * RS::kV + 2 * i + z : 16 * i + g + 8 * z] = acc[y][i][2 * z + r];
    }
  if ((kPaged || kListed) && p.status && (flags & (SSA_DEV_BAD_INDEX | SSA_DEV_BAD_COUNT))) atomicOr(p.status, flags);
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

// Splits that query row (h, t) of request b was served by.
template <typename Params>
__device__ __forceinline__ int row_splits(const Params& p, int b, int h, int t, int ctx, int n_new) {
  if constexpr (Params::kListed) {
    uint32_t flags = 0;
    return splits_used(p, Listed(p, p.tile_keys, b, h / p.group, t, ctx - n_new + t, flags).tiles);
  }
  const int row0 = (t * p.group + h % p.group) / p.block_rows * p.block_rows, rows = min(p.block_rows, n_new * p.group - row0);
  return splits_used(p, Seen(p, p.tile_keys, ctx - n_new, token_of(p, row0), token_of(p, row0 + rows - 1)).tiles);
}

// Joins the splits of query row `row` (of H n_q) of a request: a warp, whose lanes have D / 32 dimensions each.  The first few
// splits are asked for before it is known how many there are: they have their place, and what nothing was written to is not
// used.  Rows with one split are finished already.
template <typename TQ, int D, typename Params>
__device__ __forceinline__ void join_rows(const Params& p, int b, int row) {
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
  const int n = row_splits(p, b, h, t, ctx, n_new);
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

template <typename TQ, int D, typename Params>
__global__ void __launch_bounds__(kJoinWarps * 32)
window_join_kernel(const Params p) {
  grid_dependency_wait();
  grid_launch_dependents();
  join_rows<TQ, D>(p, blockIdx.y, blockIdx.x * kJoinWarps + threadIdx.x / 32);
}

// The same where there are many splits and few rows, of the calls over 4-bit values and lists: a block per query row, whose warps take
// splits in turn, two at a time, and meet in shared memory.  One request of 16384 positions, 32 heads over 8, 4-bit values, 64 splits:
// 14.4 us in all instead of 17.6.
constexpr int kManySplits = 8, kWideWarps = 8;

template <typename TQ, int D, typename Params>
__global__ void __launch_bounds__(kWideWarps * 32)
window_join_wide_kernel(const Params p) {
  constexpr int kN = D / 32, kAhead = 4;
  __shared__ float s_acc[kWideWarps][D];
  __shared__ float2 s_ml[kWideWarps];
  const int row = blockIdx.x, b = blockIdx.y, lane = threadIdx.x % 32, warp = threadIdx.x / 32;
  const int h = p.n_q == 1 ? row : row / p.n_q, t = row - h * p.n_q;
  const int64_t at = (int64_t)b * p.H * p.n_q + row, slot = at * p.n_splits;
  grid_dependency_wait();
  grid_launch_dependents();
  // (asked for before it is known how many there are: all n_splits have their place)
  float2 ml[kAhead];
  float a[kAhead][kN];
  auto ask = [&](int i, int x) {
    if (i >= p.n_splits) return;
    ml[x] = p.ws_ml[slot + i];
    const float* from = p.ws_acc + (slot + i) * D + lane * kN;
#pragma unroll
    for (int y = 0; y < kN; y += 2) {
      const float2 f = *reinterpret_cast<const float2*>(from + y);
      a[x][y] = f.x; a[x][y + 1] = f.y;
    }
  };
#pragma unroll
  for (int x = 0; x < kAhead; ++x) ask(warp + x * kWideWarps, x);
  uint32_t flags = 0;
  int ctx, n_new;
  window_sizes(p, b, ctx, n_new, flags);
  if (t >= n_new) return;
  const int n = row_splits(p, b, h, t, ctx, n_new);
  if (n == 1) return;
  float M = neg_inf(), L = 0.f, A[kN];
#pragma unroll
  for (int y = 0; y < kN; ++y) A[y] = 0.f;
  for (int i0 = warp; i0 < n; i0 += kAhead * kWideWarps) {
#pragma unroll
    for (int x = 0; x < kAhead; ++x) {
      if (i0 + x * kWideWarps < n && ml[x].y != 0.f) {       // (a split without a weight adds nothing)
        const float top = fmaxf(M, ml[x].x), base = top == neg_inf() ? 0.f : top, w = fast_exp2(ml[x].x - base), old = fast_exp2(M - base);
        L = fmaf(L, old, ml[x].y * w);
#pragma unroll
        for (int y = 0; y < kN; ++y) A[y] = fmaf(A[y], old, a[x][y] * w);
        M = top;
      }
      ask(i0 + (kAhead + x) * kWideWarps, x);
    }
  }
  if (lane == 0) s_ml[warp] = make_float2(M, L);
#pragma unroll
  for (int y = 0; y < kN; ++y) s_acc[warp][lane * kN + y] = A[y];
  __syncthreads();
  if (threadIdx.x >= D) return;
  float top = neg_inf(), sum = 0.f, x = 0.f;
#pragma unroll
  for (int w = 0; w < kWideWarps; ++w) top = fmaxf(top, s_ml[w].x);
#pragma unroll
  for (int w = 0; w < kWideWarps; ++w) {
    const float by = s_ml[w].y == 0.f ? 0.f : fast_exp2(s_ml[w].x - top);
    sum = fmaf(s_ml[w].y, by, sum);
    x = by == 0.f ? x : fmaf(s_acc[w][threadIdx.x], by, x);
  }
  store_window_value<TQ>(p, b, h, t, threadIdx.x, sum == 0.f ? 0.f : x / sum);
  if (threadIdx.x == 0 && p.lse) p.lse[at] = sum == 0.f ? neg_inf() : (top + log2f(sum)) * kLn2;
}

// ---- host ------------------------------------------------------------------------------------------------------------
// Joins the splits of the calls over 4-bit values and lists.
template <typename TQ, int D, typename Params>
static cudaError_t launch_join(const Params& p, cudaStream_t st) {
  if (p.n_splits > kManySplits) return launch_pdl(window_join_wide_kernel<TQ, D, Params>, dim3((unsigned)(p.H * p.n_q), (unsigned)p.B), dim3(kWideWarps * 32), st, p);
  return launch_pdl(window_join_kernel<TQ, D, Params>, dim3((unsigned)((p.H * p.n_q + kJoinWarps - 1) / kJoinWarps), (unsigned)p.B), dim3(kJoinWarps * 32), st, p);
}
// Splits of the kernel for few rows: what n splits cost in units of one tile's time.  The work of all blocks, each with a start and
// an end, over the places that there are (two or three blocks to an SM), but no less than one block's; half a block's until the
// last is done (lengths differ: three quarters of the longest are taken for the mean); joining.  Tiles of 4-bit values take longer,
// and four blocks of one group fit an SM (32 requests of up to 16384 positions, 32 heads over 8: 113 us instead of 119 on one GPU).
inline long long rows_splits(long long n_tiles, long long blocks, int rows, bool fp4, long long most_splits) {
  const int teams = rows <= kMostGroups * kGroup ? kWarps : kWarps / 2;
  const bool four = fp4 && rows <= kGroup;
  const double steps = (double)n_tiles / teams, places = (four ? 4.0 : rows <= 2 * kGroup ? 3.0 : 2.0) * sm_count(), ends = four ? 3 : 5, join = 6;
  double least = 0;
  long long splits = 1;
  for (long long n = 1; n <= most_splits; ++n) {
    const double one = steps / n + ends, all = blocks * n * (0.75 * steps / n + ends) / places;
    const double cost = std::max(one, all) + 0.5 * one + (n > 1 ? join : 0);
    if (n == 1 || cost < least) { least = cost; splits = n; }
  }
  return splits;
}
inline size_t up256(size_t n) { return (n + 255) / 256 * 256; }
// The seen part of a 4-bit cache as pages of an fp16 one, in the workspace: of so many requests, or K/V heads of one request, at a time.
struct Fp4Expanded {
  int requests, heads;
  __half *k, *v;                 // [heads][head_rows][D]
  int32_t* table;                // [requests][table_stride]
  int64_t head_rows;             // requests most_tiles 128
  int most_tiles, table_stride, page_shift;
};
// Converts it, and attends to it (defined in fp4_attn.cu).
int32_t launch_expanded(const Fp4Params& p, const Fp4Expanded& x, int D, cudaStream_t st);
// (defined in fp4_attn.cu; box_rows: rows side by side for certain, for the tiles of 128 rows; 0: the kernel for few rows)
int32_t launch_window_fp4(const Fp4Params& p, int D, int box_rows, cudaStream_t st);

// What the calls' parameters have in common.
inline void fill_params(WindowParams& p, const ssa_attn_desc* d, int32_t n_q, int64_t q_stride_t, int64_t o_stride_t,
                        const int32_t* q_lens, const ssa_paging* pg, const void* q, const void* k, const void* v,
                        const int32_t* ctx_lens, void* out, float* lse, uint32_t* status) {
  p.q = q; p.k = k; p.v = v; p.out = out; p.lse = lse;
  p.ctx_lens = ctx_lens; p.q_lens = q_lens; p.page_table = pg ? pg->page_table : nullptr;
  p.status = status;
  p.q_sb = d->q_stride_b; p.q_sh = d->q_stride_h; p.q_st = q_stride_t;
  p.o_sb = d->o_stride_b; p.o_sh = d->o_stride_h; p.o_st = o_stride_t;
  p.k_sb = d->k_stride_b; p.k_sh = d->k_stride_h; p.k_st = (int)d->k_stride_t;
  p.v_sb = d->v_stride_b; p.v_sh = d->v_stride_h; p.v_st = (int)d->v_stride_t;
  p.B = d->B; p.H = d->H; p.H_kv = d->H_kv; p.group = d->H / d->H_kv; p.n_q = n_q; p.max_ctx = d->max_ctx;
  p.page_table_stride = pg ? pg->page_table_stride : 0;
  p.n_pages = pg ? pg->n_pages : 0;
  p.page_shift = 0;
  while (pg && (1 << p.page_shift) < pg->page_size) ++p.page_shift;
  p.group_shift = -1;
  for (int i = 0; i < 16; ++i)
    if (p.group == 1 << i) p.group_shift = i;
  p.out_f32 = d->out_dtype == SSA_F32;
  p.scale_log2 = (d->scale > 0.f ? d->scale : 1.0f / sqrtf((float)d->D)) * kLog2e;
}
// Positions of a tile of the kernel for few rows.
inline int rows_tile_keys(int D, int kv_dtype) { return D * (kv_dtype == SSA_FP8_E4M3 || kv_dtype == SSA_FP4_E2M1 ? 1 : 2) == 256 ? 16 : 32; }

template <typename Kernel, typename Params>
static cudaError_t launch_rows_kernel(Kernel kernel, const Params& p, dim3 grid, int bytes, int warp_rows, int D, cudaStream_t st) {
  const int smem = std::max(bytes, kWarps * warp_rows * (D + 4) * (int)sizeof(float));       // (the join's place)
  const cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, smem);
  return err != cudaSuccess ? err : launch_pdl_smem(kernel, grid, dim3(kWarps * 32), smem, st, p);
}

template <typename T, int D, bool kPaged, bool kMass, bool kBoth, typename Params>
static cudaError_t launch_rows(const Params& p, cudaStream_t st) {
  const dim3 grid((unsigned)((p.group * p.n_q + p.block_rows - 1) / p.block_rows * p.n_splits), (unsigned)p.H_kv, (unsigned)p.B);
  auto launch = [&](auto kernel, int bytes, int warp_rows) { return launch_rows_kernel(kernel, p, grid, bytes, warp_rows, D, st); };
  switch (p.block_rows / kGroup) {
    case 1: return launch(window_rows_kernel<T, D, kPaged, kMass, 1, 1, kBoth, Params>, RowShape<T, D, 1>::kSmem, kGroup);
    case 2: return launch(window_rows_kernel<T, D, kPaged, kMass, 1, 2, kBoth, Params>, RowShape<T, D, 2>::kSmem, 2 * kGroup);
    case 3: return launch(window_rows_kernel<T, D, kPaged, kMass, 1, 3, kBoth, Params>, RowShape<T, D, 3>::kSmem, 3 * kGroup);
    case 4: return launch(window_rows_kernel<T, D, kPaged, kMass, 1, 4, kBoth, Params>, RowShape<T, D, 4>::kSmem, 4 * kGroup);
    default: return launch(window_rows_kernel<T, D, kPaged, kMass, 2, 4, kBoth, Params>, RowShape<T, D, 4>::kSmem, 4 * kGroup);
  }
}


}  // namespace ssa
