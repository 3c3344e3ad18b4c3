// Attention of the newest tokens of every request, each over its own past: causal, within a sliding window, with the first
// positions (sinks) visible to all; and the same with the softmax weight of every position added up.
//
//   token t of n at position pos = ctx - n + t sees V(t) = { j <= pos : j > pos - window or j < sinks }
//   s_j = scale <q_t, K_j>,  out = sum_{V(t)} softmax(s)_j V_j,  lse = log sum_{V(t)} exp(s_j)
//   mass_out[j] = decay mass_in[j] + sum over heads and tokens of exp(s_j - lse)
//
// window_rows_kernel serves few query rows per K/V head (decode steps, drafted tokens): all of a K/V head's query heads and
// tokens are rows of one warp-level m16n8k16 tile, so a cached row is read once for sixteen of them.  HBM bounds it.
// window_tile_kernel (window_tile.cuh) serves many: prompt chunks.  The tensor cores bound it.
#include <algorithm>

#include "mma.cuh"
#include "window_tile.cuh"

namespace ssa {

constexpr int kRows = 16;              // query rows of a block: (token, head of the group) pairs
constexpr int kKeys = 16;              // positions of a warp's tile
constexpr int kWarps = 4;              // of a block; they take the block's tiles in turn
constexpr int kSplitTiles = 16;        // fewest tiles worth a split of their own

// The weights enter the second contraction as a 16-bit value plus the 16-bit rest, so that the sums keep 16 bits (bf16) or 22
// (fp16) of each.  fp16 has little range below 1: its weights are scaled by 2^13, which the sum divides out again.
template <typename T> struct Weight { using Type = __half; static constexpr float kShift = 13.f; };
template <> struct Weight<__nv_bfloat16> { using Type = __nv_bfloat16; static constexpr float kShift = 0.f; };

// How a lane's pieces of a cache row are cut.  The order of the dimensions within a contraction is free as long as both sides
// agree, so lanes take whole 16-byte pieces.
template <typename T, int D>
struct RowPieces {
  static constexpr int kK = kIsFp8<T> ? 16 : 8;                        // elements of a piece of K, 4 lanes per row
  static constexpr int kNK = D / (4 * kK);
  static constexpr int kV = kIsFp8<T> && D == 128 ? 16 : 8;            // elements of a piece of V, 8 lanes per row
  static constexpr int kNV = D / (8 * kV);
  static constexpr int kVWords = kV * (kIsFp8<T> ? 1 : 2) / 4;
};

template <int kWords>
__device__ __forceinline__ void load_words(uint32_t (&w)[kWords], const void* p) {
  if constexpr (kWords == 4) {
    const uint4 x = ld_stream_16B(p);
    w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
  } else {
    static_assert(kWords == 2, "");
    asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0,%1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
  }
}

// Two e4m3 values -> two bf16 or two fp16 values (exact).
__device__ __forceinline__ uint32_t e4m3x2_to_half2(uint32_t pair) {
  uint32_t h2;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(h2) : "h"((unsigned short)pair));
  return h2;
}
__device__ __forceinline__ uint32_t e4m3x2_to_bf162(uint32_t pair) {
  const float2 f = e4m3x2_to_float2(pair);
  return pack2<__nv_bfloat16>(f.x, f.y);
}

// Whether one of two 16-bit values is infinite or NaN.
template <typename T> __device__ __forceinline__ bool pair_not_finite(uint32_t w);
template <> __device__ __forceinline__ bool pair_not_finite<__nv_bfloat16>(uint32_t w) {
  return (w & 0x7f80u) == 0x7f80u || (w & 0x7f800000u) == 0x7f800000u;
}
template <> __device__ __forceinline__ bool pair_not_finite<__half>(uint32_t w) {
  return (w & 0x7c00u) == 0x7c00u || (w & 0x7c000000u) == 0x7c000000u;
}

// grid (splits x row tiles, H_kv, B).  Fragments come straight from global memory: with the lane layout below, a load
// instruction takes whole 32-byte sectors, and no value passes through shared memory before the warps' results are joined.
//   S[16 rows, 8 keys] += Q . K^T   lane 4g+c holds key g's pieces c, c+4, ... ; step s of the contraction takes four of
//                                   their elements from every lane, and Q's registers follow the same order
//   O[16 rows, 8 dims] += P . V     lane 4g+c holds, of keys 2c, 2c+1, 2c+8, 2c+9, the pieces g, g+8, ... ; dimension e of
//                                   all lanes' pieces is one tile of eight
template <typename T, int D, bool kPaged, bool kMass>
__global__ void __launch_bounds__(kWarps * 32, 2)
window_rows_kernel(const WindowParams p) {
  using TQ = typename Storage<T>::Query;
  using TP = typename Weight<T>::Type;
  using RP = RowPieces<T, D>;
  constexpr float kShift = Weight<T>::kShift;
  constexpr int kSteps = D / 16, kBytes = kIsFp8<T> ? 1 : 2, kTiles = RP::kNV * RP::kV;
  __shared__ float s_acc[kWarps][kRows][D + 4];
  __shared__ float2 s_ml[kWarps][kRows];

  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32, g = lane / 4, c = lane % 4;
  const int split = blockIdx.x % p.n_splits, row0 = blockIdx.x / p.n_splits * kRows;
  const int hkv = blockIdx.y, b = blockIdx.z;
  grid_dependency_wait();
  grid_launch_dependents();
  uint32_t flags = 0;
  int ctx, n_new;
  window_sizes(p, b, ctx, n_new, flags);
  if (flags && p.status && split == 0 && row0 == 0 && hkv == 0 && threadIdx.x == 0) atomicOr(p.status, flags);
  const int rows = min(kRows, n_new * p.group - row0);       // rows of tokens that exist
  if (rows <= 0) return;
  const int first = ctx - n_new;
  const Seen seen(p, kKeys, first, row0 / p.group, (row0 + rows - 1) / p.group);
  const int n_splits = splits_used(p, seen.tiles);
  if (split >= n_splits) return;
  const int2 range = split_tiles(seen.tiles, split, n_splits);

  // my two rows of every tile: positions (a row that does not exist sees nothing) and the queries' registers
  int pos[2];
  uint32_t qa[kSteps][4];
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    const int row = row0 + g + 8 * r, t = row / p.group, h = hkv * p.group + row % p.group;
    const bool there = g + 8 * r < rows;
    pos[r] = there ? first + t : -1;
    const TQ* q = reinterpret_cast<const TQ*>(p.q) + (int64_t)b * p.q_sb + (int64_t)h * p.q_sh + (int64_t)t * p.q_st;
#pragma unroll
    for (int u = 0; u < RP::kNK; ++u)
#pragma unroll
      for (int i = 0; i < RP::kK / 4; ++i) {
        uint2 x = make_uint2(0, 0);
        if (there) x = *reinterpret_cast<const uint2*>(q + (u * 4 + c) * RP::kK + 4 * i);
        qa[u * (RP::kK / 4) + i][r] = x.x;
        qa[u * (RP::kK / 4) + i][r + 2] = x.y;
      }
  }
  // every row of the tile sees all of [all_lo, lo]; the sinks as well
  const int lo = first + row0 / p.group, hi = first + (row0 + rows - 1) / p.group;
  const int all_lo = p.window == 0 ? 0 : hi - p.window + 1;

  const int32_t* table = kPaged ? p.page_table + (int64_t)b * p.page_table_stride : nullptr;
  const char* kb = reinterpret_cast<const char*>(p.k) + ((kPaged ? 0 : (int64_t)b * p.k_sb) + (int64_t)hkv * p.k_sh) * kBytes;
  const char* vb = reinterpret_cast<const char*>(p.v) + ((kPaged ? 0 : (int64_t)b * p.v_sb) + (int64_t)hkv * p.v_sh) * kBytes;

  float acc[kTiles][4], m[2], l[2];
  uint32_t kw[2][RP::kNK][4], vw[4][RP::kNV][RP::kVWords];
  int64_t k_row[2], v_row[4];                                // rows of the tile that is loaded next; -1: not read
  auto find = [&](int tile) {
    const int j0 = seen.position(tile);
    // what no row sees is not read: it may hold anything, or have no page
    auto any = [&](int j) { return j <= hi && (p.window == 0 || j > lo - p.window || j < p.sinks); };
#pragma unroll
    for (int x = 0; x < 2; ++x) {
      const int j = j0 + g + 8 * x;
      k_row[x] = any(j) ? row_of<kPaged>(p, table, j) : -1;
      if (kPaged && any(j) && k_row[x] < 0) flags |= SSA_DEV_BAD_INDEX;
    }
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const int j = j0 + 2 * c + (x & 1) + 4 * (x & 2);
      v_row[x] = any(j) ? row_of<kPaged>(p, table, j) : -1;
    }
  };
  auto load_k = [&]() {
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int u = 0; u < RP::kNK; ++u) {
        if (k_row[x] >= 0) load_words(kw[x][u], kb + (k_row[x] * p.k_st + (u * 4 + c) * RP::kK) * kBytes);
        else kw[x][u][0] = kw[x][u][1] = kw[x][u][2] = kw[x][u][3] = 0;
      }
  };
  auto load_v = [&]() {
#pragma unroll
    for (int x = 0; x < 4; ++x)
#pragma unroll
      for (int u = 0; u < RP::kNV; ++u) {
        if (v_row[x] >= 0) load_words(vw[x][u], vb + (v_row[x] * p.v_st + (u * 8 + g) * RP::kV) * kBytes);
        else
#pragma unroll
          for (int i = 0; i < RP::kVWords; ++i) vw[x][u][i] = 0;
      }
  };

  // An infinite or NaN element of V must not reach rows that do not see it (0 * inf), and has to stay infinite for those that do
  // (its product with a weight's two parts may be inf - inf).  Sums that come out finite met none; else the warp goes through
  // its tiles once more and takes such elements out of the contraction, to add them to the rows that see them.
  bool careful = false;
again:
#pragma unroll
  for (int i = 0; i < kTiles; ++i)
#pragma unroll
    for (int e = 0; e < 4; ++e) acc[i][e] = 0.f;
  m[0] = m[1] = neg_inf();
  l[0] = l[1] = 0.f;
  int tile = range.x + warp;
  if (tile < range.y) { find(tile); load_k(); load_v(); }
  for (; tile < range.y; tile += kWarps) {
    const int j0 = seen.position(tile);
    float s[2][4];
#pragma unroll
    for (int x = 0; x < 2; ++x) {
#pragma unroll
      for (int e = 0; e < 4; ++e) s[x][e] = 0.f;
#pragma unroll
      for (int u = 0; u < RP::kNK; ++u) {
        if constexpr (kIsFp8<T>) {
#pragma unroll
          for (int i = 0; i < 4; ++i)
            mma_16816<TQ>(s[x], qa[u * 4 + i][0], qa[u * 4 + i][1], qa[u * 4 + i][2], qa[u * 4 + i][3],
                          e4m3x2_to_bf162(kw[x][u][i] & 0xffffu), e4m3x2_to_bf162(kw[x][u][i] >> 16), s[x]);
        } else {
#pragma unroll
          for (int i = 0; i < 2; ++i)
            mma_16816<TQ>(s[x], qa[u * 2 + i][0], qa[u * 2 + i][1], qa[u * 2 + i][2], qa[u * 2 + i][3], kw[x][u][2 * i],
                          kw[x][u][2 * i + 1], s[x]);
        }
      }
    }
    bool all_there = true;
    bool skipped[2][2] = {{false, false}, {false, false}};   // pages that do not exist: the keys of my scores
    if constexpr (kPaged) {
      const unsigned have0 = __ballot_sync(~0u, k_row[0] >= 0), have1 = __ballot_sync(~0u, k_row[1] >= 0);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        skipped[0][e] = !((have0 >> ((2 * c + e) * 4)) & 1);
        skipped[1][e] = !((have1 >> ((2 * c + e) * 4)) & 1);
      }
      all_there = (have0 & have1) == ~0u;
    }
    const int next = tile + kWarps;
    int64_t v_now[4];
#pragma unroll
    for (int x = 0; x < 4; ++x) v_now[x] = v_row[x];
    if (next < range.y) { find(next); load_k(); }

    // scores in log2 units; what a row does not see is -inf
    const bool whole = all_there && j0 + kKeys - 1 <= lo && (j0 >= all_lo || j0 + kKeys <= p.sinks);
    float top[2] = {m[0], m[1]};
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int r = e / 2;
        s[x][e] *= p.scale_log2;
        if (!whole && (skipped[x][e & 1] || !sees(p, pos[r], j0 + 8 * x + 2 * c + (e & 1)))) s[x][e] = neg_inf();
        top[r] = fmaxf(top[r], s[x][e]);
      }
    if constexpr (kMass) {
#pragma unroll
      for (int r = 0; r < 2; ++r)
        if (g + 8 * r < rows) {
          const int row = row0 + g + 8 * r, t = row / p.group, h = hkv * p.group + row % p.group;
          float* to = p.ws_s + (((int64_t)b * p.H + h) * p.n_q + t) * p.s_pitch + j0 + 2 * c;
#pragma unroll
          for (int x = 0; x < 2; ++x) *reinterpret_cast<float2*>(to + 8 * x) = make_float2(s[x][2 * r], s[x][2 * r + 1]);
        }
    }
    float shift[2], alpha[2];
#pragma unroll
    for (int r = 0; r < 2; ++r) {
      top[r] = fmaxf(top[r], __shfl_xor_sync(~0u, top[r], 1));
      top[r] = fmaxf(top[r], __shfl_xor_sync(~0u, top[r], 2));
      shift[r] = (top[r] == neg_inf() ? 0.f : top[r]) - kShift;
      alpha[r] = fast_exp2(m[r] - kShift - shift[r]);        // (m = -inf: 0)
    }
    if (__any_sync(~0u, top[0] != m[0] || top[1] != m[1])) {
#pragma unroll
      for (int i = 0; i < kTiles; ++i)
#pragma unroll
        for (int e = 0; e < 4; ++e) acc[i][e] *= alpha[e / 2];
      l[0] *= alpha[0];
      l[1] *= alpha[1];
      m[0] = top[0];
      m[1] = top[1];
    }
    uint32_t ph[4], pl[4];                                   // the weights as the A operand, and what their rounding left
#pragma unroll
    for (int x = 0; x < 2; ++x)
#pragma unroll
      for (int r = 0; r < 2; ++r) {
        const float w0 = fast_exp2(s[x][2 * r] - shift[r]), w1 = fast_exp2(s[x][2 * r + 1] - shift[r]);
        l[r] += w0 + w1;
        ph[2 * x + r] = pack2<TP>(w0, w1);
        const float2 back = unpack2<TP>(ph[2 * x + r]);
        pl[2 * x + r] = pack2<TP>(w0 - back.x, w1 - back.y);
      }
    bool odd = false;
    if (careful) {
#pragma unroll
      for (int x = 0; x < 4; ++x)
#pragma unroll
        for (int u = 0; u < RP::kNV; ++u)
#pragma unroll
          for (int i = 0; i < RP::kVWords; ++i) {
            if constexpr (kIsFp8<T>) {
#pragma unroll
              for (int y = 0; y < 32; y += 8) {
                if (((vw[x][u][i] >> y) & 0x7fu) == 0x7fu) { odd = true; vw[x][u][i] &= ~(0xffu << y); }
              }
            } else if (pair_not_finite<TQ>(vw[x][u][i])) {
              odd = true;
              if (pair_not_finite<TQ>(vw[x][u][i] & 0xffffu)) vw[x][u][i] &= 0xffff0000u;
              if (pair_not_finite<TQ>(vw[x][u][i] & 0xffff0000u)) vw[x][u][i] &= 0xffffu;
            }
          }
    }
#pragma unroll
    for (int u = 0; u < RP::kNV; ++u)
#pragma unroll
      for (int e = 0; e < RP::kV; ++e) {
        uint32_t b0, b1;
        if constexpr (kIsFp8<T>) {
          // byte e of the four keys' pieces, two keys to a word
          const uint32_t a = __byte_perm(vw[0][u][e / 4], vw[1][u][e / 4], (e % 4) | ((e % 4 + 4) << 4));
          const uint32_t z = __byte_perm(vw[2][u][e / 4], vw[3][u][e / 4], (e % 4) | ((e % 4 + 4) << 4));
          b0 = e4m3x2_to_half2(a & 0xffffu);
          b1 = e4m3x2_to_half2(z & 0xffffu);
        } else {
          constexpr uint32_t kLow = 0x5410, kHigh = 0x7632;
          b0 = __byte_perm(vw[0][u][e / 2], vw[1][u][e / 2], e & 1 ? kHigh : kLow);
          b1 = __byte_perm(vw[2][u][e / 2], vw[3][u][e / 2], e & 1 ? kHigh : kLow);
        }
        float (&o)[4] = acc[u * RP::kV + e];
        mma_16816<TP>(o, ph[0], ph[1], ph[2], ph[3], b0, b1, o);
        mma_16816<TP>(o, pl[0], pl[1], pl[2], pl[3], b0, b1, o);
      }
    if (careful && __any_sync(~0u, odd)) {                   // add what was taken out, element by element
      for (int y = 0; y < kKeys; ++y) {
        const int from = (y % 8) / 2, which = (y % 2) + 2 * (y / 8);   // the lane that holds this key's row, and which of its four
        const int64_t mine = which == 0 ? v_now[0] : which == 1 ? v_now[1] : which == 2 ? v_now[2] : v_now[3];
        const int64_t row = __shfl_sync(~0u, mine, from);
        if (row < 0) continue;
#pragma unroll
        for (int u = 0; u < RP::kNV; ++u)
#pragma unroll
          for (int e = 0; e < RP::kV; ++e)
#pragma unroll
            for (int z = 0; z < 2; ++z) {
              const int d = (u * 8 + 2 * c + z) * RP::kV + e;
              float x;
              if constexpr (kIsFp8<T>) x = e4m3x2_to_float2(reinterpret_cast<const uint8_t*>(vb)[row * p.v_st + d]).x;
              else x = to_float(reinterpret_cast<const TQ*>(vb)[row * p.v_st + d]);
              if (!isfinite(x)) {
#pragma unroll
                for (int r = 0; r < 2; ++r)
                  if (sees(p, pos[r], j0 + y)) acc[u * RP::kV + e][2 * r + z] += x;
              }
            }
      }
    }
    if (next < range.y) load_v();
  }
  if (!careful) {
    bool finite = true;
#pragma unroll
    for (int i = 0; i < kTiles; ++i)
#pragma unroll
      for (int e = 0; e < 4; ++e) finite &= fabsf(acc[i][e]) <= 3.402823466e38f;
    if (__any_sync(~0u, !finite)) {
      careful = true;
      goto again;
    }
  }

  // the warps' results, joined by the block
#pragma unroll
  for (int r = 0; r < 2; ++r) {
    l[r] += __shfl_xor_sync(~0u, l[r], 1);
    l[r] += __shfl_xor_sync(~0u, l[r], 2);
    if (c == 0) s_ml[warp][g + 8 * r] = make_float2(m[r] - kShift, l[r]);   // what acc and l are relative to
#pragma unroll
    for (int u = 0; u < RP::kNV; ++u)
#pragma unroll
      for (int z = 0; z < 2; ++z)
#pragma unroll
        for (int e = 0; e < RP::kV; ++e) s_acc[warp][g + 8 * r][(u * 8 + 2 * c + z) * RP::kV + e] = acc[u * RP::kV + e][2 * r + z];
  }
  if (kPaged && p.status && (flags & SSA_DEV_BAD_INDEX)) atomicOr(p.status, SSA_DEV_BAD_INDEX);
  __syncthreads();
  for (int i = warp; i < rows; i += kWarps) {
    float M = neg_inf(), L = 0.f, w[kWarps];
#pragma unroll
    for (int x = 0; x < kWarps; ++x) M = fmaxf(M, s_ml[x][i].x);
#pragma unroll
    for (int x = 0; x < kWarps; ++x) {
      w[x] = s_ml[x][i].y == 0.f ? 0.f : fast_exp2(s_ml[x][i].x - M);
      L += s_ml[x][i].y * w[x];
    }
    const int row = row0 + i, t = row / p.group, h = hkv * p.group + row % p.group;
    const int64_t at = ((int64_t)b * p.H + h) * p.n_q + t, slot = at * p.n_splits + split;
    for (int d = lane; d < D; d += 32) {
      float A = 0.f;
#pragma unroll
      for (int x = 0; x < kWarps; ++x) A += s_acc[x][i][d] * w[x];
      if (n_splits == 1) store_window_value<TQ>(p, b, h, t, d, L == 0.f ? 0.f : A / L);
      else p.ws_acc[slot * D + d] = A;
    }
    if (lane == 0) {
      if (n_splits == 1 && p.lse) p.lse[at] = L == 0.f ? neg_inf() : (M + log2f(L)) * kLn2;
      if (n_splits > 1 || kMass) p.ws_ml[slot] = make_float2(M, L);
    }
  }
}

// Joins the splits of query row (b, h, t): a thread per dimension.  Rows with one split are finished already.
template <typename TQ, int D>
__device__ void join_row(const WindowParams& p, int b, int h, int t) {
  uint32_t flags = 0;
  int ctx, n_new;
  window_sizes(p, b, ctx, n_new, flags);
  if (t >= n_new) return;
  const int row0 = (t * p.group + h % p.group) / p.block_rows * p.block_rows, rows = min(p.block_rows, n_new * p.group - row0);
  const Seen seen(p, p.tile_keys, ctx - n_new, row0 / p.group, (row0 + rows - 1) / p.group);
  const int n = splits_used(p, seen.tiles), d = threadIdx.x;
  if (n == 1 || d >= D) return;
  const int64_t at = ((int64_t)b * p.H + h) * p.n_q + t, slot = at * p.n_splits;
  float M = neg_inf(), L = 0.f, A = 0.f;
  for (int i = 0; i < n; ++i) M = fmaxf(M, p.ws_ml[slot + i].x);
#pragma unroll 8
  for (int i = 0; i < n; ++i) {
    const float2 ml = p.ws_ml[slot + i];
    const float w = ml.y == 0.f ? 0.f : fast_exp2(ml.x - M);
    L = fmaf(ml.y, w, L);
    A = fmaf(p.ws_acc[(slot + i) * D + d], w, A);
  }
  store_window_value<TQ>(p, b, h, t, d, L == 0.f ? 0.f : A / L);
  if (d == 0 && p.lse) p.lse[at] = L == 0.f ? neg_inf() : (M + log2f(L)) * kLn2;
}

template <typename TQ, int D>
__global__ void __launch_bounds__(D)
window_join_kernel(const WindowParams p) {
  grid_dependency_wait();
  grid_launch_dependents();
  join_row<TQ, D>(p, blockIdx.y, blockIdx.x / p.n_q, blockIdx.x % p.n_q);
}

constexpr int kMassThreads = 256;

// Blocks x < mass_blocks of a request: one position per thread, its weights summed over tokens, then heads, in that order.
// The others join the splits of one query row each.
template <typename TQ, int D>
__global__ void __launch_bounds__(kMassThreads)
window_mass_kernel(const WindowParams p, const int mass_blocks) {
  __shared__ float s_lse[SSA_MASS_MAX_ROWS];
  const int b = blockIdx.y;
  grid_dependency_wait();
  grid_launch_dependents();
  if ((int)blockIdx.x >= mass_blocks) {
    const int row = blockIdx.x - mass_blocks;
    join_row<TQ, D>(p, b, row / p.n_q, row % p.n_q);
    return;
  }
  uint32_t flags = 0;
  int ctx, n_new;
  window_sizes(p, b, ctx, n_new, flags);
  const int j0 = blockIdx.x * kMassThreads;
  if (j0 >= ctx) return;
  const int n_rows = p.H * p.n_q, first = ctx - n_new;
  for (int i = threadIdx.x / 32; i < n_rows; i += kMassThreads / 32) {       // normalisers, a warp each
    const int h = i / p.n_q, t = i % p.n_q, lane = threadIdx.x % 32;
    if (t >= n_new) continue;
    const int row0 = (t * p.group + h % p.group) / kRows * kRows, rows = min(kRows, n_new * p.group - row0);
    const Seen seen(p, kKeys, first, row0 / p.group, (row0 + rows - 1) / p.group);
    const int n = splits_used(p, seen.tiles);
    const float2* ml = p.ws_ml + (((int64_t)b * p.H + h) * p.n_q + t) * p.n_splits;
    float M = neg_inf(), L = 0.f;
    for (int x = lane; x < n; x += 32) M = fmaxf(M, ml[x].x);
    for (int o = 16; o; o /= 2) M = fmaxf(M, __shfl_xor_sync(~0u, M, o));
    for (int x = lane; x < n; x += 32) L += ml[x].y == 0.f ? 0.f : ml[x].y * fast_exp2(ml[x].x - M);
    for (int o = 16; o; o /= 2) L += __shfl_xor_sync(~0u, L, o);
    if (lane == 0) s_lse[i] = L == 0.f ? __int_as_float(0x7f800000) : M + log2f(L);   // +inf: nothing seen, weights of zero
  }
  __syncthreads();
  const int j = j0 + threadIdx.x;
  if (j >= ctx) return;
  float sum = 0.f;
  for (int t = 0; t < n_new; ++t) {
    if (!sees(p, first + t, j)) continue;
    const float* s = p.ws_s + ((int64_t)b * p.H * p.n_q + t) * p.s_pitch + j;
    float part = 0.f;
#pragma unroll 8
    for (int h = 0; h < p.H; ++h) part += fast_exp2(s[(int64_t)h * p.n_q * p.s_pitch] - s_lse[h * p.n_q + t]);
    sum += part;
  }
  if (p.mass_in && j < first) sum = fmaf(p.decay, p.mass_in[(int64_t)b * p.mass_stride + j], sum);
  p.mass_out[(int64_t)b * p.mass_stride + j] = sum;
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
struct WindowPlan { bool tiles; int n_splits, s_pitch; size_t ml_bytes, acc_bytes, s_bytes, total_bytes; };

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
  if (w->n_q <= 0 || w->window < 0 || w->sinks < 0 || w->q_stride_t < 0 || w->o_stride_t < 0) return SSA_ERR_SHAPE;
  if (w->q_stride_t % 8 != 0 || w->o_stride_t % 8 != 0) return SSA_ERR_ALIGN;
  if ((long long)d->H * w->n_q > (mass ? (long long)SSA_MASS_MAX_ROWS : 1ll << 24)) return SSA_ERR_SHAPE;
  return w->paging ? check_paging(w->paging, d->max_ctx) : SSA_OK;
}

static size_t up256(size_t n) { return (n + 255) / 256 * 256; }

// More than two row tiles of the kernel for few rows (which would read the cache once for each) go to the tiles of 256.
static bool tiles_pay(const ssa_attn_desc* d, const ssa_window* w, bool mass) {
  return !mass && d->kv_dtype != SSA_FP8_E4M3 && (long long)(d->H / d->H_kv) * w->n_q > 2 * kRows &&
         (!w->paging || w->paging->page_size >= 8);          // (a box of a copy is eight rows at least)
}

static bool plan_window(const ssa_attn_desc* d, const ssa_window* w, bool mass, bool tiles, WindowPlan* pl) {
  pl->tiles = tiles;
  const int rows = tiles ? kBlockRows : kRows, keys = tiles ? kTileKeys : kKeys, fewest = tiles ? kTileSplit : kSplitTiles;
  const long long group = d->H / d->H_kv, row_tiles = (group * w->n_q + rows - 1) / rows;
  const long long blocks = row_tiles * d->H_kv * d->B, tokens = (rows - 1) / group + 2;
  const long long most = w->window == 0 ? d->max_ctx : std::min<long long>(d->max_ctx, (long long)w->window + w->sinks + tokens);
  const long long n_tiles = (most + keys - 1) / keys + 2;
  const long long wanted = tiles ? sm_count() / blocks : (4ll * sm_count() + blocks - 1) / blocks;
  pl->n_splits = (int)std::max(1ll, std::min({wanted, n_tiles / fewest, 256ll}));
  const size_t slots = (size_t)d->B * d->H * w->n_q * pl->n_splits;
  pl->ml_bytes = up256(slots * sizeof(float2));
  pl->acc_bytes = pl->n_splits > 1 ? up256(slots * d->D * sizeof(float)) : 0;
  pl->s_pitch = mass ? (d->max_ctx + kKeys - 1) / kKeys * kKeys : 0;
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
  const dim3 grid((unsigned)((p.group * p.n_q + kBlockRows - 1) / kBlockRows * p.n_splits), (unsigned)p.H_kv, (unsigned)p.B);
  auto kernel = p.page_table ? window_tile_kernel<T, D, true> : window_tile_kernel<T, D, false>;
  constexpr int kSmem = TileShape<D>::kSmem;
  const cudaError_t err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kSmem);
  if (err != cudaSuccess) return err;
  return launch_pdl_smem(kernel, grid, dim3(kTileThreads), kSmem, st, p, k_map, v_map, box_rows);
}

template <typename T, int D>
static int32_t launch_window(const WindowParams& p, bool mass, const CUtensorMap* maps, int box_rows, cudaStream_t st) {
  using TQ = typename Storage<T>::Query;
  const dim3 grid((unsigned)((p.group * p.n_q + kRows - 1) / kRows * p.n_splits), (unsigned)p.H_kv, (unsigned)p.B);
  cudaEvent_t begin, end;
  take_kernel_events(&begin, &end);
  if (begin) cudaEventRecord(begin, st);
  cudaError_t err = cudaErrorInvalidValue;
  if (maps) {
    if constexpr (!kIsFp8<T>) err = launch_tiles<T, D>(p, maps[0], maps[1], box_rows, st);
  } else if (p.page_table) {
    err = mass ? launch_pdl(window_rows_kernel<T, D, true, true>, grid, dim3(kWarps * 32), st, p)
               : launch_pdl(window_rows_kernel<T, D, true, false>, grid, dim3(kWarps * 32), st, p);
  } else {
    err = mass ? launch_pdl(window_rows_kernel<T, D, false, true>, grid, dim3(kWarps * 32), st, p)
               : launch_pdl(window_rows_kernel<T, D, false, false>, grid, dim3(kWarps * 32), st, p);
  }
  if (err != cudaSuccess) return SSA_ERR_CUDA;
  if (end) cudaEventRecord(end, st);
  note_launches(1);
  if (mass) {
    const int mass_blocks = (p.max_ctx + kMassThreads - 1) / kMassThreads;
    err = launch_pdl(window_mass_kernel<TQ, D>, dim3((unsigned)(mass_blocks + (p.n_splits > 1 ? p.H * p.n_q : 0)), (unsigned)p.B),
                     dim3(kMassThreads), st, p, mass_blocks);
  } else if (p.n_splits > 1) {
    err = launch_pdl(window_join_kernel<TQ, D>, dim3((unsigned)(p.H * p.n_q), (unsigned)p.B), dim3(D), st, p);
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
  p.block_rows = tiles ? kBlockRows : kRows;
  p.tile_keys = tiles ? kTileKeys : kKeys;
  p.split_tiles = tiles ? kTileSplit : kSplitTiles;
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
