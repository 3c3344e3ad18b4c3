// What the kernels of the window attention, and of attention over lists of blocks, share: parameters, and which positions a run
// of query rows sees.
#pragma once
#include "ssa_common.cuh"

namespace ssa {

struct WindowParams {
  static constexpr bool kListed = false;
  const void *q, *k, *v;
  void* out;
  float* lse;
  const int32_t *ctx_lens, *q_lens, *page_table;
  float2* ws_ml;            // [B][H][n_q][n_splits]: running maximum (log2 units) and sum of a split
  float* ws_acc;            // [B][H][n_q][n_splits][D]
  float* ws_s;              // [B][H][n_q][s_pitch]: scores in log2 units, for the kernel that adds the weights up
  const float* mass_in;
  float* mass_out;
  uint32_t* status;
  int64_t q_sb, q_sh, q_st, o_sb, o_sh, o_st, k_sb, k_sh, v_sb, v_sh, mass_stride;
  int k_st, v_st;
  int B, H, H_kv, group, n_q, max_ctx, window, sinks, n_splits, s_pitch;
  int page_table_stride, page_shift, n_pages, out_f32;
  int group_shift;                           // log2 of group, -1 where it is no power of two
  int block_rows, tile_keys, split_tiles;    // of the kernel that runs: query rows of a block, positions of a tile, see splits_used
  float scale_log2, decay;
};

// A 4-bit cache's scales, those of the row that starts at value o from byte o / 16 on.
struct Fp4Params : WindowParams { const uint8_t *k_scales, *v_scales; };

// Every token of a K/V head over its own list of blocks: no window, no sinks.
struct ListParams : Fp4Params {
  static constexpr bool kListed = true;
  const int32_t *list, *list_counts;         // [B][H_kv][n_q][budget], [B][H_kv][n_q]
  int budget, block_shift, parts;            // parts: runs of block_rows query heads that a K/V head's are cut into
};

// Context length and new tokens of a request, clamped to what the call allows.
template <typename Params>
__device__ __forceinline__ void window_sizes(const Params& p, int b, int& ctx, int& n_new, uint32_t& flags) {
  ctx = p.ctx_lens[b];
  n_new = p.q_lens ? p.q_lens[b] : p.n_q;
  if (ctx > p.max_ctx || n_new > p.n_q) flags |= SSA_DEV_BAD_COUNT;
  ctx = max(0, min(ctx, p.max_ctx));
  n_new = max(0, min(n_new, p.n_q));
}

// The positions that tokens t0..t1 of a request see between them, as tiles of `size` positions: `front` tiles from 0 (the
// sinks), then those from w0 on.  Where the two meet there is one run, from 0.  Token t sits at position first + t.
struct Seen {
  int size, front, w0, tiles;
  __device__ __forceinline__ Seen(const WindowParams& p, int size_, int first, int t0, int t1) : size(size_) {
    const int lo = first + t0, hi = first + t1;            // the first token's position may be negative: it sees nothing
    front = w0 = tiles = 0;
    if (t1 < t0 || hi < 0) return;
    const int from = p.window == 0 ? 0 : max(0, lo - p.window + 1);
    const int sinks = min(p.sinks, hi + 1);
    w0 = from / size * size;
    front = (sinks + size - 1) / size;
    if (front * size >= w0) front = w0 = 0;
    tiles = front + (hi - w0) / size + 1;
  }
  __device__ __forceinline__ int position(int tile) const { return tile < front ? tile * size : w0 + (tile - front) * size; }
};

// The blocks that token t of a K/V head has on its list, as tiles of 1 << tile_shift positions.
struct Listed {
  const int32_t* list;
  int count, per_shift, tile_shift, tiles, pos;              // pos: the token's own position
  int first = 0, mine = 0;                                   // entries first ... first + 31 are in the warp's lanes
  __device__ __forceinline__ Listed(const ListParams& p, int tile_size, int b, int hkv, int t, int pos_, uint32_t& flags) : pos(pos_) {
    const int64_t r = ((int64_t)b * p.H_kv + hkv) * p.n_q + t;
    list = p.list + r * p.budget;
    const int lane = threadIdx.x % 32;
    mine = lane < p.budget ? list[lane] : -1;                // (asked for before it is known how many there are)
    count = p.list_counts[r];
    if (count > p.budget) flags |= SSA_DEV_BAD_COUNT;
    count = pos < 0 ? 0 : max(0, min(count, p.budget));
    tile_shift = 31 - __clz(tile_size);
    per_shift = p.block_shift - tile_shift;
    tiles = count << per_shift;
  }
  // Where a tile starts; behind every position where its block is none that the token sees.  All lanes of a warp ask together.
  __device__ __forceinline__ int position(int tile, uint32_t& flags) {
    const int e = tile >> per_shift;
    if ((unsigned)(e - first) >= 32u) {
      first = e;
      mine = e + (int)(threadIdx.x % 32) < count ? list[e + threadIdx.x % 32] : -1;
    }
    const int block = __shfl_sync(~0u, mine, e - first);
    if ((unsigned)block > (unsigned)(pos >> (per_shift + tile_shift))) {
      flags |= SSA_DEV_BAD_INDEX;
      return kNowhere;
    }
    return (block << (per_shift + tile_shift)) + ((tile & ((1 << per_shift) - 1)) << tile_shift);
  }
  static constexpr int kNowhere = 1 << 30;
};

// A split works on at least split_tiles tiles, whatever the launch has room for.
__device__ __forceinline__ int splits_used(const WindowParams& p, int tiles) {
  return max(1, min(p.n_splits, tiles / p.split_tiles));
}

// The token of a row of a K/V head: rows are ordered by token, then head of the group.
__device__ __forceinline__ int token_of(const WindowParams& p, int row) {
  return p.group_shift >= 0 ? row >> p.group_shift : row / p.group;
}

// Tiles [x, y) of split s of n.
__device__ __forceinline__ int2 split_tiles(int tiles, int s, int n) {
  if (n == 1) return make_int2(0, tiles);
  return make_int2((int)((long long)tiles * s / n), (int)((long long)tiles * (s + 1) / n));
}

__device__ __forceinline__ bool sees(const WindowParams& p, int pos, int j) {
  return j <= pos && (p.window == 0 || j > pos - p.window || j < p.sinks);
}

// Pool row of logical position j, -1 where its page does not exist.
template <bool kPaged, typename Params>
__device__ __forceinline__ int64_t row_of(const Params& p, const int32_t* table, int j) {
  if constexpr (!kPaged) return j;
  const int page = table[j >> p.page_shift];
  if ((unsigned)page >= (unsigned)p.n_pages) return -1;
  return ((int64_t)page << p.page_shift) + (j & ((1 << p.page_shift) - 1));
}

template <typename TQ>
__device__ __forceinline__ void store_window_value(const WindowParams& p, int b, int h, int t, int d, float x) {
  const int64_t o = (int64_t)b * p.o_sb + (int64_t)h * p.o_sh + (int64_t)t * p.o_st + d;
  if (p.out_f32) reinterpret_cast<float*>(p.out)[o] = x;
  else reinterpret_cast<TQ*>(p.out)[o] = from_float<TQ>(x);
}

}  // namespace ssa
