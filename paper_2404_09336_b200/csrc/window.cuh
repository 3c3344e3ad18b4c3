// What the kernels of the window attention share: parameters, and which positions a run of query rows sees.
#pragma once
#include "ssa_common.cuh"

namespace ssa {

struct WindowParams {
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

// Context length and new tokens of a request, clamped to what the call allows.
__device__ __forceinline__ void window_sizes(const WindowParams& p, int b, int& ctx, int& n_new, uint32_t& flags) {
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
template <bool kPaged>
__device__ __forceinline__ int64_t row_of(const WindowParams& p, const int32_t* table, int j) {
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
