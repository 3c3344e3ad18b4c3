// Window attention over a cache of 4-bit values (ssa_attn_window_fp4): the kernels of window_rows.cuh and window_tile.cuh for such rows.
#include "window_tile.cuh"

namespace ssa {

// ---- the seen part of a 4-bit cache in fp16 ---------------------------------------------------------------------------------
// Every block of 128 query rows that works on tiles converts the K and V rows that it sees.  Where many share them (prompt chunks)
// they are converted once instead, into pages of the workspace that the tiles then read: products of a code and a scale have six
// significant bits and are multiples of 2^-10 up to 2688, so that nothing is rounded, and outputs are those of tiles that convert.
// They take 512 MB of the workspace at most: requests, or K/V heads of one, go through it in turn.  HBM bounds it: 2.56 bytes a value.
// 8 requests' chunks of up to 509 tokens within a window of 4096, 8 K/V heads: some 36 us (5.4 TB/s), and 177 to 183 for the tiles; 49
// with 16 bytes of codes to a thread, whose stores then lie 64 bytes apart.  (To bf16, with weights of eight bits, the tiles took 5 us
// less: no queries to bring to fp16.)
constexpr int kExpandThreads = 256;

// grid (tiles of 128 positions that a request's tokens see between them, H_kv, B).  Page tables of the pages made: tile i of request b
// is rows (b most_tiles + i) 128 ...; where the cache has smaller pages these are as small, and missing where they are.
template <int D, bool kPaged>
__global__ void __launch_bounds__(kExpandThreads)
fp4_expand_kernel(const Fp4Params p, const Fp4Expanded x) {
  constexpr int kC = D / 8, kStep = kExpandThreads / kC, kEach = kTileKeys / kStep;    // pieces of a row; rows at a time; of a thread
  grid_dependency_wait();
  grid_launch_dependents();
  const int b = blockIdx.z, hkv = blockIdx.y, tile = blockIdx.x, tid = threadIdx.x;
  uint32_t flags = 0;
  int ctx, n_new;
  window_sizes(p, b, ctx, n_new, flags);
  const int first = ctx - n_new, hi = ctx - 1, from = p.window == 0 ? 0 : max(0, first - p.window + 1);
  const Seen seen(p, kTileKeys, first, 0, n_new - 1);
  if (tile >= seen.tiles) return;
  const int j0 = seen.position(tile);
  const int64_t to_row = ((int64_t)b * x.most_tiles + tile) * kTileKeys;
  const int32_t* table = kPaged ? p.page_table + (int64_t)b * p.page_table_stride : nullptr;
  auto is_seen = [&](int j) { return j <= hi && (j >= from || j < p.sinks); };
  if (hkv == 0 && tid < kTileKeys >> x.page_shift) {
    const int ja = j0 + (tid << x.page_shift), jz = ja + (1 << x.page_shift) - 1;
    const bool used = ja <= hi && (jz >= from || ja < p.sinks);
    if (used) x.table[(int64_t)b * x.table_stride + (ja >> x.page_shift)] = row_of<kPaged>(p, table, ja) < 0 ? -1 : (int)(to_row >> x.page_shift) + tid;
  }
  // a thread has eight values of every kStep-th row, so that a warp stores whole lines
  const int r0 = tid / kC, c = tid % kC;
  uint32_t w[2][kEach], scale[2][kEach];
#pragma unroll
  for (int y = 0; y < kEach; ++y) {
    const int r = r0 + y * kStep;
    const int64_t row = is_seen(j0 + r) ? row_of<kPaged>(p, table, j0 + r) : -1;
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      w[z][y] = scale[z][y] = 0;
      if (row >= 0) {
        const int64_t o = (kPaged ? 0 : (int64_t)b * (z ? p.v_sb : p.k_sb)) + (int64_t)hkv * (z ? p.v_sh : p.k_sh) + row * (z ? p.v_st : p.k_st) + c * 8;
        w[z][y] = *reinterpret_cast<const uint32_t*>(static_cast<const uint8_t*>(z ? p.v : p.k) + o / 2);
        scale[z][y] = (z ? p.v_scales : p.k_scales)[o / kScaleDims];
      }
    }
  }
#pragma unroll
  for (int y = 0; y < kEach; ++y) {
    const int r = r0 + y * kStep;
    if (!is_seen(j0 + r)) continue;                          // (may hold anything: the tiles do not use it)
#pragma unroll
    for (int z = 0; z < 2; ++z) {
      const uint32_t by = __byte_perm(e4m3x2_to_half2(scale[z][y]), 0, 0x1010);
      uint32_t h[4];
      e2m1x8_to_half2(w[z][y], h);
#pragma unroll
      for (int e = 0; e < 4; ++e) h[e] = half2_mul(h[e], by);
      *reinterpret_cast<uint4*>((z ? x.v : x.k) + ((int64_t)hkv * x.head_rows + to_row + r) * D + c * 8) = make_uint4(h[0], h[1], h[2], h[3]);
    }
  }
}

template <int D>
static int32_t launch_expanded(const Fp4Params& all, const Fp4Expanded& x, cudaStream_t st) {
  const int page = 1 << x.page_shift;
  const int64_t head = x.head_rows * D;
  CUtensorMap maps[2];
  if (!tile_map(&maps[0], x.k, SSA_F16, D, x.head_rows, D, x.heads, head, 1, 0, page) ||
      !tile_map(&maps[1], x.v, SSA_F16, D, x.head_rows, D, x.heads, head, 1, 0, page))
    return SSA_ERR_CUDA;
  cudaEvent_t begin, end;
  take_kernel_events(&begin, &end);
  if (begin) cudaEventRecord(begin, st);                     // (what the tiles read is part of their time)
  for (int b0 = 0; b0 < all.B; b0 += x.requests)
    for (int h0 = 0; h0 < all.H_kv; h0 += x.heads) {         // (in parts only where they are one request's: rows of lse lie side by side)
      Fp4Params p = all;
      p.B = std::min(x.requests, all.B - b0);
      p.H_kv = std::min(x.heads, all.H_kv - h0);
      p.H = p.H_kv * p.group;
      const int64_t first = (int64_t)h0 * p.group, k0 = (p.page_table ? 0 : b0 * p.k_sb) + h0 * p.k_sh, v0 = (p.page_table ? 0 : b0 * p.v_sb) + h0 * p.v_sh;
      p.q = static_cast<const __nv_bfloat16*>(all.q) + b0 * p.q_sb + first * p.q_sh;
      p.out = static_cast<char*>(all.out) + (b0 * p.o_sb + first * p.o_sh) * (p.out_f32 ? 4 : 2);
      if (p.lse) p.lse += ((int64_t)b0 * all.H + first) * p.n_q;
      p.ctx_lens += b0;
      if (p.q_lens) p.q_lens += b0;
      if (p.page_table) p.page_table += (int64_t)b0 * p.page_table_stride;
      p.k = static_cast<const uint8_t*>(all.k) + k0 / 2;
      p.v = static_cast<const uint8_t*>(all.v) + v0 / 2;
      p.k_scales += k0 / kScaleDims;
      p.v_scales += v0 / kScaleDims;
      const dim3 grid((unsigned)x.most_tiles, (unsigned)p.H_kv, (unsigned)p.B);
      if (launch_pdl(p.page_table ? fp4_expand_kernel<D, true> : fp4_expand_kernel<D, false>, grid, dim3(kExpandThreads), st, p, x) != cudaSuccess)
        return SSA_ERR_CUDA;
      note_launches(1);
      WindowParams t = p;
      t.k = x.k; t.v = x.v;
      t.page_table = x.table; t.page_table_stride = x.table_stride; t.page_shift = x.page_shift;
      t.n_pages = (int)(x.head_rows >> x.page_shift);
      t.k_sb = t.v_sb = 0; t.k_sh = t.v_sh = head; t.k_st = t.v_st = D;
      if (launch_tiles<Fp4AsHalf, D>(t, maps[0], maps[1], page, st) != cudaSuccess) return SSA_ERR_CUDA;
      if (end) cudaEventRecord(end, st);                     // (the last one counts)
      note_launches(1);
      if (p.n_splits == 1) continue;
      if (launch_join<__nv_bfloat16, D>(t, st) != cudaSuccess) return SSA_ERR_CUDA;
      note_launches(1);
    }
  return SSA_OK;
}

int32_t launch_expanded(const Fp4Params& p, const Fp4Expanded& x, int D, cudaStream_t st) {
  return D == 128 ? launch_expanded<128>(p, x, st) : launch_expanded<64>(p, x, st);
}

template <int D>
static int32_t launch(const Fp4Params& p, int box_rows, cudaStream_t st) {
  cudaEvent_t begin, end;
  take_kernel_events(&begin, &end);
  if (begin) cudaEventRecord(begin, st);
  cudaError_t err = box_rows    ? launch_tiles<Fp4E2M1, D>(p, CUtensorMap{}, CUtensorMap{}, box_rows, st)
                    : p.out_f32 ? (p.page_table ? launch_rows<Fp4E2M1, D, true, false, true>(p, st) : launch_rows<Fp4E2M1, D, false, false, true>(p, st))
                                : (p.page_table ? launch_rows<Fp4E2M1, D, true, false, false>(p, st) : launch_rows<Fp4E2M1, D, false, false, false>(p, st));
  if (err != cudaSuccess) return SSA_ERR_CUDA;
  if (end) cudaEventRecord(end, st);
  note_launches(1);
  if (p.n_splits == 1) return SSA_OK;
  err = launch_join<__nv_bfloat16, D>(p, st);
  if (err != cudaSuccess) return SSA_ERR_CUDA;
  note_launches(1);
  return SSA_OK;
}

int32_t launch_window_fp4(const Fp4Params& p, int D, int box_rows, cudaStream_t st) {
  return D == 128 ? launch<128>(p, box_rows, st) : launch<64>(p, box_rows, st);
}

}  // namespace ssa
