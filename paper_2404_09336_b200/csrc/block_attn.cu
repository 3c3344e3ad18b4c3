// Attention of every token over its own list of blocks (ssa_attn_blocks): out = sum_j softmax(s)_j V_j over the positions j <= pos
// of the listed blocks, s_j = scale <q, K_j>.
//
// The kernel for few rows of window_rows.cuh, whose rows are here the query heads of one token and K/V head: they share its list.
// HBM bounds it: the listed rows of K and V are read once, by tiles of 16 or 32 positions that never cross a block.  32 requests, 8 K/V
// heads, 32 blocks of 64 positions each: 51.4 us, 5.2 TB/s; in 8 bits 40, in 4 bits 33, where instructions bound it.
#include "window_rows.cuh"

namespace ssa {

struct BlocksPlan { int block_rows, parts, n_splits; size_t ml_bytes, total_bytes; };

static int32_t check_blocks(const ssa_attn_desc* d, const ssa_blocks* k) {
  int32_t rc = check_cache(d);
  if (rc == SSA_OK) rc = check_block_sizes(d, k);
  if (rc != SSA_OK) return rc;
  if (k->q_stride_t < 0 || k->o_stride_t < 0 || (long long)d->H * k->n_q > 1ll << 24) return SSA_ERR_SHAPE;
  if (k->q_stride_t % 8 != 0 || k->o_stride_t % 8 != 0) return SSA_ERR_ALIGN;
  if (k->budget <= 0 || (long long)k->budget * k->block_size > 0x7fffffffll) return SSA_ERR_CAPACITY;
  return k->paging ? check_paging(k->paging, d->max_ctx) : SSA_OK;
}

static bool plan_blocks(const ssa_attn_desc* d, const ssa_blocks* k, BlocksPlan* pl) {
  const int keys = rows_tile_keys(d->D, d->kv_dtype), group = d->H / d->H_kv, groups = std::min((group + kGroup - 1) / kGroup, kMostGroups);
  pl->block_rows = kGroup * (groups == 3 ? 4 : groups);
  pl->parts = (group + pl->block_rows - 1) / pl->block_rows;
  const long long blocks = (long long)pl->parts * k->n_q * d->H_kv * d->B;
  const long long listed = std::min<long long>(k->budget, (d->max_ctx + k->block_size - 1ll) / k->block_size);
  const long long n_tiles = listed * (k->block_size / keys);
  pl->n_splits = (int)rows_splits(n_tiles, blocks, pl->block_rows, d->kv_dtype == SSA_FP4_E2M1,
                                  std::max(1ll, std::min(n_tiles / (kSplitKeys / keys), 64ll)));
  const size_t slots = (size_t)d->B * d->H * k->n_q * pl->n_splits;
  pl->ml_bytes = up256(slots * sizeof(float2));
  pl->total_bytes = pl->ml_bytes + (pl->n_splits > 1 ? up256(slots * d->D * sizeof(float)) : 0);
  return (long long)pl->parts * k->n_q * pl->n_splits <= 0x7fffffffll;
}

template <typename T, int D, bool kPaged, bool kBoth>
static cudaError_t launch_lists(const ListParams& p, cudaStream_t st) {
  const dim3 grid((unsigned)(p.n_q * p.parts * p.n_splits), (unsigned)p.H_kv, (unsigned)p.B);
  auto launch = [&](auto kernel, int bytes) { return launch_rows_kernel(kernel, p, grid, bytes, p.block_rows, D, st); };
  switch (p.block_rows / kGroup) {
    case 1: return launch(window_rows_kernel<T, D, kPaged, false, 1, 1, kBoth, ListParams>, RowShape<T, D, 1>::kSmem);
    case 2: return launch(window_rows_kernel<T, D, kPaged, false, 1, 2, kBoth, ListParams>, RowShape<T, D, 2>::kSmem);
    default: return launch(window_rows_kernel<T, D, kPaged, false, 1, 4, kBoth, ListParams>, RowShape<T, D, 4>::kSmem);
  }
}

template <typename T, int D>
static int32_t launch(const ListParams& p, cudaStream_t st) {
  cudaEvent_t begin, end;
  take_kernel_events(&begin, &end);
  if (begin) cudaEventRecord(begin, st);
  const bool one = kIsFp4<T> && !p.out_f32;                  // (fp16 weights of one part)
  cudaError_t err = one ? (p.page_table ? launch_lists<T, D, true, !kIsFp4<T>>(p, st) : launch_lists<T, D, false, !kIsFp4<T>>(p, st))
                        : (p.page_table ? launch_lists<T, D, true, true>(p, st) : launch_lists<T, D, false, true>(p, st));
  if (err != cudaSuccess) return SSA_ERR_CUDA;
  if (end) cudaEventRecord(end, st);
  note_launches(1);
  if (p.n_splits == 1) return SSA_OK;
  using TQ = typename Storage<T>::Query;
  err = launch_join<TQ, D>(p, st);
  if (err != cudaSuccess) return SSA_ERR_CUDA;
  note_launches(1);
  return SSA_OK;
}

}  // namespace ssa

extern "C" {

size_t ssa_attn_blocks_workspace_bytes(const ssa_attn_desc* desc, const ssa_blocks* blocks) {
  ssa::BlocksPlan pl;
  return desc && blocks && ssa::check_blocks(desc, blocks) == SSA_OK && ssa::plan_blocks(desc, blocks, &pl) ? pl.total_bytes : 0;
}

int32_t ssa_attn_blocks(const ssa_attn_desc* desc, const ssa_blocks* blocks, const void* q, const void* k_cache,
                        const void* v_cache, const void* k_scales, const void* v_scales, const int32_t* ctx_lens,
                        const int32_t* index, const int32_t* counts, void* out, float* lse, void* workspace,
                        size_t workspace_bytes, uint32_t* dev_status, void* stream) {
  using namespace ssa;
  if (!desc || !blocks || !q || !k_cache || !v_cache || !ctx_lens || !index || !counts || !out) return SSA_ERR_NULL;
  const bool fp4 = desc->kv_dtype == SSA_FP4_E2M1;
  if (fp4 && (!k_scales || !v_scales)) return SSA_ERR_NULL;
  const int32_t rc = check_blocks(desc, blocks);
  if (rc != SSA_OK) return rc;
  if (!aligned16(q) || !aligned16(k_cache) || !aligned16(v_cache) || !aligned16(out) || !aligned16(workspace) ||
      (fp4 && (!aligned16(k_scales) || !aligned16(v_scales))))
    return SSA_ERR_ALIGN;
  BlocksPlan pl;
  if (!plan_blocks(desc, blocks, &pl)) return SSA_ERR_SHAPE;
  if (blocks->n_q > 1 && blocks->o_stride_t == 0) return SSA_ERR_UNSUPPORTED;      // (tokens would share a row of out)
  if (!workspace || workspace_bytes < pl.total_bytes) return SSA_ERR_WORKSPACE;
  ListParams p = {};
  fill_params(p, desc, blocks->n_q, blocks->q_stride_t, blocks->o_stride_t, blocks->q_lens, blocks->paging, q, k_cache, v_cache,
              ctx_lens, out, lse, dev_status);
  p.ws_ml = static_cast<float2*>(workspace);
  p.ws_acc = reinterpret_cast<float*>(static_cast<char*>(workspace) + pl.ml_bytes);
  p.n_splits = pl.n_splits;
  p.block_rows = pl.block_rows;
  p.tile_keys = rows_tile_keys(desc->D, desc->kv_dtype);
  p.split_tiles = kSplitKeys / p.tile_keys;
  p.k_scales = static_cast<const uint8_t*>(k_scales);
  p.v_scales = static_cast<const uint8_t*>(v_scales);
  p.list = index;
  p.list_counts = counts;
  p.budget = blocks->budget;
  p.parts = pl.parts;
  while ((1 << p.block_shift) < blocks->block_size) ++p.block_shift;
  cudaStream_t st = (cudaStream_t)stream;
  const bool wide = desc->D == 128;
  switch (desc->kv_dtype) {
    case SSA_FP4_E2M1: return wide ? launch<Fp4E2M1, 128>(p, st) : launch<Fp4E2M1, 64>(p, st);
    case SSA_FP8_E4M3: return wide ? launch<Fp8E4M3, 128>(p, st) : launch<Fp8E4M3, 64>(p, st);
    case SSA_BF16: return wide ? launch<__nv_bfloat16, 128>(p, st) : launch<__nv_bfloat16, 64>(p, st);
    default: return wide ? launch<__half, 128>(p, st) : launch<__half, 64>(p, st);
  }
}

}  // extern "C"
