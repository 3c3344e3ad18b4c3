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
#include "window_rows.cuh"
#include "window_tile.cuh"

namespace ssa {

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
      const int n = row_splits(p, b, h, t, ctx, n_new);
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

static int32_t check_window(const ssa_attn_desc* d, const ssa_window* w, bool mass, bool fp4) {
  if (fp4 && d->kv_dtype != SSA_FP4_E2M1) return SSA_ERR_DTYPE;
  const int32_t rc = fp4 ? check_cache(d) : check_desc(d);
  if (rc != SSA_OK) return rc;
  if (d->max_ctx > kMostContext || w->n_q <= 0 || w->window < 0 || w->sinks < 0 || w->q_stride_t < 0 || w->o_stride_t < 0) return SSA_ERR_SHAPE;
  if (w->q_stride_t % 8 != 0 || w->o_stride_t % 8 != 0) return SSA_ERR_ALIGN;
  if ((long long)d->H * w->n_q > (mass ? (long long)SSA_MASS_MAX_ROWS : 1ll << 24)) return SSA_ERR_SHAPE;
  return w->paging ? check_paging(w->paging, d->max_ctx) : SSA_OK;
}

// kFewRows holds for a 4-bit cache too: with 24 rows the kernel for few rows takes 85, 52, 81 and 42 us, the tiles 124, 54, 116 and 40 (8
// requests of 4100 to 16384 positions, those within a window of 4096, 32 requests of up to 4096, one of 16384; 8 K/V heads, L2 cold), in
// pages of 16 89, 56, 91 and 42 against 163, 66, 155 and 44; with 25 to 32 rows 122, 71, 119 and 54 against 124, 56, 117 and 40, in pages
// 133, 78, 133 and 56 against 163, 66, 155 and 44.
// Rows above which it is converted once for all of them, instead of by every block of 128 rows: for the same requests that takes 247,
// 110, 235 and 73 us with 256 rows, 361, 134, 286 and 97 with 512, 441, 196, 452 and 99 with 768, 562, 216, 478 and 116 with 1024, each
// block for itself 212, 89, 191 and 62, then 389, 127, 264 and 93, then 467, 199, 453 and 101, then 649, 231, 498 and 128.  In pages each
// piece of a row costs a block more instructions: 273, 116, 255 and 75 against 280, 108, 248 and 71 with 256 rows, 386, 142, 308 and 87
// against 463, 158, 330 and 87 with 384.
constexpr int kExpandRows = 768, kExpandRowsPaged = 256;

// Whether the tiles of 128 rows serve a call.
static bool tiles_pay(const ssa_attn_desc* d, const ssa_window* w, bool mass) {
  return !mass && d->kv_dtype != SSA_FP8_E4M3 &&
         (long long)(d->H / d->H_kv) * w->n_q > kFewRows &&
         (!w->paging || w->paging->page_size >= 8);          // (a box of a copy is eight rows at least, or a lane's run of 4-bit ones)
}

static bool plan_window(const ssa_attn_desc* d, const ssa_window* w, bool mass, bool tiles, WindowPlan* pl) {
  pl->tiles = tiles;
  const long long per_head = (long long)(d->H / d->H_kv) * w->n_q;
  const int keys = tiles ? kTileKeys : rows_tile_keys(d->D, d->kv_dtype), fewest = tiles ? kTileSplit : kSplitKeys / keys;
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
  if (!tiles) splits = rows_splits(n_tiles, blocks, rows, d->kv_dtype == SSA_FP4_E2M1, most_splits);
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

// Most bytes of converted rows that a call has in its workspace at a time.  (A 4-bit cache is held for its size: all rows at once would
// take 3.6 times that.)  Parts of a call are few blocks for the GPU: 32 chunks of 512 tokens over 16384 positions, 32 heads over 8, take
// 4333 us with all 2 GB, 4198 with 1 GB, 4633 with 512 MB, 4749 with 256; 32 K/V heads of 8 requests 1669, 1745, 1790 and 2076; 4 chunks
// of 128 over 131072 positions 1799, 1819, 1816 and 2036.
constexpr long long kExpandBytes = 1 << 29;

// Where the rows of a 4-bit cache that the tokens see have places in fp16; bytes of all of it, 0 where the call has no use for that, or a
// K/V head of a request does not fit most_bytes.  Few blocks of 128 rows convert what they see themselves.
static size_t plan_expanded(const ssa_attn_desc* d, const ssa_window* w, long long most_bytes, Fp4Expanded* x) {
  const long long rows = (long long)(d->H / d->H_kv) * w->n_q;
  if (rows <= (w->paging ? kExpandRowsPaged : kExpandRows)) return 0;
  const long long all = (d->max_ctx + kTileKeys - 1ll) / kTileKeys;
  const long long seen = ((long long)w->sinks + kTileKeys - 1) / kTileKeys + ((long long)w->window + w->n_q + kTileKeys - 1) / kTileKeys + 1;
  const long long tiles = w->window == 0 ? all : std::min(all, seen), fit = most_bytes / (tiles * kTileKeys * d->D * 2 * (long long)sizeof(__half));
  if (fit == 0) return 0;
  // as many requests as fit, or heads of one, in parts of one size
  const long long per = std::max(1ll, fit / d->H_kv), parts = (d->B + per - 1) / per;
  const long long most = std::min<long long>(fit, d->H_kv), head_parts = (d->H_kv + most - 1) / most;
  x->requests = (int)((d->B + parts - 1) / parts);
  x->heads = (int)((d->H_kv + head_parts - 1) / head_parts);
  const int page = w->paging ? std::min(w->paging->page_size, kTileKeys) : kTileKeys;
  x->most_tiles = (int)tiles;
  x->head_rows = tiles * x->requests * kTileKeys;
  x->page_shift = 0;
  while ((1 << x->page_shift) < page) ++x->page_shift;
  x->table_stride = (int)((d->max_ctx + (long long)page - 1) / page);
  return up256((size_t)x->requests * x->table_stride * sizeof(int32_t)) + 2 * up256((size_t)x->head_rows * x->heads * d->D * 2);
}

// The part of the call that is served at a time.
static ssa_attn_desc part_of(const ssa_attn_desc* d, const Fp4Expanded& x) {
  ssa_attn_desc part = *d;
  part.B = x.requests;
  part.H = d->H / d->H_kv * x.heads;
  part.H_kv = x.heads;
  return part;
}

// Room for either kernel: which one runs may depend on the cache's strides (of a 4-bit cache: does not).
static size_t window_bytes(const ssa_attn_desc* d, const ssa_window* w, bool mass, bool fp4) {
  WindowPlan pl;
  if (!d || !w || check_window(d, w, mass, fp4) != SSA_OK || !plan_window(d, w, mass, false, &pl)) return 0;
  const size_t few = pl.total_bytes;
  if (!tiles_pay(d, w, mass) || !plan_window(d, w, mass, true, &pl)) return few;
  return fp4 ? pl.total_bytes : std::max(few, pl.total_bytes);
}
// The same for a call that converts once, and where in it the converted rows start, in parts that have room in ws_bytes; 0 where it
// does not, or the smallest have none.
static size_t expanded_bytes(const ssa_attn_desc* d, const ssa_window* w, size_t ws_bytes, Fp4Expanded* x, size_t* start) {
  if (!tiles_pay(d, w, false)) return 0;
  for (long long most = kExpandBytes;; most /= 2) {
    const size_t more = plan_expanded(d, w, most, x);
    if (!more) return 0;
    const ssa_attn_desc part = part_of(d, *x);               // (whose rows may be split further than the whole call's)
    *start = std::max(window_bytes(d, w, false, true), window_bytes(&part, w, false, true));
    if (*start + more <= ws_bytes) return *start + more;
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
    err = p.page_table ? (mass ? launch_rows<T, D, true, true, true>(p, st) : launch_rows<T, D, true, false, true>(p, st))
                       : (mass ? launch_rows<T, D, false, true, true>(p, st) : launch_rows<T, D, false, false, true>(p, st));
  }
  if (err != cudaSuccess) return SSA_ERR_CUDA;
  if (end) cudaEventRecord(end, st);
  note_launches(1);
  if (mass) {
    const int mass_blocks = (p.max_ctx + kMassKeys - 1) / kMassKeys, joins = p.n_splits > 1 ? (p.H * p.n_q + kMassWarps - 1) / kMassWarps : 0;
    err = launch_pdl(window_mass_kernel<TQ, D>, dim3((unsigned)(mass_blocks + joins), (unsigned)p.B), dim3(kMassThreads), st, p, mass_blocks);
  } else if (p.n_splits > 1) {
    err = launch_pdl(window_join_kernel<TQ, D, WindowParams>, dim3((unsigned)((p.H * p.n_q + kJoinWarps - 1) / kJoinWarps), (unsigned)p.B),
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
                          int64_t mass_stride, float decay, bool fp4, const void* k_scales, const void* v_scales, void* ws,
                          size_t ws_bytes, uint32_t* status, void* stream) {
  if (!d || !w || !q || !k || !v || !ctx_lens || !out || (mass && !mass_out) || (fp4 && (!k_scales || !v_scales))) return SSA_ERR_NULL;
  const int32_t rc = check_window(d, w, mass, fp4);
  if (rc != SSA_OK) return rc;
  if (mass && mass_stride < d->max_ctx) return SSA_ERR_SHAPE;
  if (!aligned16(q) || !aligned16(k) || !aligned16(v) || !aligned16(out) || !aligned16(ws) || !aligned16(k_scales) || !aligned16(v_scales))
    return SSA_ERR_ALIGN;
  if (!ws || ws_bytes < window_bytes(d, w, mass, fp4)) return SSA_ERR_WORKSPACE;
  const ssa_paging* pg = w->paging;
  CUtensorMap maps[2];
  const int box_rows = pg ? std::min(pg->page_size, kTileKeys) : kTileKeys;
  const int64_t pool_rows = pg ? (int64_t)pg->n_pages * pg->page_size : d->max_ctx;
  WindowPlan pl;
  auto mapped = [&](CUtensorMap* map, const void* cache, int64_t st, int64_t sh, int64_t sb) {
    return tile_map(map, cache, d->kv_dtype, d->D, pool_rows, st, d->H_kv, sh, pg ? 1 : d->B, sb, box_rows);
  };
  const bool tiles = tiles_pay(d, w, mass) && plan_window(d, w, mass, true, &pl) &&
                     (fp4 || (mapped(&maps[0], k, d->k_stride_t, d->k_stride_h, d->k_stride_b) &&
                              mapped(&maps[1], v, d->v_stride_t, d->v_stride_h, d->v_stride_b)));
  if (!tiles && !plan_window(d, w, mass, false, &pl)) return SSA_ERR_SHAPE;
  WindowParams p;
  p.block_rows = pl.block_rows;
  p.tile_keys = pl.keys;
  p.split_tiles = pl.fewest;
  fill_params(p, d, w->n_q, w->q_stride_t, w->o_stride_t, w->q_lens, pg, q, k, v, ctx_lens, out, lse, status);
  char* at = static_cast<char*>(ws);
  p.ws_ml = reinterpret_cast<float2*>(at);
  p.ws_acc = reinterpret_cast<float*>(at + pl.ml_bytes);
  p.ws_s = reinterpret_cast<float*>(at + pl.ml_bytes + pl.acc_bytes);
  p.mass_in = mass_in; p.mass_out = mass_out;
  p.mass_stride = mass_stride;
  p.window = w->window >= d->max_ctx ? 0 : w->window;                  // (no window at all; and no overflow in sums with it)
  p.sinks = std::min(w->sinks, d->max_ctx);
  p.n_splits = pl.n_splits; p.s_pitch = pl.s_pitch;
  p.decay = decay;
  cudaStream_t st = (cudaStream_t)stream;
  if (fp4) {
    Fp4Params f;
    static_cast<WindowParams&>(f) = p;
    f.k_scales = static_cast<const uint8_t*>(k_scales);
    f.v_scales = static_cast<const uint8_t*>(v_scales);
    Fp4Expanded x;
    size_t start = 0;
    if (expanded_bytes(d, w, ws_bytes, &x, &start)) {
      // the rows that are seen in fp16, behind the partial results, and the tiles of a cache of such rows in pages
      const ssa_attn_desc part = part_of(d, x);
      if (!plan_window(&part, w, false, true, &pl)) return SSA_ERR_SHAPE;
      f.n_splits = pl.n_splits;
      f.ws_acc = reinterpret_cast<float*>(at + pl.ml_bytes);
      char* to = at + start;
      x.table = reinterpret_cast<int32_t*>(to);
      to += up256((size_t)x.requests * x.table_stride * sizeof(int32_t));
      x.k = reinterpret_cast<__half*>(to);
      x.v = reinterpret_cast<__half*>(to + up256((size_t)x.head_rows * x.heads * d->D * 2));
      return launch_expanded(f, x, d->D, st);
    }
    return launch_window_fp4(f, d->D, tiles ? box_rows : 0, st);
  }
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
  return ssa::window_bytes(desc, window, false, false);
}

size_t ssa_attn_mass_workspace_bytes(const ssa_attn_desc* desc, const ssa_window* window) {
  return ssa::window_bytes(desc, window, true, false);
}

int32_t ssa_attn_window(const ssa_attn_desc* desc, const ssa_window* window, const void* q, const void* k_cache,
                        const void* v_cache, const int32_t* ctx_lens, void* out, float* lse, void* workspace,
                        size_t workspace_bytes, uint32_t* dev_status, void* stream) {
  return ssa::run_window(desc, window, q, k_cache, v_cache, ctx_lens, out, lse, false, nullptr, nullptr, 0, 0.f, false, nullptr, nullptr,
                         workspace, workspace_bytes, dev_status, stream);
}

int32_t ssa_attn_mass(const ssa_attn_desc* desc, const ssa_window* window, const void* q, const void* k_cache,
                      const void* v_cache, const int32_t* ctx_lens, void* out, float* lse, const float* mass_in,
                      float* mass_out, int64_t mass_stride, float decay, void* workspace, size_t workspace_bytes,
                      uint32_t* dev_status, void* stream) {
  return ssa::run_window(desc, window, q, k_cache, v_cache, ctx_lens, out, lse, true, mass_in, mass_out, mass_stride, decay, false,
                         nullptr, nullptr, workspace, workspace_bytes, dev_status, stream);
}

size_t ssa_attn_window_fp4_workspace_bytes(const ssa_attn_desc* desc, const ssa_window* window) {
  const size_t need = ssa::window_bytes(desc, window, false, true);
  ssa::Fp4Expanded x;
  size_t start;
  return need ? std::max(need, ssa::expanded_bytes(desc, window, ~(size_t)0, &x, &start)) : 0;
}

int32_t ssa_attn_window_fp4(const ssa_attn_desc* desc, const ssa_window* window, const void* q, const void* k_cache,
                            const void* v_cache, const void* k_scales, const void* v_scales, const int32_t* ctx_lens,
                            void* out, float* lse, void* workspace, size_t workspace_bytes, uint32_t* dev_status,
                            void* stream) {
  return ssa::run_window(desc, window, q, k_cache, v_cache, ctx_lens, out, lse, false, nullptr, nullptr, 0, 0.f, true, k_scales,
                         v_scales, workspace, workspace_bytes, dev_status, stream);
}

}  // extern "C"
