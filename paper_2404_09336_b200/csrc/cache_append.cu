// A step's keys and values into the cache, rotated by position on the way, and its queries rotated (ssa_cache_append).
//
//   pairs (x, y) of rotary dimensions -> (x c - y s, y c + x s);  16-bit, e4m3 or e2m1 with an e4m3 scale for 16 dimensions
//
// HBM bounds it: every row is read and written once.  The products of 16-bit values and fp32 cosines are exact in fp64, so that what
// is stored is the formula's value rounded: to fp32, then to the cache's type.  (8- and 4-bit values lie next to borders, where an
// error of an fp32 rounding would be half a step.)  4 x 4096 tokens, 32 heads, pages of 16: 148 to 163 us by the GPU, 5.0 to 5.5 TB/s
// (without rotation 135); conversions to and from fp64 fill a third of their pipe.  In 8 bits, 6 x 4096 tokens, 32 heads over 8: 110
// us; in 4 bits 151.
#include <algorithm>
#include <type_traits>

#include "mma.cuh"
#include "window.cuh"

namespace ssa {

constexpr int kAppendThreads = 64;

struct AppendParams {
  const void *q, *k_new, *v_new;
  void *q_out, *k, *v;
  uint8_t *k_scales, *v_scales;
  const float* cos_sin;
  const int32_t *positions, *ctx_lens, *q_lens, *page_table;
  uint32_t* status;
  int64_t q_sb, q_sh, q_st, qo_sb, qo_sh, qo_st, kn_sb, kn_sh, kn_st, vn_sb, vn_sh, vn_st;
  int64_t k_sb, k_sh, k_st, v_sb, v_sh, v_st;                // values
  int B, H, H_kv, n_q, max_ctx, rotary, interleaved, n_positions;
  int page_table_stride, page_shift, n_pages;
  int slots, tokens;                                         // threads' places for a token's rows; tokens of a thread block
  float k_factor, v_factor;
};

// Two values as e4m3, two as e2m1; the first in the low half.
__device__ __forceinline__ uint32_t to_e4m3x2(float lo, float hi) {
  uint16_t w;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %2, %1;" : "=h"(w) : "f"(lo), "f"(hi));
  return w;
}
__device__ __forceinline__ uint32_t to_e2m1x8(const float (&f)[8]) {
  uint32_t w;
  asm("{ .reg .b8 b0, b1, b2, b3; cvt.rn.satfinite.e2m1x2.f32 b0, %2, %1; cvt.rn.satfinite.e2m1x2.f32 b1, %4, %3; "
      "cvt.rn.satfinite.e2m1x2.f32 b2, %6, %5; cvt.rn.satfinite.e2m1x2.f32 b3, %8, %7; mov.b32 %0, {b0, b1, b2, b3}; }"
      : "=r"(w) : "f"(f[0]), "f"(f[1]), "f"(f[2]), "f"(f[3]), "f"(f[4]), "f"(f[5]), "f"(f[6]), "f"(f[7]));
  return w;
}
// A new row's piece.  (volatile: asked for where it stands.  Not read-only memory: queries may be rotated in their place.)
__device__ __forceinline__ uint4 ld_row(const void* p) {
  uint4 r;
  asm volatile("ld.global.L1::no_allocate.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(r.x), "=r"(r.y), "=r"(r.z), "=r"(r.w) : "l"(p) : "memory");
  return r;
}
template <typename TQ>
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
  return make_uint4(pack2<TQ>(f[0], f[1]), pack2<TQ>(f[2], f[3]), pack2<TQ>(f[4], f[5]), pack2<TQ>(f[6], f[7]));
}

// grid (tokens / p.tokens, parts, B).  A row has D / 16 lanes with two pieces of eight dimensions each: the pieces that are rotated
// with one another, which are neighbours where pairs are.  A thread has up to kEach rows of a token, all asked for before anything
// else is: lengths, pages and cosines arrive meanwhile, and are made ready once for all of them.
template <typename T, int D, bool kPaged, int kEach>
__global__ void __launch_bounds__(kAppendThreads, 12)
cache_append_kernel(const AppendParams p) {
  using TQ = typename Storage<T>::Query;
  constexpr int kLanes = D / 16, kRows = kAppendThreads / kLanes;
  const int b = blockIdx.z, lane = threadIdx.x % kLanes, place = blockIdx.y * kRows + threadIdx.x / kLanes;
  const int part = p.tokens == 1 ? 0 : place / p.slots, slot = place - part * p.slots, t = blockIdx.x * p.tokens + part;
  const int R = p.rotary, turned = R / 16;                   // lanes that rotate
  const bool apart = lane < turned && !p.interleaved;        // the two pieces are R / 2 dimensions apart
  const int piece0 = apart ? lane : !p.interleaved && R ? R / 8 + 2 * (lane - turned) : 2 * lane;
  const int piece1 = apart ? lane + R / 16 : piece0 + 1;
  const int queries = p.q ? p.H : 0, rows = queries + 2 * p.H_kv;
  const bool placed = part < p.tokens && slot < p.slots && t < p.n_q;
  grid_dependency_wait();
  grid_launch_dependents();
  uint4 w[kEach][2];
#pragma unroll
  for (int y = 0; y < kEach; ++y) {
    const int i = slot + y * p.slots;
    const bool is_q = i < queries, is_v = i >= queries + p.H_kv;
    w[y][0] = w[y][1] = make_uint4(0, 0, 0, 0);
    if (placed && i < rows) {
      const TQ* from = is_q ? static_cast<const TQ*>(p.q) + b * p.q_sb + i * p.q_sh + t * p.q_st
                       : is_v ? static_cast<const TQ*>(p.v_new) + b * p.vn_sb + (i - queries - p.H_kv) * p.vn_sh + t * p.vn_st
                              : static_cast<const TQ*>(p.k_new) + b * p.kn_sb + (i - queries) * p.kn_sh + t * p.kn_st;
      w[y][0] = ld_row(from + piece0 * 8);
      w[y][1] = ld_row(from + piece1 * 8);
    }
  }
  uint32_t flags = 0;
  int ctx, n_new;
  window_sizes(p, b, ctx, n_new, flags);
  const int pos = ctx - n_new + t;
  if (flags && p.status && blockIdx.x == 0 && blockIdx.y == 0 && threadIdx.x == 0) atomicOr(p.status, flags);
  bool live = placed && t < n_new && pos >= 0;
  int64_t row = -1;
  int angle = 0;
  if (live) {
    row = row_of<kPaged>(p, kPaged ? p.page_table + (int64_t)b * p.page_table_stride : nullptr, pos);
    angle = R == 0 ? 0 : p.positions ? p.positions[(int64_t)b * p.n_q + t] : pos;
    const bool known = R == 0 || (unsigned)angle < (unsigned)p.n_positions;
    if ((!known || row < 0) && slot == 0 && lane == 0 && p.status) atomicOr(p.status, SSA_DEV_BAD_INDEX);
    live = known;
  }
  if (!__any_sync(~0u, live)) return;
  double c[8], s[8];                                         // of pairs 8 lane ...
#pragma unroll
  for (int e = 0; e < 8; ++e) c[e] = s[e] = 0.0;
  if (live && lane < turned) {
    const float* at = p.cos_sin + (int64_t)angle * R + 8 * lane;
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
      const float4 x = *reinterpret_cast<const float4*>(at + e), y = *reinterpret_cast<const float4*>(at + R / 2 + e);
      c[e] = x.x; c[e + 1] = x.y; c[e + 2] = x.z; c[e + 3] = x.w;
      s[e] = y.x; s[e + 1] = y.y; s[e + 2] = y.z; s[e + 3] = y.w;
    }
  }
#pragma unroll
  for (int y = 0; y < kEach; ++y) {                          // (a warp's rows together: neighbouring lanes exchange their largest values)
    const int i = slot + y * p.slots;
    const bool there = live && i < rows, is_q = i < queries, is_v = i >= queries + p.H_kv;
    if (!__any_sync(~0u, there)) break;
    const int h = is_q ? i : is_v ? i - queries - p.H_kv : i - queries;
    float x[2][8];
    unpack8<TQ>(w[y][0], x[0]);
    unpack8<TQ>(w[y][1], x[1]);
    if (!is_v && lane < turned) {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float& u = p.interleaved ? x[e / 4][e % 4 * 2] : x[0][e];
        float& v = p.interleaved ? x[e / 4][e % 4 * 2 + 1] : x[1][e];
        const double du = u, dv = v;
        u = (float)(du * c[e] - dv * s[e]);
        v = (float)(dv * c[e] + du * s[e]);
      }
    }
    if (is_q) {
      if (there) {
        TQ* to = static_cast<TQ*>(p.q_out) + b * p.qo_sb + h * p.qo_sh + t * p.qo_st;
        *reinterpret_cast<uint4*>(to + piece0 * 8) = pack8<TQ>(x[0]);
        *reinterpret_cast<uint4*>(to + piece1 * 8) = pack8<TQ>(x[1]);
      }
    }
    const float factor = is_v ? p.v_factor : p.k_factor;
    const int64_t o = (kPaged ? 0 : b * (is_v ? p.v_sb : p.k_sb)) + h * (is_v ? p.v_sh : p.k_sh) + row * (is_v ? p.v_st : p.k_st);
    const bool stored = there && !is_q && row >= 0;
#pragma unroll
    for (int z = 0; z < 2; ++z)
#pragma unroll
      for (int e = 0; e < 8; ++e) x[z][e] *= factor;
    if constexpr (kIsFp4<T>) {
      float top[2], by[2];
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        top[z] = max3_or_nan(fabsf(x[z][0]), fabsf(x[z][1]), fabsf(x[z][2]));
        top[z] = max3_or_nan(top[z], fabsf(x[z][3]), fabsf(x[z][4]));
        top[z] = max3_or_nan(top[z], fabsf(x[z][5]), max_or_nan(fabsf(x[z][6]), fabsf(x[z][7])));
      }
      // sixteen dimensions are a neighbouring lane's piece, or both of this lane's
      const float their0 = __shfl_xor_sync(~0u, top[0], 1), their1 = __shfl_xor_sync(~0u, top[1], 1);
      by[0] = max_or_nan(top[0], apart ? their0 : top[1]);
      by[1] = max_or_nan(top[1], apart ? their1 : top[0]);
      uint32_t bits[2];
#pragma unroll
      for (int z = 0; z < 2; ++z) {
        bits[z] = to_e4m3x2(__fdiv_rn(by[z], 6.f), 0.f) & 0xffu;
        // Quotients by one reciprocal and a residual step (Markstein): exact where they lie halfway between two codes, and never on the
        // wrong side of that: the scale has four bits, so that fp32 values next to half of a step are told from it.
        const float scale = e4m3x2_to_float2(bits[z]).x, inverse = scale == 0.f ? 0.f : __frcp_rn(scale);
        if (by[z] == __int_as_float(0x7f800000)) {           // (an infinity has no residual)
#pragma unroll
          for (int e = 0; e < 8; ++e)
            if (isinf(x[z][e])) { x[z][e] = copysignf(6.f * scale, x[z][e]); }
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float near = x[z][e] * inverse;
          x[z][e] = fmaf(fmaf(-near, scale, x[z][e]), inverse, near);
        }
      }
      if (stored) {
        uint8_t* codes = static_cast<uint8_t*>(is_v ? p.v : p.k) + o / 2;
        uint8_t* scales = (is_v ? p.v_scales : p.k_scales) + o / kScaleDims;
        *reinterpret_cast<uint32_t*>(codes + piece0 * 4) = bits[0] ? to_e2m1x8(x[0]) : 0;
        *reinterpret_cast<uint32_t*>(codes + piece1 * 4) = bits[1] ? to_e2m1x8(x[1]) : 0;
        if (!apart || lane % 2 == 0) scales[piece0 / 2] = (uint8_t)bits[0];
        if (apart && lane % 2 == 0) scales[piece1 / 2] = (uint8_t)bits[1];
      }
    } else if constexpr (kIsFp8<T>) {
      if (stored) {
        uint8_t* to = static_cast<uint8_t*>(is_v ? p.v : p.k) + o;
#pragma unroll
        for (int z = 0; z < 2; ++z)
          *reinterpret_cast<uint2*>(to + (z ? piece1 : piece0) * 8) =
              make_uint2(to_e4m3x2(x[z][0], x[z][1]) | to_e4m3x2(x[z][2], x[z][3]) << 16, to_e4m3x2(x[z][4], x[z][5]) | to_e4m3x2(x[z][6], x[z][7]) << 16);
      }
    } else if (stored) {
      TQ* to = static_cast<TQ*>(is_v ? p.v : p.k) + o;
      *reinterpret_cast<uint4*>(to + piece0 * 8) = pack8<TQ>(x[0]);
      *reinterpret_cast<uint4*>(to + piece1 * 8) = pack8<TQ>(x[1]);
    }
  }
}

template <typename T, int D>
static cudaError_t launch_append(const AppendParams& p, cudaStream_t st) {
  constexpr int kRows = kAppendThreads / (D / 16);
  const int rows = (p.q ? p.H : 0) + 2 * p.H_kv;
  auto launch = [&](auto kernel, int each) {
    AppendParams x = p;
    x.slots = (rows + each - 1) / each;
    x.tokens = std::max(1, std::min(kRows / x.slots, p.n_q));
    const dim3 grid((unsigned)((p.n_q + x.tokens - 1) / x.tokens), (unsigned)((x.slots * x.tokens + kRows - 1) / kRows), (unsigned)p.B);
    return launch_pdl(kernel, grid, dim3(kAppendThreads), st, x);
  };
  // Where rows take more blocks than the GPU holds at a time (12 to an SM), three a thread: cosines are made ready once for them, and more
  // of them are under way.  One against three, L2 cold: 32 heads over 8 of 128, 6 blocks to an SM 8.2 against 9.2 us (4 bits 8.3 against
  // 10.3), 10 blocks 9.2 against 10.2, 24 both 12.3; 8 heads of 64, 8 blocks 8.2 against 10.2, 24 13.2 against 12.3, 48 18.4 against 16.4;
  // 4 x 4096 tokens, 32 heads of 128, 206 against 155.
  const bool many = rows >= 3 && (long long)rows * p.n_q * p.B > 12ll * sm_count() * kRows;
  if (p.page_table) return many ? launch(cache_append_kernel<T, D, true, 3>, 3) : launch(cache_append_kernel<T, D, true, 1>, 1);
  return many ? launch(cache_append_kernel<T, D, false, 3>, 3) : launch(cache_append_kernel<T, D, false, 1>, 1);
}

}  // namespace ssa

extern "C" int32_t ssa_cache_append(const ssa_attn_desc* desc, const ssa_append* append, const void* k_new, const void* v_new,
                                    const int32_t* ctx_lens, void* k_cache, void* v_cache, const void* q, void* q_out,
                                    void* k_scales, void* v_scales, uint32_t* dev_status, void* stream) {
  using namespace ssa;
  const ssa_append* a = append;
  if (!desc || !a || !k_new || !v_new || !ctx_lens || !k_cache || !v_cache || !q != !q_out) return SSA_ERR_NULL;
  const bool fp4 = desc->kv_dtype == SSA_FP4_E2M1;
  if (fp4 && (!k_scales || !v_scales)) return SSA_ERR_NULL;
  int32_t rc = check_cache(desc);
  if (rc == SSA_OK && a->paging) rc = check_paging(a->paging, desc->max_ctx);
  if (rc != SSA_OK) return rc;
  if (a->n_q <= 0 || (long long)desc->H * a->n_q > 1ll << 24 || desc->max_ctx > kMostContext) return SSA_ERR_SHAPE;
  if (a->rotary_dims < 0 || a->rotary_dims > desc->D || a->rotary_dims % 32 != 0) return SSA_ERR_SHAPE;
  if (a->rotary_dims > 0 && !a->cos_sin) return SSA_ERR_NULL;
  if (a->rotary_dims > 0 && a->n_positions <= 0) return SSA_ERR_SHAPE;
  for (int64_t s : {a->q_stride_t, a->qo_stride_b, a->qo_stride_h, a->qo_stride_t, a->kn_stride_b, a->kn_stride_h, a->kn_stride_t,
                    a->vn_stride_b, a->vn_stride_h, a->vn_stride_t}) {
    if (s < 0) return SSA_ERR_SHAPE;
    if (s % 8 != 0) return SSA_ERR_ALIGN;
  }
  for (const void* x : {k_new, v_new, (const void*)k_cache, (const void*)v_cache, q, (const void*)q_out, (const void*)a->cos_sin})
    if (!aligned16(x)) return SSA_ERR_ALIGN;
  if (fp4 && (!aligned16(k_scales) || !aligned16(v_scales))) return SSA_ERR_ALIGN;
  // rows that several heads or requests share, or that K and V do, would be written more than once
  if (k_cache == v_cache || (fp4 && k_scales == v_scales) || desc->k_stride_t == 0 || desc->v_stride_t == 0 ||
      (desc->H_kv > 1 && (desc->k_stride_h == 0 || desc->v_stride_h == 0)) ||
      (desc->B > 1 && !a->paging && (desc->k_stride_b == 0 || desc->v_stride_b == 0)) ||
      (q && ((desc->B > 1 && a->qo_stride_b == 0) || (desc->H > 1 && a->qo_stride_h == 0) || (a->n_q > 1 && a->qo_stride_t == 0))))
    return SSA_ERR_UNSUPPORTED;
  const ssa_paging* pg = a->paging;
  AppendParams p = {};
  p.q = q; p.k_new = k_new; p.v_new = v_new; p.q_out = q_out; p.k = k_cache; p.v = v_cache;
  p.k_scales = static_cast<uint8_t*>(k_scales); p.v_scales = static_cast<uint8_t*>(v_scales);
  p.cos_sin = a->cos_sin; p.positions = a->positions; p.ctx_lens = ctx_lens; p.q_lens = a->q_lens;
  p.page_table = pg ? pg->page_table : nullptr; p.status = dev_status;
  p.q_sb = desc->q_stride_b; p.q_sh = desc->q_stride_h; p.q_st = a->q_stride_t;
  p.qo_sb = a->qo_stride_b; p.qo_sh = a->qo_stride_h; p.qo_st = a->qo_stride_t;
  p.kn_sb = a->kn_stride_b; p.kn_sh = a->kn_stride_h; p.kn_st = a->kn_stride_t;
  p.vn_sb = a->vn_stride_b; p.vn_sh = a->vn_stride_h; p.vn_st = a->vn_stride_t;
  p.k_sb = desc->k_stride_b; p.k_sh = desc->k_stride_h; p.k_st = desc->k_stride_t;
  p.v_sb = desc->v_stride_b; p.v_sh = desc->v_stride_h; p.v_st = desc->v_stride_t;
  p.B = desc->B; p.H = desc->H; p.H_kv = desc->H_kv; p.n_q = a->n_q; p.max_ctx = desc->max_ctx;
  p.rotary = a->rotary_dims; p.interleaved = a->interleaved != 0; p.n_positions = a->n_positions;
  p.page_table_stride = pg ? pg->page_table_stride : 0; p.n_pages = pg ? pg->n_pages : 0;
  while (pg && (1 << p.page_shift) < pg->page_size) ++p.page_shift;
  p.k_factor = a->k_factor > 0.f ? a->k_factor : 1.f;
  p.v_factor = a->v_factor > 0.f ? a->v_factor : 1.f;
  cudaStream_t st = (cudaStream_t)stream;
  const bool wide = desc->D == 128;
  cudaError_t err;
  switch (desc->kv_dtype) {
    case SSA_FP4_E2M1: err = wide ? launch_append<Fp4E2M1, 128>(p, st) : launch_append<Fp4E2M1, 64>(p, st); break;
    case SSA_FP8_E4M3: err = wide ? launch_append<Fp8E4M3, 128>(p, st) : launch_append<Fp8E4M3, 64>(p, st); break;
    case SSA_BF16: err = wide ? launch_append<__nv_bfloat16, 128>(p, st) : launch_append<__nv_bfloat16, 64>(p, st); break;
    default: err = wide ? launch_append<__half, 128>(p, st) : launch_append<__half, 64>(p, st);
  }
  if (err != cudaSuccess) return SSA_ERR_CUDA;
  note_launches(1);
  return SSA_OK;
}
