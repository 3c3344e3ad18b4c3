// Window attention of many query rows per K/V head (prompt chunks): tcgen05 tiles.  Included by window_attn.cu.
//
// A block serves 128 (token, head of the group) rows of one K/V head and goes through the tiles of 128 positions that they see
// between them.  Both contractions are tcgen05.mma in steps of 16 with fp32 accumulators:
//   S = Q . K^T   128 x 128; Q and K in shared memory (128-byte swizzle, K by TMA), S in TMEM
//   O += P . V    128 x D; P, the weights as 16-bit values, in TMEM over the first half of S (two parts: over both); V in
//                 shared memory as it lies
// Warps 0-3 do the softmax, a thread per row; warp 4 issues the matrix instructions, warp 5 the copies (6 and 7 make up its group
// of four).  A tile's chain - scores, softmax, sums, the next scores - takes some 3500 cycles, of which the tensor cores work
// 1024 and the softmax 2000; two blocks share an SM (half its TMEM each, a K and a V tile in flight besides the one at work), so
// that one's chain, start and end fill the other's gaps.  Whole prompts (4 x 4096 tokens, 32 heads, window 1024, 64 sinks) in runs
// of many calls, at the clock that the power limit leaves:
//   452 us, 561 TFLOP/s of visible pairs; full causal prompts 707 us, 778 TFLOP/s; fp32 outputs 609 and 976 us.
// In 20 calls in a row, where clocks are higher, 407 us; there with one block of 256 rows to an SM, its halves alternating, 446 (a
// block's start and end, a third of its time, stood alone); with tiles of 64 positions and two S in turn 524, when this form took
// 485 (an instruction of 128 x 64 takes as long as one of 128 x 128: the 128 rows of Q are read either way).
//
// The running maximum that weights are relative to follows the true one only where that is more than 2^8 above it, so that O
// is rescaled in a few tiles at the start and hardly ever after that; weights are then at most 2^8 (fp16: times 2^6, which
// the sum divides out again, because fp16 has little range below 1).  For a 16-bit output they are rounded once to 16 bits: as much
// as that output is rounded.  An fp32 output keeps the rest of each weight as a second 16-bit part, over the other half of S, with
// a contraction of its own, as in the kernel for few rows.  (Instructions, not the special function unit, bound the softmax: with a
// quarter of the powers on the FMA units prompts took 7 % longer.)
#pragma once
#include <cuda.h>

#include <type_traits>

#include "mma.cuh"
#include "window.cuh"

namespace ssa {

constexpr int kTileRows = 128, kTileKeys = 128;
constexpr int kTileThreads = 256;
constexpr int kSoftmaxRegs = 200, kOtherRegs = 56;  // of a thread; 128 x 200 + 128 x 56 = 256 x 128, what the launch has
constexpr int kTileSplit = 4;                       // fewest tiles worth a split of their own
constexpr float kLazy = 8.f;                        // log2 of how far weights may exceed 1

template <int D>
struct TileShape {
  static constexpr int kQHalf = kTileRows * 128, kHalf = kTileKeys * 128;   // bytes of 64 dimensions of a Q tile, of a K or V tile
  static constexpr int kQBytes = kQHalf * (D / 64), kTileBytes = kHalf * (D / 64);
  static constexpr int kStages = D == 64 ? 4 : 2;                   // K and V tiles of the ring: two blocks fit an SM
  static constexpr int kSmem = kQBytes + kStages * kTileBytes + 1024;   // (1024: room to align)
};

// ---- PTX ------------------------------------------------------------------------------------------------------------
__device__ __forceinline__ uint32_t smem_at(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void mbar_init(uint32_t bar, int count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" ::"r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint32_t bar, int bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;" ::"r"(bar), "r"(bytes) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ bool mbar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile("{ .reg .pred p; mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2; selp.u32 %0, 1, 0, p; }"
               : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok;
}
constexpr long long kPatience = 4000000000;         // cycles
// Waits end: after some two seconds the block gives up (*dead), and everything in it runs to its end without waiting, asking for
// no more copies.  What is under way then is still waited for (mbar_drain): nothing arrives in memory that is another block's by
// that time.
__device__ __forceinline__ bool mbar_wait(uint32_t bar, uint32_t parity, volatile int* dead) {      // false: given up
  if (mbar_try(bar, parity)) return true;
  if (*dead) return false;                                   // (a try may last: one for each wait that is left)
  for (int i = 0; i < 64; ++i)
    if (mbar_try(bar, parity)) return true;
  const long long since = clock64();
  while (!mbar_try(bar, parity)) {
    if (*dead) return false;
    if (clock64() - since > kPatience) { *dead = 1; return false; }
  }
  return true;
}
__device__ __forceinline__ void mbar_drain(uint32_t bar, uint32_t parity) {
  for (const long long since = clock64(); !mbar_try(bar, parity) && clock64() - since <= kPatience;) {}
}
__device__ __forceinline__ void tma_load(uint32_t to, const CUtensorMap* map, int x, int row, int head, int b, uint32_t bar) {
  asm volatile("cp.async.bulk.tensor.4d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}], [%6];"
               ::"r"(to), "l"(map), "r"(x), "r"(row), "r"(head), "r"(b), "r"(bar) : "memory");
}
__device__ __forceinline__ bool elect_one() {
  uint32_t is;
  asm volatile("{ .reg .pred p; elect.sync _|p, 0xffffffff; selp.u32 %0, 1, 0, p; }" : "=r"(is));
  return is;
}
__device__ __forceinline__ void tc_commit(uint32_t bar) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile("{ .reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p; }"
               ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"((int)add) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, bool add) {
  asm volatile("{ .reg .pred p; setp.ne.b32 p, %4, 0; tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p; }"
               ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"((int)add) : "memory");
}
#define SSA_R8(v, i) "=r"(v[i]), "=r"(v[i + 1]), "=r"(v[i + 2]), "=r"(v[i + 3]), "=r"(v[i + 4]), "=r"(v[i + 5]), "=r"(v[i + 6]), "=r"(v[i + 7])
#define SSA_W8(v, i) "r"(v[i]), "r"(v[i + 1]), "r"(v[i + 2]), "r"(v[i + 3]), "r"(v[i + 4]), "r"(v[i + 5]), "r"(v[i + 6]), "r"(v[i + 7])
// 32 columns of this warp's 32 lanes: a thread has its row's.
__device__ __forceinline__ void tc_ld32(uint32_t (&v)[32], uint32_t at) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,"
               "%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
               : SSA_R8(v, 0), SSA_R8(v, 8), SSA_R8(v, 16), SSA_R8(v, 24) : "r"(at));
}
__device__ __forceinline__ void tc_st32(uint32_t at, const uint32_t (&v)[32]) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,"
               "%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31};"
               ::SSA_W8(v, 0), SSA_W8(v, 8), SSA_W8(v, 16), SSA_W8(v, 24), "r"(at) : "memory");
}
#undef SSA_R8
#undef SSA_W8

__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b) {
  float2 y;
  asm("add.rn.f32x2 %0, %1, %2;"
      : "=l"(*reinterpret_cast<unsigned long long*>(&y))
      : "l"(*reinterpret_cast<unsigned long long*>(&a)), "l"(*reinterpret_cast<unsigned long long*>(&b)));
  return y;
}
// The lowest n of 32 bits, for any n.
__device__ __forceinline__ uint32_t bits_below(int n) { return n <= 0 ? 0u : n >= 32 ? ~0u : (1u << n) - 1; }

// Shared-memory operand with 128-byte swizzle.  Rows of 128 bytes, groups of eight rows 1024 bytes apart; `lead`: bytes from
// one 64-element part of the contiguous dimension to the next, where one instruction spans several (V).
__device__ __forceinline__ uint64_t tile_desc(uint32_t at, uint32_t lead) {
  return (uint64_t)((at & 0x3ffffu) >> 4) | (uint64_t)(lead >> 4) << 16 | (uint64_t)(1024 >> 4) << 32 | 1ull << 46 | 2ull << 61;
}
// fp32 accumulators of 128 rows and N columns; A along its rows; B along its rows (K) or across them (V).
template <typename T, int N, bool kAcross>
__device__ constexpr uint32_t tile_idesc() {
  const uint32_t type = sizeof(T) == 2 && std::is_same<T, __nv_bfloat16>::value ? 1 : 0;
  return 1u << 4 | type << 7 | type << 10 | (kAcross ? 1u << 16 : 0u) | (uint32_t)(N / 8) << 17 | (uint32_t)(kTileRows / 16) << 24;
}

// One row again in fp32, by a warp, with the infinities and NaNs of V kept to where they are seen: lane i's dimensions i D/32 ...
template <typename T, int D, bool kPaged>
__device__ __noinline__ void careful_row(const WindowParams& p, const Seen& seen, int2 range, int b, int h, int t, int pos, float& m,
                                         float& l, float (&acc)[D / 32]) {
  constexpr int kN = D / 32;
  const int lane = threadIdx.x % 32, hkv = h / p.group;
  const T* q = reinterpret_cast<const T*>(p.q) + (int64_t)b * p.q_sb + (int64_t)h * p.q_sh + (int64_t)t * p.q_st + lane * kN;
  const T* k = reinterpret_cast<const T*>(p.k) + (kPaged ? 0 : (int64_t)b * p.k_sb) + (int64_t)hkv * p.k_sh + lane * kN;
  const T* v = reinterpret_cast<const T*>(p.v) + (kPaged ? 0 : (int64_t)b * p.v_sb) + (int64_t)hkv * p.v_sh + lane * kN;
  const int32_t* table = kPaged ? p.page_table + (int64_t)b * p.page_table_stride : nullptr;
  float odd[kN], qf[kN];
  m = neg_inf();
  l = 0.f;
#pragma unroll
  for (int i = 0; i < kN; ++i) { acc[i] = odd[i] = 0.f; qf[i] = to_float(q[i]); }
  for (int it = range.x; it < range.y; ++it)
    for (int j = seen.position(it); j < seen.position(it) + kTileKeys; ++j) {
      if (!sees(p, pos, j)) continue;
      const int64_t row = row_of<kPaged>(p, table, j);
      if (row < 0) continue;
      float s = 0.f;
#pragma unroll
      for (int i = 0; i < kN; ++i) s = fmaf(qf[i], to_float(k[row * p.k_st + i]), s);
#pragma unroll
      for (int o = 16; o; o /= 2) s += __shfl_xor_sync(~0u, s, o);
      s *= p.scale_log2;
      const float top = fmaxf(m, s), base = top == neg_inf() ? 0.f : top, a = fast_exp2(m - base), w = fast_exp2(s - base);
      m = top;
      l = fmaf(l, a, w);
#pragma unroll
      for (int i = 0; i < kN; ++i) {
        const float x = to_float(v[row * p.v_st + i]);
        if (isfinite(x)) acc[i] = fmaf(acc[i], a, w * x);
        else { acc[i] *= a; odd[i] += x; }
      }
    }
#pragma unroll
  for (int i = 0; i < kN; ++i) acc[i] += odd[i];
}

// grid (splits x row blocks, H_kv, B), the last row blocks first: they see most.  kBoth: weights in two 16-bit parts.
template <typename T, int D, bool kPaged, bool kBoth>
__global__ void __launch_bounds__(kTileThreads, 2)
window_tile_kernel(const WindowParams p, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map,
                   const int box_rows) {
  using Shape = TileShape<D>;
  constexpr int kStages = Shape::kStages;
  constexpr float kShift = std::is_same<T, __half>::value ? 6.f : 0.f;
  extern __shared__ uint8_t smem_raw[];
  __shared__ __align__(8) uint64_t s_bar[3 * kStages + 4];
  __shared__ uint32_t s_tmem;
  __shared__ int64_t s_row[2][kTileRows];                              // where a row starts in q and in out
  __shared__ int s_dead, s_asked;                                      // the block has given up; copies asked for
  const uint32_t base = (smem_at(smem_raw) + 1023) & ~1023u;
  uint8_t* const smem = smem_raw + (base - smem_at(smem_raw));
  const uint32_t full = smem_at(s_bar), empty = full + 8 * kStages, fixed = empty + 8 * kStages, s_full = fixed + 8 * kStages,
                 p_full = s_full + 8, o_full = p_full + 16;            // p_full: of each half
  const int warp = threadIdx.x / 32, lane = threadIdx.x % 32;
  grid_dependency_wait();
  grid_launch_dependents();
  const int block = p.n_splits == 1 ? blockIdx.x : blockIdx.x / p.n_splits, split = blockIdx.x - block * p.n_splits;
  const int row0 = ((p.group * p.n_q - 1) / kTileRows - block) * kTileRows, hkv = blockIdx.y, b = blockIdx.z;
  uint32_t flags = 0;
  int ctx, n_new;
  window_sizes(p, b, ctx, n_new, flags);
  if (flags && p.status && split == 0 && row0 == 0 && hkv == 0 && threadIdx.x == 0) atomicOr(p.status, flags);
  const int rows = min(kTileRows, n_new * p.group - row0);            // rows of tokens that exist
  if (rows <= 0) return;
  const int first = ctx - n_new;
  const int t_lo = token_of(p, row0), t_hi = token_of(p, row0 + rows - 1), lo = first + t_lo, hi = first + t_hi;
  const Seen seen(p, kTileKeys, first, t_lo, t_hi);
  const int n_splits = splits_used(p, seen.tiles);
  if (split >= n_splits) return;
  const int2 range = split_tiles(seen.tiles, split, n_splits);
  // whether the tile has positions that no token sees: their rows of V may hold anything, and are made zero
  const int from = p.window == 0 ? 0 : max(0, lo - p.window + 1);
  auto unseen = [&](int it) {
    const int j0 = seen.position(it), jz = j0 + kTileKeys - 1;
    return jz > hi || !(j0 >= from || jz < p.sinks || from <= p.sinks);
  };
  const uint32_t kv = base + Shape::kQBytes;
  const int n_tiles = range.y - range.x, n_loads = 2 * n_tiles;
  volatile int* dead = &s_dead;

  // ---- copies, by warp 5: K(0), V(0), K(1), ... into a ring of stages ----
  auto load = [&](int i) {
    const int stage = i % kStages, j0 = seen.position(range.x + i / 2);
    if (lane == 0) mbar_expect(full + 8 * stage, Shape::kTileBytes);
    __syncwarp();
    if (lane < kTileKeys / box_rows) {
      int row = j0, batch = b;
      if constexpr (kPaged) {
        // pages that no token sees a position of, and pages that do not exist, are read as zeros: a row behind the last
        const int ja = j0 + lane * box_rows, jz = ja + box_rows - 1;
        const bool used = ja <= hi && (jz >= from || ja < p.sinks);
        const int64_t at = used ? row_of<true>(p, p.page_table + (int64_t)b * p.page_table_stride, ja) : -1;
        row = at < 0 ? p.n_pages << p.page_shift : (int)at;
        batch = 0;
      }
      const uint32_t to = kv + stage * Shape::kTileBytes + lane * box_rows * 128;
#pragma unroll
      for (int x = 0; x < D / 64; ++x)
        tma_load(to + x * Shape::kHalf, i & 1 ? &v_map : &k_map, x * 64, row, hkv, batch, full + 8 * stage);
    }
  };
  // Rows of V that no token sees become zero.  A copy's turn comes after the next one has been asked for (which needs no more of V).
  int settled = 1;
  auto settle = [&](int upto) {
    for (; settled <= upto; settled += 2) {
      if (!unseen(range.x + settled / 2)) continue;
      const int stage = settled % kStages, j0 = seen.position(range.x + settled / 2);
      mbar_wait(full + 8 * stage, (settled / kStages) & 1, dead);
      for (int r = lane / 8; r < kTileKeys; r += 4) {
        const int j = j0 + r;
        if (j <= hi && (j >= from || j < p.sinks)) continue;
#pragma unroll
        for (int x = 0; x < D / 64; ++x)
          *reinterpret_cast<uint4*>(smem + (kv - base) + stage * Shape::kTileBytes + x * Shape::kHalf + r * 128 + lane % 8 * 16) =
              make_uint4(0, 0, 0, 0);
      }
      asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
      mbar_arrive(fixed + 8 * stage);
    }
  };
  if (warp == 5) {
    if (lane == 0) {
      for (int i = 0; i < kStages; ++i) { mbar_init(full + 8 * i, 1); mbar_init(empty + 8 * i, 1); mbar_init(fixed + 8 * i, 32); }
      mbar_init(s_full, 1);
      mbar_init(o_full, 1);
      for (int half = 0; half < 2; ++half) mbar_init(p_full + 8 * half, kTileRows);
      s_dead = 0;
      s_asked = n_loads;
      asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncwarp();
    for (int i = 0; i < min(kStages, n_loads); ++i) load(i);
  }
  if (warp == 4) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_at(&s_tmem)), "n"(256) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;");
  }
  if (warp < 4) {                                                      // queries: a warp's 32 rows, D / 8 lanes to a row, swizzled
    constexpr int kLanes = D / 8, kAtOnce = 32 / kLanes;
    const int i = lane % kLanes;
    {
      const int row = row0 + (int)threadIdx.x, t = token_of(p, row), h = hkv * p.group + row - t * p.group;
      s_row[0][threadIdx.x] = (int64_t)b * p.q_sb + (int64_t)h * p.q_sh + (int64_t)t * p.q_st;
      s_row[1][threadIdx.x] = (int64_t)b * p.o_sb + (int64_t)h * p.o_sh + (int64_t)t * p.o_st;
    }
    __syncwarp();
    uint4 w[32 / kAtOnce];
#pragma unroll
    for (int y = 0; y < 32 / kAtOnce; ++y) {
      const int r = warp * 32 + y * kAtOnce + lane / kLanes;
      w[y] = make_uint4(0, 0, 0, 0);
      if (r < rows) w[y] = *reinterpret_cast<const uint4*>(reinterpret_cast<const T*>(p.q) + s_row[0][r] + i * 8);
    }
#pragma unroll
    for (int y = 0; y < 32 / kAtOnce; ++y) {
      const int r = warp * 32 + y * kAtOnce + lane / kLanes;
      *reinterpret_cast<uint4*>(smem + i / 8 * Shape::kQHalf + r * 128 + ((i % 8) ^ (r & 7)) * 16) = w[y];
    }
    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
  }
  tc_before();
  __syncthreads();
  tc_after();
  const uint32_t tmem = s_tmem;

  if (warp == 5) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    settle(min(kStages, n_loads) - 2);
    for (int i = kStages; i < n_loads; ++i) {
      if (!__all_sync(~0u, mbar_wait(empty + 8 * (i % kStages), (i / kStages - 1) & 1, dead))) {
        s_asked = i;
        break;
      }
      load(i);
      settle(i - 1);
    }
    settle(n_loads - 1);
  } else if (warp == 4) {
    // ---- matrix instructions: the whole warp goes through this, so that addresses stay in uniform registers; one lane issues ----
    constexpr uint32_t kIdS = tile_idesc<T, kTileKeys, false>(), kIdO = tile_idesc<T, D, true>();
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
    const bool leader = elect_one();
    uint32_t fixes = 0;                                      // phases of `fixed`
    const uint64_t q_desc = tile_desc(base, 16), k_desc = tile_desc(kv, 16), v_desc = tile_desc(kv, Shape::kHalf);
    auto wait_full = [&](int i) { mbar_wait(full + 8 * (i % kStages), (i / kStages) & 1, dead); };
    auto scores = [&](int tile) {
      const int stage = 2 * tile % kStages;
      wait_full(2 * tile);
      tc_after();
      const uint64_t kd = k_desc + stage * (Shape::kTileBytes >> 4);
      if (leader) {
#pragma unroll
        for (int s = 0; s < D / 16; ++s)
          mma_ss(tmem, q_desc + (s / 4 * (Shape::kQHalf >> 4) + s % 4 * 2), kd + (s / 4 * (Shape::kHalf >> 4) + s % 4 * 2), kIdS, s > 0);
        tc_commit(s_full);
        tc_commit(empty + 8 * stage);
      }
      __syncwarp();
    };
    if (n_tiles > 0) scores(0);
    for (int tile = 0; tile < n_tiles; ++tile) {
      const int i = 2 * tile + 1, stage = i % kStages;
      wait_full(i);
      if (unseen(range.x + tile)) {
        mbar_wait(fixed + 8 * stage, fixes >> stage & 1, dead);
        fixes ^= 1u << stage;
      }
      const uint64_t vd = v_desc + stage * (Shape::kTileBytes >> 4);
#pragma unroll
      for (int half = 0; half < 2; ++half) {                 // the weights come in two halves
        mbar_wait(p_full + 8 * half, tile & 1, dead);
        tc_after();
        if (leader) {
#pragma unroll
          for (int s = 4 * half; s < 4 * half + 4; ++s) {
            mma_ts(tmem + 128, tmem + s * 8, vd + s * (2048 >> 4), kIdO, tile > 0 || s > 0);
            if constexpr (kBoth) mma_ts(tmem + 128, tmem + 64 + s * 8, vd + s * (2048 >> 4), kIdO, true);
          }
          if (half) {
            tc_commit(empty + 8 * stage);
            if (tile + 1 == n_tiles) tc_commit(o_full);
          }
        }
        __syncwarp();
      }
      if (tile + 1 < n_tiles) scores(tile + 1);              // over weights that the contraction just issued takes
    }
  } else if (warp < 4) {
    // ---- softmax: a thread per row ----
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kSoftmaxRegs));
    const int row = row0 + (int)threadIdx.x;
    const bool there = (int)threadIdx.x < rows;
    const int t = token_of(p, row), h = hkv * p.group + row - t * p.group, pos = there ? first + t : -1;
    const uint32_t s_at = tmem + ((uint32_t)(warp * 32) << 16), o_at = s_at + 128;
    const int all_lo = p.window == 0 ? 0 : hi - p.window + 1;          // every row sees [all_lo, lo]
    const int window_lo = p.window == 0 ? 0 : pos - p.window + 1;
    const int32_t* table = kPaged ? p.page_table + (int64_t)b * p.page_table_stride : nullptr;
    float m = neg_inf(), l = 0.f;
    int n = 0;                                               // tiles so far
    for (int it = range.x; it < range.y; ++it) {
      const int j0 = seen.position(it);
      unsigned have = ~0u;                                   // positions 4 i ... 4 i + 3 have a page
      if constexpr (kPaged) {
        const int j = j0 + lane * 4;
        bool used = false;
        for (int y = j; y < j + 4; ++y) used |= y <= hi && (y >= from || y < p.sinks);
        const bool gone = used && row_of<true>(p, table, j) < 0;
        have = __ballot_sync(~0u, !gone);
        if (gone) flags |= SSA_DEV_BAD_INDEX;
      }
      mbar_wait(s_full, n & 1, dead);
      tc_after();
      uint32_t s[4][32];
#pragma unroll
      for (int c = 0; c < 4; ++c) tc_ld32(s[c], s_at + c * 32);
      tc_wait_ld();
      const bool whole = have == ~0u && j0 + kTileKeys - 1 <= lo && (j0 >= all_lo || j0 + kTileKeys <= p.sinks);
      if (!whole) {
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          // a bit per position: up to the row's own, and from its window on or below the sinks
          const int j = j0 + c * 32;
          uint32_t seen_bits = bits_below(pos + 1 - j) & (~bits_below(window_lo - j) | bits_below(p.sinks - j));
          if constexpr (kPaged) {
            if (have != ~0u) {
#pragma unroll
              for (int y = 0; y < 8; ++y)
                if (!(have >> (c * 8 + y) & 1)) seen_bits &= ~(15u << (4 * y));
            }
          }
#pragma unroll
          for (int i = 0; i < 32; ++i)
            if (!(seen_bits >> i & 1)) s[c][i] = 0xff800000u;
        }
      }
      float top[4] = {neg_inf(), neg_inf(), neg_inf(), neg_inf()};
#pragma unroll
      for (int c = 0; c < 128; c += 2)
        top[c / 2 % 4] = max3(top[c / 2 % 4], __uint_as_float(s[c / 32][c % 32]), __uint_as_float(s[c / 32][c % 32 + 1]));
      const float now = fmaxf(max3(top[0], top[1], top[2]), top[3]) * p.scale_log2;
      const bool higher = now > m + kLazy;                   // (m = -inf: anything)
      if (__any_sync(~0u, higher)) {
        const float to = higher ? now : m;
        const float a = m == to ? 1.f : fast_exp2(m - to);
        m = to;
        l *= a;
        if (n > 0) {                                         // S is there, so the contraction before it has ended
#pragma unroll 1
          for (int c = 0; c < D / 32; ++c) {
            uint32_t o[32];
            tc_ld32(o, o_at + c * 32);
            tc_wait_ld();
#pragma unroll
            for (int i = 0; i < 32; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * a);
            tc_st32(o_at + c * 32, o);
          }
        }
      }
      const float off1 = (m == neg_inf() ? 0.f : -m) + kShift;
      const float2 off = make_float2(off1, off1), by = make_float2(p.scale_log2, p.scale_log2);
      float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
#pragma unroll
      for (int half = 0; half < 2; ++half) {
        uint32_t w[32], rest[kBoth ? 32 : 1];
#pragma unroll
        for (int i = 0; i < 32; ++i) {
          const int e = half * 64 + 2 * i;
          float2 y = fma2(make_float2(__uint_as_float(s[e / 32][e % 32]), __uint_as_float(s[e / 32][e % 32 + 1])), by, off);
          y = make_float2(fast_exp2(y.x), fast_exp2(y.y));
          sum[i & 1] = add2(sum[i & 1], y);
          w[i] = pack2<T>(y.x, y.y);
          if constexpr (kBoth) {
            const float2 back = unpack2<T>(w[i]);
            rest[i] = pack2<T>(y.x - back.x, y.y - back.y);
          }
        }
        tc_st32(s_at + half * 32, w);
        if constexpr (kBoth) tc_st32(s_at + 64 + half * 32, rest);
        tc_wait_st();
        tc_before();
        mbar_arrive(p_full + 8 * half);             // its contraction starts meanwhile
      }
      l += (sum[0].x + sum[0].y) + (sum[1].x + sum[1].y);
      ++n;
    }
    if (n > 0) mbar_wait(o_full, 0, dead);
    tc_after();

    // ---- the row: out, or a split's part of it ----
    const int64_t at = ((int64_t)b * p.H + h) * p.n_q + t, slot = at * p.n_splits + split;
    const bool finished = n_splits == 1;
    const float scale = finished ? (l == 0.f ? 0.f : 1.f / l) : 1.f;
    float2 test = make_float2(l * 0.f, 0.f);
    float* out32 = finished ? reinterpret_cast<float*>(p.out) + s_row[1][threadIdx.x] : p.ws_acc + slot * D;
    const bool staged = finished && !p.out_f32;              // 16-bit rows go through the queries' place, to be stored whole
    const int rw = threadIdx.x;
    uint8_t* stage = smem;
#pragma unroll 1
    for (int c = 0; c < D / 32; ++c) {
      uint32_t o[32];
      tc_ld32(o, o_at + c * 32);
      tc_wait_ld();
      float f[32];
#pragma unroll
      for (int i = 0; i < 32; i += 2) {                      // (0 times an infinity or a NaN is NaN)
        const float2 y = fma2(make_float2(__uint_as_float(o[i]), __uint_as_float(o[i + 1])), make_float2(scale, scale), make_float2(0.f, 0.f));
        test = fma2(y, make_float2(0.f, 0.f), test);
        f[i] = l == 0.f ? 0.f : y.x;
        f[i + 1] = l == 0.f ? 0.f : y.y;
      }
      if (staged) {
#pragma unroll
        for (int i = 0; i < 32; i += 8) {
          const int at16 = c * 4 + i / 8;
          *reinterpret_cast<uint4*>(stage + at16 / 8 * Shape::kQHalf + rw * 128 + ((at16 % 8) ^ (rw & 7)) * 16) =
              make_uint4(pack2<T>(f[i], f[i + 1]), pack2<T>(f[i + 2], f[i + 3]), pack2<T>(f[i + 4], f[i + 5]), pack2<T>(f[i + 6], f[i + 7]));
        }
      } else if (there) {
#pragma unroll
        for (int i = 0; i < 32; i += 4) *reinterpret_cast<float4*>(out32 + c * 32 + i) = make_float4(f[i], f[i + 1], f[i + 2], f[i + 3]);
      }
    }
    if (staged) {
      __syncwarp();
      constexpr int kLanes = D / 8, kAtOnce = 32 / kLanes;
      const int i = lane % kLanes;
      uint4 w[32 / kAtOnce];
#pragma unroll
      for (int y = 0; y < 32 / kAtOnce; ++y) {
        const int yr = warp * 32 + y * kAtOnce + lane / kLanes;
        w[y] = *reinterpret_cast<const uint4*>(stage + i / 8 * Shape::kQHalf + yr * 128 + ((i % 8) ^ (yr & 7)) * 16);
      }
#pragma unroll
      for (int y = 0; y < 32 / kAtOnce; ++y) {
        const int yr = warp * 32 + y * kAtOnce + lane / kLanes;
        if (yr < rows) *reinterpret_cast<uint4*>(reinterpret_cast<T*>(p.out) + s_row[1][yr] + i * 8) = w[y];
      }
    }
    if (there) {
      if (finished) {
        if (p.lse) p.lse[at] = l == 0.f ? neg_inf() : (m - kShift + log2f(l)) * kLn2;
      } else {
        p.ws_ml[slot] = make_float2(m - kShift, l);
      }
    }
    unsigned again = __ballot_sync(~0u, there && l != 0.f && !(test.x + test.y == 0.f) && !*dead);
    __syncwarp();
    while (again) {                                          // rows that met an infinity or a NaN, or what they must not see
      const int i = __ffs(again) - 1;
      again &= again - 1;
      const int rt = __shfl_sync(~0u, t, i), rh = __shfl_sync(~0u, h, i), rpos = __shfl_sync(~0u, pos, i);
      const int64_t rat = ((int64_t)b * p.H + rh) * p.n_q + rt, rslot = rat * p.n_splits + split;
      float rm, rl, acc[D / 32];
      careful_row<T, D, kPaged>(p, seen, range, b, rh, rt, rpos, rm, rl, acc);
      __syncwarp();
#pragma unroll
      for (int d = 0; d < D / 32; ++d) {
        if (finished) store_window_value<T>(p, b, rh, rt, lane * (D / 32) + d, rl == 0.f ? 0.f : acc[d] / rl);
        else p.ws_acc[rslot * D + lane * (D / 32) + d] = acc[d];
      }
      if (lane == 0) {
        if (!finished) p.ws_ml[rslot] = make_float2(rm, rl);
        else if (p.lse) p.lse[rat] = rl == 0.f ? neg_inf() : (rm + log2f(rl)) * kLn2;
      }
    }
    if (kPaged && p.status && (flags & SSA_DEV_BAD_INDEX)) atomicOr(p.status, SSA_DEV_BAD_INDEX);
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kOtherRegs));
  }
  tc_before();
  __syncthreads();
  tc_after();
  if (s_dead) {                                              // (otherwise all that was asked for has been waited for)
    for (int i = max(0, s_asked - kStages); i < s_asked; ++i) mbar_drain(full + 8 * (i % kStages), (i / kStages) & 1);
    if (n_tiles > 0) mbar_drain(o_full, 0);                  // instructions end in order: these have all
    if (threadIdx.x == 0 && p.status) atomicOr(p.status, SSA_DEV_GAVE_UP);
    __syncthreads();
    tc_after();
  }
  if (warp == 4) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(256));
}

// ---- host ------------------------------------------------------------------------------------------------------------
// A cache or pool as (D, rows, heads, requests), read in boxes of 64 elements x box_rows rows.  False where the strides are
// none that the copies take (the call is then left to the kernel for few rows).
inline bool tile_map(CUtensorMap* map, const void* base, int32_t dtype, int D, int64_t rows, int64_t row_stride, int heads,
                     int64_t head_stride, int B, int64_t b_stride, int box_rows) {
  using Encode = CUresult (*)(CUtensorMap*, CUtensorMapDataType, cuuint32_t, void*, const cuuint64_t*, const cuuint64_t*,
                              const cuuint32_t*, const cuuint32_t*, CUtensorMapInterleave, CUtensorMapSwizzle,
                              CUtensorMapL2promotion, CUtensorMapFloatOOBfill);
  static const Encode encode = [] {
    void* f = nullptr;
    cudaDriverEntryPointQueryResult found = cudaDriverEntryPointSymbolNotFound;
    if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess) {
      cudaGetLastError();
      f = nullptr;
    }
    return reinterpret_cast<Encode>(f);
  }();
  if (!encode) return false;
  const int64_t strides[3] = {row_stride * 2, heads > 1 ? head_stride * 2 : row_stride * 2, B > 1 ? b_stride * 2 : row_stride * 2};
  cuuint64_t dims[4] = {(cuuint64_t)D, (cuuint64_t)rows, (cuuint64_t)heads, (cuuint64_t)B}, steps[3];
  for (int i = 0; i < 3; ++i) {
    if (strides[i] <= 0 || strides[i] >= 1ll << 40) return false;
    steps[i] = (cuuint64_t)strides[i];
  }
  const cuuint32_t box[4] = {64, (cuuint32_t)box_rows, 1, 1}, ones[4] = {1, 1, 1, 1};
  return encode(map, dtype == SSA_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 4, const_cast<void*>(base),
                dims, steps, box, ones, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

}  // namespace ssa
