// Window attention over a cache of 4-bit values (ssa_attn_window_fp4): the kernels of window_rows.cuh and window_tile.cuh for such rows.
#include "window_tile.cuh"

namespace ssa {

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
  err = launch_pdl(window_join_kernel<__nv_bfloat16, D, Fp4Params>, dim3((unsigned)((p.H * p.n_q + kJoinWarps - 1) / kJoinWarps), (unsigned)p.B),
                   dim3(kJoinWarps * 32), st, p);
  if (err != cudaSuccess) return SSA_ERR_CUDA;
  note_launches(1);
  return SSA_OK;
}

int32_t launch_window_fp4(const Fp4Params& p, int D, int box_rows, cudaStream_t st) {
  return D == 128 ? launch<128>(p, box_rows, st) : launch<64>(p, box_rows, st);
}

}  // namespace ssa
