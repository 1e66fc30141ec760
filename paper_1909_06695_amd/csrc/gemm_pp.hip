// bf16 MFMA contraction on 256x256 tiles in which the two waves of a SIMD take turns: while one runs its
// matrix instructions the other reads fragments from LDS and requests tiles from memory.
//
// What bounds it: the clock first.  With random operands the chip runs these loops at 1.54 (A B^T) and 1.69 GHz (A^T B) against
// 2.4 GHz nominal, and at that clock the matrix pipe is busy 82 and 77 % of the cycles (LDS conflicts 1 %): the rest are the
// barriers between the phases and the epilogue.  8192^3 takes 780-830 us in either form, 1.33-1.41 PFLOP/s; in the 24-layer
// 1024-wide step dh_L = G V goes 874 -> 589 us, dV_o
// 670 -> 592 us, a layer's weight gradients 255 -> 170-178 us.  The same tile with one barrier per K-tile, all eight waves in step
// (the form this one replaced), needs 895 and 912 us: fragment reads and requests then stand between the matrix
// instructions instead of beside them.  Tried on the way, same products: BK = 32 with a four-stage ring 883 / 829 us (a
// row-form request then fetches half cache lines), five stages the same (latency is not the limit), requests between the
// matrix instructions 856 / 833 us, four waves with 128x128 wave tiles and one barrier per K-tile 861 / 820 us.
//
// A workgroup has eight waves (two per SIMD).  The tile consists of two 128-row halves of A and two 128-column halves of
// B; waves 0-3 own the first 64 rows of each row half, waves 4-7 the other 64; wave % 4 owns 32 columns of each column
// half.  LDS holds two stages of the four halves (K-tile 64).  A K-tile is two phases of 16 matrix instructions:
//
//   phase  reads                 multiplies            requests
//     1    A0, B1                A0 x B0, A0 x B1      A1 of K-tile kt+1, B0 of kt+2     (both halves were last read in the phase before)
//     2    A1, B0 of kt+1        A1 x B1, A1 x B0      A0 and B1 of kt+2                 (likewise)
//
// and a phase is: read the fragments and wait for them; request; wait for the halves that the next phase reads; barrier;
// multiply; barrier (requests ahead of the reads delay them: 3 % on dV_o).  Waves 4-7 run one barrier behind waves 0-3, so one group's multiplications coincide with the other group's
// reads.  Every wave waits for its fragments before the barrier inside the phase: a wave that has begun the next phase
// knows that all eight have read what this phase reads, which is what the refill needs.  A request has two phases of both
// groups' matrix work to arrive in.
#include "gemm_pp.h"

namespace ouro {

template <bool TA, bool TB>
__global__ __launch_bounds__(512, 2) void gemm_pp_kernel(GemmParams p) {
  extern __shared__ uint4 smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  batch_offsets(p);
  int m0, n0, kbeg;
  tile_of_block(p, 256, 256, blockIdx.x, gridDim.x, m0, n0, kbeg);
  const int nk = (min(p.K, kbeg + p.kchunk) - kbeg + PP_BK - 1) / PP_BK;
  f32x16 acc[4][2];
  pp_mainloop<TA, TB>(p, m0, n0, kbeg, nk, reinterpret_cast<char*>(smem), acc);
  const int m_w = m0 + 64 * (wave >> 2), n_w = n0 + 32 * (wave & 3);
  mfma_epilogue<4, 2, !TA && TB, 128, 128>(p, acc, smem, m_w, n_w, lane, wave);
}

// Several accumulating products in one launch (weight gradients of a layer).  Product i owns the work items
// [first[i], first[i+1]), a multiple of 8 so that the low bits of a work item still name its XCD.
struct PpGroupParams {
  int n;
  int first[GEMM_GROUP_MAX + 1];
  GemmParams p[GEMM_GROUP_MAX];
};
static_assert(sizeof(PpGroupParams) <= 4096, "kernel arguments are limited to 4 KiB");
__global__ __launch_bounds__(512, 2) void gemm_pp_group_kernel(PpGroupParams g) {
  extern __shared__ uint4 smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int bid = blockIdx.x;
  int i = 0;
  while (i + 1 < g.n && bid >= g.first[i + 1]) ++i;
  const GemmParams& p = g.p[i];
  int m0, n0, kbeg;
  tile_of_block(p, 256, 256, bid - g.first[i], g.first[i + 1] - g.first[i], m0, n0, kbeg);
  if (kbeg >= p.K) return;                         // a work item past the last K range (the item count is rounded up)
  f32x16 acc[4][2];
  pp_mainloop<true, false>(p, m0, n0, kbeg, (min(p.K, kbeg + p.kchunk) - kbeg + PP_BK - 1) / PP_BK, reinterpret_cast<char*>(smem), acc);
  mfma_accumulate<4, 2, 128, 128>(p, acc, m0 + 64 * (wave >> 2), n0 + 32 * (wave & 3), lane);
}

hipError_t launch_gemm_pp(hipStream_t s, GemmParams& p, int transA, int transB, int splits) {
  static_assert((size_t)8 * epilogue_stage_floats<2>() * sizeof(float) <= PP_LDS, "the epilogue's patches fit the ring");
  p.tilesM = (p.M + 255) / 256;
  p.tilesN = (p.N + 255) / 256;
  p.ntiles = p.tilesM * p.tilesN;
  p.mfast = splits > 1 && p.N > p.M;
  p.band = splits == 1 && p.tilesM % 8 == 0 && p.tilesN % 8 == 0 && p.tilesN > 8;
  dim3 grid(p.ntiles * splits, p.by, p.bz), block(512);
#define OURO_LAUNCH(TA_, TB_)                                                                       \
  do {                                                                                              \
    static bool allowed = false;                                                                    \
    hipError_t e = pp_allow_lds((const void*)gemm_pp_kernel<TA_, TB_>, PP_LDS, allowed);            \
    if (e != hipSuccess) return e;                                                                  \
    hipLaunchKernelGGL((gemm_pp_kernel<TA_, TB_>), grid, block, PP_LDS, s, p);                      \
  } while (0)
  if (!transA && !transB) OURO_LAUNCH(false, false);
  else if (!transA && transB) OURO_LAUNCH(false, true);
  else if (transA && !transB) OURO_LAUNCH(true, false);
  else OURO_LAUNCH(true, true);
#undef OURO_LAUNCH
  return hipGetLastError();
}

// ps: kchunk set; accumulate as mfma_accumulate takes it.
hipError_t launch_gemm_pp_group(hipStream_t s, const GemmParams* ps, int n) {
  if (n < 1 || n > GEMM_GROUP_MAX) return hipErrorInvalidValue;
  PpGroupParams g;
  memset(&g, 0, sizeof g);
  g.n = n;
  for (int i = 0; i < n; ++i) {
    GemmParams p = ps[i];
    p.tilesM = (p.M + 255) / 256;
    p.tilesN = (p.N + 255) / 256;
    p.ntiles = p.tilesM * p.tilesN;
    p.mfast = p.N > p.M;                           // neighbouring tiles share the larger operand's columns
    p.band = 0;
    g.p[i] = p;
    g.first[i + 1] = g.first[i] + (p.ntiles * ((p.K + p.kchunk - 1) / p.kchunk) + 7) / 8 * 8;
  }
  static bool allowed = false;
  hipError_t e = pp_allow_lds((const void*)gemm_pp_group_kernel, PP_LDS, allowed);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(gemm_pp_group_kernel, dim3(g.first[n]), dim3(512), PP_LDS, s, g);
  return hipGetLastError();
}

}  // namespace ouro
