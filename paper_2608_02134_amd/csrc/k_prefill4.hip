// Attention of the newest tokens of each sequence over a paged cache of 4 bits.
//
// The products are those over pages of the type (k_prefill.hip): a tile of keys in
// shared memory serves 128 rows, so its values are formed once, as bf16, between the
// pages and shared memory, while the codes of the next tile are on their way to a place
// of their own there.  A tile so costs a thread 32 conversions and 8 writes more than
// one of bf16 pages: 16448 tokens, window 4096, 28 heads on 4 of 128 in bf16 1.00 ms, 845
// TFLOP/s (bf16 pages 0.96 on the same card).
// fp32 queries and weights enter as three bf16 (gmc_prefill.h): 4096 tokens, 28 heads
// on 4 of 128, 0.63 ms; products of fp32 took 1.82.  bf16 weights are rounded to bf16 once
// for the second product, as over pages of bf16 (and not as in decode, which has the
// matrix cores to spare for two parts): the outputs' error against 64 bits, relative to
// their size, is 0.0018 to 0.0022, where two parts of each weight have the 0.0016 of the
// output's own rounding and take 1.28 ms for the 16448 tokens where this takes 1.00.
#include "gmc_prefill.h"

namespace gmc {

template <typename T, int DH>
__global__ void __launch_bounds__(64 * kPreWaves, sizeof(T) == 2 && DH <= 128 ? 2 : 1)
prefill4_kernel(CacheView c, CacheScales s, AttendArgs a, PreScratch sc, int row_blocks) {
  prefill_block<T, DH, true>(c, s, a, sc, row_blocks);
}

hipError_t launch_cache4_prefill(const CacheView& c, const CacheScales& s, const AttendArgs& a, void* scratch,
                                 hipStream_t st) {
  int row_blocks;
  const PreScratch sc = pre_plan(c, a, true, scratch, &row_blocks);
#define GMC_PREFILL4(T, DH)                                                                                       \
  case DH:                                                                                                        \
    hipLaunchKernelGGL((prefill4_kernel<T, DH>), dim3(static_cast<unsigned>(sc.grid.blocks)), dim3(64 * kPreWaves), 0, st, \
                       c, s, a, sc, row_blocks);                                                                  \
    break;
#define GMC_PREFILL4_ALL(T)                                                                                       \
  switch (c.dh) {                                                                                                 \
    GMC_PREFILL4(T, 32) GMC_PREFILL4(T, 64) GMC_PREFILL4(T, 96) GMC_PREFILL4(T, 128)                              \
    GMC_PREFILL4(T, 160) GMC_PREFILL4(T, 192) GMC_PREFILL4(T, 224) GMC_PREFILL4(T, 256)                           \
    default: return hipErrorInvalidValue;                                                                         \
  }
  if (c.dtype == 0) { GMC_PREFILL4_ALL(float) } else { GMC_PREFILL4_ALL(bf16_t) }
#undef GMC_PREFILL4_ALL
#undef GMC_PREFILL4
  const hipError_t err = hipGetLastError();
  if (err != hipSuccess) return err;   // (there is nothing to join)
  return sc.nsplit > 1 ? launch_prefill_join(c, a, sc, st) : hipSuccess;
}

}  // namespace gmc
