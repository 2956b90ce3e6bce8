// The grouped GEMM on 8-bit integers with a scale for each row of X and of W (kModeSwigluI8, kModeStoreI8): the tiles of bf16
// operands, chosen by the same rule.
//
// Why the rule carries over: a tile's time is that of its bytes (weights and rows, LDS reads) or of its MFMAs, and both are what a bf16
// product of half the depth has: 16 bytes of a row are one MFMA operand, of as many cycles.  The rule therefore gets the depth in
// pairs of integers, as the kernels do.
#include "gemm_launch.hpp"

namespace semmoe {

int32_t launch_gemm_i8(int mode, const GemmArgs& a, int max_rows, int est_rows_per_group, hipStream_t stream) {
  if (a.nq <= 0 || max_rows <= 0) return SEMMOE_OK;
  if (a.nq > 512) return SEMMOE_EUNSUPPORTED;
  const int bpc = tuning_value(SEMMOE_TUNE_BLOCKS_PER_CU);
  return mode == kModeSwigluI8 ? launch_by_rule<kModeSwigluI8>(a, max_rows, est_rows_per_group, bpc, stream)
                               : launch_by_rule<kModeStoreI8>(a, max_rows, est_rows_per_group, bpc, stream);
}

}  // namespace semmoe
