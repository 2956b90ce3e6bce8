// The grouped GEMM on 8-bit integers with a scale for each row of X and of W (kModeSwigluI8, kModeStoreI8).
#include "gemm_launch.hpp"

namespace semmoe {

int32_t launch_gemm_i8(int mode, const GemmArgs& a, int max_rows, int est_rows_per_group, hipStream_t stream) {
  if (a.nq <= 0 || max_rows <= 0) return SEMMOE_OK;
  if (a.nq > 512) return SEMMOE_EUNSUPPORTED;
  if (mode == kModeSwigluI8) return launch_bf16<kModeSwigluI8, 2, 2, 2, 2, 64>(a, max_rows, 2, stream);
  return launch_bf16<kModeStoreI8, 2, 2, 2, 2, 64>(a, max_rows, 2, stream);
}

}  // namespace semmoe
