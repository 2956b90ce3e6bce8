// Kernel instantiations and the host launcher of the grouped NN GEMM.
#include "gemm_nn.hpp"

namespace semmoe {

static int nn_grid(long long bound, int per_cu) {
  DeviceInfo d;
  const long long cap = (long long)(device_info(&d) == SEMMOE_OK ? d.num_cu : 256) * per_cu;
  bound = (bound + 7) / 8 * 8;  // whole rounds over the XCDs
  return int(bound < cap ? bound : cap);
}

template <int MODE, int NWF, int NWT, int TF, int TT, int BK, int NSTAGE>
static int32_t launch_nn_ring(const GemmArgs& a, int max_rows, int per_cu, hipStream_t s) {
  using C = NnCfg<NWF, NWT, TF, TT, BK, NSTAGE>;
  auto kern = gemm_nn_ring_kernel<MODE, NWF, NWT, TF, TT, BK, NSTAGE>;
  static std::atomic<uint64_t> allowed{0};
  const int32_t st = allow_max_dynamic_lds(&allowed, reinterpret_cast<const void*>(kern));
  if (st != SEMMOE_OK) return st;
  const long long bound = (long long)(max_rows / C::BT + a.nq) * cdiv(a.N, C::BW);
  hipLaunchKernelGGL(kern, dim3(nn_grid(bound, per_cu)), dim3(C::kThreads), C::kLdsBytes, s, a);
  SEMMOE_LAUNCH_CHECK();
  return SEMMOE_OK;
}

template <int MODE, int TT>
static int32_t launch_nn_f32(const GemmArgs& a, int max_rows, hipStream_t s) {
  const long long bound = (long long)(max_rows / (32 * TT) + a.nq) * cdiv(a.N, 128);
  hipLaunchKernelGGL((gemm_nn_f32_kernel<MODE, TT>), dim3(nn_grid(bound, 2)), dim3(256), 0, s, a);
  SEMMOE_LAUNCH_CHECK();
  return SEMMOE_OK;
}

template <int MODE>
static int32_t launch_nn(int dtype, const GemmArgs& a, int max_rows, int est, hipStream_t s) {
  if (dtype == SEMMOE_FP32) return est <= 32 ? launch_nn_f32<MODE, 1>(a, max_rows, s) : launch_nn_f32<MODE, 2>(a, max_rows, s);
  if (est < 96) return launch_nn_ring<MODE, 2, 2, 2, 1, 64, 3>(a, max_rows, 2, s);
  return launch_nn_ring<MODE, 2, 4, 4, 2, 64, 2>(a, max_rows, 1, s);
}

int32_t launch_gemm_nn(int mode, int dtype, const GemmArgs& a, int max_rows, int est, hipStream_t s) {
  if (a.nq <= 0 || max_rows <= 0) return SEMMOE_OK;
  if (a.nq > 512) return SEMMOE_EUNSUPPORTED;
  return mode == kNnSwigluGrad ? launch_nn<kNnSwigluGrad>(dtype, a, max_rows, est, s) : launch_nn<kNnStore>(dtype, a, max_rows, est, s);
}

}  // namespace semmoe
