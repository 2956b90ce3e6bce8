// The grouped GEMM's launcher for fp32 and bf16 operands, and its tuning knobs.
#include "gemm_launch.hpp"

namespace semmoe {

// Tuning knobs (semmoe_set_tuning): process-wide, read by every call from every thread; meant for tests and sweeps.
static std::atomic<int> g_tune[8] = {{-1}, {-1}, {-1}, {-1}, {-1}, {-1}, {-1}, {-1}};

int tuning_value(int key) { return (key >= 0 && key < 8) ? g_tune[key].load(std::memory_order_relaxed) : -1; }

int32_t launch_ksplit_gemm(const void* X, const void* W, int T, int N, int d, int n_parts, float* partial,
                           hipStream_t stream) {
  if (T <= 0 || N <= 0 || n_parts < 1 || n_parts > 64 || N % 4 != 0) return SEMMOE_EUNSUPPORTED;
  if (d % (64 * n_parts) != 0 || (long long)T * n_parts > 0x3fffffffLL) return SEMMOE_EUNSUPPORTED;
  GemmArgs a{};
  a.X = X; a.ldx = d;
  a.W = W; a.ldw = d; a.w_group_stride = size_t(d / n_parts);
  a.N = N; a.K = d / n_parts;
  a.offsets = nullptr; a.q_lo = 0; a.nq = n_parts; a.n_rows_single = T;
  a.group_to_weight = nullptr;
  a.out = partial; a.ldo = N;
  a.ksplit_rows = T;
  return launch_w4<kModeLogits, 64, 2, 2>(a, T * n_parts, stream);
}

int32_t launch_gemm(int mode, int dtype, const GemmArgs& a, int max_rows, int est_rows_per_group,
                    hipStream_t stream) {
  if (a.nq <= 0 || max_rows <= 0) return SEMMOE_OK;
  if (a.nq > 512) return SEMMOE_EUNSUPPORTED;
  if (dtype == SEMMOE_BF16) {
    const int bpc = tuning_value(SEMMOE_TUNE_BLOCKS_PER_CU);
    switch (mode) {
      case kModeLogits: return launch_bf16<kModeLogits, 2, 2, 2, 1, 64>(a, max_rows, 2, stream);  // 128 experts x 64 tokens
      case kModeSwiglu: return launch_by_rule<kModeSwiglu>(a, max_rows, est_rows_per_group, bpc, stream);
      case kModeSwigluGrad: return launch_by_rule<kModeSwigluGrad>(a, max_rows, est_rows_per_group, bpc, stream);
      default: return launch_by_rule<kModeStore>(a, max_rows, est_rows_per_group, bpc, stream);
    }
  }
  const int gate_id = tuning_value(SEMMOE_TUNE_GATEUP_TILE), down_id = tuning_value(SEMMOE_TUNE_DOWN_TILE);
  switch (mode) {
    case kModeLogits: return launch_f32<kModeLogits>(gate_id, a, max_rows, est_rows_per_group, stream);
    case kModeSwiglu: return launch_f32<kModeSwiglu>(gate_id, a, max_rows, est_rows_per_group, stream);
    case kModeSwigluGrad: return launch_f32<kModeSwigluGrad>(gate_id, a, max_rows, est_rows_per_group, stream);
    default: return launch_f32<kModeStore>(down_id, a, max_rows, est_rows_per_group, stream);
  }
}

}  // namespace semmoe

extern "C" int32_t semmoe_set_tuning(int32_t key, int32_t value) {
  if (key < 0 || key >= 8) return SEMMOE_EINVAL;
  semmoe::g_tune[key].store(value, std::memory_order_relaxed);
  return SEMMOE_OK;
}

extern "C" int32_t semmoe_get_tuning(int32_t key, int32_t* value_out) {
  if (key < 0 || key >= 8 || !value_out) return SEMMOE_EINVAL;
  *value_out = semmoe::tuning_value(key);
  return SEMMOE_OK;
}
