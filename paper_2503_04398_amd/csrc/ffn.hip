// expert_ffn / shared_ffn: the expert FFN (Sec. 2) in SwiGLU form as two grouped GEMMs over the rows
// that dispatch made contiguous per expert:  H = silu(X_perm W_gate^T) * (X_perm W_up^T),  Y = H W_down^T.
#include "gemm_core.hpp"
#include "gemm_nn.hpp"

namespace semmoe {

static int32_t run_ffn(const semmoe_config* cfg, hipStream_t s, const void* X, const int32_t* offsets, int q_lo,
                       int nq, int n_rows_single, int max_rows, int est_rows, const int32_t* group_to_weight, const void* W_gu,
                       const void* W_down, void* Y, void* H) {
  GemmArgs a{};
  a.X = X; a.ldx = cfg->d;
  a.W = W_gu; a.w_group_stride = size_t(2) * cfg->F * cfg->d; a.ldw = cfg->d;
  a.N = cfg->F; a.K = cfg->d;
  a.offsets = offsets; a.q_lo = q_lo; a.nq = nq; a.n_rows_single = n_rows_single;
  a.group_to_weight = group_to_weight;
  a.out = H; a.ldo = cfg->F;
  int32_t st = launch_gemm(kModeSwiglu, cfg->dtype, a, max_rows, est_rows, s);
  if (st != SEMMOE_OK) return st;
  GemmArgs b = a;
  b.X = H; b.ldx = cfg->F;
  b.W = W_down; b.w_group_stride = size_t(cfg->d) * cfg->F; b.ldw = cfg->F;
  b.N = cfg->d; b.K = cfg->F;
  b.out = Y; b.ldo = cfg->d;
  return launch_gemm(kModeStore, cfg->dtype, b, max_rows, est_rows, s);
}

// The gradient towards the rows, the weights standing still:  dh = dY W_down;  [dg | du] from dh and the gate and up products,
// taken again and never written down;  dX = [dg | du] W_gu.  dh stays fp32 on its way to the second product's epilogue; dg and
// du are rounded to the act type, which the third product's operands are.  With that and the result's rounding bf16 rows are off by
// 2.35e-3 of their norm, where the result's alone is 1.66e-3; in two bf16 parts each they would double the last product
// (16 experts of 1300 rows, d 2048, F 768: 142 to 160 of 400 us).
static int32_t run_ffn_grad(const semmoe_config* cfg, hipStream_t s, const void* X, const void* dY, const int32_t* offsets,
                            int q_lo, int nq, int n_rows_single, int max_rows, int est_rows, const int32_t* group_to_weight,
                            const void* W_gu, const void* W_down, void* dX, float* dH, void* dGU) {
  GemmArgs h{};
  h.X = dY; h.ldx = cfg->d;
  h.W = W_down; h.w_group_stride = size_t(cfg->d) * cfg->F; h.ldw = cfg->F;
  h.N = cfg->F; h.K = cfg->d;
  h.offsets = offsets; h.q_lo = q_lo; h.nq = nq; h.n_rows_single = n_rows_single;
  h.group_to_weight = group_to_weight;
  h.out = dH;  // blocks of 32 rows
  int32_t st = launch_gemm_nn(kNnSums, cfg->dtype, h, max_rows, est_rows, s);
  if (st != SEMMOE_OK) return st;
  GemmArgs a = h;
  a.X = X;
  a.W = W_gu; a.w_group_stride = size_t(2) * cfg->F * cfg->d; a.ldw = cfg->d;
  a.b_g = dH;
  a.out = dGU; a.ldo = 2 * cfg->F;
  st = launch_gemm(kModeSwigluGrad, cfg->dtype, a, max_rows, est_rows, s);
  if (st != SEMMOE_OK) return st;
  GemmArgs b = a;
  b.X = dGU; b.ldx = 2 * cfg->F;
  b.N = cfg->d; b.K = 2 * cfg->F;
  b.out = dX; b.ldo = cfg->d;
  b.sched_reverse = 1;  // W_gu from where the second product left off: 128 experts of 62 rows 468 -> 460 us
  return launch_gemm_nn(kNnStore, cfg->dtype, b, max_rows, est_rows, s);
}

size_t ws_ffn(const semmoe_config* cfg) {
  return align_up(size_t(cfg->T) * cfg->k * cfg->F * act_bytes(cfg), 256) + 256;  // hidden activation H[P,F]
}

}  // namespace semmoe

using namespace semmoe;

extern "C" int32_t semmoe_expert_ffn(const semmoe_config* cfg, void* stream, int32_t rank, const void* X_perm,
                                     const int32_t* expert_offsets, const int32_t* expert_of_phys, const void* W_gu,
                                     const void* W_down, void* Y, void* ws, size_t ws_bytes) {
  int32_t st = validate_config(cfg, true, true, true);
  if (st != SEMMOE_OK) return st;
  if (!X_perm || !expert_offsets || !expert_of_phys || !W_gu || !W_down || !Y) return SEMMOE_EINVAL;
  if (rank < -1 || rank >= cfg->D) return SEMMOE_EINVAL;
  if (!aligned16(X_perm) || !aligned16(W_gu) || !aligned16(W_down) || !aligned16(Y)) return SEMMOE_EINVAL;
  Carver c(ws, ws_bytes);
  void* H = c.take<char>(size_t(cfg->T) * cfg->k * cfg->F * act_bytes(cfg));
  if (!c.ok) return SEMMOE_EWORKSPACE;
  const int m = cfg->E / cfg->D;
  const int q_lo = rank < 0 ? 0 : rank * m;
  const int nq = rank < 0 ? cfg->E : m;
  return run_ffn(cfg, static_cast<hipStream_t>(stream), X_perm, expert_offsets, q_lo, nq, 0, cfg->T * cfg->k,
                 cfg->T * cfg->k / cfg->E, expert_of_phys, W_gu, W_down, Y, H);
}

extern "C" int32_t semmoe_shared_ffn(const semmoe_config* cfg, void* stream, const void* X, int32_t n_tokens,
                                     const void* W_gu_sh, const void* W_down_sh, void* Y_shared, void* ws,
                                     size_t ws_bytes) {
  int32_t st = validate_config(cfg, true, true, true);
  if (st != SEMMOE_OK) return st;
  if (!X || !W_gu_sh || !W_down_sh || !Y_shared || n_tokens < 0) return SEMMOE_EINVAL;
  if ((long long)n_tokens > (long long)cfg->T * cfg->k) return SEMMOE_ESHAPE;
  if (!aligned16(X) || !aligned16(W_gu_sh) || !aligned16(W_down_sh) || !aligned16(Y_shared)) return SEMMOE_EINVAL;
  Carver c(ws, ws_bytes);
  void* H = c.take<char>(size_t(n_tokens) * cfg->F * act_bytes(cfg));
  if (!c.ok) return SEMMOE_EWORKSPACE;
  if (n_tokens == 0) return SEMMOE_OK;
  return run_ffn(cfg, static_cast<hipStream_t>(stream), X, nullptr, 0, 1, n_tokens, n_tokens, n_tokens, nullptr, W_gu_sh,
                 W_down_sh, Y_shared, H);
}

extern "C" int32_t semmoe_expert_ffn_grad(const semmoe_config* cfg, void* stream, int32_t rank, const void* X_perm,
                                          const void* dY, const int32_t* expert_offsets, const int32_t* expert_of_phys,
                                          const void* W_gu, const void* W_down, void* dX_perm, void* ws, size_t ws_bytes) {
  int32_t st = validate_config(cfg, true, true, true);
  if (st != SEMMOE_OK) return st;
  if (!X_perm || !dY || !expert_offsets || !expert_of_phys || !W_gu || !W_down || !dX_perm) return SEMMOE_EINVAL;
  if (rank < -1 || rank >= cfg->D) return SEMMOE_EINVAL;
  if (!aligned16(X_perm) || !aligned16(dY) || !aligned16(W_gu) || !aligned16(W_down) || !aligned16(dX_perm)) return SEMMOE_EINVAL;
  Carver c(ws, ws_bytes);
  float* dH = c.take<float>(align_up(size_t(cfg->T) * cfg->k, 32) * cfg->F);
  void* dGU = c.take<char>(size_t(cfg->T) * cfg->k * 2 * cfg->F * act_bytes(cfg));
  if (!c.ok) return SEMMOE_EWORKSPACE;
  const int m = cfg->E / cfg->D;
  const int q_lo = rank < 0 ? 0 : rank * m;
  const int nq = rank < 0 ? cfg->E : m;
  return run_ffn_grad(cfg, static_cast<hipStream_t>(stream), X_perm, dY, expert_offsets, q_lo, nq, 0, cfg->T * cfg->k,
                      cfg->T * cfg->k / cfg->E, expert_of_phys, W_gu, W_down, dX_perm, dH, dGU);
}

extern "C" int32_t semmoe_shared_ffn_grad(const semmoe_config* cfg, void* stream, const void* X, const void* dY,
                                          int32_t n_tokens, const void* W_gu_sh, const void* W_down_sh, void* dX, void* ws,
                                          size_t ws_bytes) {
  int32_t st = validate_config(cfg, true, true, true);
  if (st != SEMMOE_OK) return st;
  if (!X || !dY || !W_gu_sh || !W_down_sh || !dX || n_tokens < 0) return SEMMOE_EINVAL;
  if ((long long)n_tokens > (long long)cfg->T * cfg->k) return SEMMOE_ESHAPE;
  if (!aligned16(X) || !aligned16(dY) || !aligned16(W_gu_sh) || !aligned16(W_down_sh) || !aligned16(dX)) return SEMMOE_EINVAL;
  Carver c(ws, ws_bytes);
  float* dH = c.take<float>(align_up(size_t(n_tokens), 32) * cfg->F);
  void* dGU = c.take<char>(size_t(n_tokens) * 2 * cfg->F * act_bytes(cfg));
  if (!c.ok) return SEMMOE_EWORKSPACE;
  if (n_tokens == 0) return SEMMOE_OK;
  return run_ffn_grad(cfg, static_cast<hipStream_t>(stream), X, dY, nullptr, 0, 1, n_tokens, n_tokens, n_tokens, nullptr,
                      W_gu_sh, W_down_sh, dX, dH, dGU);
}
