// Products of 8-bit integers with a scale for each token and each channel: linear_i8, and the SwiGLU FFN of one rank's experts or of
// the shared expert on them.
//   y[t,n] = xs[t] ws[n] sum_c x[t,c] w[n,c]   (the sum in int32, exact);
//   FFN: h = silu(gate) up of two such products, rounded to bf16 and then to 8 bits with a scale for each row, and a third.
// h lies in memory as bf16 between its product and its 8-bit form, as expert_ffn's does, since its largest magnitude is known only when
// the row is whole.  That rounding raises the error of the 8-bit form from 1.904e-2 of a row's norm to 1.911e-2 (silu(g) u of normal
// numbers, F 768; 2.243e-2 to 2.249e-2 at F 2048); fp32 would double the bytes of the pass.
// What bounds them: weights' bytes where rows are few (128 experts of 8 rows, d 2048, F 768: 604 MB in 71 + 46 us, 5.2 TB/s), the matrix
// pipes where they are many (8192 rows 7168 -> 4096: 207 us, 2.3 POP/s, busy in 58 % of the cycles at 1.9 GHz), a tile's epilogue where K is
// short (20865 rows 768 -> 2048: 64 us, 1.0 POP/s).
#include "gemm_core.hpp"
#include "rows.hpp"

namespace semmoe {

// K, ldx and the like in pairs of integers (gemm_core.hpp)
static GemmArgs i8_args(const void* Xq, int64_t ldx, const float* x_scale, const void* Wq, const float* w_scale, int w_rows, int K,
                        int N, void* out, int ldo) {
  GemmArgs a{};
  a.X = Xq; a.ldx = int(ldx / 2); a.x_scale = x_scale;
  a.W = Wq; a.ldw = K / 2; a.w_group_stride = size_t(w_rows) * K / 2; a.w_scale = w_scale;
  a.N = N; a.K = K / 2;
  a.out = out; a.ldo = ldo;
  return a;
}

struct FfnI8 {
  const void* Xq; const float* x_scale;
  const void* Wq_gu; const float* w_scale_gu;
  const void* Wq_down; const float* w_scale_down;
  void* Y;
  void* H; void* Hq; float* h_scale;  // workspace: the hidden rows in bf16 and in 8 bits
};

static int32_t run_ffn_i8(const semmoe_config* cfg, hipStream_t s, const FfnI8& f, const int32_t* offsets, int q_lo, int nq,
                          int n_rows_single, int max_rows, int est_rows, const int32_t* group_to_weight) {
  auto groups = [&](GemmArgs a) {
    a.offsets = offsets; a.q_lo = q_lo; a.nq = nq; a.n_rows_single = n_rows_single;
    a.group_to_weight = group_to_weight;
    return a;
  };
  const int d = cfg->d, F = cfg->F;
  int32_t st = launch_gemm_i8(kModeSwigluI8, groups(i8_args(f.Xq, d, f.x_scale, f.Wq_gu, f.w_scale_gu, 2 * F, d, F, f.H, F)),
                              max_rows, est_rows, s);
  if (st != SEMMOE_OK) return st;
  st = launch_quantize_rows(true, f.H, F, max_rows, F, offsets ? offsets + q_lo : nullptr, nq, f.Hq, f.h_scale, s);
  if (st != SEMMOE_OK) return st;
  return launch_gemm_i8(kModeStoreI8, groups(i8_args(f.Hq, F, f.h_scale, f.Wq_down, f.w_scale_down, d, F, d, f.Y, d)), max_rows,
                        est_rows, s);
}

static int32_t check_i8(int dtype, int64_t K) {
  if (dtype != SEMMOE_BF16) return SEMMOE_EUNSUPPORTED;
  if (K % 16 != 0) return SEMMOE_ESHAPE;
  return K > SEMMOE_MAX_I8_DEPTH ? SEMMOE_EUNSUPPORTED : SEMMOE_OK;
}

static bool carve_ffn_i8(FfnI8* f, void* ws, size_t bytes, size_t rows, int F) {
  Carver c(ws, bytes);
  f->H = c.take<bf16_t>(rows * F);
  f->Hq = c.take<char>(rows * F);
  f->h_scale = c.take<float>(rows);
  return c.ok;
}

static int32_t check_ffn_i8(const semmoe_config* cfg, const FfnI8& f) {
  int32_t st = validate_config(cfg, true, true, true);
  if (st == SEMMOE_OK) st = check_i8(cfg->dtype, cfg->d);
  if (st == SEMMOE_OK) st = check_i8(cfg->dtype, cfg->F);
  if (st != SEMMOE_OK) return st;
  if (!f.Xq || !f.x_scale || !f.Wq_gu || !f.w_scale_gu || !f.Wq_down || !f.w_scale_down || !f.Y) return SEMMOE_EINVAL;
  if (!aligned16(f.Xq) || !aligned16(f.Wq_gu) || !aligned16(f.w_scale_gu) || !aligned16(f.Wq_down) || !aligned16(f.w_scale_down) ||
      !aligned16(f.Y))
    return SEMMOE_EINVAL;
  return SEMMOE_OK;
}

}  // namespace semmoe

using namespace semmoe;

extern "C" int32_t semmoe_linear_i8(const semmoe_config* cfg, void* stream, const semmoe_linear_shape* shape, const void* Xq,
                                    const float* x_scale, const void* Wq, const float* w_scale, void* Y) {
  if (!cfg || !shape) return SEMMOE_EINVAL;
  const semmoe_linear_shape n = *shape;
  if (n.n_rows < 0 || n.d_in <= 0 || n.d_out <= 0 || n.ldx < 0 || n.ldy < 0) return SEMMOE_EINVAL;
  const int32_t st = check_i8(cfg->dtype, n.d_in);
  if (st != SEMMOE_OK) return st;
  if (n.d_out % 8 != 0 || n.ldx % 16 != 0 || n.ldy % 8 != 0 || (n.ldx > 0 && n.ldx < n.d_in) || (n.ldy > 0 && n.ldy < n.d_out))
    return SEMMOE_ESHAPE;
  if (n.n_rows > 0x3fffffff || n.ldx > 0x7fffffff || n.ldy >= 1 << 26 || n.d_out >= 1 << 26) return SEMMOE_EUNSUPPORTED;
  if (!Xq || !x_scale || !Wq || !w_scale || !Y) return SEMMOE_EINVAL;
  if (!aligned16(Xq) || !aligned16(Wq) || !aligned16(w_scale) || !aligned16(Y)) return SEMMOE_EINVAL;
  if (n.n_rows == 0) return SEMMOE_OK;
  GemmArgs a = i8_args(Xq, n.ldx ? n.ldx : n.d_in, x_scale, Wq, w_scale, n.d_out, n.d_in, n.d_out, Y, int(n.ldy ? n.ldy : n.d_out));
  a.nq = 1;
  a.n_rows_single = n.n_rows;
  return launch_gemm_i8(kModeStoreI8, a, n.n_rows, n.n_rows, static_cast<hipStream_t>(stream));
}

extern "C" int32_t semmoe_expert_ffn_i8(const semmoe_config* cfg, void* stream, int32_t rank, const void* Xq_perm,
                                        const float* x_scale_perm, const int32_t* expert_offsets, const int32_t* expert_of_phys,
                                        const void* Wq_gu, const float* w_scale_gu, const void* Wq_down, const float* w_scale_down,
                                        void* Y, void* ws, size_t ws_bytes) {
  FfnI8 f{Xq_perm, x_scale_perm, Wq_gu, w_scale_gu, Wq_down, w_scale_down, Y, nullptr, nullptr, nullptr};
  const int32_t st = check_ffn_i8(cfg, f);
  if (st != SEMMOE_OK) return st;
  if (!expert_offsets || !expert_of_phys || rank < -1 || rank >= cfg->D) return SEMMOE_EINVAL;
  const int P = cfg->T * cfg->k, m = cfg->E / cfg->D;
  if (!carve_ffn_i8(&f, ws, ws_bytes, P, cfg->F)) return SEMMOE_EWORKSPACE;
  if (P == 0) return SEMMOE_OK;
  return run_ffn_i8(cfg, static_cast<hipStream_t>(stream), f, expert_offsets, rank < 0 ? 0 : rank * m, rank < 0 ? cfg->E : m, 0, P,
                    P / cfg->E, expert_of_phys);
}

extern "C" int32_t semmoe_shared_ffn_i8(const semmoe_config* cfg, void* stream, const void* Xq, const float* x_scale, int32_t n_tokens,
                                        const void* Wq_gu_sh, const float* w_scale_gu_sh, const void* Wq_down_sh,
                                        const float* w_scale_down_sh, void* Y_shared, void* ws, size_t ws_bytes) {
  FfnI8 f{Xq, x_scale, Wq_gu_sh, w_scale_gu_sh, Wq_down_sh, w_scale_down_sh, Y_shared, nullptr, nullptr, nullptr};
  const int32_t st = check_ffn_i8(cfg, f);
  if (st != SEMMOE_OK) return st;
  if (n_tokens < 0) return SEMMOE_EINVAL;
  if ((long long)n_tokens > (long long)cfg->T * cfg->k) return SEMMOE_ESHAPE;
  if (!carve_ffn_i8(&f, ws, ws_bytes, n_tokens, cfg->F)) return SEMMOE_EWORKSPACE;
  if (n_tokens == 0) return SEMMOE_OK;
  return run_ffn_i8(cfg, static_cast<hipStream_t>(stream), f, nullptr, 0, 1, n_tokens, n_tokens, n_tokens, nullptr);
}
