// Rows in 8-bit integers with a scale each: quantize_rows and the row moves of dispatch on such rows.
//
//   scale = max |x| * (1 / 127),   q = rint(x * ((1 / max |x|) * 127))
// Both stream: a row is read once into registers, its largest magnitude found, and written as a byte a number.  A number's error is
// at most half a step, max |x| / 254, beside which the roundings of the factor and the product (2^-24 each) are nothing but for a
// number on the border of two steps, such as half of the largest one, which may go either way.
// Measured: 8192 rows of 7168 bf16 34 to 36 us, 5.0 to 5.2 TB/s; the moves of 8192 rows of 2048 to 8 places each 25.5 us, 5.9 TB/s.
#include "rows.hpp"

namespace semmoe {

// NP pieces a thread; 0: a row too long for that is read twice, the second time from the caches.
template <bool BF16, int NP>
__global__ __launch_bounds__(1024) void quantize_rows_kernel(const void* __restrict__ X, int64_t ldx, int n_rows, int n_cols,
                                                            const int32_t* __restrict__ row_range, int n_range, int tr,
                                                            uint8_t* __restrict__ Xq, float* __restrict__ x_scale) {
  using E = Piece<BF16>;
  constexpr int N = E::N;
  __shared__ uint32_t part[16];
  const int teams = blockDim.x / tr, team = threadIdx.x / tr, t = threadIdx.x % tr, pieces = n_cols / N;
  const int lo = row_range ? row_range[0] : 0, hi = row_range ? min(row_range[n_range], n_rows) : n_rows;
  for (int row0 = lo + int(blockIdx.x) * teams; row0 < hi; row0 += int(gridDim.x) * teams) {
    const int row = row0 + team;
    const bool have = row < hi;
    const size_t at = size_t(have ? row : row0) * ldx;
    E v[NP ? NP : 1];
    uint32_t m[1] = {0};
    if constexpr (NP > 0) {
#pragma unroll
      for (int p = 0; p < NP; ++p) {
        const int c = t + p * tr;
        if (c < pieces) v[p].load(X, at + size_t(c) * N);
        else v[p].zero();
      }
#pragma unroll
      for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int x = 0; x < N; ++x) m[0] = max(m[0], magnitude_bits(v[p][x]));
    } else {
      for (int c = t; c < pieces; c += tr) {
        v[0].load(X, at + size_t(c) * N);
#pragma unroll
        for (int x = 0; x < N; ++x) m[0] = max(m[0], magnitude_bits(v[0][x]));
      }
    }
    team_join(m, part, tr >> 6, [](uint32_t a, uint32_t b) { return max(a, b); });
    const RowScale s(m[0]);
    auto put = [&](const E& e, int c) __attribute__((always_inline)) {
      float f[N];
#pragma unroll
      for (int x = 0; x < N; ++x) f[x] = e[x];
      if (have) s.put(Xq + size_t(row) * n_cols + size_t(c) * N, f);
    };
    if constexpr (NP > 0) {
#pragma unroll
      for (int p = 0; p < NP; ++p)
        if (t + p * tr < pieces) put(v[p], t + p * tr);
    } else {
      for (int c = t; c < pieces; c += tr) {
        v[0].load(X, at + size_t(c) * N);
        put(v[0], c);
      }
    }
    if (have && t == 0) x_scale[row] = s.scale;
    if (tr > 64) __syncthreads();  // `part` has been read
  }
}

int32_t launch_quantize_rows(bool bf16, const void* X, int64_t ldx, int n_rows, int n_cols, const int32_t* row_range, int n_range,
                             void* Xq, float* x_scale, hipStream_t stream) {
  DeviceInfo dev;
  const int32_t st = device_info(&dev);
  if (st != SEMMOE_OK) return st;
  // A wave a row where four pieces a thread hold it: no barrier (20865 rows of 768: 13.7 -> 11.2 us, 8192 of 2048: 12.3 -> 11.8; few
  // rows: no difference).
  const bool short_rows = n_cols <= (bf16 ? 2048 : 1024);
  const RowTeams g = short_rows ? RowTeams(bf16, n_cols, 64) : RowTeams(bf16, n_cols);
  const long long groups = cdiv(n_rows, g.teams), most = (long long)dev.num_cu * 8;
  const int grid = int(groups < most ? groups : most);
#define SEMMOE_QUANTIZE(BF_, NP_)                                                                                             \
  hipLaunchKernelGGL((quantize_rows_kernel<BF_, NP_>), dim3(grid), dim3(g.tr * g.teams), 0, stream, X, ldx, n_rows, n_cols, \
                     row_range, n_range, g.tr, static_cast<uint8_t*>(Xq), x_scale)
  if (bf16) {
    if (g.np == 1) SEMMOE_QUANTIZE(true, 1);
    else if (g.np == 2) SEMMOE_QUANTIZE(true, 2);
    else if (g.np == 4) SEMMOE_QUANTIZE(true, 4);
    else SEMMOE_QUANTIZE(true, 0);
  } else {
    if (g.np == 1) SEMMOE_QUANTIZE(false, 1);
    else if (g.np == 2) SEMMOE_QUANTIZE(false, 2);
    else if (g.np == 4) SEMMOE_QUANTIZE(false, 4);
    else SEMMOE_QUANTIZE(false, 0);
  }
#undef SEMMOE_QUANTIZE
  SEMMOE_LAUNCH_CHECK();
  return SEMMOE_OK;
}

// One workgroup a token, a 16-byte piece a thread and pass, read once and written to the token's k rows; the scale goes with it.
template <int KU>
__global__ __launch_bounds__(512) void dispatch_rows_i8_kernel(int k, int pieces, int P, const row_u32x4_t* __restrict__ Xq,
                                                               const float* __restrict__ x_scale,
                                                               const int32_t* __restrict__ slot_of_pair,
                                                               row_u32x4_t* __restrict__ Xq_perm, float* __restrict__ x_scale_perm) {
  const size_t tok = blockIdx.x;
  int slot[KU];
#pragma unroll
  for (int j = 0; j < KU; ++j) {
    const int s = slot_of_pair[tok * k + min(j, k - 1)];
    slot[j] = j < k && unsigned(s) < unsigned(P) ? s : -1;
  }
  for (int c = threadIdx.x; c < pieces; c += blockDim.x) {
    const row_u32x4_t v = Xq[tok * pieces + c];
#pragma unroll
    for (int j = 0; j < KU; ++j)
      if (slot[j] >= 0) Xq_perm[size_t(slot[j]) * pieces + c] = v;
  }
  if (threadIdx.x == 0) {
    const float s = x_scale[tok];
#pragma unroll
    for (int j = 0; j < KU; ++j)
      if (slot[j] >= 0) x_scale_perm[slot[j]] = s;
  }
}

}  // namespace semmoe

using namespace semmoe;

extern "C" int32_t semmoe_quantize_rows(const semmoe_config* cfg, void* stream, const void* X, int32_t n_rows, int32_t n_cols,
                                        int64_t ldx, void* Xq, float* x_scale) {
  if (!cfg) return SEMMOE_EINVAL;
  if (cfg->dtype != SEMMOE_FP32 && cfg->dtype != SEMMOE_BF16) return SEMMOE_EUNSUPPORTED;
  if (!X || !Xq || !x_scale || n_rows < 0 || n_cols <= 0 || ldx < 0) return SEMMOE_EINVAL;
  if (n_cols % 8 != 0 || ldx % 8 != 0 || (ldx > 0 && ldx < n_cols)) return SEMMOE_ESHAPE;
  if (n_rows > 0x3fffffff) return SEMMOE_EUNSUPPORTED;
  if (!aligned16(X) || !aligned16(Xq)) return SEMMOE_EINVAL;
  if (n_rows == 0) return SEMMOE_OK;
  return launch_quantize_rows(cfg->dtype == SEMMOE_BF16, X, ldx ? ldx : n_cols, n_rows, n_cols, nullptr, 0, Xq, x_scale,
                              static_cast<hipStream_t>(stream));
}

extern "C" int32_t semmoe_dispatch_rows_i8(const semmoe_config* cfg, void* stream, const void* Xq, const float* x_scale,
                                           const int32_t* slot_of_pair, void* Xq_perm, float* x_scale_perm) {
  const int32_t st = validate_config(cfg, true, true, false);
  if (st != SEMMOE_OK) return st;
  if (!Xq || !x_scale || !slot_of_pair || !Xq_perm || !x_scale_perm) return SEMMOE_EINVAL;
  if (cfg->d % 16 != 0) return SEMMOE_ESHAPE;
  if (!aligned16(Xq) || !aligned16(Xq_perm)) return SEMMOE_EINVAL;
  if (cfg->T == 0) return SEMMOE_OK;
  const int pieces = cfg->d / 16, threads = row_walk_threads(pieces), P = cfg->T * cfg->k;
  const row_u32x4_t* X = static_cast<const row_u32x4_t*>(Xq);
  const int per = rows_a_launch(1, threads);
#define SEMMOE_ROWS_I8(KU_)                                                                                                    \
  hipLaunchKernelGGL(dispatch_rows_i8_kernel<KU_>, dim3(left < per ? left : per), dim3(threads), 0, static_cast<hipStream_t>(stream), \
                     cfg->k, pieces, P, X, x_scale, slot_of_pair, static_cast<row_u32x4_t*>(Xq_perm), x_scale_perm)
  for (int left = cfg->T; left > 0; left -= per) {
    if (cfg->k <= 2) SEMMOE_ROWS_I8(2);
    else if (cfg->k <= 4) SEMMOE_ROWS_I8(4);
    else if (cfg->k <= 8) SEMMOE_ROWS_I8(8);
    else SEMMOE_ROWS_I8(16);
    SEMMOE_LAUNCH_CHECK();
    X += size_t(per) * pieces;
    x_scale += per;
    slot_of_pair += size_t(per) * cfg->k;
  }
#undef SEMMOE_ROWS_I8
  return SEMMOE_OK;
}
