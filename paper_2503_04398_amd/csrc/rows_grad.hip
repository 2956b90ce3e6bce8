// The gradient of the row moves of a layer.  combine is Out[i] = sum_j w[i,j] Y[slot(i,j)], so towards its rows and weights
//   dY[slot(i,j)] = w[i,j] dOut[i],   dw[i,j] = <dOut[i], Y[slot(i,j)]>;
// dispatch copies X[i] to k places, so dX[i] = sum_j dX_perm[slot(i,j)] (combine.hip's kernel with weights of one).
//
// Both stream: combine's gradient reads P + T rows and writes P, one workgroup a token, a 16-byte piece a thread and pass, the
// k rows of a piece requested before the first is used.  The k dot products are kept in registers over the walk and meet once
// at its end, in a fixed order.  Y is read past the caches: it comes once, and dY is what the next kernel reads.
// Measured, bf16, 16384 tokens of 7168, 8 rows each: 4.0 GB in 767 to 775 us, 5.2 TB/s where a copy of that size reaches 4.8.
#include "common.hpp"

namespace semmoe {

typedef unsigned int u32x4_t __attribute__((ext_vector_type(4)));

template <bool BF16>
struct Piece {  // 16 bytes as floats
  static constexpr int N = BF16 ? 8 : 4;
  float f[N];
  __device__ __forceinline__ explicit Piece(u32x4_t v) {
    if constexpr (BF16) {
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        f[2 * x] = __uint_as_float(v[x] << 16);
        f[2 * x + 1] = __uint_as_float(v[x] & 0xffff0000u);
      }
    } else {
#pragma unroll
      for (int x = 0; x < 4; ++x) f[x] = __uint_as_float(v[x]);
    }
  }
  __device__ __forceinline__ u32x4_t times(float w) const {
    u32x4_t v;
#pragma unroll
    for (int x = 0; x < 4; ++x) v[x] = BF16 ? cvt_pk_bf16(w * f[2 * x], w * f[2 * x + 1]) : __float_as_uint(w * f[x]);
    return v;
  }
  __device__ __forceinline__ float dot(const Piece& o, float s) const {
#pragma unroll
    for (int x = 0; x < N; ++x) s = fmaf(f[x], o.f[x], s);
    return s;
  }
};

// ROWS: dY is asked for; DOTS: dtopk_w is.
template <bool BF16, int KU, bool ROWS, bool DOTS>
__global__ __launch_bounds__(512) void combine_grad_kernel(int k, int row_chunks, int P, const u32x4_t* __restrict__ dOut,
                                                           const u32x4_t* Y, const int32_t* __restrict__ slot_of_pair,
                                                           const float* __restrict__ topk_w, u32x4_t* dY,
                                                           float* __restrict__ dw) {
  __shared__ float part[KU][8];
  const size_t tok = blockIdx.x;
  int sl[KU];
  float wt[KU], acc[KU];
#pragma unroll
  for (int j = 0; j < KU; ++j) {
    sl[j] = -1;
    wt[j] = acc[j] = 0.0f;
    if (j < k) {
      const int s = slot_of_pair[tok * k + j];
      if (unsigned(s) < unsigned(P)) sl[j] = s;
      if constexpr (ROWS) wt[j] = topk_w[tok * k + j];
    }
  }
  constexpr int G = KU < 8 ? KU : 8;  // rows in flight per thread
  for (int c = threadIdx.x; c < row_chunks; c += blockDim.x) {
    const Piece<BF16> g(dOut[tok * row_chunks + c]);
#pragma unroll
    for (int g0 = 0; g0 < KU; g0 += G) {
      u32x4_t v[G];
      if constexpr (DOTS) {
#pragma unroll
        for (int j = 0; j < G; ++j)
          v[j] = sl[g0 + j] >= 0 ? __builtin_nontemporal_load(&Y[size_t(sl[g0 + j]) * row_chunks + c]) : u32x4_t{0, 0, 0, 0};
      }
#pragma unroll
      for (int j = 0; j < G; ++j) {
        if constexpr (DOTS)  // zeros in the place of a missing row would be NaN beside an infinite number
          if (sl[g0 + j] >= 0) acc[g0 + j] = g.dot(Piece<BF16>(v[j]), acc[g0 + j]);
        if constexpr (ROWS)
          if (sl[g0 + j] >= 0) dY[size_t(sl[g0 + j]) * row_chunks + c] = g.times(wt[g0 + j]);
      }
    }
  }
  if constexpr (DOTS) {
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
#pragma unroll
    for (int j = 0; j < KU; ++j) {
      float v = acc[j];
#pragma unroll
      for (int off = 32; off; off >>= 1) v += __shfl_xor(v, off);
      if (lane == 0) part[j][wave] = v;
    }
    __syncthreads();
    for (int j = threadIdx.x; j < k; j += blockDim.x) {
      float v = part[j][0];
      for (int w = 1; w < int(blockDim.x >> 6); ++w) v += part[j][w];
      dw[tok * k + j] = v;
    }
  }
}

template <bool BF16, bool ROWS, bool DOTS>
static void launch_combine_grad(int k, int T, int row_chunks, hipStream_t s, const u32x4_t* dOut, const u32x4_t* Y,
                                const int32_t* slot, const float* w, u32x4_t* dY, float* dw) {
  const int threads = row_walk_threads(row_chunks);
#define SEMMOE_COMBINE_GRAD(KU_)                                                                                              \
  hipLaunchKernelGGL((combine_grad_kernel<BF16, KU_, ROWS, DOTS>), dim3(T), dim3(threads), 0, s, k, row_chunks, T * k, dOut, \
                     Y, slot, w, dY, dw)
  if (k <= 1) SEMMOE_COMBINE_GRAD(1);
  else if (k <= 2) SEMMOE_COMBINE_GRAD(2);
  else if (k <= 4) SEMMOE_COMBINE_GRAD(4);
  else if (k <= 8) SEMMOE_COMBINE_GRAD(8);
  else SEMMOE_COMBINE_GRAD(16);
#undef SEMMOE_COMBINE_GRAD
}

}  // namespace semmoe

using namespace semmoe;

extern "C" int32_t semmoe_combine_grad(const semmoe_config* cfg, void* stream, const void* dOut, const void* Y,
                                       const int32_t* slot_of_pair, const float* topk_w, void* dY, float* dtopk_w) {
  const int32_t st = validate_config(cfg, true, true, false);
  if (st != SEMMOE_OK) return st;
  if (!dOut || !slot_of_pair || (!dY && !dtopk_w) || (dY && !topk_w) || (dtopk_w && !Y)) return SEMMOE_EINVAL;
  if (!aligned16(dOut) || !aligned16(Y) || !aligned16(dY)) return SEMMOE_EINVAL;
  if (cfg->T == 0) return SEMMOE_OK;
  const int row_chunks = int(size_t(cfg->d) * act_bytes(cfg) / 16);
  const bool bf = cfg->dtype == SEMMOE_BF16;
  auto* const launch = dY && dtopk_w ? (bf ? launch_combine_grad<true, true, true> : launch_combine_grad<false, true, true>)
                       : dY          ? (bf ? launch_combine_grad<true, true, false> : launch_combine_grad<false, true, false>)
                                     : (bf ? launch_combine_grad<true, false, true> : launch_combine_grad<false, false, true>);
  launch(cfg->k, cfg->T, row_chunks, static_cast<hipStream_t>(stream), static_cast<const u32x4_t*>(dOut),
         static_cast<const u32x4_t*>(Y), slot_of_pair, topk_w, static_cast<u32x4_t*>(dY), dtopk_w);
  SEMMOE_LAUNCH_CHECK();
  return SEMMOE_OK;
}
