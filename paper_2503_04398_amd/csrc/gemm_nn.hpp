// Grouped "NN" GEMM core for gfx950:  OUT[row, n] = sum_k X[row, k] * W[g][k, n]
// The products of the expert FFN's gradient walk the forward's weights along their other dimension: a token row's k meets
// weight row k, so the weights' rows are K and their columns the output.  Groups, tile list and walk are those of gemm_core.hpp.
//
// bf16: the slice of a weight panel goes to LDS as it lies in memory, BK rows of BW consecutive numbers, and the MFMA
// operand (8 consecutive k of one column a lane) is read across it with ds_read_b64_tr_b16: 16 lanes read 4 rows x 16
// columns, and each gets the 4 numbers of its column.
// fp32: see gemm_nn_f32_kernel.
#pragma once
#include "gemm_core.hpp"
#include "gemm_w4.hpp"

namespace semmoe {

// kModeSwigluGrad: the sums are dh = d(silu(g) u); out holds [g | u] of a row (ldo = 2N) and takes [dg | du] in their place.
enum NnMode { kNnStore = 0, kNnSwigluGrad = 1 };

typedef __attribute__((ext_vector_type(4))) short i16x4_t;
typedef __attribute__((ext_vector_type(8))) short i16x8_t;

// d silu(g) = sigmoid(g) (1 + g (1 - sigmoid(g)))
__device__ __forceinline__ void swiglu_grad(float dh, float g, float u, float* dg, float* du) {
  const float sig = 1.0f / (1.0f + __expf(-g));
  *dg = dh * u * sig * (1.0f + g * (1.0f - sig));
  *du = dh * g * sig;
}

// v[e] belongs to features feat + e of `row`
template <int MODE, bool F32>
__device__ __forceinline__ void nn_store4(const GemmArgs& a, size_t row, int feat, f32x4_t v) {
  if constexpr (F32) {
    float* o = static_cast<float*>(a.out) + row * a.ldo + feat;
    if constexpr (MODE == kNnSwigluGrad) {
      const f32x4_t g = *reinterpret_cast<const f32x4_t*>(o), u = *reinterpret_cast<const f32x4_t*>(o + a.N);
      f32x4_t dg, du;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const float sig = 1.0f / (1.0f + expf(-g[e]));
        dg[e] = v[e] * u[e] * sig * (1.0f + g[e] * (1.0f - sig));
        du[e] = v[e] * g[e] * sig;
      }
      *reinterpret_cast<f32x4_t*>(o) = dg;
      *reinterpret_cast<f32x4_t*>(o + a.N) = du;
    } else {
      *reinterpret_cast<f32x4_t*>(o) = v;
    }
  } else {
    bf16_t* o = static_cast<bf16_t*>(a.out) + row * a.ldo + feat;
    if constexpr (MODE == kNnSwigluGrad) {
      const uint2 g = *reinterpret_cast<const uint2*>(o), u = *reinterpret_cast<const uint2*>(o + a.N);
      float dg[4], du[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const uint32_t gw = e < 2 ? g.x : g.y, uw = e < 2 ? u.x : u.y;
        const float gf = __uint_as_float(e & 1 ? gw & 0xffff0000u : gw << 16);
        const float uf = __uint_as_float(e & 1 ? uw & 0xffff0000u : uw << 16);
        swiglu_grad(v[e], gf, uf, &dg[e], &du[e]);
      }
      *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16x2(dg[0], dg[1]), pack_bf16x2(dg[2], dg[3]));
      *reinterpret_cast<uint2*>(o + a.N) = make_uint2(pack_bf16x2(du[0], du[1]), pack_bf16x2(du[2], du[3]));
    } else {
      *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    }
  }
}

// Where lane `lane` reads its 8 bytes of a 32-column MFMA tile at column f0 (a multiple of 32) of a weight slice, k-step ks,
// half h: 4 rows x 16 columns for each 16 lanes, which then hold k = 16 ks + 8 (lane / 32) + 4 h + 0..3 of column
// f0 + lane % 32.  Row k's 16-byte piece c lies at position c ^ 4 (k % 4), so the four rows that 16 lanes read are 64 bytes
// apart modulo the 256 bytes of the banks.
template <int RBW>
__device__ __forceinline__ unsigned nn_frag_at(int lane, int f0, int ks, int h) {
  const int i = lane & 15, k = ks * 16 + (lane >> 5) * 8 + h * 4 + (i >> 2);
  const int c = (f0 >> 3) + ((lane >> 4) & 1) * 2 + ((i & 3) >> 1);
  return unsigned(k * RBW + ((c ^ ((k & 3) << 2)) << 4) + (i & 1) * 8);
}

typedef __attribute__((address_space(3))) i16x4_t lds_i16x4;

__device__ __forceinline__ bf16x8_t nn_frag(unsigned at0, unsigned at1) {
  const i16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_i16x4*>(at0));
  const i16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_i16x4*>(at1));
  return __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// ------------------------------------------------------------------------------------------------
// bf16, ring of NSTAGE LDS stages filled by direct global->LDS loads, one barrier per slice (gemm_bf16_dma_body with the
// weights' slice the other way round).
// ------------------------------------------------------------------------------------------------
template <int NWF, int NWT, int TF, int TT, int BK, int NSTAGE>
struct NnCfg {
  static constexpr int NW = NWF * NWT, kThreads = 64 * NW;
  static constexpr int BW = NWF * TF * 32, BT = NWT * TT * 32;
  static constexpr int RBW = BW * 2;           // bytes of a weight row of a slice
  static constexpr int CPW = BW / 8;           // 16-byte pieces of it
  static constexpr int RBX = BK * 2, CPX = BK / 8, RPBX = 256 / RBX;
  static constexpr int kWBytes = BK * RBW, kXBytes = BT * RBX;
  static constexpr int kStageBytes = kWBytes + kXBytes;
  static constexpr int WI = kWBytes / 1024, XI = kXBytes / 1024;  // load instructions
  static constexpr int IPW = (WI + XI) / NW;
  static constexpr int KS = BK / 16;
  static constexpr size_t kRingBytes = size_t(NSTAGE) * kStageBytes;
  static constexpr size_t kLdsBytes = kRingBytes + 520 * 4;
  static_assert(BK == 32 || BK == 64, "row of 64 or 128 bytes");
  static_assert(CPW >= 16 && CPW <= 64, "the swizzle moves pieces inside 16; a row is at most an instruction");
  static_assert((WI + XI) % NW == 0 && (NSTAGE - 1) * IPW < 64, "instructions divide over the waves; vmcnt range");
  static_assert(NSTAGE >= 2 && NSTAGE <= 4, "ring depth");
};

template <int MODE, int NWF, int NWT, int TF, int TT, int BK, int NSTAGE>
__global__ __launch_bounds__(64 * NWF * NWT, 1) void gemm_nn_ring_kernel(GemmArgs a) {
  using C = NnCfg<NWF, NWT, TF, TT, BK, NSTAGE>;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
  int* pre = reinterpret_cast<int*>(lds_raw + C::kRingBytes);
  const unsigned lds_base = static_cast<unsigned>(reinterpret_cast<size_t>(lds_raw));
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wf = wave % NWF, wt = wave / NWF;
  const TileWalk walk = make_walk(a, pre, C::BT, C::BW);
  const int nk = (a.K + BK - 1) / BK, k_tail = a.K - (nk - 1) * BK;

  const int x_swz = ((lane & 31) / C::RPBX) % C::CPX;
  const ItemWalk my = xcd_share(walk.total);
  for (int r = 0; r < my.count; ++r) {
    TileAt at;
    if (!walk_tile(a, walk, pre, my.item(r), C::BT, C::BW, &at)) continue;  // uniform: no barrier is skipped
    const int widx = a.group_to_weight ? a.group_to_weight[a.q_lo + at.q] : (a.q_lo + at.q);
    const bf16_t* Wg = static_cast<const bf16_t*>(a.W) + size_t(widx) * a.w_group_stride;
    const bf16_t* Xg = static_cast<const bf16_t*>(a.X) + size_t(at.row_lo) * a.ldx;

    // this lane's source of each of the wave's load instructions, at the first slice; in_k: its k inside a slice
    const bf16_t* src[C::IPW];
    int in_k[C::IPW];
#pragma unroll
    for (int i = 0; i < C::IPW; ++i) {
      const int n = wave * C::IPW + i;  // instruction of the stage: weights first, then tokens
      if (n < C::WI) {
        const int k = n * (64 / C::CPW) + lane / C::CPW, c = (lane % C::CPW) ^ ((k & 3) << 2);
        in_k[i] = k;
        src[i] = Wg + size_t(k) * a.ldw + min(at.f0 + c * 8, a.N - 8);
      } else {
        const int t = (n - C::WI) * (64 / C::CPX) + lane / C::CPX, c = (lane % C::CPX) ^ ((t / C::RPBX) % C::CPX);
        in_k[i] = c * 8;
        src[i] = Xg + size_t(min(t, at.n_tok - 1)) * a.ldx + c * 8;
      }
    }
    auto issue = [&](int slice, int stage) {
#pragma unroll
      for (int i = 0; i < C::IPW; ++i) {
        const int n = wave * C::IPW + i;
        const unsigned dst = lds_base + stage * C::kStageBytes + n * 1024;
        const size_t step = n < C::WI ? size_t(slice) * BK * a.ldw : size_t(slice) * BK;
        if (slice + 1 < nk || in_k[i] < k_tail) lds_dma16(src[i] + step, dst);
        else *reinterpret_cast<uint4*>(lds_raw + (dst - lds_base) + lane * 16) = make_uint4(0, 0, 0, 0);
      }
    };

    f32x16_t acc[TF][TT];
#pragma unroll
    for (int i = 0; i < TF; ++i)
#pragma unroll
      for (int j = 0; j < TT; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;

#pragma unroll
    for (int s = 0; s < NSTAGE - 1; ++s)
      if (s < nk) issue(s, s);
    int stage = 0;
    for (int it = 0; it < nk; ++it) {
      const int younger = min(NSTAGE - 2, nk - 1 - it);
      if (younger >= 2) wait_vmcnt<2 * C::IPW>();
      else if (younger == 1) wait_vmcnt<1 * C::IPW>();
      else wait_vmcnt<0>();
      __syncthreads();  // slice `it` is complete in LDS; every wave is done with slice it - 1
      const int fill = stage == 0 ? NSTAGE - 1 : stage - 1;
      if (it + NSTAGE - 1 < nk) issue(it + NSTAGE - 1, fill);
      const unsigned Ws = lds_base + stage * C::kStageBytes;
      const unsigned char* xrow = lds_raw + stage * C::kStageBytes + C::kWBytes + (wt * TT * 32 + (lane & 31)) * C::RBX;
#pragma unroll
      for (int ks = 0; ks < C::KS; ++ks) {
        bf16x8_t af[TF], bfr[TT];
#pragma unroll
        for (int i = 0; i < TF; ++i)
          af[i] = nn_frag(Ws + nn_frag_at<C::RBW>(lane, (wf * TF + i) * 32, ks, 0), Ws + nn_frag_at<C::RBW>(lane, (wf * TF + i) * 32, ks, 1));
#pragma unroll
        for (int j = 0; j < TT; ++j)
          bfr[j] = *reinterpret_cast<const bf16x8_t*>(xrow + j * 32 * C::RBX + (((ks * 2 + (lane >> 5)) ^ x_swz) * 16));
#pragma unroll
        for (int i = 0; i < TF; ++i)
#pragma unroll
          for (int j = 0; j < TT; ++j)
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(af[i], bfr[j], acc[i][j], 0, 0, 0);
      }
      stage = stage + 1 == NSTAGE ? 0 : stage + 1;
    }
    __syncthreads();  // the next tile's loads overwrite the ring
#pragma unroll
    for (int j = 0; j < TT; ++j) {
      const int t = (wt * TT + j) * 32 + (lane & 31);
      if (t >= at.n_tok) continue;
#pragma unroll
      for (int i = 0; i < TF; ++i)
#pragma unroll
        for (int g4 = 0; g4 < 4; ++g4) {
          const int feat = at.f0 + (wf * TF + i) * 32 + g4 * 8 + (lane >> 5) * 4;
          if (feat < a.N)
            nn_store4<MODE, false>(a, size_t(at.row_lo) + t, feat,
                                   f32x4_t{acc[i][j][g4 * 4], acc[i][j][g4 * 4 + 1], acc[i][j][g4 * 4 + 2], acc[i][j][g4 * 4 + 3]});
        }
    }
  }
}

// ------------------------------------------------------------------------------------------------
// fp32 (v_mfma_f32_16x16x4_f32: full fp32 products and sums).  128 weight columns x 32 TT tokens, four waves as 2 x 2.  A lane
// reads 16 bytes of a weight row: four consecutive columns, which are row l16 of four MFMA tiles (tile i has the columns
// 4 m + i), and 16 bytes of a token row: the k of four MFMAs in turn.  So a lane ends with four consecutive columns of a token.
// ------------------------------------------------------------------------------------------------
template <int MODE, int TT>
__global__ __launch_bounds__(256) void gemm_nn_f32_kernel(GemmArgs a) {
  constexpr int BW = 128, BT = 32 * TT, BK = 32, LDX = BK + 4;
  __shared__ __attribute__((aligned(16))) float Ws[BK * BW];
  __shared__ __attribute__((aligned(16))) float Xs[BT * LDX];
  __shared__ int pre[520];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, wf = wave & 1, wt = wave >> 1;
  const int l16 = lane & 15, g = lane >> 4;
  const TileWalk walk = make_walk(a, pre, BT, BW);
  const ItemWalk my = xcd_share(walk.total);
  for (int r = 0; r < my.count; ++r) {
    TileAt at;
    if (!walk_tile(a, walk, pre, my.item(r), BT, BW, &at)) continue;
    const int widx = a.group_to_weight ? a.group_to_weight[a.q_lo + at.q] : (a.q_lo + at.q);
    const float* Wg = static_cast<const float*>(a.W) + size_t(widx) * a.w_group_stride + min(at.f0 + (tid & 31) * 4, a.N - 4);
    const float* Xg = static_cast<const float*>(a.X) + size_t(at.row_lo) * a.ldx;
    f32x4_t acc[4][TT];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t < TT; ++t) acc[i][t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    f32x4_t w[4], x[TT];
    const f32x4_t zero = {0.0f, 0.0f, 0.0f, 0.0f};
    auto fetch = [&](int k0) {
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int k = k0 + i * 8 + (tid >> 5);
        w[i] = k < a.K ? *reinterpret_cast<const f32x4_t*>(Wg + size_t(k) * a.ldw) : zero;
      }
#pragma unroll
      for (int t = 0; t < TT; ++t) {
        const int row = min(t * 32 + (tid >> 3), at.n_tok - 1), k = k0 + (tid & 7) * 4;
        x[t] = k < a.K ? *reinterpret_cast<const f32x4_t*>(Xg + size_t(row) * a.ldx + k) : zero;
      }
    };
    fetch(0);
    for (int k0 = 0; k0 < a.K; k0 += BK) {
      __syncthreads();
#pragma unroll
      for (int i = 0; i < 4; ++i) *reinterpret_cast<f32x4_t*>(Ws + (i * 8 + (tid >> 5)) * BW + (tid & 31) * 4) = w[i];
#pragma unroll
      for (int t = 0; t < TT; ++t) *reinterpret_cast<f32x4_t*>(Xs + (t * 32 + (tid >> 3)) * LDX + (tid & 7) * 4) = x[t];
      __syncthreads();
      if (k0 + BK < a.K) fetch(k0 + BK);
#pragma unroll
      for (int h = 0; h < BK / 16; ++h) {
        f32x4_t xf[TT];
#pragma unroll
        for (int t = 0; t < TT; ++t)
          xf[t] = *reinterpret_cast<const f32x4_t*>(Xs + ((wt * TT + t) * 16 + l16) * LDX + h * 16 + g * 4);
#pragma unroll
        for (int s = 0; s < 4; ++s) {
          const f32x4_t wv = *reinterpret_cast<const f32x4_t*>(Ws + (h * 16 + g * 4 + s) * BW + wf * 64 + l16 * 4);
#pragma unroll
          for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int t = 0; t < TT; ++t) acc[i][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(wv[i], xf[t][s], acc[i][t], 0, 0, 0);
        }
      }
    }
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      const int tok = (wt * TT + t) * 16 + l16;
      if (tok >= at.n_tok) continue;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int feat = at.f0 + wf * 64 + g * 16 + e * 4;
        if (feat < a.N) nn_store4<MODE, true>(a, size_t(at.row_lo) + tok, feat, f32x4_t{acc[0][t][e], acc[1][t][e], acc[2][t][e], acc[3][t][e]});
      }
    }
  }
}

// host-side launcher; `mode` an NnMode
int32_t launch_gemm_nn(int mode, int dtype, const GemmArgs& a, int max_rows, int est_rows_per_group, hipStream_t stream);

}  // namespace semmoe
