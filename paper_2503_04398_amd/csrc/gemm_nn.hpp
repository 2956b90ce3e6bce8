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

// kNnStore: act type.  kNnSums: the fp32 sums themselves, in fours (quad_at).
enum NnMode { kNnStore = 0, kNnSums = 1 };

typedef __attribute__((ext_vector_type(4))) short i16x4_t;

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
      // slices issued after this one may stay in flight.  Of a partial slice a wave may have no load at all (its rows lie past K), so
      // that the loads behind this slice's are fewer than they are counted: once it has been issued, all of them are waited for.
      const bool counted = k_tail == BK || it + NSTAGE - 2 < nk - 1;
      const int younger = counted ? min(NSTAGE - 2, nk - 1 - it) : 0;
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
      const size_t row = size_t(at.row_lo) + t;
#pragma unroll
      for (int i = 0; i < TF; ++i)
#pragma unroll
        for (int g4 = 0; g4 < 4; ++g4) {
          const int feat = at.f0 + (wf * TF + i) * 32 + g4 * 8 + (lane >> 5) * 4;
          if (feat >= a.N) continue;
          const f32x4_t v = {acc[i][j][g4 * 4], acc[i][j][g4 * 4 + 1], acc[i][j][g4 * 4 + 2], acc[i][j][g4 * 4 + 3]};
          if constexpr (MODE == kNnSums)
            *reinterpret_cast<f32x4_t*>(static_cast<float*>(a.out) + quad_at(a.N, int(row), feat)) = v;
          else
            *reinterpret_cast<uint2*>(static_cast<bf16_t*>(a.out) + row * a.ldo + feat) = make_uint2(cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]));
        }
    }
  }
}

// ------------------------------------------------------------------------------------------------
// bf16, four waves as 2 x 2 on a tile of 64 TI columns x 64 TJ tokens (a wave: TI x TJ MFMA tiles), one wave per SIMD, slices
// of 64 through a ring of NSTAGE: the K loop of gemm_bf16_w4_body for weights that lie the other way round.  Loads of a slice
// go out one by one behind the MFMAs, fragments are read a k-step ahead, the one barrier of a slice sits before its last k-step,
// and the stream of slices runs on into the workgroup's next tile.  What differs: a slice of the weight panel is 64 rows of
// 128 TI bytes, its rows advance by 64 ldw a slice, and a weight fragment is two transposing reads of 8 bytes a lane.
// Where K is no multiple of 64 the last slice is the last 64 rows of K once more in part: what the slice before held is masked out of
// its fragments (K % 8 == 0: whole halves of a wave).  Needs more than NSTAGE slices.
// Measured, 16 experts of 1300 rows, d 2048, F 768, 256 x 256 tiles and pieces: dh (K 2048) 94 to 105 us, 0.62 to 0.70 PFLOP/s; dX (K
// 1536) 142 to 160 us, 0.82 to 0.93.  128 experts of 62 rows, 128 x 128: 102 and 172 us at best, 4.5 and 5.0 TB/s of weights, rows and sums.
// ------------------------------------------------------------------------------------------------
template <int TI, int TJ, int NSTAGE>
struct NnW4Cfg {
  static constexpr int kThreads = 256, BW = 64 * TI, BT = 64 * TJ;
  static constexpr int RBW = BW * 2, CPW = BW / 8, RBX = 128;
  static constexpr int kWBytes = 64 * RBW, kStageBytes = kWBytes + BT * RBX;
  static constexpr int WI = 8 * TI, XI = 8 * TJ, IPW = (WI + XI) / 4;  // loads of a slice: weights, tokens, a wave
  static constexpr int kSplit = WI % IPW == 0 ? IPW : WI - 2 * IPW;    // wave 2's weight loads where a wave has both
  static constexpr size_t kRingBytes = size_t(NSTAGE) * kStageBytes;
  static constexpr int NB = TI == 4 && TJ == 2 ? 1 : 2;  // 64-byte blocks of a staged row
  static constexpr int kStgRow = NB * 64 + 16, kStgWave = 32 * kStgRow;
  static constexpr size_t lds_bytes(int nq) { return kRingBytes + 4 * kStgWave + (4 * size_t(nq) + 8) * 4; }
  static_assert(IPW * 4 == WI + XI && (kSplit == IPW || (kSplit > 0 && kSplit < IPW)), "how loads are dealt out to the waves");
  static_assert(NSTAGE >= 2 && (NSTAGE - 1) * IPW < 64, "vmcnt range");
};

template <int MODE, int TI, int TJ, int NSTAGE, int DMA_EVERY>
__device__ __forceinline__ void gemm_nn_w4_body(const GemmArgs& a, unsigned char* lds_raw) {
  using C = NnW4Cfg<TI, TJ, NSTAGE>;
  constexpr int M = TI * TJ;  // MFMAs of a k-step
  static_assert(4 * M / DMA_EVERY >= C::IPW, "the loads of a slice fit between two barriers");
  const unsigned lds_base = static_cast<unsigned>(reinterpret_cast<size_t>(lds_raw));
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wf = wave & 1, wt = wave >> 1;
  unsigned char* stg = lds_raw + C::kRingBytes + wave * C::kStgWave;
  int* pre = reinterpret_cast<int*>(lds_raw + C::kRingBytes + 4 * C::kStgWave);
  int* gtab = pre + a.nq + 1;  // per group: first row, row after the last, weights
  for (int q = tid; q < a.nq; q += C::kThreads) {
    gtab[3 * q] = a.offsets ? a.offsets[a.q_lo + q] : 0;
    gtab[3 * q + 1] = a.offsets ? a.offsets[a.q_lo + q + 1] : a.n_rows_single;
    gtab[3 * q + 2] = a.group_to_weight ? a.group_to_weight[a.q_lo + q] : a.q_lo + q;
  }
  const TileWalk walk = make_walk(a, pre, C::BT, C::BW);  // ends with a barrier
  const int nk = (a.K + 63) / 64, again = nk * 64 - a.K;  // rows of the last slice that the slice before held
  const ItemWalk my = xcd_share(__builtin_amdgcn_readfirstlane(walk.total));

  struct Tile {
    int row_lo, n_tok, f0, widx;
  };
  auto locate = [&](int item, Tile* t) __attribute__((always_inline)) {
    const int pieces = walk.sub_t * walk.sub_f;
    int tile = walk.tail ? walk.cutoff + item / pieces : item;
    if (a.sched_reverse) tile = pre[a.nq] - 1 - tile;
    const int q = __builtin_amdgcn_readfirstlane(find_group(pre, a.nq, tile));
    const int local = tile - __builtin_amdgcn_readfirstlane(pre[q]);
    const int g_lo = __builtin_amdgcn_readfirstlane(gtab[3 * q]), row_hi = __builtin_amdgcn_readfirstlane(gtab[3 * q + 1]);
    int ft, tt;
    decode_tile(local, (row_hi - g_lo + walk.bt_list - 1) / walk.bt_list, walk.n_ftiles_list, &tt, &ft);
    if (walk.tail) {
      const int piece = item % pieces;
      tt = tt * walk.sub_t + piece / walk.sub_f;
      ft = ft * walk.sub_f + piece % walk.sub_f;
    }
    tt = __builtin_amdgcn_readfirstlane(tt);
    ft = __builtin_amdgcn_readfirstlane(ft);
    if (g_lo + tt * C::BT >= row_hi || ft * C::BW >= a.N) return false;  // a piece outside the matrix
    t->row_lo = g_lo + tt * C::BT;
    t->n_tok = min(C::BT, row_hi - t->row_lo);
    t->f0 = ft * C::BW;
    t->widx = __builtin_amdgcn_readfirstlane(gtab[3 * q + 2]);
    return true;
  };

  // ---- load stream
  int s_round = -1, s_tiles = 0;  // tiles that the stream has entered
  Tile s_tile;
  auto next_tile = [&]() __attribute__((always_inline)) {
    while (++s_round < my.count)
      if (locate(my.item(s_round), &s_tile)) {
        ++s_tiles;
        return true;
      }
    return false;
  };
  if (!next_tile()) return;  // the whole workgroup leaves; no barrier is pending

  int i_slice = 0, i_k = 0, i_stage = 0;
  bool i_done = false;
  unsigned i_dst = 0;
  const unsigned char *i_base = nullptr, *i_base2 = nullptr;
  uint32_t i_off[C::IPW];
  const bool loads_w = wave < 2, first_w = C::kSplit == C::IPW ? loads_w : wave < 3;
  auto aim = [&]() __attribute__((always_inline)) {
    const unsigned char* w_panel = reinterpret_cast<const unsigned char*>(static_cast<const bf16_t*>(a.W) + size_t(s_tile.widx) * a.w_group_stride);
    const unsigned char* x_panel = reinterpret_cast<const unsigned char*>(static_cast<const bf16_t*>(a.X) + size_t(s_tile.row_lo) * a.ldx);
    i_k = again ? 0 : first_step(a, s_tile.widx, 2, nk);  // the last slice has to come last
    w_panel += size_t(i_k) * 64 * a.ldw * 2;
    x_panel += size_t(i_k) * 128;
    i_base = first_w ? w_panel : x_panel;
    i_base2 = loads_w ? w_panel : x_panel;
    auto w_off = [&](int n) __attribute__((always_inline)) {
      const int k = n * (64 / C::CPW) + lane / C::CPW, c = (lane % C::CPW) ^ ((k & 3) << 2);
      return uint32_t(k) * uint32_t(a.ldw) * 2u + uint32_t(min(s_tile.f0 + c * 8, a.N - 8)) * 2u;
    };
    auto x_off = [&](int n) __attribute__((always_inline)) {
      const int t = n * 8 + (lane >> 3), c = (lane & 7) ^ ((t >> 1) & 7);
      return uint32_t(min(t, s_tile.n_tok - 1)) * uint32_t(a.ldx) * 2u + uint32_t(c) * 16u;
    };
    if (first_w) {
#pragma unroll
      for (int i = 0; i < C::kSplit; ++i) i_off[i] = w_off(wave * C::IPW + i);
    } else {
#pragma unroll
      for (int i = 0; i < C::kSplit; ++i) i_off[i] = x_off(wave * C::IPW + i - C::WI);
    }
    if constexpr (C::kSplit < C::IPW) {
      if (loads_w) {
#pragma unroll
        for (int i = C::kSplit; i < C::IPW; ++i) i_off[i] = w_off(wave * C::IPW + i);
      } else {
#pragma unroll
        for (int i = C::kSplit; i < C::IPW; ++i) i_off[i] = x_off(wave * C::IPW + i - C::WI);
      }
    }
  };
  auto move = [&](long long rows) __attribute__((always_inline)) {  // along K
    i_base += rows * (first_w ? 2ll * a.ldw : 2ll);
    if constexpr (C::kSplit < C::IPW) i_base2 += rows * (loads_w ? 2ll * a.ldw : 2ll);
  };
  // After the last slice there is nothing new to fetch: the stream stands still and its loads fetch the same bytes again.
  auto next_slice = [&]() __attribute__((always_inline)) {
    if (i_slice + 1 == nk) {
      if (i_done || !next_tile()) {
        i_done = true;
        return;
      }
      i_slice = 0;
      aim();
    } else {
      ++i_slice;
      if (++i_k == nk) {
        i_k = 0;
        move(64 * (1 - nk));
      } else {
        move(i_k + 1 == nk ? 64 - again : 64);
      }
    }
    i_stage = i_stage + 1 == NSTAGE ? 0 : i_stage + 1;
    i_dst = lds_base + i_stage * C::kStageBytes + wave * C::IPW * 1024;
  };
  auto issue = [&](auto idx) __attribute__((always_inline)) {
    constexpr int i = decltype(idx)::value;
    lds_dma16_imm<i * 1024>(i < C::kSplit ? i_base : i_base2, i_off[i], i_dst);
    if constexpr (i == C::IPW - 1) next_slice();
  };

  // ---- fragments: the XOR of a weight piece's place is a lane's own (k % 4 = lane % 16 / 4), k-steps are constants
  bf16x8_t af[2][TI], bfr[2][TJ];
  unsigned w_at[TI];
#pragma unroll
  for (int i = 0; i < TI; ++i) w_at[i] = nn_frag_at<C::RBW>(lane, (wf * TI + i) * 32, 0, 0);
  const unsigned x_at = C::kWBytes + (wt * 32 + (lane & 31)) * C::RBX;
  const int x_swz = ((lane & 31) >> 1) & 7;
  constexpr int R = 2 * TI + TJ;  // reads of a k-step
  i16x4_t w_lo[TI];
  auto read = [&](unsigned S, int ks, int r, bf16x8_t(&fa)[TI], bf16x8_t(&fb)[TJ]) __attribute__((always_inline)) {
    if (r < 2 * TI) {
      const i16x4_t v = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
          reinterpret_cast<lds_i16x4*>(S + w_at[r >> 1] + (ks * 16 + (r & 1) * 4) * C::RBW));
      if (r & 1) fa[r >> 1] = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(w_lo[r >> 1], v, 0, 1, 2, 3, 4, 5, 6, 7));
      else w_lo[r >> 1] = v;
    } else {
      const int j = r - 2 * TI;
      fb[j] = *reinterpret_cast<const bf16x8_t*>(lds_raw + (S - lds_base) + x_at + j * 64 * C::RBX + (((ks * 2 + (lane >> 5)) ^ x_swz) * 16));
    }
  };

  // ---- prologue: the first NSTAGE slices
  aim();
  i_dst = lds_base + wave * C::IPW * 1024;
  for (int s = 0; s < NSTAGE; ++s) {
#pragma unroll
    for (int i = 0; i < C::IPW; ++i)
      lds_dma16_s(i < C::kSplit ? i_base : i_base2, i_off[i], i_dst + i * 1024);
    if (s + 1 < NSTAGE) next_slice();
  }
  // where the loads of a window do not fit its first k-step, the k-steps before the first barrier carry the window's tail:
  // they fetch the rest of the standing slice once more, and the stream moves on when they are through
  if constexpr (C::IPW * DMA_EVERY <= M) next_slice();
  wait_vmcnt<(NSTAGE - 1) * C::IPW>();
  __syncthreads();
#pragma unroll
  for (int r = 0; r < R; ++r) read(lds_base, 0, r, af[0], bfr[0]);
  int c_stage = 0, c_tiles = 0;

  do {
    const Tile t = s_tile;  // more than NSTAGE slices: the stream is still in this tile
    const int nj = min(TJ, max(0, (t.n_tok - wt * 32 + 63) >> 6));
    f32x16_t acc[TI][TJ];
#pragma unroll
    for (int i = 0; i < TI; ++i)
#pragma unroll
      for (int j = 0; j < TJ; ++j)
#pragma unroll
        for (int e = 0; e < 16; ++e) acc[i][j][e] = 0.0f;
    for (int it = 0; it < nk; ++it) {
      const int n_stage = c_stage + 1 == NSTAGE ? 0 : c_stage + 1;
      auto k_step = [&](auto ks_tag) __attribute__((always_inline)) {
        constexpr int ks = decltype(ks_tag)::value, cur = ks & 1, nxt = ks == 3 ? 0 : ks + 1;
        if constexpr (ks == 3) {
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // this wave's reads of the slice are complete
          if (!i_done) wait_vmcnt<(NSTAGE - 2) * C::IPW>(); else wait_vmcnt<0>();
          __syncthreads();
        }
        const unsigned S = lds_base + (ks == 3 ? n_stage : c_stage) * C::kStageBytes;
        if (again && it + 1 == nk) {
          const bool mine = ks * 16 + (lane >> 5) * 8 >= again;
          const bf16x8_t none = {};
#pragma unroll
          for (int i = 0; i < TI; ++i) af[cur][i] = mine ? af[cur][i] : none;
#pragma unroll
          for (int j = 0; j < TJ; ++j) bfr[cur][j] = mine ? bfr[cur][j] : none;
        }
        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
        for (int j = 0; j < TJ; ++j) {
#pragma unroll
          for (int i = 0; i < TI; ++i) {
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(af[cur][i], bfr[cur][j], acc[i][j], 0, 0, 0);
            const int p = j * TI + i;  // constant after unrolling
            const int r0 = R <= M ? p : p * R / M, r1 = R <= M ? (p < R ? p + 1 : p) : (p + 1) * R / M;
#pragma unroll
            for (int r = r0; r < r1; ++r) read(S, nxt, r, af[cur ^ 1], bfr[cur ^ 1]);
            const int m = (ks == 3 ? 0 : (ks + 1) * M) + p;  // MFMAs since the barrier
            if (m % DMA_EVERY == DMA_EVERY - 1 && m / DMA_EVERY < C::IPW) {
              switch (m / DMA_EVERY) {
#define SEMMOE_NN_CASE(n) case n: if constexpr (n < C::IPW) issue(std::integral_constant<int, n>{}); break;
                SEMMOE_NN_CASE(0) SEMMOE_NN_CASE(1) SEMMOE_NN_CASE(2) SEMMOE_NN_CASE(3)
                SEMMOE_NN_CASE(4) SEMMOE_NN_CASE(5) SEMMOE_NN_CASE(6) SEMMOE_NN_CASE(7)
                SEMMOE_NN_CASE(8) SEMMOE_NN_CASE(9) SEMMOE_NN_CASE(10) SEMMOE_NN_CASE(11)
                SEMMOE_NN_CASE(12) SEMMOE_NN_CASE(13) SEMMOE_NN_CASE(14) SEMMOE_NN_CASE(15)
#undef SEMMOE_NN_CASE
                default: break;
              }
            }
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      };
      k_step(std::integral_constant<int, 0>{});
      k_step(std::integral_constant<int, 1>{});
      k_step(std::integral_constant<int, 2>{});
      k_step(std::integral_constant<int, 3>{});
      c_stage = n_stage;
    }

    // ---- epilogue: no barrier; the ring already holds the next tile's first slices
    const int tok_in = lane & 31, half = lane >> 5;
    if constexpr (MODE == kNnSums) {
#pragma unroll
      for (int j = 0; j < TJ; ++j) {
        if (j >= nj) break;
        const int row = (j * 2 + wt) * 32 + tok_in;
#pragma unroll
        for (int i = 0; i < TI; ++i) {
          asm volatile("" : "+a"(acc[i][j]));
#pragma unroll
          for (int g4 = 0; g4 < 4; ++g4) {
            const int feat = t.f0 + (wf * TI + i) * 32 + g4 * 8 + half * 4;
            if (row < t.n_tok && feat < a.N)
              *reinterpret_cast<f32x4_t*>(static_cast<float*>(a.out) + quad_at(a.N, t.row_lo + row, feat)) =
                  f32x4_t{acc[i][j][g4 * 4], acc[i][j][g4 * 4 + 1], acc[i][j][g4 * 4 + 2], acc[i][j][g4 * 4 + 3]};
          }
        }
      }
    } else {
      // 32 tokens x NB * 32 features at a time go through the wave's staging area, so that neighbouring lanes store one row
      constexpr int kLpr = 4 * C::NB, kRpr = 64 / kLpr;  // lanes of a staged row, rows of a read-back
      const int b_row = lane / kLpr, b_chunk = lane % kLpr;
#pragma unroll
      for (int j = 0; j < TJ; ++j) {
        if (j >= nj) break;
#pragma unroll
        for (int h = 0; h < TI / C::NB; ++h) {
          __builtin_amdgcn_sched_barrier(0);
          unsigned char* wp = stg + tok_in * C::kStgRow + half * 8;
#pragma unroll
          for (int b = 0; b < C::NB; ++b) asm volatile("" : "+a"(acc[C::NB * h + b][j]));
#pragma unroll
          for (int b = 0; b < C::NB; ++b) {
            const f32x16_t& c = acc[C::NB * h + b][j];
#pragma unroll
            for (int g4 = 0; g4 < 4; ++g4)
              *reinterpret_cast<uint2*>(wp + (b * 4 + g4) * 16) =
                  make_uint2(cvt_pk_bf16(c[g4 * 4], c[g4 * 4 + 1]), cvt_pk_bf16(c[g4 * 4 + 2], c[g4 * 4 + 3]));
          }
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          __builtin_amdgcn_wave_barrier();
          const int feat = t.f0 + wf * 32 * TI + h * C::NB * 32 + b_chunk * 8;
#pragma unroll
          for (int p = 0; p < 32 / kRpr; ++p) {
            const int sr = p * kRpr + b_row, row = (j * 2 + wt) * 32 + sr;
            const uint4 v = *reinterpret_cast<const uint4*>(stg + sr * C::kStgRow + b_chunk * 16);
            if (row < t.n_tok && feat < a.N)
              *reinterpret_cast<uint4*>(static_cast<bf16_t*>(a.out) + (size_t(t.row_lo) + row) * a.ldo + feat) = v;
          }
          asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
          __builtin_amdgcn_wave_barrier();
        }
      }
    }
  } while (++c_tiles < s_tiles);
  wait_vmcnt<0>();  // nothing may still be writing into this workgroup's LDS when it ends
}

template <int MODE, int TI, int TJ, int NSTAGE, int DMA_EVERY>
__global__ __launch_bounds__(256, 1) void gemm_nn_w4_kernel(GemmArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
  gemm_nn_w4_body<MODE, TI, TJ, NSTAGE, DMA_EVERY>(a, lds_raw);
}

// The tiles of the full rounds, then the rest as 128 x 128 pieces, in one launch (as gemm_bf16_w4_split_kernel).
template <int MODE, int TJ, int NSTAGE>
__global__ __launch_bounds__(256, 1) void gemm_nn_split_kernel(GemmArgs head, GemmArgs tail) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
  gemm_nn_w4_body<MODE, 4, TJ, NSTAGE, 2>(head, lds_raw);
  __syncthreads();  // every wave is done with the head's LDS
  gemm_nn_w4_body<MODE, 2, 2, 3, 1>(tail, lds_raw);
}

// ------------------------------------------------------------------------------------------------
// fp32 (v_mfma_f32_16x16x4_f32: full fp32 products and sums).  64 weight columns x 16 TT tokens; NW waves cut K between them, 16
// weight rows at a time: four, or eight where the tiles do not fill the chip.  A lane's 16 bytes of a weight row are four
// consecutive columns, which are row l16 of four MFMA tiles (tile i has the columns 4 m + i), and its 16 bytes of a token row the
// k of four MFMAs in turn, so the operands come from memory as they are used, a weight row in runs of 256 bytes, AHEAD steps
// ahead and without a barrier; a lane ends with four consecutive columns.
// What bounds it: the matrix pipe, 32 cycles an instruction, on tiles that ragged groups half fill, and with few rows the walk's
// start and end.  Measured, 16 experts of 32 rows, d 512, F 1024: K 512 18 us, K 2048 31 us, of which the products are 14.  (As 128 x 32
// tiles that share LDS slices that was 64 workgroups: 62 us for K 2048.)
// ------------------------------------------------------------------------------------------------
template <int MODE, int TT, int NW>
__global__ __launch_bounds__(64 * NW) void gemm_nn_f32_kernel(GemmArgs a) {
  constexpr int BW = 64, BT = 16 * TT, AHEAD = TT <= 2 ? 4 : 2;
  __shared__ f32x4_t red[NW * 4 * 64];  // [wave][tile][lane]
  __shared__ int pre[520];
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const TileWalk walk = make_walk(a, pre, BT, BW);
  const ItemWalk my = xcd_share(walk.total);
  const f32x4_t zero = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int r = 0; r < my.count; ++r) {
    TileAt at;
    if (!walk_tile(a, walk, pre, my.item(r), BT, BW, &at)) continue;  // uniform: no barrier is skipped
    const int widx = a.group_to_weight ? a.group_to_weight[a.q_lo + at.q] : (a.q_lo + at.q);
    const float* Wg = static_cast<const float*>(a.W) + size_t(widx) * a.w_group_stride + size_t(g * 4) * a.ldw + min(at.f0 + l16 * 4, a.N - 4);
    const float* Xg = static_cast<const float*>(a.X) + size_t(at.row_lo) * a.ldx + g * 4;
    uint32_t x_at[TT];
#pragma unroll
    for (int t = 0; t < TT; ++t) x_at[t] = uint32_t(min(t * 16 + l16, at.n_tok - 1)) * uint32_t(a.ldx);
    f32x4_t acc[4][TT];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int t = 0; t < TT; ++t) acc[i][t] = zero;
    struct Step {
      f32x4_t w[4], x[TT];
    };
    auto fetch = [&](int k0, Step& s) __attribute__((always_inline)) {
      const bool in = k0 + g * 4 < a.K;  // K % 8 == 0: four rows of a lane are there or not
#pragma unroll
      for (int e = 0; e < 4; ++e) s.w[e] = in ? *reinterpret_cast<const f32x4_t*>(Wg + size_t(k0 + e) * a.ldw) : zero;
#pragma unroll
      for (int t = 0; t < TT; ++t) s.x[t] = in ? *reinterpret_cast<const f32x4_t*>(Xg + x_at[t] + k0) : zero;
    };
    auto multiply = [&](const Step& s) __attribute__((always_inline)) {
#pragma unroll
      for (int e = 0; e < 4; ++e)
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int t = 0; t < TT; ++t) acc[i][t] = __builtin_amdgcn_mfma_f32_16x16x4f32(s.w[e][i], s.x[t][e], acc[i][t], 0, 0, 0);
    };
    Step s[AHEAD];
#pragma unroll
    for (int i = 0; i < AHEAD; ++i) fetch((wave + i * NW) * 16, s[i]);
    for (int k0 = wave * 16; k0 < a.K; k0 += AHEAD * NW * 16) {
#pragma unroll
      for (int i = 0; i < AHEAD; ++i) {
        multiply(s[i]);  // zeros where the wave has no such step
        fetch(k0 + (AHEAD + i) * NW * 16, s[i]);
      }
    }
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      __syncthreads();  // what was read of the tokens before
#pragma unroll
      for (int i = 0; i < 4; ++i) red[(wave * 4 + i) * 64 + lane] = acc[i][t];
      __syncthreads();
      f32x4_t v = zero;
      if (wave < 4) {  // tile `wave`
#pragma unroll
        for (int w = 0; w < NW; ++w) v += red[(w * 4 + wave) * 64 + lane];
      }
      __syncthreads();
      if (wave < 4) red[wave * 64 + lane] = v;
      __syncthreads();
      if (wave >= 4) continue;
      const float* rs = reinterpret_cast<const float*>(red) + lane * 4 + wave;  // row 4 g + `wave` of the four tiles
      const f32x4_t o = {rs[0], rs[256], rs[512], rs[768]};
      const int tok = t * 16 + l16, feat = at.f0 + g * 16 + wave * 4, row = at.row_lo + tok;
      if (tok < at.n_tok && feat < a.N)
        *reinterpret_cast<f32x4_t*>(static_cast<float*>(a.out) + (MODE == kNnSums ? quad_at(a.N, row, feat) : size_t(row) * a.ldo + feat)) = o;
    }
  }
}

// host-side launcher; `mode` an NnMode
int32_t launch_gemm_nn(int mode, int dtype, const GemmArgs& a, int max_rows, int est_rows_per_group, hipStream_t stream);

}  // namespace semmoe
