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

// more slices than the ring holds, and a table that fits beside the ring
template <int TI, int TJ, int NSTAGE>
static bool nn_w4_fits(const GemmArgs& a) {
  using C = NnW4Cfg<TI, TJ, NSTAGE>;
  DeviceInfo d;
  if (cdiv(a.K, 64) <= NSTAGE || device_info(&d) != SEMMOE_OK) return false;
  // per-lane offsets are 32-bit
  return C::lds_bytes(a.nq) <= size_t(d.max_lds) && 128ull * a.ldw < (1ull << 31) && 2ull * C::BT * a.ldx < (1ull << 31);
}

template <int MODE, int TI, int TJ, int NSTAGE, int DMA_EVERY>
static int32_t launch_nn_w4(const GemmArgs& a, int max_rows, hipStream_t s) {
  using C = NnW4Cfg<TI, TJ, NSTAGE>;
  auto kern = gemm_nn_w4_kernel<MODE, TI, TJ, NSTAGE, DMA_EVERY>;
  static std::atomic<uint64_t> allowed{0};
  const int32_t st = allow_max_dynamic_lds(&allowed, reinterpret_cast<const void*>(kern));
  if (st != SEMMOE_OK) return st;
  const long long bound = (long long)(max_rows / C::BT + a.nq) * cdiv(a.N, C::BW);
  hipLaunchKernelGGL(kern, dim3(nn_grid(bound, 1)), dim3(256), C::lds_bytes(a.nq), s, a);
  SEMMOE_LAUNCH_CHECK();
  return SEMMOE_OK;
}

template <int MODE, int TJ, int NSTAGE>
static int32_t launch_nn_split(const GemmArgs& a, int max_rows, hipStream_t s) {
  using CH = NnW4Cfg<4, TJ, NSTAGE>;
  using CP = NnW4Cfg<2, 2, 3>;
  auto kern = gemm_nn_split_kernel<MODE, TJ, NSTAGE>;
  static std::atomic<uint64_t> allowed{0};
  const int32_t st = allow_max_dynamic_lds(&allowed, reinterpret_cast<const void*>(kern));
  if (st != SEMMOE_OK) return st;
  const long long bound = (long long)(max_rows / CH::BT + a.nq) * cdiv(a.N, CH::BW);
  const int grid = nn_grid(bound, 1);
  GemmArgs h = a;
  h.sched_mode = 1;
  h.sched_thr = 8;
  GemmArgs t = h;
  t.sched_mode = 2;
  t.sched_g = grid;
  t.sched_sub_t = CH::BT / CP::BT;
  t.sched_sub_f = CH::BW / CP::BW;
  const size_t lds = CH::lds_bytes(a.nq) > CP::lds_bytes(a.nq) ? CH::lds_bytes(a.nq) : CP::lds_bytes(a.nq);
  hipLaunchKernelGGL(kern, dim3(grid), dim3(256), lds, s, h, t);
  SEMMOE_LAUNCH_CHECK();
  return SEMMOE_OK;
}

template <int MODE, int TT, int NW>
static int32_t launch_nn_f32_as(const GemmArgs& a, int max_rows, hipStream_t s) {
  const long long bound = (long long)(max_rows / (16 * TT) + a.nq) * cdiv(a.N, 64);
  hipLaunchKernelGGL((gemm_nn_f32_kernel<MODE, TT, NW>), dim3(nn_grid(bound, NW == 8 ? 1 : 2)), dim3(64 * NW), 0, s, a);
  SEMMOE_LAUNCH_CHECK();
  return SEMMOE_OK;
}

template <int MODE, int TT>
static int32_t launch_nn_f32(const GemmArgs& a, int max_rows, int est, hipStream_t s) {
  DeviceInfo d;
  const int32_t st = device_info(&d);
  if (st != SEMMOE_OK) return st;
  // eight waves while the tiles (a ragged group's last one half full) have a compute unit each and K repays the sum over them: 16
  // experts of 32 rows, K 2048, 192 tiles 31 us, 34 with four waves; K 512, 384 tiles 23 and 17
  const long long tiles = (long long)a.nq * (2 * est / (16 * TT) + 1) * cdiv(a.N, 64) / 2;
  if (tiles <= d.num_cu && a.K >= 1024) return launch_nn_f32_as<MODE, TT, 8>(a, max_rows, s);
  return launch_nn_f32_as<MODE, TT, 4>(a, max_rows, s);
}

template <int MODE>
static int32_t launch_nn_f32(const GemmArgs& a, int max_rows, int est, hipStream_t s) {
  if (64ull * a.ldx >= (1ull << 31)) return SEMMOE_EUNSUPPORTED;  // 32-bit offsets of a tile's rows
  DeviceInfo d;
  const int32_t st = device_info(&d);
  if (st != SEMMOE_OK) return st;
  // 64 tokens where the tiles have a compute unit each (16 experts of 61 rows, K 1280, 376 columns, 96 tiles: 33 us, 22 as 16-token tiles)
  if (est > 48 && (long long)a.nq * cdiv(est, 64) * cdiv(a.N, 64) >= d.num_cu) return launch_nn_f32<MODE, 4>(a, max_rows, est, s);
  if (est > 16) return launch_nn_f32<MODE, 2>(a, max_rows, est, s);
  return launch_nn_f32<MODE, 1>(a, max_rows, est, s);
}

// Tile shapes.  Means of rows an expert, groups spread lognormally by 0.3; FFN gradients in us with one of the two products as 128 x 128 /
// 256 x 128 and pieces / 256 x 256 and pieces:
//   * 128 x 128 up to 80 rows (128 experts of 40, d 2048, F 768: 407 / 411 / 427) and while they have a compute unit each (16
//     experts of 90, d 4096, F 1536, dh: 263 / 283 / 312; 130 rows 327 / 314 / 341).  128 x 64 tiles are behind these even where they leave
//     half the chip idle, 64 x 64 ones too: a slice costs a wave much the same (one expert of 64 rows, d 7168, F 2048, dh: 172, 187 as
//     128 x 64, 170 as 64 x 64, dX 180 / 187 / 178; 8 of 90 rows, dX: 368 / 423; 16 of 48, d 2048, F 768, dX: 71 / 90 / 94)
//   * 256 x 256 from 192 rows on with four fifths of a round of them (tiles a compute unit: 0.42, 8 experts of 300, d 2048, F 768, dX 101 /
//     97 / 105; 0.46, 8 of 500, d 4096, F 1536, dh 374 / 346 / 372; 0.84, 16 of 300, d 2048, F 768, dX 150 / 154 / 145; 1.0, 8 of 900,
//     dX 170 / 161 / 153); 256 x 128 else
// Over 269 calls (8 to 64 experts of 60 to 2000 rows, five pairs of widths, all experts or one rank of eight) these lines are 0.4 % behind
// the best of the three for dh and 0.7 % for dX; with half a round in the place of four fifths 0.6 and 1.0.
// Shapes whose K is shorter than a ring, or with more groups than the tables hold, take 128 x 64 tiles with a barrier a slice.
template <int MODE>
static int32_t launch_nn_bf16(const GemmArgs& a, int max_rows, int est, hipStream_t s) {
  DeviceInfo d;
  const int32_t st = device_info(&d);
  if (st != SEMMOE_OK) return st;
  const long long cus = d.num_cu;
  // The mean is that of all experts.  A rank that an affinity placement loads has some twice as many rows, so a rank's mean is taken
  // twice.  140 calls of one rank of eight: with as many rows as the others it is 0.6 (dh) and 1.0 % (dX) behind the best tiles so, 0.7 and
  // 1.3 with the mean once; with twice as many 0.5 and 0.5, 1.2 and 1.8 once.
  if (a.offsets && (long long)a.nq * (est + 1) < max_rows) est *= 2;
  // a ragged group's last tile is half full in the mean; times 100
  auto tiles = [&](int bw, int bt) {
    const long long rows = !a.offsets ? 100ll * cdiv(est, bt) : (est * 2 <= bt ? 100ll : 100ll * est / bt + 50);
    return a.nq * rows * cdiv(a.N, bw);
  };
  if (nn_w4_fits<2, 2, 3>(a)) {
    if (est < 80 || tiles(128, 128) <= 110 * cus) return launch_nn_w4<MODE, 2, 2, 3, 1>(a, max_rows, s);
    const long long big = tiles(256, 256);
    if (est >= 192 && big >= 80 * cus && nn_w4_fits<4, 4, 2>(a))
      return launch_nn_split<MODE, 4, 2>(a, max_rows, s);
    if (nn_w4_fits<4, 2, 3>(a)) return launch_nn_split<MODE, 2, 3>(a, max_rows, s);
    return launch_nn_w4<MODE, 2, 2, 3, 1>(a, max_rows, s);
  }
  return launch_nn_ring<MODE, 2, 2, 2, 1, 64, 3>(a, max_rows, 2, s);
}

int32_t launch_gemm_nn(int mode, int dtype, const GemmArgs& a, int max_rows, int est, hipStream_t s) {
  if (a.nq <= 0 || max_rows <= 0) return SEMMOE_OK;
  if (a.nq > 512) return SEMMOE_EUNSUPPORTED;
  if (dtype == SEMMOE_FP32) return mode == kNnSums ? launch_nn_f32<kNnSums>(a, max_rows, est, s) : launch_nn_f32<kNnStore>(a, max_rows, est, s);
  return mode == kNnSums ? launch_nn_bf16<kNnSums>(a, max_rows, est, s) : launch_nn_bf16<kNnStore>(a, max_rows, est, s);
}

}  // namespace semmoe
