// Rows held in the registers of a team of waves: how they are read, written, summed and rounded to 8 bits.
//
// A team of `tr` threads (whole waves) owns a row; thread t holds the pieces t, t + tr, ... of 16 bytes.  The teams of a workgroup
// go through the same number of rows, so that their barriers match; a team without a row counts zeros and stores nothing.
#pragma once
#include "common.hpp"

namespace semmoe {

typedef __attribute__((ext_vector_type(4))) uint32_t row_u32x4_t;

template <bool BF16>
struct Piece {  // 16 bytes of a row as they lie in memory
  static constexpr int N = BF16 ? 8 : 4;
  row_u32x4_t v;
  __device__ __forceinline__ void load(const void* base, size_t at) {
    v = *reinterpret_cast<const row_u32x4_t*>(static_cast<const char*>(base) + at * (BF16 ? 2 : 4));
  }
  __device__ __forceinline__ void zero() { v = row_u32x4_t{0, 0, 0, 0}; }
  __device__ __forceinline__ float operator[](int x) const {
    if constexpr (BF16) return __uint_as_float(x & 1 ? v[x >> 1] & 0xffff0000u : v[x >> 1] << 16);
    else return __uint_as_float(v[x]);
  }
  __device__ __forceinline__ void round(const float (&f)[N]) {
#pragma unroll
    for (int x = 0; x < 4; ++x) v[x] = BF16 ? cvt_pk_bf16(f[(2 * x) % N], f[(2 * x + 1) % N]) : __float_as_uint(f[x]);
  }
  __device__ __forceinline__ void store(void* base, size_t at) const {
    *reinterpret_cast<row_u32x4_t*>(static_cast<char*>(base) + at * (BF16 ? 2 : 4)) = v;
  }
  // keeps the numbers packed from here on: unpacked ahead of time they take twice the registers
  __device__ __forceinline__ void stay() { asm volatile("" : "+v"(v)); }
};

// The sum (or, of bits, the maximum) over a team, the same in all of its threads, in an order that depends on the team's size alone.
// `part` is LDS of N numbers a wave of the workgroup, of this use alone until another join's barrier has passed.
template <int N, typename V, typename F>
__device__ __forceinline__ void team_join(V (&v)[N], V* part, int team_waves, F f) {
#pragma unroll
  for (int off = 32; off; off >>= 1)
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = f(v[n], __shfl_xor(v[n], off));
  if (team_waves == 1) return;  // uniform
  const int wave = threadIdx.x >> 6, first = wave / team_waves * team_waves;
  if ((threadIdx.x & 63) == 0)
#pragma unroll
    for (int n = 0; n < N; ++n) part[wave * N + n] = v[n];
  __syncthreads();
#pragma unroll
  for (int n = 0; n < N; ++n) v[n] = part[first * N + n];
  for (int w = 1; w < team_waves; ++w)
#pragma unroll
    for (int n = 0; n < N; ++n) v[n] = f(v[n], part[(first + w) * N + n]);
}

__device__ __forceinline__ uint32_t magnitude_bits(float f) { return __float_as_uint(f) & 0x7fffffffu; }

// A row in 8 bits: scale = amax * (1 / 127), q = rint(x * ((1 / amax) * 127)), ties to even; amax by its bits, so that NaN is more than
// any number.  A row with an infinity or a NaN has scale NaN and q = 0: whatever is multiplied with it is NaN.  The reciprocal keeps
// its bits where amax lies between 2^-64 and 2^64; rows beyond are taken times 2^64 or 2^-64, which loses nothing that q holds.
struct RowScale {
  float scale, r, pre;
  bool bad;
  __device__ __forceinline__ explicit RowScale(uint32_t amax_bits) {
    const float amax = __uint_as_float(amax_bits);
    bad = amax_bits >= 0x7f800000u;
    pre = amax < 0x1p-64f ? 0x1p64f : amax > 0x1p64f ? 0x1p-64f : 1.0f;
    r = amax > 0.0f ? 1.0f / (amax * pre) * 127.0f : 0.0f;
    scale = bad ? __uint_as_float(0x7fc00000u) : amax * (1.0f / 127.0f);
  }
  __device__ __forceinline__ uint32_t q(float x) const {
    const int v = bad ? 0 : __float2int_rn(x * pre * r);
    return uint32_t(v) & 255u;
  }
  // N numbers at `to`, which lies on N bytes
  template <int N>
  __device__ __forceinline__ void put(uint8_t* to, const float (&f)[N]) const {
    const uint32_t lo = q(f[0]) | q(f[1]) << 8 | q(f[2]) << 16 | q(f[3]) << 24;
    if constexpr (N == 4) *reinterpret_cast<uint32_t*>(to) = lo;
    else *reinterpret_cast<uint2*>(to) = make_uint2(lo, q(f[4]) | q(f[5]) << 8 | q(f[6]) << 16 | q(f[7]) << 24);
  }
};

// Threads of a team for rows of n_cols numbers, pieces a thread (1, 2 or 4; 0: too long for registers), teams of a workgroup.
struct RowTeams {
  int tr, np, teams;
  RowTeams(bool bf16, int n_cols, int most) {  // most: threads of a team
    const int pieces = n_cols / (bf16 ? 8 : 4);
    np = pieces <= most ? 1 : pieces <= 2 * most ? 2 : pieces <= 4 * most ? 4 : 0;
    tr = np ? cdiv(cdiv(pieces, np), 64) * 64 : most;
    teams = tr >= 256 ? 1 : 256 / tr;
  }
  // 512 threads where four pieces each hold the row: several such teams a compute unit are at different steps (norms of 20297 rows of
  // 3632 in fp32 228 us, 276 with up to 1024 threads; of 16384 rows of 7168 in bf16 194 and 244;
  // 20297 rows of 3632 in fp32 to 8 bits 72 and 88).  Four pieces a thread, norms of 1.1e8 numbers in bf16, widths 8208, 10240, 12288, 14336
  // and 16384: 222, 195, 190, 185 and 176 us, as 1024 threads of two 248, 221, 204, 215 and 209; of 5.5e7 in fp32, widths 4104, 5120, 6144, 7168 and
  // 8192: 178, 163, 160, 158 and 151, as 1024 threads of two 164, 157, 153, 165 and 153; to 8 bits within 5 % of one another, 7 % at 4104.
  // 1024 beyond it: 4096 rows of 32768 in bf16 to 8 bits 88 us, read twice 102.
  RowTeams(bool bf16, int n_cols) : RowTeams(bf16, n_cols, n_cols / (bf16 ? 8 : 4) <= 2048 ? 512 : 1024) {}
};

// Rows that one launch takes where every `teams` rows are a workgroup of `threads`: a grid has fewer than 2^32 threads.  More rows are
// more launches (narrow rows from 2^25 on).
inline int rows_a_launch(int teams, int threads) { return int((1u << 31) / unsigned(threads)) * teams; }

// Rows of `n_cols` activations in 8 bits, see semmoe_quantize_rows.  row_range (device, nullable): only the rows from row_range[0] up
// to row_range[n_range] exist, n_rows is then the most there can be.
int32_t launch_quantize_rows(bool bf16, const void* X, int64_t ldx, int n_rows, int n_cols, const int32_t* row_range, int n_range,
                             void* Xq, float* x_scale, hipStream_t stream);

}  // namespace semmoe
