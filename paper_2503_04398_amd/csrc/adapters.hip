// Low-rank adapters of many requests at once beside a projection that all of them share: the index that orders a batch's
// tokens by adapter, the forward form Y = Y_base + s_a B_a (A_a x), and its gradient.
//
// With u = s_a A_a x (rank numbers a token) and v = s_a B_a^T dY:
//   Y  = Y_base + B_a u          dX = dX_base + A_a^T v
//   dA_a = sum over a's tokens of v x^T        dB_a = sum of dY u^T
// so everything is made of three kernels over the ordered tokens: `shrink` (rows times a factor, down to rank numbers),
// `expand` (rank numbers times a factor, added to rows) and `outer` (sums over tokens).  u and v are fp32 sums in the
// workspace; as operands of the matrix instructions of bf16 rows they are rounded to bf16 once, as the rows and factors are.
//
// A 16-byte piece of a row is the unit throughout: eight bf16 (v_mfma_f32_16x16x32_bf16) or four fp32 (four times
// v_mfma_f32_16x16x4_f32, a lane's four numbers in turn: any order of k will do as long as both operands use it).
#include "common.hpp"

namespace semmoe {

typedef __attribute__((ext_vector_type(8))) __bf16 bf16x8_t;
typedef __attribute__((ext_vector_type(4))) float f32x4_t;
typedef __attribute__((ext_vector_type(4))) uint32_t u32x4_t;

template <bool F32>
__device__ __forceinline__ f32x4_t piece_mfma(u32x4_t a, u32x4_t b, f32x4_t c) {
  if constexpr (F32) {
#pragma unroll
    for (int j = 0; j < 4; ++j)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[j]), __uint_as_float(b[j]), c, 0, 0, 0);
    return c;
  } else {
    return __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8_t, a), __builtin_bit_cast(bf16x8_t, b), c, 0,
                                                   0, 0);
  }
}

template <bool F32>
struct Elem {
  using type = float;
  static constexpr int kSize = 4, kPer16 = 4, kStep = 16;  // bytes; numbers in 16 bytes; depth of a piece_mfma
};
template <>
struct Elem<false> {
  using type = bf16_t;
  static constexpr int kSize = 2, kPer16 = 8, kStep = 32;
};

template <bool F32>
__device__ __forceinline__ typename Elem<F32>::type to_act(float f) {
  if constexpr (F32) return f; else return f32_to_bf16(f);
}

// 16 bytes whose numbers lie `stride` elements apart in LDS (a fragment along the other dimension)
template <bool F32>
__device__ __forceinline__ u32x4_t gather_piece(const typename Elem<F32>::type* p, int stride) {
  u32x4_t v;
  if constexpr (F32) {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = __float_as_uint(p[e * stride]);
  } else {
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = uint32_t(p[2 * e * stride]) | (uint32_t(p[(2 * e + 1) * stride]) << 16);
  }
  return v;
}

// The ordered tokens of group g: positions [lo, hi).  Group n_adapters: tokens of requests without an adapter, and -1
// behind them.  Offsets are clamped, so that no position lies outside the order whatever they hold.
struct Span {
  int lo, hi;
};
__device__ __forceinline__ Span group_span(const int32_t* __restrict__ offsets, int n_adapters, int T, int g) {
  Span s;
  s.lo = min(max(offsets[g], 0), T);
  s.hi = g < n_adapters ? min(max(offsets[g + 1], s.lo), T) : T;
  return s;
}

// Items of the groups: group g has max(least, ceil(tokens / per)) of them; pre[g] = items before it (LDS, n_groups + 1).
// Wave 0 scans; ends with a barrier.
__device__ __forceinline__ int build_items(const int32_t* __restrict__ offsets, int n_adapters, int n_groups, int T, int per,
                                           int least, int* pre) {
  const int tid = threadIdx.x;
  if (tid < 64) {
    const int each = (n_groups + 63) / 64;
    const int lo = min(tid * each, n_groups), hi = min(lo + each, n_groups);
    int s = 0;
    for (int g = lo; g < hi; ++g) {
      const Span sp = group_span(offsets, n_adapters, T, g);
      s += max(least, (sp.hi - sp.lo + per - 1) / per);
    }
    int incl = s;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int v = __shfl_up(incl, off);
      if (tid >= off) incl += v;
    }
    int run = incl - s;
    if (tid == 0) pre[0] = 0;
    for (int g = lo; g < hi; ++g) {
      const Span sp = group_span(offsets, n_adapters, T, g);
      run += max(least, (sp.hi - sp.lo + per - 1) / per);
      pre[g + 1] = run;
    }
  }
  __syncthreads();
  return pre[n_groups];
}

__device__ __forceinline__ int item_group(const int* pre, int n_groups, int item) {
  int lo = 0, hi = n_groups;  // pre[lo] <= item < pre[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) >> 1;
    if (pre[mid] <= item) lo = mid; else hi = mid;
  }
  return lo;
}

struct AdapterArgs {
  const int32_t* order;    // [T] ordered tokens, -1: none
  const int32_t* offsets;  // [n_adapters + 1]
  int T, n_adapters, rank;
};

// ---- shrink: U[part][position][j] = s_a * sum over the part's k of R[token, k] F_a(j, k) ------------------------------
// TR = false: F_a = A_a [rank][K], rows along k.  TR = true: F_a = B_a [K][rank].
struct ShrinkArgs {
  AdapterArgs ad;
  const void* R;       // rows, act type
  size_t ldr;          // elements
  const void* F;       // act, n_adapters panels of rank * K
  const float* scale;  // [n_adapters] or nullptr
  int K, part_k, parts;  // part_k: depth of a part, a multiple of 128 bytes
  float* U;            // [parts][T][rank]
};

template <bool F32, int RT, int TT, bool TR>
__global__ __launch_bounds__(256) void shrink_kernel(const ShrinkArgs a) {
  using E = Elem<F32>;
  using elem = typename E::type;
  constexpr int BT = 16 * TT, KSL = 128 / E::kSize;  // tokens of a tile; numbers in 128 bytes of a row
  extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
  const int n_ad = a.ad.n_adapters, r = a.ad.rank;
  int* pre = reinterpret_cast<int*>(lds_raw);
  unsigned char* body = lds_raw + ((n_ad + 2) * 4 + 15) / 16 * 16;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, g4 = lane >> 4;

  const int items = build_items(a.ad.offsets, n_ad, n_ad, a.ad.T, BT, 0, pre);
  const int item = blockIdx.x / a.parts, part = blockIdx.x % a.parts;
  if (item >= items) return;
  const int g = item_group(pre, n_ad, item);
  const Span sp = group_span(a.ad.offsets, n_ad, a.ad.T, g);
  const int p0 = sp.lo + (item - pre[g]) * BT, n_tok = min(BT, sp.hi - p0);
  if (n_tok <= 0) return;

  const elem* row[TT];
#pragma unroll
  for (int t = 0; t < TT; ++t) {
    const int tok = a.ad.order[p0 + min(t * 16 + l16, n_tok - 1)];
    row[t] = static_cast<const elem*>(a.R) + size_t(min(max(tok, 0), a.ad.T - 1)) * a.ldr;
  }
  const elem* F = static_cast<const elem*>(a.F) + size_t(g) * r * a.K;

  f32x4_t acc[RT][TT];
#pragma unroll
  for (int j = 0; j < RT; ++j)
#pragma unroll
    for (int t = 0; t < TT; ++t) acc[j][t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};

  const int k_lo = part * a.part_k, k_hi = min(a.K, k_lo + a.part_k);
  elem* stg = reinterpret_cast<elem*>(body) + size_t(wave) * KSL * (16 * RT + E::kPer16);  // TR: a wave's slice of B
  constexpr int LDB = 16 * RT + E::kPer16;
  for (int k0 = k_lo + wave * KSL; k0 < k_hi; k0 += 4 * KSL) {
    if constexpr (TR) {  // [KSL][rank] of B is one run of memory
      const int per_row = r / E::kPer16, n_k = min(KSL, k_hi - k0);
      for (int c = lane; c < KSL * per_row; c += 64) {
        const int kk = c / per_row, jj = c % per_row;
        const u32x4_t v = kk < n_k ? *reinterpret_cast<const u32x4_t*>(F + size_t(k0 + kk) * r + jj * E::kPer16)
                                   : u32x4_t{0, 0, 0, 0};
        *reinterpret_cast<u32x4_t*>(stg + kk * LDB + jj * E::kPer16) = v;
      }
      asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
    }
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int kk = h * E::kStep + g4 * E::kPer16, k = k0 + kk;
      const bool in = k < k_hi;
      u32x4_t x[TT];
#pragma unroll
      for (int t = 0; t < TT; ++t) x[t] = in ? *reinterpret_cast<const u32x4_t*>(row[t] + k) : u32x4_t{0, 0, 0, 0};
#pragma unroll
      for (int j = 0; j < RT; ++j) {
        u32x4_t f;
        if constexpr (TR)
          f = gather_piece<F32>(stg + kk * LDB + min(j * 16 + l16, r - 1), LDB);
        else
          f = in ? *reinterpret_cast<const u32x4_t*>(F + size_t(min(j * 16 + l16, r - 1)) * a.K + k) : u32x4_t{0, 0, 0, 0};
#pragma unroll
        for (int t = 0; t < TT; ++t) acc[j][t] = piece_mfma<F32>(f, x[t], acc[j][t]);
      }
    }
    if constexpr (TR) asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
  }

  // the four waves' sums meet in LDS, a tile of tokens at a time
  const float s = a.scale ? a.scale[g] : 1.0f;
  f32x4_t* red = reinterpret_cast<f32x4_t*>(body);  // [wave][RT][64]
  float* U = a.U + size_t(part) * a.ad.T * r;
#pragma unroll
  for (int t = 0; t < TT; ++t) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < RT; ++j) red[(wave * RT + j) * 64 + lane] = acc[j][t];
    __syncthreads();
    for (int j = wave; j < RT; j += 4) {
      f32x4_t v = red[j * 64 + lane];
#pragma unroll
      for (int w = 1; w < 4; ++w) v += red[(w * RT + j) * 64 + lane];
      const int tok = t * 16 + l16, jj = j * 16 + g4 * 4;
      if (tok < n_tok && jj < r) *reinterpret_cast<f32x4_t*>(U + size_t(p0 + tok) * r + jj) = v * s;
    }
  }
}

// ---- expand: Out[token, n] = Base[token, n] + sum over j of F_a(n, j) U[position][j] -----------------------------------
// TR = false: F_a = B_a [N][rank].  TR = true: F_a = A_a [rank][N].  Group n_adapters: Out = Base.
struct ExpandArgs {
  AdapterArgs ad;
  const float* U;
  int parts;
  const void* F;
  int N;
  const void* Base;  // act or nullptr (zero)
  size_t ld_base;
  void* Out;
  size_t ldo;
};

constexpr int kExpandCols = 128;

template <bool F32, int RT, int TT, bool TR>
__global__ __launch_bounds__(256) void expand_kernel(const ExpandArgs a) {
  using E = Elem<F32>;
  using elem = typename E::type;
  constexpr int BT = 16 * TT, NC = kExpandCols, LDD = NC + 4;
  constexpr int RP = (16 * RT + E::kStep - 1) / E::kStep * E::kStep, LDU = RP + E::kPer16, KS = RP / E::kStep;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
  const int n_ad = a.ad.n_adapters, r = a.ad.rank;
  int* pre = reinterpret_cast<int*>(lds_raw);
  float* delta = reinterpret_cast<float*>(lds_raw + ((n_ad + 2) * 4 + 15) / 16 * 16);  // [BT][LDD]
  elem* Us = reinterpret_cast<elem*>(delta + BT * LDD);                                // [BT][LDU]
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, g4 = lane >> 4;

  const int items = build_items(a.ad.offsets, n_ad, n_ad + 1, a.ad.T, BT, 0, pre);
  const int n_chunks = (a.N + NC - 1) / NC;
  const int item = blockIdx.x / n_chunks, n0 = (blockIdx.x % n_chunks) * NC;
  if (item >= items) return;
  const int g = item_group(pre, n_ad + 1, item);
  const Span sp = group_span(a.ad.offsets, n_ad, a.ad.T, g);
  const int p0 = sp.lo + (item - pre[g]) * BT, n_tok = min(BT, sp.hi - p0);
  if (n_tok <= 0) return;
  const bool none = g == n_ad;
  if (none && a.Base == a.Out && a.ld_base == a.ldo) return;

  if (!none) {
    for (int i = tid; i < BT * (RP / 4); i += 256) {
      const int t = i / (RP / 4), j = i % (RP / 4) * 4;
      f32x4_t v = {0.0f, 0.0f, 0.0f, 0.0f};
      if (t < n_tok && j < r)
        for (int p = 0; p < a.parts; ++p)
          v += *reinterpret_cast<const f32x4_t*>(a.U + (size_t(p) * a.ad.T + p0 + t) * r + j);
#pragma unroll
      for (int e = 0; e < 4; ++e) Us[t * LDU + j + e] = to_act<F32>(v[e]);
    }
    __syncthreads();
    const elem* F = static_cast<const elem*>(a.F) + size_t(g) * r * a.N;
    f32x4_t acc[2][TT];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int t = 0; t < TT; ++t) acc[i][t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      const int k = ks * E::kStep + g4 * E::kPer16;
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const int n = min(n0 + wave * 32 + i * 16 + l16, a.N - 1);
        u32x4_t f = {0, 0, 0, 0};
        if (k < r) {
          if constexpr (TR) f = gather_piece<F32>(F + size_t(k) * a.N + n, a.N);
          else f = *reinterpret_cast<const u32x4_t*>(F + size_t(n) * r + k);
        }
#pragma unroll
        for (int t = 0; t < TT; ++t)
          acc[i][t] = piece_mfma<F32>(f, *reinterpret_cast<const u32x4_t*>(Us + (t * 16 + l16) * LDU + k), acc[i][t]);
      }
    }
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int t = 0; t < TT; ++t)
        *reinterpret_cast<f32x4_t*>(delta + (t * 16 + l16) * LDD + wave * 32 + i * 16 + g4 * 4) = acc[i][t];
    __syncthreads();
  }

  constexpr int CPR = NC / E::kPer16;  // 16-byte pieces of a row
  for (int i = tid; i < n_tok * CPR; i += 256) {
    const int t = i / CPR, c = i % CPR * E::kPer16, n = n0 + c;
    const int tok = a.ad.order[p0 + t];
    if (n >= a.N || unsigned(tok) >= unsigned(a.ad.T)) continue;
    u32x4_t v = {0, 0, 0, 0};
    if (a.Base) v = *reinterpret_cast<const u32x4_t*>(static_cast<const elem*>(a.Base) + size_t(tok) * a.ld_base + n);
    if (!none) {
      const float* dl = delta + t * LDD + c;
      if constexpr (F32) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) + dl[e]);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
          v[e] = pack_bf16x2(__uint_as_float(v[e] << 16) + dl[2 * e], __uint_as_float(v[e] & 0xffff0000u) + dl[2 * e + 1]);
      }
    }
    *reinterpret_cast<u32x4_t*>(static_cast<elem*>(a.Out) + size_t(tok) * a.ldo + n) = v;
  }
}

// ---- outer: dF_a = sum over a's tokens of U[position][j] R[token][c] ---------------------------------------------------
// SWAP = false: dF_a [rank][C] (c along a row).  SWAP = true: dF_a [C][rank].  An adapter's tokens are cut into segments;
// one with several of them leaves fp32 sums, which `outer_join` adds in the order of the segments.
struct OuterArgs {
  AdapterArgs ad;
  const float* U;
  int parts;
  const void* R;
  size_t ldr;
  int C, seg;      // columns; tokens of a segment
  int max_items;   // items that `partial` holds
  float* partial;  // [max_items][rank * C]
  void* dF;        // act [n_adapters][rank * C]
};

constexpr int kOuterCols = 64, kOuterTok = 64;

template <bool F32, int RT, bool SWAP>
__global__ __launch_bounds__(256) void outer_kernel(const OuterArgs a) {
  using E = Elem<F32>;
  using elem = typename E::type;
  constexpr int NC = kOuterCols, KT = kOuterTok, LDR = NC + E::kPer16, LDU = 16 * RT + E::kPer16;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
  const int n_ad = a.ad.n_adapters, r = a.ad.rank;
  int* pre = reinterpret_cast<int*>(lds_raw);
  elem* Rs = reinterpret_cast<elem*>(lds_raw + ((n_ad + 2) * 4 + 15) / 16 * 16);  // [KT][LDR]
  elem* Us = Rs + KT * LDR;                                                        // [KT][LDU]
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, g4 = lane >> 4;

  const int items = build_items(a.ad.offsets, n_ad, n_ad, a.ad.T, a.seg, 1, pre);
  const int n_chunks = (a.C + NC - 1) / NC;
  const int item = blockIdx.x / n_chunks, c0 = (blockIdx.x % n_chunks) * NC;
  if (item >= items) return;
  const int g = item_group(pre, n_ad, item);
  const Span sp = group_span(a.ad.offsets, n_ad, a.ad.T, g);
  const int p0 = sp.lo + (item - pre[g]) * a.seg, p1 = min(sp.hi, p0 + a.seg);
  const bool whole = pre[g + 1] - pre[g] == 1;

  f32x4_t acc[RT];
#pragma unroll
  for (int j = 0; j < RT; ++j) acc[j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  for (int p = p0; p < p1; p += KT) {
    constexpr int CPR = NC / E::kPer16;
    for (int i = tid; i < KT * CPR; i += 256) {
      const int t = i / CPR, c = i % CPR * E::kPer16;
      u32x4_t v = {0, 0, 0, 0};
      if (p + t < p1 && c0 + c < a.C) {
        const int tok = a.ad.order[p + t];
        if (unsigned(tok) < unsigned(a.ad.T))
          v = *reinterpret_cast<const u32x4_t*>(static_cast<const elem*>(a.R) + size_t(tok) * a.ldr + c0 + c);
      }
      *reinterpret_cast<u32x4_t*>(Rs + t * LDR + c) = v;
    }
    for (int i = tid; i < KT * RT * 4; i += 256) {
      const int t = i / (RT * 4), j = i % (RT * 4) * 4;
      f32x4_t v = {0.0f, 0.0f, 0.0f, 0.0f};
      if (p + t < p1 && j < r)
        for (int q = 0; q < a.parts; ++q)
          v += *reinterpret_cast<const f32x4_t*>(a.U + (size_t(q) * a.ad.T + p + t) * r + j);
#pragma unroll
      for (int e = 0; e < 4; ++e) Us[t * LDU + j + e] = to_act<F32>(v[e]);
    }
    __syncthreads();
#pragma unroll
    for (int ks = 0; ks < KT / E::kStep; ++ks) {
      const int k = ks * E::kStep + g4 * E::kPer16;
      const u32x4_t x = gather_piece<F32>(Rs + k * LDR + wave * 16 + l16, LDR);
#pragma unroll
      for (int j = 0; j < RT; ++j) {
        const u32x4_t u = gather_piece<F32>(Us + k * LDU + j * 16 + l16, LDU);
        acc[j] = SWAP ? piece_mfma<F32>(u, x, acc[j]) : piece_mfma<F32>(x, u, acc[j]);
      }
    }
    __syncthreads();
  }

  // SWAP = false: lane holds columns 4 g4 + 0..3 of its wave's 16 for rank number l16 of tile j; SWAP = true: rank numbers
  // 4 g4 + 0..3 of tile j for column l16
#pragma unroll
  for (int j = 0; j < RT; ++j) {
    const int c = c0 + wave * 16 + (SWAP ? l16 : g4 * 4), jj = j * 16 + (SWAP ? g4 * 4 : l16);
    if (c >= a.C || jj >= r) continue;
    const size_t at = SWAP ? size_t(c) * r + jj : size_t(jj) * a.C + c;
    if (!whole) {
      *reinterpret_cast<f32x4_t*>(a.partial + size_t(item) * r * a.C + at) = acc[j];
      continue;
    }
    elem* o = static_cast<elem*>(a.dF) + size_t(g) * r * a.C + at;
    if constexpr (F32) {
      *reinterpret_cast<f32x4_t*>(o) = acc[j];
    } else {
      *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16x2(acc[j][0], acc[j][1]), pack_bf16x2(acc[j][2], acc[j][3]));
    }
  }
}

template <bool F32>
__global__ __launch_bounds__(256) void outer_join_kernel(const OuterArgs a) {
  using elem = typename Elem<F32>::type;
  extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
  const int n_ad = a.ad.n_adapters;
  int* pre = reinterpret_cast<int*>(lds_raw);
  build_items(a.ad.offsets, n_ad, n_ad, a.ad.T, a.seg, 1, pre);
  const int g = blockIdx.y, first = pre[g], n = min(pre[g + 1], a.max_items) - first;
  if (n <= 1) return;
  const size_t size = size_t(a.ad.rank) * a.C;
  for (size_t i = (size_t(blockIdx.x) * 256 + threadIdx.x) * 4; i < size; i += size_t(gridDim.x) * 1024) {
    f32x4_t v = *reinterpret_cast<const f32x4_t*>(a.partial + first * size + i);
    for (int q = 1; q < n; ++q) v += *reinterpret_cast<const f32x4_t*>(a.partial + (first + q) * size + i);
    elem* o = static_cast<elem*>(a.dF) + g * size + i;
    if constexpr (F32) {
      *reinterpret_cast<f32x4_t*>(o) = v;
    } else {
      *reinterpret_cast<uint2*>(o) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
    }
  }
}

// ---- index ---------------------------------------------------------------------------------------------------------------
// A stable counting sort without counters: a request's place is the sum of the lengths of all requests that come before it
// by (adapter, number), which a wave adds up 64 requests at a time.  One launch, no workspace, no atomics, the same bits
// whatever runs first; n_req^2 / 64 steps over the chip, which beats a pass per digit for the batches of a serving step.
__device__ __forceinline__ int wave_sum(int v) {
#pragma unroll
  for (int off = 32; off; off >>= 1) v += __shfl_xor(v, off);
  return v;
}

struct IndexArgs {
  const int32_t* req_offsets;
  const int32_t* adapter_of_req;
  int n_req, n_adapters, T, per_block;
  int32_t* order;
  int32_t* offsets;
};

__global__ __launch_bounds__(256) void adapter_index_kernel(const IndexArgs a, int token_blocks) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  auto start_of = [&](int q) { return q == 0 ? 0 : min(max(a.req_offsets[q], 0), a.T); };
  auto key_of = [&](int q) {
    const int v = a.adapter_of_req[q];
    return unsigned(v) < unsigned(a.n_adapters) ? v : a.n_adapters;
  };
  // tokens of all requests whose (key, number) is below (key, q)
  auto before = [&](int key, int q) {
    int s = 0;
#pragma unroll 4
    for (int i = lane; i < a.n_req; i += 64) {
      const int k = key_of(i), len = max(0, start_of(i + 1) - start_of(i));
      s += k < key || (k == key && i < q) ? len : 0;
    }
    return wave_sum(s);
  };
  if (int(blockIdx.x) >= token_blocks) {
    const int g = (blockIdx.x - token_blocks) * 4 + wave;
    if (g > a.n_adapters) return;
    const int s = before(g, 0);
    if (lane == 0) a.offsets[g] = min(s, a.T);
    return;
  }
  const int t0 = blockIdx.x * a.per_block, t1 = min(a.T, t0 + a.per_block);
  const int end = start_of(a.n_req);
  for (int t = max(t0, end) + int(threadIdx.x); t < t1; t += 256) a.order[t] = -1;  // behind the last request
  if (t0 >= end) return;
  // the last request that begins at or before t0, 64 probes at a time
  int lo = 0, hi = a.n_req;  // start_of(lo) <= t0; answer in [lo, hi)
  while (hi - lo > 1) {
    const int step = (hi - lo + 63) / 64;
    const int at = lo + (lane + 1) * step;
    const unsigned long long m = __ballot(at < hi && start_of(at) <= t0);
    const int n = __popcll(m);
    const int nlo = lo + n * step;
    hi = min(hi, nlo + step);
    lo = nlo;
  }
  for (int q = lo + wave; q < a.n_req; q += 4) {
    const int b = start_of(q), e = min(start_of(q + 1), t1);
    if (b >= t1) break;
    if (e <= max(b, t0)) continue;
    const int pos = before(key_of(q), q) - b;
    for (int t = max(b, t0) + lane; t < e; t += 64)
      if (unsigned(pos + t) < unsigned(a.T)) a.order[pos + t] = t;
  }
}

// ---- host ----------------------------------------------------------------------------------------------------------------
struct AdapterPlan {
  int shrink_tt, expand_tt;       // 16-token tiles a workgroup takes
  int part_k_in, parts_in;        // shrink over d_in
  int part_k_out, parts_out;      // shrink over d_out
  int seg;                        // tokens of a segment of `outer`
  long long tiles(int tt, int T, int groups) const { return T / (16 * tt) + (groups < T ? groups : T); }
};

// K cut into parts until the tiles fill the chip about twice, each part at least 1 KB of a row
static void cut_k(int K, int es, long long tiles, int* part_k, int* parts) {
  const int unit = 512 / es;  // a slice for each of the four waves
  const int units = cdiv(K, unit);
  long long want = tiles > 0 ? 512 / tiles : 1;
  want = want < 1 ? 1 : (want > 16 ? 16 : want);
  const int most = units < 2 ? 1 : units / 2;
  int n = int(want < most ? want : most);
  const int per = cdiv(units, n);
  *part_k = per * unit;
  *parts = cdiv(units, per);
}

static AdapterPlan plan_of(const semmoe_config* cfg, const semmoe_adapter_shape* s) {
  AdapterPlan p;
  const int T = cfg->T, es = int(act_bytes(cfg));
  const int mean = T / s->n_adapters;
  const int rt = cdiv(s->rank, 16);
  p.shrink_tt = mean <= 24 ? 1 : (rt > 4 || mean <= 48 ? 2 : 4);
  p.expand_tt = mean <= 24 ? 1 : (mean <= 48 ? 2 : 4);
  const long long tiles = p.tiles(p.shrink_tt, T, s->n_adapters);
  cut_k(s->d_in, es, tiles, &p.part_k_in, &p.parts_in);
  cut_k(s->d_out, es, tiles, &p.part_k_out, &p.parts_out);
  const long long chunks = cdiv(s->d_in < s->d_out ? s->d_in : s->d_out, kOuterCols);
  long long segs = 1024 / (chunks > 0 ? chunks : 1);
  segs = segs < 1 ? 1 : segs;
  long long seg = T / segs;
  seg = (seg + 255) / 256 * 256;
  p.seg = int(seg < 256 ? 256 : seg);
  return p;
}

static size_t u_floats(const semmoe_config* cfg, const semmoe_adapter_shape* s, int parts) {
  return size_t(parts) * cfg->T * s->rank;
}
static size_t partial_items(const semmoe_config* cfg, const semmoe_adapter_shape* s, const AdapterPlan& p) {
  return size_t(cfg->T) / p.seg + s->n_adapters;
}

static int32_t check_shape(const semmoe_config* cfg, const semmoe_adapter_shape* s) {
  const int32_t st = validate_config(cfg, true, false, false);
  if (st != SEMMOE_OK) return st;
  if (!s) return SEMMOE_EINVAL;
  if (s->n_adapters <= 0 || s->rank <= 0 || s->d_in <= 0 || s->d_out <= 0) return SEMMOE_EINVAL;
  if (s->ldx < 0 || s->ldy < 0 || s->ld_base < 0 || s->ld_out < 0) return SEMMOE_EINVAL;
  if (s->rank % 8 || s->d_in % 8 || s->d_out % 8) return SEMMOE_ESHAPE;
  if (s->ldx % 8 || s->ldy % 8 || s->ld_base % 8 || s->ld_out % 8) return SEMMOE_ESHAPE;
  if (s->n_adapters > SEMMOE_MAX_ADAPTERS || s->rank > SEMMOE_MAX_RANK) return SEMMOE_EUNSUPPORTED;
  if (s->d_in > (1 << 20) || s->d_out > (1 << 20)) return SEMMOE_EUNSUPPORTED;
  return SEMMOE_OK;
}

// a leading dimension: `ld` or, where that is 0, `width`; rows must not overlap
static bool take_ld(int64_t ld, int width, size_t* out) {
  *out = size_t(ld ? ld : width);
  return *out >= size_t(width);
}

template <typename F>
static int32_t with_rank_tiles(int rank, F f) {
  const int rt = cdiv(rank, 16);
  if (rt <= 1) return f(std::integral_constant<int, 1>{});
  if (rt <= 2) return f(std::integral_constant<int, 2>{});
  if (rt <= 4) return f(std::integral_constant<int, 4>{});
  static_assert(SEMMOE_MAX_RANK == 128, "the widths here");
  return f(std::integral_constant<int, 8>{});
}
template <typename F>
static int32_t with_token_tiles(int tt, F f) {
  if (tt <= 1) return f(std::integral_constant<int, 1>{});
  if (tt <= 2) return f(std::integral_constant<int, 2>{});
  return f(std::integral_constant<int, 4>{});
}

static size_t pre_bytes(int n_ad) { return ((size_t(n_ad) + 2) * 4 + 15) / 16 * 16; }

// One launch of 256 threads a workgroup.  `allowed`: the kernel's own flag word (allow_max_dynamic_lds).
template <typename K, typename A>
static int32_t launch_groups(K kern, std::atomic<uint64_t>* allowed, long long groups, size_t lds, hipStream_t s, const A& a) {
  if (groups <= 0) return SEMMOE_OK;
  if (groups >= (1ll << 24)) return SEMMOE_EUNSUPPORTED;  // 2^32 threads a launch
  if (lds > 48 * 1024) {
    DeviceInfo d;
    int32_t st = device_info(&d);
    if (st != SEMMOE_OK) return st;
    if (lds > size_t(d.max_lds)) return SEMMOE_EUNSUPPORTED;
    st = allow_max_dynamic_lds(allowed, reinterpret_cast<const void*>(kern));
    if (st != SEMMOE_OK) return st;
  }
  hipLaunchKernelGGL(kern, dim3(unsigned(groups)), dim3(256), lds, s, a);
  SEMMOE_LAUNCH_CHECK();
  return SEMMOE_OK;
}

template <bool F32, bool TR>
static int32_t launch_shrink(const ShrinkArgs& a, int tt, long long tiles, hipStream_t s) {
  return with_rank_tiles(a.ad.rank, [&](auto rt) {
    return with_token_tiles(tt, [&](auto t4) -> int32_t {
      constexpr int RT = decltype(rt)::value, TT = decltype(t4)::value;
      using E = Elem<F32>;
      auto kern = shrink_kernel<F32, RT, TT, TR>;
      const size_t red = size_t(4) * RT * 1024;
      const size_t stage = TR ? size_t(4) * (128 / E::kSize) * (16 * RT + E::kPer16) * E::kSize : 0;
      const size_t lds = pre_bytes(a.ad.n_adapters) + (red > stage ? red : stage);
      static std::atomic<uint64_t> allowed{0};
      return launch_groups(kern, &allowed, tiles * a.parts, lds, s, a);
    });
  });
}

template <bool F32, bool TR>
static int32_t launch_expand(const ExpandArgs& a, int tt, long long tiles, hipStream_t s) {
  return with_rank_tiles(a.ad.rank, [&](auto rt) {
    return with_token_tiles(tt, [&](auto t4) -> int32_t {
      constexpr int RT = decltype(rt)::value, TT = decltype(t4)::value;
      using E = Elem<F32>;
      auto kern = expand_kernel<F32, RT, TT, TR>;
      const size_t rp = (16 * RT + E::kStep - 1) / E::kStep * E::kStep;
      const size_t lds = pre_bytes(a.ad.n_adapters) + size_t(16 * TT) * (kExpandCols + 4) * 4 + size_t(16 * TT) * (rp + E::kPer16) * E::kSize;
      static std::atomic<uint64_t> allowed{0};
      return launch_groups(kern, &allowed, tiles * cdiv(a.N, kExpandCols), lds, s, a);
    });
  });
}

template <bool F32, bool SWAP>
static int32_t launch_outer(const OuterArgs& a, size_t items, hipStream_t s) {
  const int32_t st = with_rank_tiles(a.ad.rank, [&](auto rt) -> int32_t {
    constexpr int RT = decltype(rt)::value;
    using E = Elem<F32>;
    auto kern = outer_kernel<F32, RT, SWAP>;
    const size_t lds = pre_bytes(a.ad.n_adapters) + size_t(kOuterTok) * (kOuterCols + E::kPer16 + 16 * RT + E::kPer16) * E::kSize;
    static std::atomic<uint64_t> allowed{0};
    return launch_groups(kern, &allowed, (long long)items * cdiv(a.C, kOuterCols), lds, s, a);
  });
  if (st != SEMMOE_OK) return st;
  if (a.ad.T <= a.seg) return SEMMOE_OK;  // no adapter has a second segment
  const size_t size = size_t(a.ad.rank) * a.C;
  const unsigned gx = unsigned((size + 4095) / 4096);
  hipLaunchKernelGGL((outer_join_kernel<F32>), dim3(gx, a.ad.n_adapters), dim3(256), pre_bytes(a.ad.n_adapters), s, a);
  SEMMOE_LAUNCH_CHECK();
  return SEMMOE_OK;
}

template <bool F32>
static int32_t run_adapters(const semmoe_config* cfg, const semmoe_adapter_shape* sh, const AdapterPlan& p, hipStream_t s,
                            const void* X, const AdapterArgs& ad, const void* A, const void* B, const float* scale,
                            const void* Y_base, void* Y, float* U, size_t ldx, size_t ld_base, size_t ldo) {
  ShrinkArgs sa{ad, X, ldx, A, scale, sh->d_in, p.part_k_in, p.parts_in, U};
  const int32_t st = launch_shrink<F32, false>(sa, p.shrink_tt, p.tiles(p.shrink_tt, cfg->T, sh->n_adapters), s);
  if (st != SEMMOE_OK) return st;
  ExpandArgs ea{ad, U, p.parts_in, B, sh->d_out, Y_base, ld_base, Y, ldo};
  return launch_expand<F32, false>(ea, p.expand_tt, p.tiles(p.expand_tt, cfg->T, sh->n_adapters + 1), s);
}

template <bool F32>
static int32_t run_adapters_grad(const semmoe_config* cfg, const semmoe_adapter_shape* sh, const AdapterPlan& p, hipStream_t s,
                                 const void* X, const void* dY, const AdapterArgs& ad, const void* A, const void* B,
                                 const float* scale, const void* dX_base, void* dX, void* dA, void* dB, float* U, float* V,
                                 float* partial, size_t ldx, size_t ldy, size_t ld_base, size_t ldo) {
  const long long tiles = p.tiles(p.shrink_tt, cfg->T, sh->n_adapters);
  const size_t items = partial_items(cfg, sh, p);
  int32_t st;
  if (dX || dA) {
    ShrinkArgs sa{ad, dY, ldy, B, scale, sh->d_out, p.part_k_out, p.parts_out, V};
    st = launch_shrink<F32, true>(sa, p.shrink_tt, tiles, s);
    if (st != SEMMOE_OK) return st;
  }
  if (dX) {
    ExpandArgs ea{ad, V, p.parts_out, A, sh->d_in, dX_base, ld_base, dX, ldo};
    st = launch_expand<F32, true>(ea, p.expand_tt, p.tiles(p.expand_tt, cfg->T, sh->n_adapters + 1), s);
    if (st != SEMMOE_OK) return st;
  }
  if (dA) {
    OuterArgs oa{ad, V, p.parts_out, X, ldx, sh->d_in, p.seg, int(items), partial, dA};
    st = launch_outer<F32, false>(oa, items, s);
    if (st != SEMMOE_OK) return st;
  }
  if (dB) {
    ShrinkArgs sa{ad, X, ldx, A, scale, sh->d_in, p.part_k_in, p.parts_in, U};
    st = launch_shrink<F32, false>(sa, p.shrink_tt, tiles, s);  // nothing to launch where T is 0
    if (st != SEMMOE_OK) return st;
    OuterArgs oa{ad, U, p.parts_in, dY, ldy, sh->d_out, p.seg, int(items), partial, dB};
    st = launch_outer<F32, true>(oa, items, s);
    if (st != SEMMOE_OK) return st;
  }
  return SEMMOE_OK;
}

}  // namespace semmoe

using namespace semmoe;

extern "C" int32_t semmoe_adapter_index(const semmoe_config* cfg, void* stream, const int32_t* req_offsets, int32_t n_req,
                                        const int32_t* adapter_of_req, int32_t n_adapters, int32_t* order,
                                        int32_t* adapter_offsets) {
  const int32_t st = validate_config(cfg, true, false, false);
  if (st != SEMMOE_OK) return st;
  if (n_req < 0 || n_adapters <= 0 || !order || !adapter_offsets || (n_req > 0 && (!req_offsets || !adapter_of_req)))
    return SEMMOE_EINVAL;
  if (n_adapters > SEMMOE_MAX_ADAPTERS || n_req > SEMMOE_MAX_REQUESTS) return SEMMOE_EUNSUPPORTED;
  IndexArgs a{req_offsets, adapter_of_req, n_req, n_adapters, cfg->T, 0, order, adapter_offsets};
  // about four requests a workgroup, one for each wave
  const long long tokens = n_req > 0 ? 4ll * cfg->T / n_req : 256;
  a.per_block = int(tokens < 4 ? 4 : (tokens > 256 ? 256 : tokens));
  const int token_blocks = cdiv(cfg->T, a.per_block);
  hipLaunchKernelGGL(adapter_index_kernel, dim3(token_blocks + cdiv(n_adapters + 1, 4)), dim3(256), 0,
                     static_cast<hipStream_t>(stream), a, token_blocks);
  SEMMOE_LAUNCH_CHECK();
  return SEMMOE_OK;
}

extern "C" int32_t semmoe_adapter_workspace_bytes(const semmoe_config* cfg, const semmoe_adapter_shape* shape,
                                                  size_t* bytes_out) {
  if (!bytes_out) return SEMMOE_EINVAL;
  const int32_t st = check_shape(cfg, shape);
  if (st != SEMMOE_OK) return st;
  const AdapterPlan p = plan_of(cfg, shape);
  const size_t widest = size_t(shape->d_in > shape->d_out ? shape->d_in : shape->d_out);
  *bytes_out = align_up(u_floats(cfg, shape, p.parts_in) * 4, 256) + align_up(u_floats(cfg, shape, p.parts_out) * 4, 256) +
               (cfg->T > p.seg ? align_up(partial_items(cfg, shape, p) * shape->rank * widest * 4, 256) : 0) + 256;
  return SEMMOE_OK;
}

extern "C" int32_t semmoe_adapters(const semmoe_config* cfg, void* stream, const semmoe_adapter_shape* shape, const void* X,
                                   const int32_t* order, const int32_t* adapter_offsets, const void* A, const void* B,
                                   const float* scale, const void* Y_base, void* Y, void* ws, size_t ws_bytes) {
  const int32_t st = check_shape(cfg, shape);
  if (st != SEMMOE_OK) return st;
  if (!X || !order || !adapter_offsets || !A || !B || !Y) return SEMMOE_EINVAL;
  if (!aligned16(X) || !aligned16(A) || !aligned16(B) || !aligned16(Y_base) || !aligned16(Y)) return SEMMOE_EINVAL;
  size_t ldx, ld_base, ldo;
  if (!take_ld(shape->ldx, shape->d_in, &ldx) || !take_ld(shape->ld_base, shape->d_out, &ld_base) ||
      !take_ld(shape->ld_out, shape->d_out, &ldo))
    return SEMMOE_ESHAPE;
  if (Y_base == Y && ld_base != ldo) return SEMMOE_ESHAPE;
  const AdapterPlan p = plan_of(cfg, shape);
  Carver c(ws, ws_bytes);
  float* U = c.take<float>(u_floats(cfg, shape, p.parts_in));
  if (!c.ok) return SEMMOE_EWORKSPACE;
  if (cfg->T == 0) return SEMMOE_OK;
  const AdapterArgs ad{order, adapter_offsets, cfg->T, shape->n_adapters, shape->rank};
  auto* const run = cfg->dtype == SEMMOE_BF16 ? run_adapters<false> : run_adapters<true>;
  return run(cfg, shape, p, static_cast<hipStream_t>(stream), X, ad, A, B, scale, Y_base, Y, U, ldx, ld_base, ldo);
}

extern "C" int32_t semmoe_adapters_grad(const semmoe_config* cfg, void* stream, const semmoe_adapter_shape* shape,
                                        const void* X, const void* dY, const int32_t* order, const int32_t* adapter_offsets,
                                        const void* A, const void* B, const float* scale, const void* dX_base, void* dX,
                                        void* dA, void* dB, void* ws, size_t ws_bytes) {
  const int32_t st = check_shape(cfg, shape);
  if (st != SEMMOE_OK) return st;
  if (!X || !dY || !order || !adapter_offsets || !A || !B || (!dX && !dA && !dB)) return SEMMOE_EINVAL;
  if (!aligned16(X) || !aligned16(dY) || !aligned16(A) || !aligned16(B) || !aligned16(dX_base) || !aligned16(dX) ||
      !aligned16(dA) || !aligned16(dB))
    return SEMMOE_EINVAL;
  size_t ldx, ldy, ld_base, ldo;
  if (!take_ld(shape->ldx, shape->d_in, &ldx) || !take_ld(shape->ldy, shape->d_out, &ldy) ||
      !take_ld(shape->ld_base, shape->d_in, &ld_base) || !take_ld(shape->ld_out, shape->d_in, &ldo))
    return SEMMOE_ESHAPE;
  if (dX && dX_base == dX && ld_base != ldo) return SEMMOE_ESHAPE;
  const AdapterPlan p = plan_of(cfg, shape);
  const size_t widest = size_t(shape->d_in > shape->d_out ? shape->d_in : shape->d_out);
  Carver c(ws, ws_bytes);
  float* U = c.take<float>(u_floats(cfg, shape, p.parts_in));
  float* V = c.take<float>(u_floats(cfg, shape, p.parts_out));
  float* partial = c.take<float>(cfg->T > p.seg ? partial_items(cfg, shape, p) * shape->rank * widest : 0);
  if (!c.ok) return SEMMOE_EWORKSPACE;
  const AdapterArgs ad{order, adapter_offsets, cfg->T, shape->n_adapters, shape->rank};
  auto* const run = cfg->dtype == SEMMOE_BF16 ? run_adapters_grad<false> : run_adapters_grad<true>;
  return run(cfg, shape, p, static_cast<hipStream_t>(stream), X, dY, ad, A, B, scale, dX_base, dX, dA, dB, U, V, partial, ldx,
             ldy, ld_base, ldo);
}
