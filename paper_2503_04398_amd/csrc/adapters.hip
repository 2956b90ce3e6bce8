// Low-rank adapters of many requests at once beside a projection that all of them share: the index that orders a batch's
// tokens by adapter, the forward form Y = Y_base + s_a B_a (A_a x), and its gradient.
//
// With u = s_a A_a x (rank numbers a token) and v = s_a B_a^T dY:
//   Y  = Y_base + B_a u          dX = dX_base + A_a^T v
//   dA_a = sum over a's tokens of v x^T        dB_a = sum of dY u^T
// so everything is made of three kernels over the ordered tokens: `shrink` (rows times a factor, down to rank numbers),
// `expand` (rank numbers times a factor, added to rows) and `outer` (sums over tokens).  u and v are fp32 sums in the
// workspace.  As operands of the matrix instructions of bf16 rows they are taken in two parts, the upper half and what that leaves,
// 16 bits between them: half a step of the result's type is then the whole error, where one rounding of u would add as much again
// (8192 tokens x 4096, rank 16, against 64 bits: 1.66e-3, and 2.35e-3 with u and v in bf16).
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

// operands made of fp32 numbers: the numbers themselves, or parts of them
template <bool F32>
constexpr int kParts = F32 ? 1 : 2;

// The upper halves of a and b in hi, and what these leave, as bf16, in lo.  Cut off and not rounded, so that what is left has the
// number's sign: beside an infinity in the other operand both products are infinite the same way.  For that, too, nothing left
// becomes 2^-60 of the number, and an infinity leaves an infinity; NaN leaves NaN.  2^-16 of a number is lost at most.
__device__ __forceinline__ float left_of(float a) {
  const float r = a - __uint_as_float(__float_as_uint(a) & 0xffff0000u);
  return fabsf(a) == __builtin_huge_valf() ? a : (r == 0.0f ? a * 0x1p-60f : r);
}
__device__ __forceinline__ void two_parts(float a, float b, uint32_t* hi, uint32_t* lo) {
  *hi = __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
  *lo = cvt_pk_bf16(left_of(a), left_of(b));
}

__device__ __forceinline__ u32x4_t load_piece(const void* p) { return *reinterpret_cast<const u32x4_t*>(p); }

// the compiler keeps LDS accesses on both sides in place; a wave's own LDS operations complete in order
__device__ __forceinline__ void lds_fence() { asm volatile("" ::: "memory"); }

typedef __attribute__((ext_vector_type(4))) short i16x4_t;
typedef __attribute__((address_space(3))) i16x4_t lds_i16x4;

__device__ __forceinline__ unsigned lds_address(const void* p) { return static_cast<unsigned>(reinterpret_cast<size_t>(p)); }

// Fragment across the rows of a matrix in LDS: lane gets the kPer16 numbers of one column in rows row0 + kPer16 * (lane / 16) + 0, 1, ...
// at(row, col): address of a number.  bf16: two ds_read_b64_tr_b16, where lane i of 16 points at four consecutive columns
// 4 (i % 4) of row i / 4 and gets four rows of column i; fp32: a number a row.
template <bool F32, typename At>
__device__ __forceinline__ u32x4_t column_piece(int lane, At at) {
  const int l16 = lane & 15, g4 = lane >> 4;
  if constexpr (F32) {
    u32x4_t v;
#pragma unroll
    for (int e = 0; e < 4; ++e) v[e] = *reinterpret_cast<const uint32_t*>(at(g4 * 4 + e, l16));
    return v;
  } else {
    const unsigned a0 = lds_address(at(g4 * 8 + (l16 >> 2), (l16 & 3) * 4));
    const unsigned a1 = lds_address(at(g4 * 8 + 4 + (l16 >> 2), (l16 & 3) * 4));
    const i16x4_t lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_i16x4*>(a0));
    const i16x4_t hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(reinterpret_cast<lds_i16x4*>(a1));
    return __builtin_bit_cast(u32x4_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
  }
}

struct AdapterArgs {
  const int32_t* order;    // [T] ordered tokens, -1: none
  const int32_t* offsets;  // [n_adapters + 1]
  int T, n_adapters, rank;
};

// Group g: the ordered tokens [lo, hi) of adapter g; group n_adapters: tokens of requests without an adapter, and -1 behind them.
// A group has max(least, ceil(tokens / per)) items.  Every wave finds an item by itself, 64 groups at a time: one load and a
// scan across the lanes, no LDS and no barrier in front of a kernel of a few microseconds.  Offsets are clamped, so that no
// position lies outside the order whatever they hold.
struct Item {
  int g, lo, hi, first, count;  // group, its positions, its first item and their number
};
__device__ __forceinline__ bool find_item(const AdapterArgs& a, int n_groups, int per, int least, int item, Item* it) {
  const int lane = threadIdx.x & 63;
  int before = 0;
  for (int g0 = 0; g0 < n_groups; g0 += 64) {
    const int g = min(g0 + lane, n_groups - 1);
    const int lo = min(max(a.offsets[g], 0), a.T);
    const int end = g < a.n_adapters ? min(max(a.offsets[min(g + 1, a.n_adapters)], lo), a.T) : a.T;
    const int c = g0 + lane < n_groups ? max(least, (end - lo + per - 1) / per) : 0;
    int incl = c;
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) {
      const int v = __shfl_up(incl, off);
      if (lane >= off) incl += v;
    }
    const int total = __builtin_amdgcn_readlane(incl, 63);
    if (item < before + total) {
      const int l = __builtin_amdgcn_readfirstlane(__ffsll((unsigned long long)__ballot(before + incl > item)) - 1);
      it->g = g0 + l;
      it->lo = __builtin_amdgcn_readlane(lo, l);
      it->hi = __builtin_amdgcn_readlane(end, l);
      it->count = __builtin_amdgcn_readlane(c, l);
      it->first = before + __builtin_amdgcn_readlane(incl, l) - it->count;
      return true;
    }
    before += total;
  }
  return false;
}

// ---- shrink: U[part][position][j] = s_a * sum over the part's k of R[token, k] F_a(j, k) ------------------------------
// TR = false: F_a = A_a [rank][K], rows along k.  TR = true: F_a = B_a [K][rank].
//
// A read stream with matrix instructions attached.  A workgroup's four waves share a tile of 16 TT tokens and cut the part's k
// between them, 128 bytes of every row at a time, so that no wave waits for another inside the tile.  A load covers 8 rows x 128
// bytes (four neighbouring lanes in one 64-byte segment; fragments loaded as they are put them into four rows), one step ahead
// into registers, and goes through LDS of the wave's own to become fragments.  A slice of B is one run of memory and is read
// across (column_piece).  Few tiles: k in parts over workgroups, whose planes `expand` and `outer` add.
// Measured, bf16: 16384 tokens x 7168, rank 64 (235 MB) 49 to 53 us, 4.4 to 4.8 TB/s, the rate of a large copy; both shrinks of
// 8192 tokens x 4096, rank 16 (134 MB, in the memory-side cache) 22 us, 6.0 TB/s; 256 tokens x 4096 of 64 adapters (10.5 MB) 4.5 us.  A
// second step ahead changes none of them.
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
__device__ __forceinline__ void shrink_body(const ShrinkArgs& a, int block, unsigned char* lds_raw) {
  using E = Elem<F32>;
  using elem = typename E::type;
  constexpr int BT = 16 * TT, KSL = 128 / E::kSize;  // tokens of a tile; numbers in 128 bytes of a row
  const int r = a.ad.rank;
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  Item it;
  const int item = block / a.parts, part = block - item * a.parts;
  if (!find_item(a.ad, a.ad.n_adapters, BT, 0, item, &it)) return;  // the whole workgroup
  const int p0 = it.lo + (item - it.first) * BT, n_tok = min(BT, it.hi - p0);

  // load layout: row lane / 8 of 8, 16 bytes at lane % 8 of 128
  const int l_row = lane >> 3, l_k = (lane & 7) * E::kPer16;
  const elem* x_row[2 * TT];
#pragma unroll
  for (int i = 0; i < 2 * TT; ++i) {
    const int tok = a.ad.order[p0 + min(i * 8 + l_row, n_tok - 1)];
    x_row[i] = static_cast<const elem*>(a.R) + size_t(min(max(tok, 0), a.ad.T - 1)) * a.ldr;
  }
  const elem* F = static_cast<const elem*>(a.F) + size_t(it.g) * r * a.K;
  const int k_hi = min(a.K, part * a.part_k + a.part_k);

  f32x4_t acc[RT][TT];
#pragma unroll
  for (int j = 0; j < RT; ++j)
#pragma unroll
    for (int t = 0; t < TT; ++t) acc[j][t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  u32x4_t xb[2 * TT], fb[2 * RT];
  const u32x4_t zero = {0, 0, 0, 0};
  auto fetch = [&](int k0) __attribute__((always_inline)) {
    const bool in = k0 + l_k < k_hi;
#pragma unroll
    for (int i = 0; i < 2 * RT; ++i) {  // the factor first: the first step's rows wait for the order
      if constexpr (TR) {
        const int at = (i * 64 + lane) * E::kPer16;
        fb[i] = at < min(KSL, k_hi - k0) * r ? load_piece(F + size_t(k0) * r + at) : zero;
      } else {
        fb[i] = in ? load_piece(F + size_t(min(i * 8 + l_row, r - 1)) * a.K + k0 + l_k) : zero;
      }
    }
#pragma unroll
    for (int i = 0; i < 2 * TT; ++i) xb[i] = in ? load_piece(x_row[i] + k0 + l_k) : zero;
  };

  unsigned char* const stg = lds_raw + wave * (TT + RT) * 2048;
  unsigned char* const f_stg = stg + TT * 2048;
  // rows of 128 bytes; piece c of row i lies at c ^ (i / 2 % 8)
  const int put0 = l_row * 128 + (((lane & 7) ^ ((l_row >> 1) & 7)) * 16);
  const int put1 = (l_row + 8) * 128 + (((lane & 7) ^ ((l_row >> 1) + 4)) * 16);
  int k0 = part * a.part_k + wave * KSL;
  if (k0 < k_hi) fetch(k0);
  while (k0 < k_hi) {
#pragma unroll
    for (int i = 0; i < 2 * TT; ++i) *reinterpret_cast<u32x4_t*>(stg + (i >> 1) * 2048 + (i & 1 ? put1 : put0)) = xb[i];
#pragma unroll
    for (int i = 0; i < 2 * RT; ++i)
      *reinterpret_cast<u32x4_t*>(f_stg + (TR ? i * 1024 + lane * 16 : (i >> 1) * 2048 + (i & 1 ? put1 : put0))) = fb[i];
    lds_fence();
    k0 += 4 * KSL;
    if (k0 < k_hi) fetch(k0);
    lds_fence();
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      const int at = l16 * 128 + (((h * 4 + g4) ^ ((l16 >> 1) & 7)) * 16);
      u32x4_t x[TT];
#pragma unroll
      for (int t = 0; t < TT; ++t) x[t] = *reinterpret_cast<const u32x4_t*>(stg + t * 2048 + at);
#pragma unroll
      for (int j = 0; j < RT; ++j) {
        u32x4_t f;
        if constexpr (TR)  // rank numbers from r on are of the next row, and in results that nobody stores
          f = column_piece<F32>(lane, [&](int row, int col) { return f_stg + size_t((h * E::kStep + row) * r + (F32 ? min(j * 16 + col, r - 1) : j * 16 + col)) * E::kSize; });
        else
          f = *reinterpret_cast<const u32x4_t*>(f_stg + j * 2048 + at);
#pragma unroll
        for (int t = 0; t < TT; ++t) acc[j][t] = piece_mfma<F32>(f, x[t], acc[j][t]);
      }
    }
    lds_fence();
  }

  // the four waves' sums meet in the staging areas' place
  f32x4_t* red = reinterpret_cast<f32x4_t*>(lds_raw);  // [wave][RT * TT][64]
  __syncthreads();
#pragma unroll
  for (int j = 0; j < RT; ++j)
#pragma unroll
    for (int t = 0; t < TT; ++t) red[((wave * RT + j) * TT + t) * 64 + lane] = acc[j][t];
  __syncthreads();
  const float s = a.scale ? a.scale[it.g] : 1.0f;
  float* U = a.U + size_t(part) * a.ad.T * r;
  for (int u = wave; u < RT * TT; u += 4) {
    f32x4_t v = red[u * 64 + lane];
#pragma unroll
    for (int w = 1; w < 4; ++w) v += red[(w * RT * TT + u) * 64 + lane];
    const int tok = (u % TT) * 16 + l16, j = (u / TT) * 16 + g4 * 4;
    if (tok < n_tok && j < r) *reinterpret_cast<f32x4_t*>(U + size_t(p0 + tok) * r + j) = v * s;
  }
}

template <bool F32, int RT, int TT>
__global__ __launch_bounds__(256) void shrink_kernel(const ShrinkArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
  shrink_body<F32, RT, TT, false>(a, blockIdx.x, lds_raw);
}

// v of dY and B, and u of X and A, side by side: each alone leaves part of the chip idle
template <bool F32, int RT, int TT>
__global__ __launch_bounds__(256) void shrink_both_kernel(const ShrinkArgs v, int v_blocks, const ShrinkArgs u) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
  if (int(blockIdx.x) < v_blocks) shrink_body<F32, RT, TT, true>(v, blockIdx.x, lds_raw);
  else shrink_body<F32, RT, TT, false>(u, blockIdx.x - v_blocks, lds_raw);
}

// ---- expand: Out[token, n] = Base[token, n] + sum over j of F_a(n, j) U[position][j] -----------------------------------
// TR = false: F_a = B_a [N][rank].  TR = true: F_a = A_a [rank][N].  Group n_adapters: Out = Base.
//
// Streams rows of Base in and rows of Out out.  A wave keeps the fragments of u for its 16 TT tokens and walks over 32 columns at a
// time (its workgroup over 128), the next columns' Base and factor requested before the present ones are multiplied.  Loads and
// stores are as memory lies: four neighbouring lanes a 64-byte segment of a row, the factor as runs; its fragments and the products
// change places in LDS of the wave's own, no barrier.  (Fragments loaded and products stored as the matrix instruction has them, a
// segment's pieces 16 lanes apart, kept the address units busy for 74 % of 134 us: 16384 tokens, 7168 columns, rank 64.)
// Out is stored past the caches (8192 tokens x 4096, rank 16, with both products before it: 81 us, 85 otherwise); Base read past
// them costs 94.  Measured, bf16: 16384 tokens x 7168, rank 64 (474 MB) 132 to 142 us, 3.4 to 3.6 TB/s: 64-token tiles wait for Base with
// the few waves they leave room for, and 32-token ones read the factors twice as often (with shrink 228 us, 199 then).  8192 x 4096,
// rank 16: 30 to 31 us, 4.4 TB/s (29 with u as one bf16).
struct ExpandArgs {
  AdapterArgs ad;
  const float* U;
  int parts;
  const void* F;
  int N, chunks;     // 128-column steps of a workgroup
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
  constexpr int BT = 16 * TT;
  constexpr int KS = (16 * RT + E::kStep - 1) / E::kStep;
  constexpr int LPR = 2 * E::kSize, NP = 16 * LPR / 64;  // lanes of a token's 32 columns, 16 bytes each; pieces a lane has of 16 tokens
  constexpr int RB = 32 * E::kSize;                      // TR: bytes of a factor's row in LDS
  constexpr int NF = RT * E::kSize / 2;                  // loads of a step's factor, 32 * 16 RT numbers
  constexpr int kDelta = 16 * 144;                       // 16 tokens x 32 products, rows padded against bank conflicts
  extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
  const int n_ad = a.ad.n_adapters, r = a.ad.rank;
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int cuts = (a.N + a.chunks * kExpandCols - 1) / (a.chunks * kExpandCols);
  const int item = blockIdx.x / cuts, cut = blockIdx.x - item * cuts;
  Item it;
  if (!find_item(a.ad, n_ad + 1, BT, 0, item, &it)) return;
  const int p0 = it.lo + (item - it.first) * BT, n_tok = min(BT, it.hi - p0);
  const bool none = it.g == n_ad;
  if (none && a.Base == a.Out) return;  // the same rows
  const int c_hi = min(a.N, (cut + 1) * a.chunks * kExpandCols);
  int c0 = cut * a.chunks * kExpandCols + wave * 32;
  if (c0 >= c_hi) return;  // no barrier below

  // what does not wait for the tokens' numbers is requested while they are on their way
  int tok[TT][NP];
#pragma unroll
  for (int t = 0; t < TT; ++t)
#pragma unroll
    for (int q = 0; q < NP; ++q) {
      const int at = t * 16 + q * (64 / LPR) + lane / LPR;
      tok[t][q] = at < n_tok ? a.ad.order[p0 + at] : -1;
    }
  const u32x4_t zero = {0, 0, 0, 0};
  const elem* F = static_cast<const elem*>(a.F) + size_t(none ? 0 : it.g) * r * a.N;
  unsigned char* const delta = lds_raw + wave * kDelta;
  unsigned char* const stg = lds_raw + 4 * kDelta + wave * (TR ? KS * E::kStep * RB : 32 * (16 * RT + E::kPer16) * E::kSize);
  // where the lane's pieces of the factor come from and go to.  TR: rows of 32 columns.  Else the 32 columns' runs of r numbers are
  // one run; in LDS a piece's width apart, so that 16 of them start in different banks.
  int f_row[NF], f_col[NF], f_put[NF];
#pragma unroll
  for (int i = 0; i < NF; ++i) {
    const int n = i * 64 + lane, per_row = TR ? LPR : r / E::kPer16;
    f_row[i] = n / per_row;
    f_col[i] = (n - f_row[i] * per_row) * E::kPer16;
    f_put[i] = TR ? n * 16 : (f_row[i] * (r + E::kPer16) + f_col[i]) * E::kSize;
  }
  u32x4_t fb[NF], bs[TT][NP];
  auto fetch_factor = [&](int c) __attribute__((always_inline)) {
    if (none) return;
#pragma unroll
    for (int i = 0; i < NF; ++i) {
      if constexpr (TR) fb[i] = f_row[i] < r && c + f_col[i] < c_hi ? load_piece(F + size_t(f_row[i]) * a.N + c + f_col[i]) : zero;
      else fb[i] = f_row[i] < 32 && c + f_row[i] < c_hi ? load_piece(F + size_t(c + f_row[i]) * r + f_col[i]) : zero;
    }
  };
  fetch_factor(c0);
  if constexpr (TR) {  // rows that no load fills
    for (int i = NF * 64 + lane; i < KS * E::kStep * LPR; i += 64) *reinterpret_cast<u32x4_t*>(stg + i * 16) = zero;
  }
  u32x4_t u[kParts<F32>][KS][TT];
  {
    // all numbers of a part, up to 16 loads, on their way together; the parts in order
    constexpr int NV = KS * TT * (E::kPer16 / 4);
    f32x4_t f[NV];
#pragma unroll
    for (int i = 0; i < NV; ++i) f[i] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    auto at = [&](int i) {  // number of the i-th four, or none
      const int ks = i / (TT * (E::kPer16 / 4)), t = i / (E::kPer16 / 4) % TT, k = ks * E::kStep + g4 * E::kPer16 + i % (E::kPer16 / 4) * 4;
      return !none && k < r && t * 16 + l16 < n_tok ? (p0 + t * 16 + l16) * (long long)r + k : -1ll;
    };
    const size_t plane = size_t(a.ad.T) * r;
    constexpr int UP = NV >= 16 ? 1 : (NV >= 8 ? 2 : 4);  // parts at a time
    for (int p = 0; p < a.parts; p += UP) {
      f32x4_t v[UP][NV];
#pragma unroll
      for (int x = 0; x < UP; ++x)
#pragma unroll
        for (int i = 0; i < NV; ++i)
          v[x][i] = at(i) >= 0 ? *reinterpret_cast<const f32x4_t*>(a.U + plane * min(p + x, a.parts - 1) + at(i)) : f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
      for (int x = 0; x < UP; ++x)
#pragma unroll
        for (int i = 0; i < NV; ++i)
          if (p + x < a.parts) f[i] += v[x][i];
    }
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int t = 0; t < TT; ++t)
#pragma unroll
        for (int x = 0; x < 4; ++x) {
          if constexpr (F32) {
            u[0][ks][t][x] = __float_as_uint(f[ks * TT + t][x]);
          } else {
            const f32x4_t& four = f[(ks * TT + t) * 2 + (x >> 1)];
            uint32_t hi, lo;
            two_parts(four[(x & 1) * 2], four[(x & 1) * 2 + 1], &hi, &lo);
            u[0][ks][t][x] = hi;
            u[1][ks][t][x] = lo;
          }
        }
  }
  const int l_col = (lane % LPR) * E::kPer16;  // this lane's piece of a row's 32 columns
  const elem* base_row[TT][NP];
  elem* out_row[TT][NP];
  bool there[TT][NP];
#pragma unroll
  for (int t = 0; t < TT; ++t)
#pragma unroll
    for (int q = 0; q < NP; ++q) {
      there[t][q] = unsigned(tok[t][q]) < unsigned(a.ad.T);
      const size_t row = there[t][q] ? tok[t][q] : 0;
      base_row[t][q] = static_cast<const elem*>(a.Base) + row * a.ld_base + l_col;
      out_row[t][q] = static_cast<elem*>(a.Out) + row * a.ldo + l_col;
    }
  auto fetch_base = [&](int c) __attribute__((always_inline)) {
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int q = 0; q < NP; ++q) bs[t][q] = a.Base && there[t][q] && c + l_col < c_hi ? load_piece(base_row[t][q] + c) : zero;
  };
  fetch_base(c0);
  for (; c0 < c_hi; c0 += kExpandCols) {
    u32x4_t now[TT][NP];
#pragma unroll
    for (int t = 0; t < TT; ++t)
#pragma unroll
      for (int q = 0; q < NP; ++q) now[t][q] = bs[t][q];
    lds_fence();
    if (!none) {
#pragma unroll
      for (int i = 0; i < NF; ++i)
        if (TR || f_row[i] < 32) *reinterpret_cast<u32x4_t*>(stg + f_put[i]) = fb[i];
    }
    lds_fence();
    if (c0 + kExpandCols < c_hi) {
      fetch_factor(c0 + kExpandCols);
      fetch_base(c0 + kExpandCols);
    }
    f32x4_t acc[2][TT];
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
      for (int t = 0; t < TT; ++t) acc[i][t] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    if (!none) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          u32x4_t f;
          if constexpr (TR) {
            f = column_piece<F32>(lane, [&](int row, int col) { return stg + (ks * E::kStep + row) * RB + (i * 16 + col) * E::kSize; });
          } else {
            const int k = ks * E::kStep + g4 * E::kPer16;
            f = k < r ? *reinterpret_cast<const u32x4_t*>(stg + ((i * 16 + l16) * (r + E::kPer16) + k) * E::kSize) : zero;
          }
#pragma unroll
          for (int h = 0; h < kParts<F32>; ++h)
#pragma unroll
            for (int t = 0; t < TT; ++t) acc[i][t] = piece_mfma<F32>(f, u[h][ks][t], acc[i][t]);
        }
    }
#pragma unroll
    for (int t = 0; t < TT; ++t) {
      lds_fence();
#pragma unroll
      for (int i = 0; i < 2; ++i) *reinterpret_cast<f32x4_t*>(delta + l16 * 144 + (i * 16 + g4 * 4) * 4) = acc[i][t];
      lds_fence();
#pragma unroll
      for (int q = 0; q < NP; ++q) {
        const float* d = reinterpret_cast<const float*>(delta + (q * (64 / LPR) + lane / LPR) * 144) + l_col;
        u32x4_t v = now[t][q];
        const f32x4_t lo = *reinterpret_cast<const f32x4_t*>(d);
        if (!none) {  // else Base as it is, bit for bit
          if constexpr (F32) {
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = __float_as_uint(__uint_as_float(v[e]) + lo[e]);
          } else {
            const f32x4_t hi = *reinterpret_cast<const f32x4_t*>(d + 4);
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const f32x4_t& two = e < 2 ? lo : hi;
              v[e] = cvt_pk_bf16(__uint_as_float(v[e] << 16) + two[(e & 1) * 2], __uint_as_float(v[e] & 0xffff0000u) + two[(e & 1) * 2 + 1]);
            }
          }
        }
        if (there[t][q] && c0 + l_col < c_hi) __builtin_nontemporal_store(v, reinterpret_cast<u32x4_t*>(out_row[t][q] + c0));
      }
    }
  }
}

// ---- outer: dF_a = sum over a's tokens of U[position][j] R[token][c] ---------------------------------------------------
// SWAP = false: dF_a [rank][C] (c along a row).  SWAP = true: dF_a [C][rank].  An adapter's tokens are cut into segments;
// one with several of them leaves fp32 sums, which `outer_join` adds in the order of the segments.
// A segment that begins at position p has the place 2 (p / seg), or 2 (p / seg) + 1 if it isn't its adapter's first.  Adapters of
// several segments are longer than one, so of all positions with the same p / seg at most one begins such an adapter and at
// most one goes on with one: no place is taken twice, and there are two for every `seg` tokens, however many adapters there are.
//
// Both operands run along the tokens, so a slice of 64 rows x 256 bytes and the numbers of its tokens go to LDS and are read
// across; the next slice's rows are on their way meanwhile.  Every row is read once, the numbers once for each 256 bytes of it.
// Measured, bf16, dA and dB of 8192 tokens x 4096 x 4096, rank 16, 8 adapters: 134 MB in 26 us, 5.1 TB/s, and 5 us to join.  The numbers'
// second parts cost 1 us of it; at rank 128, where their LDS reads count as much as the rows', they take the whole gradient of 16384
// tokens of 4 adapters from 404 to 465 us.
struct OuterArgs {
  AdapterArgs ad;
  const float* U;
  int parts;
  const void* R;
  size_t ldr;
  int C, seg;      // columns; tokens of a segment
  float* partial;  // [partial_places][rank * C]
  void* dF;        // act [n_adapters][rank * C]
};

__device__ __forceinline__ int partial_place(int lo, int i, int seg) { return (lo / seg + i) * 2 + (i > 0); }  // i-th segment

constexpr int kOuterTok = 64;
template <bool F32>
constexpr int kOuterCols = 256 / Elem<F32>::kSize;

template <bool F32, int RT, bool SWAP>
__device__ __forceinline__ void outer_body(const OuterArgs& a, int block, unsigned char* lds_raw) {
  using E = Elem<F32>;
  using elem = typename E::type;
  constexpr int NC = kOuterCols<F32>, KT = kOuterTok, CT = NC / 64;  // 16-column tiles of a wave
  constexpr int RBU = 16 * RT * E::kSize + 16;                       // bytes of a token's numbers in LDS
  constexpr int NU = KT * RT * 4 / 256;                              // their loads a thread
  unsigned char* const Rs = lds_raw;               // [KT][256 bytes], 32-byte pairs of pieces swapped about by the row
  unsigned char* const Us = lds_raw + KT * 256;    // [parts][KT][RBU]
  const int r = a.ad.rank;
  const int tid = threadIdx.x, lane = tid & 63, l16 = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n_chunks = (a.C + NC - 1) / NC;
  const int item = block / n_chunks, c0 = (block - item * n_chunks) * NC;
  Item it;
  if (!find_item(a.ad, a.ad.n_adapters, a.seg, 1, item, &it)) return;
  const int p0 = it.lo + (item - it.first) * a.seg, p1 = min(it.hi, p0 + a.seg);

  // the four rows that 16 lanes read across lie 64 bytes apart modulo the banks' 256, rows 8 apart in the other half
  auto r_at = [&](int row, int col_byte) { return Rs + row * 256 + (col_byte ^ (((row & 3) ^ ((row >> 3) & 1) * 4) << 5)); };
  const int l_row = tid >> 4, l_col = (tid & 15) * E::kPer16;
  const u32x4_t zero = {0, 0, 0, 0};
  u32x4_t xb[4];
  constexpr int UP = RT <= 2 ? 4 : (RT == 4 ? 2 : 1);  // planes of the numbers that are under way with the rows
  f32x4_t ub[NU][UP];
  int tok[4];
  auto tokens = [&](int p) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i) tok[i] = p + i * 16 + l_row < p1 ? a.ad.order[p + i * 16 + l_row] : -1;
  };
  auto fetch = [&](int p) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < 4; ++i)
      xb[i] = unsigned(tok[i]) < unsigned(a.ad.T) && c0 + l_col < a.C
                  ? load_piece(static_cast<const elem*>(a.R) + size_t(tok[i]) * a.ldr + c0 + l_col) : zero;
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int t = (i * 256 + tid) / (RT * 4), j = (i * 256 + tid) % (RT * 4) * 4;
#pragma unroll
      for (int x = 0; x < UP; ++x)
        ub[i][x] = p + t < p1 && j < r && x < a.parts
                       ? *reinterpret_cast<const f32x4_t*>(a.U + (size_t(x) * a.ad.T + p + t) * r + j) : f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
    }
  };

  f32x4_t acc[CT][RT];
#pragma unroll
  for (int c = 0; c < CT; ++c)
#pragma unroll
    for (int j = 0; j < RT; ++j) acc[c][j] = f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
  tokens(p0);
  fetch(p0);
  tokens(p0 + KT);
  for (int p = p0; p < p1; p += KT) {
    __syncthreads();  // the slice before has been read
#pragma unroll
    for (int i = 0; i < 4; ++i) *reinterpret_cast<u32x4_t*>(r_at(i * 16 + l_row, (tid & 15) * 16)) = xb[i];
#pragma unroll
    for (int i = 0; i < NU; ++i) {
#pragma unroll
      for (int x = 1; x < UP; ++x) ub[i][0] += ub[i][x];
    }
    // the planes behind them, all numbers of two at a time
    for (int x0 = UP; x0 < a.parts; x0 += 2) {
      f32x4_t more[2][NU];
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int i = 0; i < NU; ++i) {
          const int t = (i * 256 + tid) / (RT * 4), j = (i * 256 + tid) % (RT * 4) * 4;
          more[x][i] = p + t < p1 && j < r && x0 + x < a.parts
                           ? *reinterpret_cast<const f32x4_t*>(a.U + (size_t(x0 + x) * a.ad.T + p + t) * r + j) : f32x4_t{0.0f, 0.0f, 0.0f, 0.0f};
        }
#pragma unroll
      for (int x = 0; x < 2; ++x)
#pragma unroll
        for (int i = 0; i < NU; ++i) ub[i][0] += more[x][i];
    }
#pragma unroll
    for (int i = 0; i < NU; ++i) {
      const int t = (i * 256 + tid) / (RT * 4), j = (i * 256 + tid) % (RT * 4) * 4;
      const f32x4_t v = ub[i][0];
      unsigned char* const o = Us + t * RBU + j * E::kSize;
      if constexpr (F32) *reinterpret_cast<f32x4_t*>(o) = v;
      else {
        uint2 hi, lo;
        two_parts(v[0], v[1], &hi.x, &lo.x);
        two_parts(v[2], v[3], &hi.y, &lo.y);
        *reinterpret_cast<uint2*>(o) = hi;
        *reinterpret_cast<uint2*>(o + KT * RBU) = lo;
      }
    }
    __syncthreads();
    if (p + KT < p1) {
      fetch(p + KT);
      tokens(p + 2 * KT);
    }
#pragma unroll
    for (int ks = 0; ks < KT / E::kStep; ++ks) {
      u32x4_t x[CT];
#pragma unroll
      for (int c = 0; c < CT; ++c)
        x[c] = column_piece<F32>(lane, [&](int row, int col) { return r_at(ks * E::kStep + row, ((wave * CT + c) * 16 + col) * E::kSize); });
#pragma unroll
      for (int j = 0; j < RT; ++j)
#pragma unroll
        for (int h = 0; h < kParts<F32>; ++h) {
          const u32x4_t u = column_piece<F32>(lane, [&](int row, int col) { return Us + (h * KT + ks * E::kStep + row) * RBU + (j * 16 + col) * E::kSize; });
#pragma unroll
          for (int c = 0; c < CT; ++c) acc[c][j] = SWAP ? piece_mfma<F32>(u, x[c], acc[c][j]) : piece_mfma<F32>(x[c], u, acc[c][j]);
        }
    }
  }

  // SWAP = false: lane holds columns 4 g4 + 0..3 of tile c for rank number l16 of tile j; SWAP = true: rank numbers 4 g4 + 0..3 of
  // tile j for column l16
#pragma unroll
  for (int ct = 0; ct < CT; ++ct)
#pragma unroll
    for (int j = 0; j < RT; ++j) {
      const int c = c0 + (wave * CT + ct) * 16 + (SWAP ? l16 : g4 * 4), jj = j * 16 + (SWAP ? g4 * 4 : l16);
      if (c >= a.C || jj >= r) continue;
      const size_t at = SWAP ? size_t(c) * r + jj : size_t(jj) * a.C + c;
      const f32x4_t v = acc[ct][j];
      if (it.count > 1) {
        *reinterpret_cast<f32x4_t*>(a.partial + size_t(partial_place(it.lo, item - it.first, a.seg)) * r * a.C + at) = v;
        continue;
      }
      elem* o = static_cast<elem*>(a.dF) + size_t(it.g) * r * a.C + at;
      if constexpr (F32) *reinterpret_cast<f32x4_t*>(o) = v;
      else *reinterpret_cast<uint2*>(o) = make_uint2(cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]));
    }
}

// dA of v and X, and dB of u and dY, side by side
template <bool F32, int RT>
__global__ __launch_bounds__(256) void outer_kernel(const OuterArgs da, int da_blocks, const OuterArgs db) {
  extern __shared__ __attribute__((aligned(16))) unsigned char lds_raw[];
  if (int(blockIdx.x) < da_blocks) outer_body<F32, RT, false>(da, blockIdx.x, lds_raw);
  else outer_body<F32, RT, true>(db, blockIdx.x - da_blocks, lds_raw);
}

template <bool F32>
__global__ __launch_bounds__(256) void outer_join_kernel(const OuterArgs da, int da_blocks, const OuterArgs db) {
  using elem = typename Elem<F32>::type;
  const bool first = int(blockIdx.x) < da_blocks;
  const OuterArgs& a = first ? da : db;
  const int own = blockIdx.y;
  const int lo = min(max(a.ad.offsets[own], 0), a.ad.T), hi = min(max(a.ad.offsets[own + 1], lo), a.ad.T);
  const int n = (hi - lo + a.seg - 1) / a.seg;
  const size_t size = size_t(a.ad.rank) * a.C;
  const size_t i = (size_t(first ? blockIdx.x : blockIdx.x - da_blocks) * 256 + threadIdx.x) * 4;
  if (n <= 1 || i >= size) return;
  f32x4_t v = *reinterpret_cast<const f32x4_t*>(a.partial + partial_place(lo, 0, a.seg) * size + i);
  for (int q = 1; q < n; ++q) v += *reinterpret_cast<const f32x4_t*>(a.partial + partial_place(lo, q, a.seg) * size + i);
  elem* o = static_cast<elem*>(a.dF) + own * size + i;
  if constexpr (F32) *reinterpret_cast<f32x4_t*>(o) = v;
  else *reinterpret_cast<uint2*>(o) = make_uint2(cvt_pk_bf16(v[0], v[1]), cvt_pk_bf16(v[2], v[3]));
}

// ---- index ---------------------------------------------------------------------------------------------------------------
// A stable counting sort without counters: a request's place is the sum of the lengths of all requests that come before it
// by (adapter, number), which a wave adds up 64 requests at a time.  One launch, no workspace, no atomics, the same bits
// whatever runs first; n_req^2 / 64 steps over the chip, which beats a pass per digit for the batches of a serving step.
// 4.0 us for 256 requests of a token each, 4.4 for 96 of 32768 tokens: a launch and three loads that wait for one another.  As a graph's
// node 5.4 us for 256 requests of a token, 6.7 for 1024, 18 for 4096, 173 for 16384, 2.4 ms for 65536: past some 4000 requests the square tells.
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
  int shrink_tt, expand_tt;    // 16-token tiles a workgroup takes
  int part_k_in, parts_in;     // shrink over d_in
  int part_k_out, parts_out;   // shrink over d_out
  int chunks_in, chunks_out;   // expand: 128-column steps of a workgroup, rows of d_in and of d_out
  int seg;                     // tokens of a segment of `outer`
  // tiles of the groups, at most: the lengths live on the device
  static long long tiles(int tt, int T, int groups) { return T / (16 * tt) + (groups < T ? groups : T); }
};

// K cut into parts until there are some 400 workgroups, 140 to 280 of ranks past 64, whose steps are longer; at most 4: every part is a
// plane that each reader of u adds, a few at a time.  4096 x 4096, us as captured graphs, with 1 / 2 / 3 / 4 / 6 / 8 parts: forward of 500 tokens of 8
// adapters, rank 64 (39 tiles) 24.4 / 17.8 / 18.0 / 16.3 / 21.0 / 20.9, gradient 35.1 / 29.1 / 28.6 / 27.2 / 30.6 / 31.1; 256 tokens of
// 64, rank 16 forward 12.9 / 10.9 / 10.5 / 10.1 / 10.1 / 10.1; 1000 tokens of 8, 2880 columns, rank 128 (70 tiles), gradient 63.0 / 62.1 /
// 67.5 / 72.7 / 73.1 / 73.5, 2000 tokens (133 tiles), 4096 columns, forward 40.8 / 32.5 / 36.3 / 36.4; but fp32, 79 tokens of one, 568 and 4808 columns, rank 128 (5 tiles) 92 / 58 / 50 / 45 / 44 / 43.
static void cut_k(int K, int es, int rank, long long tiles, int* part_k, int* parts) {
  const int unit = 512 / es;  // a slice for each of the four waves
  const int units = cdiv(K, unit);
  long long want = tiles > 0 ? (rank > 64 ? (140 + tiles - 1) / tiles : 400 / tiles) : 1;
  want = want < 1 ? 1 : (want > 4 ? 4 : want);
  const int per = cdiv(units, int(want < units ? want : units));
  *part_k = per * unit;
  *parts = cdiv(units, per);
}

// Workgroups that share a tile's columns: each reads the tile's u, so no more than fill the chip; 64-token tiles, of which a compute
// unit holds two, twice that (16384 tokens, 7168 columns: 201 us with 1024 workgroups, 177 with 2048).
static int cut_columns(int N, int tt, long long tiles) {
  const int steps = cdiv(N, kExpandCols);
  long long cuts = tiles > 0 ? (tt <= 2 ? 896 : 2048) / tiles : 1;
  if (cuts >= 6) cuts = (cuts + 2) / 8 * 8;
  cuts = cuts < 1 ? 1 : (cuts > steps ? steps : cuts);
  return cdiv(steps, int(cuts));
}

// Tokens of a tile.  A tile reads the whole of its adapter's factor, so many tokens want large tiles; few want many tiles.  us of the
// forward (gradient) with the tokens in shrink / expand, bf16, 4096 x 4096 and 4 adapters where nothing else is said:
//   * shrink 32: ranks up to 32 from 4000 tokens on (rank 16, 3000 tokens 16/32 20.7, 32/32 20.6; 4000 27.1, 24.6; 7168 x 7168: 36.4, 34.4
//     and 55.1, 46.7), up to 64 from 5000 (rank 64, 4000 39.0 (84.6), 42.8 (90.4); 6000 56.9 (109), 51.7 (104)), wider ones from T *
//     rank = 2^19 (rank 128, 3390 tokens, 688 x 800: 28.3 (60.0), 33.6 (68.2); 6000 82.4 (199), 77.7 (186))
//   * shrink 64: ranks 33 to 64 from T * rank = 14000 * 64 (rank 64, 12000 tokens 32/64 91.3 (174), 64/64 95.4 (187); 16000 110 (219),
//     106 (203); 16 adapters 118 (264), 114 (239))
//   * expand 32 from 2048 tokens on (rank 16, 2000 15.6, 17.4, 3000 20.2, 20.7; rank 64, 2000 24.0, 25.8, 3000 30.3, 28.0)
//   * expand 64 from 8192 tokens on (rank 16, 6000 32/32 39.9, 32/64 38.6, 12000 85.6, 73.1; rank 64, 8000 51.6, 59.2, 16 adapters 72.1, 74.1,
//     12000 102, 91.3), not for bf16 ranks past 64, whose u in two parts takes the registers (rank 128, 16000 tokens 32/32 151
//     (383), 32/64 187 (417), 16384 the same 226 (475) with both; rank 96, 15654 tokens of 24, 624 x 576: 31 (100), 60 (125))
static bool shrink_has_64(int rank) { return rank > 32 && rank <= 64; }  // the ranks where 64-token tiles of shrink pay
static constexpr bool expand_has_64(bool f32, int rank) { return f32 || rank <= 64; }

static AdapterPlan plan_of(const semmoe_config* cfg, const semmoe_adapter_shape* s) {
  AdapterPlan p;
  const int T = cfg->T, es = int(act_bytes(cfg));
  const int mean = T / s->n_adapters, most = mean <= 24 ? 1 : (mean <= 48 ? 2 : 4);
  const long long work = (long long)T * s->rank;
  const bool shrink_32 = s->rank <= 32 ? T >= 4000 : (s->rank <= 64 ? T >= 5000 : work >= 1 << 19);
  const int shrink_tt = work >= 14000 * 64 && shrink_has_64(s->rank) ? 4 : (shrink_32 ? 2 : 1);
  const int expand_tt = T >= 8192 && expand_has_64(es == 4, s->rank) ? 4 : (T >= 2048 ? 2 : 1);
  p.shrink_tt = shrink_tt < most ? shrink_tt : most;
  p.expand_tt = expand_tt < most ? expand_tt : most;
  const long long tiles = p.tiles(p.shrink_tt, T, s->n_adapters), e_tiles = p.tiles(p.expand_tt, T, s->n_adapters + 1);
  cut_k(s->d_in, es, s->rank, tiles, &p.part_k_in, &p.parts_in);
  cut_k(s->d_out, es, s->rank, tiles, &p.part_k_out, &p.parts_out);
  p.chunks_in = cut_columns(s->d_in, p.expand_tt, e_tiles);
  p.chunks_out = cut_columns(s->d_out, p.expand_tt, e_tiles);
  // Segments until there are some 512 workgroups; a slice of 64 tokens takes one 1 to 3 us, a segment more a launch that joins (862 tokens of
  // 3 adapters, 336 and 976 columns, rank 48: 32 us as whole adapters, 14 slices long).  Adapters of few tokens stay whole where the
  // batch is short: no launch that joins.
  const int cols = es == 2 ? kOuterCols<false> : kOuterCols<true>;
  const int wanted = 512 / (cdiv(s->d_in, cols) + cdiv(s->d_out, cols));
  const int seg = cdiv(cdiv(T, wanted < 1 ? 1 : wanted), kOuterTok) * kOuterTok, least = mean <= 192 ? 1024 : 128;
  p.seg = seg < least ? least : (seg > 8192 ? 8192 : seg);
  return p;
}

static size_t u_floats(const semmoe_config* cfg, const semmoe_adapter_shape* s, int parts) {
  return size_t(parts) * cfg->T * s->rank;
}
static size_t partial_places(const semmoe_config* cfg, const AdapterPlan& p) {
  return cfg->T > p.seg ? size_t(cdiv(cfg->T, p.seg)) * 2 : 0;  // else no adapter has a second segment
}
static size_t partial_floats(const semmoe_config* cfg, const semmoe_adapter_shape* s, const AdapterPlan& p, int width) {
  return partial_places(cfg, p) * s->rank * width;
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

// One launch of 256 threads a workgroup.  `allowed`: the kernel's own flag word (allow_max_dynamic_lds).
template <typename... P, typename... A>
static int32_t launch_groups(void (*kern)(P...), std::atomic<uint64_t>* allowed, dim3 groups, size_t lds, hipStream_t s, A... args) {
  if (lds > 48 * 1024) {
    DeviceInfo d;
    int32_t st = device_info(&d);
    if (st != SEMMOE_OK) return st;
    if (lds > size_t(d.max_lds)) return SEMMOE_EUNSUPPORTED;
    st = allow_max_dynamic_lds(allowed, reinterpret_cast<const void*>(kern));
    if (st != SEMMOE_OK) return st;
  }
  hipLaunchKernelGGL(kern, groups, dim3(256), lds, s, args...);
  SEMMOE_LAUNCH_CHECK();
  return SEMMOE_OK;
}
constexpr long long kMostGroups = 1ll << 24;  // 2^32 threads a launch

template <bool F32, int RT, int TT>
constexpr size_t kShrinkLds = 4 * (TT + RT) * 2048 > 4 * RT * TT * 1024 ? 4 * (TT + RT) * 2048 : 4 * RT * TT * 1024;

template <typename F>
static int32_t with_shrink_tiles(int rank, int tt, F f) {
  return with_rank_tiles(rank, [&](auto rt) -> int32_t {
    if (tt <= 1) return f(rt, std::integral_constant<int, 1>{});
    if constexpr (decltype(rt)::value == 4)  // shrink_has_64
      if (tt >= 4) return f(rt, std::integral_constant<int, 4>{});
    return f(rt, std::integral_constant<int, 2>{});
  });
}

template <bool F32>
static int32_t launch_shrink(const ShrinkArgs& a, int tt, hipStream_t s) {
  return with_shrink_tiles(a.ad.rank, tt, [&](auto rt, auto t4) -> int32_t {
    constexpr int RT = decltype(rt)::value, TT = decltype(t4)::value;
    const long long tiles = AdapterPlan::tiles(TT, a.ad.T, a.ad.n_adapters);
    if (tiles <= 0) return SEMMOE_OK;
    if (tiles * a.parts >= kMostGroups) return SEMMOE_EUNSUPPORTED;
    static std::atomic<uint64_t> allowed{0};
    return launch_groups(shrink_kernel<F32, RT, TT>, &allowed, dim3(unsigned(tiles * a.parts)), kShrinkLds<F32, RT, TT>, s, a);
  });
}

template <bool F32>
static int32_t launch_shrink_both(const ShrinkArgs& v, const ShrinkArgs& u, bool want_v, bool want_u, int tt, hipStream_t s) {
  return with_shrink_tiles(v.ad.rank, tt, [&](auto rt, auto t4) -> int32_t {
    constexpr int RT = decltype(rt)::value, TT = decltype(t4)::value;
    const long long tiles = AdapterPlan::tiles(TT, v.ad.T, v.ad.n_adapters);
    const long long vb = want_v ? tiles * v.parts : 0, ub = want_u ? tiles * u.parts : 0;
    if (vb + ub <= 0) return SEMMOE_OK;
    if (vb + ub >= kMostGroups) return SEMMOE_EUNSUPPORTED;
    static std::atomic<uint64_t> allowed{0};
    return launch_groups(shrink_both_kernel<F32, RT, TT>, &allowed, dim3(unsigned(vb + ub)), kShrinkLds<F32, RT, TT>, s, v, int(vb), u);
  });
}

template <bool F32, typename F>
static int32_t with_expand_tiles(int rank, int tt, F f) {
  return with_rank_tiles(rank, [&](auto rt) -> int32_t {
    if (tt <= 1) return f(rt, std::integral_constant<int, 1>{});
    if constexpr (expand_has_64(F32, 16 * decltype(rt)::value))
      if (tt >= 4) return f(rt, std::integral_constant<int, 4>{});
    return f(rt, std::integral_constant<int, 2>{});
  });
}

template <bool F32, bool TR>
static int32_t launch_expand(const ExpandArgs& a, int tt, hipStream_t s) {
  return with_expand_tiles<F32>(a.ad.rank, tt, [&](auto rt, auto t4) -> int32_t {
    constexpr int RT = decltype(rt)::value, TT = decltype(t4)::value;
    const long long groups = AdapterPlan::tiles(TT, a.ad.T, a.ad.n_adapters + 1) * cdiv(a.N, a.chunks * kExpandCols);
    if (groups <= 0) return SEMMOE_OK;
    if (groups >= kMostGroups) return SEMMOE_EUNSUPPORTED;
    using E = Elem<F32>;
    constexpr size_t rows = (16 * RT + E::kStep - 1) / E::kStep * E::kStep;
    constexpr size_t factor = TR ? rows * 32 * E::kSize : 32 * (16 * RT + E::kPer16) * E::kSize;
    static std::atomic<uint64_t> allowed{0};
    return launch_groups(expand_kernel<F32, RT, TT, TR>, &allowed, dim3(unsigned(groups)), 4 * (16 * 144 + factor), s, a);
  });
}

template <bool F32>
static int32_t launch_outer(const OuterArgs& da, const OuterArgs& db, hipStream_t s) {
  constexpr int NC = kOuterCols<F32>;
  const long long items = (long long)da.ad.T / da.seg + da.ad.n_adapters, ab = da.dF ? items * cdiv(da.C, NC) : 0, bb = db.dF ? items * cdiv(db.C, NC) : 0;
  if (ab + bb >= kMostGroups) return SEMMOE_EUNSUPPORTED;
  const int32_t st = with_rank_tiles(da.ad.rank, [&](auto rt) -> int32_t {
    constexpr int RT = decltype(rt)::value;
    using E = Elem<F32>;
    static std::atomic<uint64_t> allowed{0};
    return launch_groups(outer_kernel<F32, RT>, &allowed, dim3(unsigned(ab + bb)), kOuterTok * (256 + kParts<F32> * (16 * RT * E::kSize + 16)), s, da, int(ab), db);
  });
  if (st != SEMMOE_OK || da.ad.T <= da.seg) return st;  // no adapter has a second segment
  const int ja = da.dF ? int((size_t(da.ad.rank) * da.C + 1023) / 1024) : 0, jb = db.dF ? int((size_t(db.ad.rank) * db.C + 1023) / 1024) : 0;
  static std::atomic<uint64_t> allowed{0};
  return launch_groups(outer_join_kernel<F32>, &allowed, dim3(ja + jb, da.ad.n_adapters), 0, s, da, ja, db);
}

template <bool F32>
static int32_t run_adapters(const semmoe_config* cfg, const semmoe_adapter_shape* sh, const AdapterPlan& p, hipStream_t s,
                            const void* X, const AdapterArgs& ad, const void* A, const void* B, const float* scale,
                            const void* Y_base, void* Y, float* U, size_t ldx, size_t ld_base, size_t ldo) {
  const ShrinkArgs sa{ad, X, ldx, A, scale, sh->d_in, p.part_k_in, p.parts_in, U};
  const int32_t st = launch_shrink<F32>(sa, p.shrink_tt, s);
  if (st != SEMMOE_OK) return st;
  const ExpandArgs ea{ad, U, p.parts_in, B, sh->d_out, p.chunks_out, Y_base, ld_base, Y, ldo};
  return launch_expand<F32, false>(ea, p.expand_tt, s);
}

template <bool F32>
static int32_t run_adapters_grad(const semmoe_config* cfg, const semmoe_adapter_shape* sh, const AdapterPlan& p, hipStream_t s,
                                 const void* X, const void* dY, const AdapterArgs& ad, const void* A, const void* B,
                                 const float* scale, const void* dX_base, void* dX, void* dA, void* dB, float* U, float* V,
                                 float* partial_a, float* partial_b, size_t ldx, size_t ldy, size_t ld_base, size_t ldo) {
  const ShrinkArgs va{ad, dY, ldy, B, scale, sh->d_out, p.part_k_out, p.parts_out, V};
  const ShrinkArgs ua{ad, X, ldx, A, scale, sh->d_in, p.part_k_in, p.parts_in, U};
  int32_t st = launch_shrink_both<F32>(va, ua, dX || dA, dB, p.shrink_tt, s);
  if (st != SEMMOE_OK) return st;
  if (dA || dB) {
    const OuterArgs oa{ad, V, p.parts_out, X, ldx, sh->d_in, p.seg, partial_a, dA};
    const OuterArgs ob{ad, U, p.parts_in, dY, ldy, sh->d_out, p.seg, partial_b, dB};
    st = launch_outer<F32>(oa, ob, s);
    if (st != SEMMOE_OK) return st;
  }
  if (!dX) return SEMMOE_OK;  // last: dX may take the place of X or dY
  const ExpandArgs ea{ad, V, p.parts_out, A, sh->d_in, p.chunks_in, dX_base, ld_base, dX, ldo};
  return launch_expand<F32, true>(ea, p.expand_tt, s);
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
  *bytes_out = align_up(u_floats(cfg, shape, p.parts_in) * 4, 256) + align_up(u_floats(cfg, shape, p.parts_out) * 4, 256) +
               align_up(partial_floats(cfg, shape, p, shape->d_in) * 4, 256) + partial_floats(cfg, shape, p, shape->d_out) * 4 + 256;
  return SEMMOE_OK;
}

extern "C" int32_t semmoe_adapter_forward_workspace_bytes(const semmoe_config* cfg, const semmoe_adapter_shape* shape,
                                                          size_t* bytes_out) {
  if (!bytes_out) return SEMMOE_EINVAL;
  const int32_t st = check_shape(cfg, shape);
  if (st != SEMMOE_OK) return st;
  *bytes_out = u_floats(cfg, shape, plan_of(cfg, shape).parts_in) * 4 + 256;
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
  Carver c(ws, ws_bytes);
  float* U = c.take<float>(u_floats(cfg, shape, p.parts_in));
  float* V = c.take<float>(u_floats(cfg, shape, p.parts_out));
  float* partial_a = c.take<float>(partial_floats(cfg, shape, p, shape->d_in));
  float* partial_b = c.take<float>(partial_floats(cfg, shape, p, shape->d_out));
  if (!c.ok) return SEMMOE_EWORKSPACE;
  const AdapterArgs ad{order, adapter_offsets, cfg->T, shape->n_adapters, shape->rank};
  auto* const run = cfg->dtype == SEMMOE_BF16 ? run_adapters_grad<false> : run_adapters_grad<true>;
  return run(cfg, shape, p, static_cast<hipStream_t>(stream), X, dY, ad, A, B, scale, dX_base, dX, dA, dB, U, V, partial_a, partial_b, ldx,
             ldy, ld_base, ldo);
}
