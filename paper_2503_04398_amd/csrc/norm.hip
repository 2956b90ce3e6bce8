// The norms around a block with its gate and the residual's scale, forward and back:
//   n = Y rsqrt(mean Y^2 + e) w_post,   H = s R + gate n,   X = H rsqrt(mean H^2 + e) w_pre.
// Towards H, with xn = H rh and a = dX w_pre:  dH += rh (a - xn mean(a xn)); towards Y the same with b = dH gate w_post.  dR = s dH,
// dgate = dH n, dw_post = sum over rows of dH gate Y ry, dw_pre = sum of dX H rh.
//
// Both stream: each tensor is read or written once, a row stays in registers between its two norms.  Statistics and sums are fp32.
// Measured, bf16: 16384 rows of 7168 194 us, 4.85 TB/s as a copy; the gradient of 8192 rows of 4096 89 + 6 us, 4.7 TB/s with its partial
// sums, of 4096 rows of 7168 100 + 5.  fp32 gradient: 8192 rows of 4096 179 + 5 us, 4096 of 7168 148 + 5.  Past 8192 registers are
// spilled: 17 of four pieces a thread in bf16 (13401 rows of 8208 222 us where 178 are a copy), and below at the gradient.
#include <initializer_list>

#include "rows.hpp"

namespace semmoe {

struct NormArgs {
  int n_rows, d, tr;
  float res_scale, eps_post, eps_pre;
  const void *R, *Y, *w_post, *gate, *w_pre;
  void *H, *X;
  uint8_t* Xq;
  float* x_scale;
  int64_t ld_r, ld_y, ld_gate, ld_h, ld_x;  // ld_gate 0: one gate for all rows
  // backward
  const void *dH, *dX;
  void *dR, *dY, *dgate;
  int64_t ld_dh, ld_dx, ld_dr, ld_dy, ld_dgate;
  float* sums;  // [3][workgroups][d]: dw_post, dw_pre, dgate; nullptr: none is asked for
};

__device__ __forceinline__ float add_f(float a, float b) { return a + b; }

template <bool BF16, int NP>
__global__ __launch_bounds__(1024) void block_norm_kernel(const NormArgs a) {
  using E = Piece<BF16>;
  constexpr int N = E::N;
  __shared__ float part[2][16];
  __shared__ uint32_t part_m[16];
  const int teams = blockDim.x / a.tr, team = threadIdx.x / a.tr, t = threadIdx.x % a.tr, pieces = a.d / N, tw = a.tr >> 6;
  const int row = blockIdx.x * teams + team;
  const bool have = row < a.n_rows;
  const size_t rw = have ? row : 0;
  E r[NP], y[NP], wp[NP], g[NP], wq[NP];
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int c = t + p * a.tr;
    const bool in = c < pieces && have;
    const size_t at = size_t(c) * N;
    auto get = [&](E& e, const void* base, size_t off) __attribute__((always_inline)) {
      if (in && base) e.load(base, off + at);
      else e.zero();
    };
    get(y[p], a.Y, rw * a.ld_y);
    get(r[p], a.R, rw * a.ld_r);
    get(wp[p], a.w_post, 0);
    get(g[p], a.gate, rw * a.ld_gate);
    get(wq[p], a.w_pre, 0);
  }
  const float inv_d = 1.0f / float(a.d);
  float ry = 1.0f;
  if (a.w_post) {
    float s[1] = {0.0f};
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int x = 0; x < N; ++x) s[0] = fmaf(y[p][x], y[p][x], s[0]);
    team_join(s, part[0], tw, add_f);
    ry = 1.0f / sqrtf(s[0] * inv_d + a.eps_post);
  }
  float h[NP][N];
#pragma unroll
  for (int p = 0; p < NP; ++p)
#pragma unroll
    for (int x = 0; x < N; ++x) {
      float n = y[p][x];
      if (a.w_post) n = n * ry * wp[p][x];
      if (a.gate) n *= g[p][x];
      h[p][x] = fmaf(a.res_scale, r[p][x], n);
    }
  if (a.H) {
#pragma unroll
    for (int p = 0; p < NP; ++p)
      if (have && t + p * a.tr < pieces) {
        E e;
        e.round(h[p]);
        e.store(a.H, rw * a.ld_h + size_t(t + p * a.tr) * N);
      }
  }
  if (!a.w_pre) return;
  float s[1] = {0.0f};
#pragma unroll
  for (int p = 0; p < NP; ++p)
#pragma unroll
    for (int x = 0; x < N; ++x) s[0] = fmaf(h[p][x], h[p][x], s[0]);
  team_join(s, part[1], tw, add_f);
  const float rh = 1.0f / sqrtf(s[0] * inv_d + a.eps_pre);
#pragma unroll
  for (int p = 0; p < NP; ++p)
#pragma unroll
    for (int x = 0; x < N; ++x) h[p][x] = h[p][x] * rh * wq[p][x];
  if (a.X) {
#pragma unroll
    for (int p = 0; p < NP; ++p)
      if (have && t + p * a.tr < pieces) {
        E e;
        e.round(h[p]);
        e.store(a.X, rw * a.ld_x + size_t(t + p * a.tr) * N);
      }
  }
  if (!a.Xq) return;
  // in 8 bits: of the numbers before they are rounded to the act type
  uint32_t m[1] = {0};
#pragma unroll
  for (int p = 0; p < NP; ++p)
#pragma unroll
    for (int x = 0; x < N; ++x) m[0] = max(m[0], magnitude_bits(h[p][x]));
  team_join(m, part_m, tw, [](uint32_t u, uint32_t v) { return max(u, v); });
  const RowScale q(m[0]);
#pragma unroll
  for (int p = 0; p < NP; ++p)
    if (have && t + p * a.tr < pieces)
      q.put(a.Xq + rw * a.d + size_t(t + p * a.tr) * N, h[p]);
  if (have && t == 0) a.x_scale[row] = q.scale;
}

constexpr int kNormGradGroups = 512;  // workgroups of the backward pass at most: the rows of partial sums

// NP 1: the rows that come next are requested before this one's sums are joined; with NP 2 there are no registers for that.  GATES: a
// gate for each row.  Of 128 registers bf16 rows past 8192 spill 10 with GATES and 41 without (2048 rows of 14336: 192 us, a copy 71), fp32
// ones 191 and 238 (545 and 509 us, a copy 190 and 142).
template <bool BF16, int NP, bool GATES>
__global__ __launch_bounds__(1024, 4) void block_norm_grad_kernel(const NormArgs a) {
  using E = Piece<BF16>;
  constexpr int N = E::N;
  extern __shared__ float lds[];
  float* part = lds;  // [3][16 waves], then [16 waves]
  const int teams = blockDim.x / a.tr, team = threadIdx.x / a.tr, t = threadIdx.x % a.tr, pieces = a.d / N, tw = a.tr >> 6;
  const float inv_d = 1.0f / float(a.d);
  constexpr bool AHEAD = NP == 1;
  E wp[NP], wq[NP], g[NP];
  float sp[NP][N], sq[NP][N], sg[GATES ? 1 : NP][N];  // dw_post, dw_pre, dgate of this thread's columns
#pragma unroll
  for (int p = 0; p < NP; ++p) {
    const int c = t + p * a.tr;
    wp[p].zero();
    wq[p].zero();
    g[p].zero();
    if (c < pieces) {
      if (a.w_post) wp[p].load(a.w_post, size_t(c) * N);
      if (a.w_pre) wq[p].load(a.w_pre, size_t(c) * N);
      if (!GATES && a.gate) g[p].load(a.gate, size_t(c) * N);
    }
#pragma unroll
    for (int x = 0; x < N; ++x) {
      sp[p][x] = sq[p][x] = 0.0f;
      if constexpr (!GATES) sg[p][x] = 0.0f;
    }
  }
  struct Row {
    E h[NP], x[NP], d[NP], y[NP], g[GATES ? NP : 1];
  };
  auto fetch = [&](Row& v, int row0) __attribute__((always_inline)) {
    const int row = row0 + team;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int c = t + p * a.tr;
      const bool in = row < a.n_rows && c < pieces;
      const size_t at = size_t(c) * N, rw = row;
      auto get = [&](E& e, const void* base, int64_t ld) __attribute__((always_inline)) {
        if (in && base) e.load(base, rw * ld + at);
        else e.zero();
      };
      get(v.x[p], a.dX, a.ld_dx);
      get(v.h[p], a.dX ? a.H : nullptr, a.ld_h);
      get(v.d[p], a.dH, a.ld_dh);
      get(v.y[p], a.Y, a.ld_y);
      if constexpr (GATES) get(v.g[p], a.gate, a.ld_gate);
    }
  };
  Row next;
  if constexpr (AHEAD) fetch(next, blockIdx.x * teams);
  for (int row0 = blockIdx.x * teams; row0 < a.n_rows; row0 += gridDim.x * teams) {
    const int row = row0 + team;
    const bool have = row < a.n_rows;
    const size_t rw = have ? row : row0;
    Row v;
    if constexpr (AHEAD) {
      v = next;
      fetch(next, row0 + gridDim.x * teams);
    } else {
      fetch(v, row0);
    }
    if constexpr (GATES)
#pragma unroll
      for (int p = 0; p < NP; ++p) g[p] = v.g[p];
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      wp[p].stay();
      wq[p].stay();
      g[p].stay();
    }
    // sums over the row: H^2, a H, Y^2
    float s[3] = {0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int p = 0; p < NP; ++p)
#pragma unroll
      for (int x = 0; x < N; ++x) {
        s[0] = fmaf(v.h[p][x], v.h[p][x], s[0]);
        s[1] = fmaf(v.x[p][x] * wq[p][x], v.h[p][x], s[1]);
        s[2] = fmaf(v.y[p][x], v.y[p][x], s[2]);
      }
    team_join(s, part, tw, add_f);
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      v.h[p].stay();
      v.x[p].stay();
      v.y[p].stay();
      wq[p].stay();
    }
    const float rh = 1.0f / sqrtf(s[0] * inv_d + a.eps_pre), ch = s[1] * rh * inv_d;
    const float ry = a.w_post ? 1.0f / sqrtf(s[2] * inv_d + a.eps_post) : 1.0f;
    float dh[NP][N], e[1] = {0.0f};
    // A team without a row adds nothing to the sums: its zeros times the root's reciprocal, infinite where eps is 0, or times an infinite
    // weight would be NaN.
    if (have) {
#pragma unroll
      for (int p = 0; p < NP; ++p)
#pragma unroll
        for (int x = 0; x < N; ++x) {
          float u = v.d[p][x];
          if (a.dX) {
            const float xn = v.h[p][x] * rh;
            u += rh * (v.x[p][x] * wq[p][x] - xn * ch);
            sq[p][x] = fmaf(v.x[p][x], xn, sq[p][x]);
          }
          dh[p][x] = u;
          const float yn = v.y[p][x] * ry, b = a.gate ? u * g[p][x] : u;
          if (a.w_post) {
            e[0] = fmaf(b * wp[p][x], yn, e[0]);
            sp[p][x] = fmaf(b, yn, sp[p][x]);
          }
          if constexpr (!GATES) sg[p][x] = fmaf(u, a.w_post ? yn * wp[p][x] : yn, sg[p][x]);
        }
    }
    if (a.w_post) team_join(e, part + 48, tw, add_f);
    else if (tw > 1) __syncthreads();  // `part` has been read
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      v.y[p].stay();
      wp[p].stay();
      g[p].stay();
    }
    const float cy = e[0] * inv_d;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const size_t at = size_t(t + p * a.tr) * N;
      if (!have || t + p * a.tr >= pieces) continue;
      float f[N];
      E o;
      if (a.dR) {
#pragma unroll
        for (int x = 0; x < N; ++x) f[x] = a.res_scale * dh[p][x];
        o.round(f);
        o.store(a.dR, rw * a.ld_dr + at);
      }
      if (GATES && a.dgate) {
#pragma unroll
        for (int x = 0; x < N; ++x) f[x] = dh[p][x] * (a.w_post ? v.y[p][x] * ry * wp[p][x] : v.y[p][x]);
        o.round(f);
        o.store(a.dgate, rw * a.ld_dgate + at);
      }
      if (a.dY) {
#pragma unroll
        for (int x = 0; x < N; ++x) {
          const float b = a.gate ? dh[p][x] * g[p][x] : dh[p][x];
          f[x] = a.w_post ? ry * (b * wp[p][x] - v.y[p][x] * ry * cy) : b;
        }
        o.round(f);
        o.store(a.dY, rw * a.ld_dy + at);
      }
    }
  }
  if (!a.sums) return;
  // the teams' sums meet in LDS, in the order of the teams
  float* meet = lds + 64;
#pragma unroll
  for (int which = 0; which < (GATES ? 2 : 3); ++which) {
#pragma unroll
    for (int p = 0; p < NP; ++p) {
      const int c = t + p * a.tr;
      float v[N];
#pragma unroll
      for (int x = 0; x < N; ++x) v[x] = which == 0 ? sp[p][x] : which == 1 ? sq[p][x] : sg[GATES ? 0 : p][x];
      if (teams > 1) {
        __syncthreads();
#pragma unroll
        for (int x = 0; x < N; ++x) meet[(team * a.tr + t) * N + x] = v[x];
        __syncthreads();
        if (team == 0)
          for (int w = 1; w < teams; ++w)
#pragma unroll
            for (int x = 0; x < N; ++x) v[x] += meet[(w * a.tr + t) * N + x];
      }
      if (team == 0 && c < pieces) {
        float* const to = a.sums + (size_t(which) * gridDim.x + blockIdx.x) * a.d + size_t(c) * N;
#pragma unroll
        for (int x = 0; x < N; x += 4)
          *reinterpret_cast<row_u32x4_t*>(to + x) = row_u32x4_t{__float_as_uint(v[x]), __float_as_uint(v[x + 1]),
                                                                __float_as_uint(v[x + 2]), __float_as_uint(v[x + 3])};
      }
    }
  }
}

// Columns of the workgroups' sums: 64 columns, four a thread, and 16 runs of the rows a workgroup, the runs joined in order.
template <bool BF16>
__global__ __launch_bounds__(256) void norm_sums_kernel(const float* __restrict__ sums, int groups, int d, void* dw_post, void* dw_pre,
                                                        void* dgate) {
  typedef __attribute__((ext_vector_type(4))) float f4;
  __shared__ f4 part[16][16];
  const int which = blockIdx.y, quad = threadIdx.x & 15, run = threadIdx.x >> 4, col = blockIdx.x * 64 + quad * 4;
  void* const out = which == 0 ? dw_post : which == 1 ? dw_pre : dgate;
  if (!out) return;  // the whole workgroup
  const f4* from = reinterpret_cast<const f4*>(sums + size_t(which) * groups * d + min(col, d - 4));
  const int per = (groups + 15) / 16, lo = run * per, hi = min(lo + per, groups);
  f4 s = {0.0f, 0.0f, 0.0f, 0.0f};
  for (int r = lo; r < hi; r += 8) {
    f4 v[8];
#pragma unroll
    for (int u = 0; u < 8; ++u) v[u] = r + u < hi ? from[size_t(r + u) * d / 4] : f4{0.0f, 0.0f, 0.0f, 0.0f};
#pragma unroll
    for (int u = 0; u < 8; ++u) s += v[u];
  }
  part[run][quad] = s;
  __syncthreads();
  if (run || col >= d) return;
#pragma unroll
  for (int w = 1; w < 16; ++w) s += part[w][quad];
  if constexpr (BF16) {
    *reinterpret_cast<uint2*>(static_cast<bf16_t*>(out) + col) = make_uint2(cvt_pk_bf16(s[0], s[1]), cvt_pk_bf16(s[2], s[3]));
  } else {
    *reinterpret_cast<f4*>(static_cast<float*>(out) + col) = s;
  }
}

static int32_t check_norm(const semmoe_config* cfg, const semmoe_norm_shape* n, std::initializer_list<int64_t> lds) {
  if (!cfg || !n) return SEMMOE_EINVAL;
  if (cfg->dtype != SEMMOE_FP32 && cfg->dtype != SEMMOE_BF16) return SEMMOE_EUNSUPPORTED;
  if (cfg->T < 0 || cfg->d <= 0) return SEMMOE_EINVAL;
  if (!(n->eps_post >= 0.0f) || !(n->eps_pre >= 0.0f)) return SEMMOE_EINVAL;
  if (cfg->d % 8 != 0) return SEMMOE_ESHAPE;
  if (cfg->d > SEMMOE_MAX_NORM_D || cfg->T > 0x3fffffff) return SEMMOE_EUNSUPPORTED;
  for (int64_t ld : lds) {
    if (ld < 0) return SEMMOE_EINVAL;
    if (ld % 8 != 0 || (ld > 0 && ld < cfg->d)) return SEMMOE_ESHAPE;
  }
  return SEMMOE_OK;
}

// The backward pass' kernel holds 128 registers a thread: 16 waves a compute unit.  Workgroups of 8 waves, two a compute unit, as many
// teams in each as fit: their sums meet in LDS, and the rows of partial sums are fewer (16384 rows of 2048: 94 us, one team a workgroup
// of 4 waves 112; as 16 waves 103).  A team of more than 8 waves is a workgroup, one a compute unit (4096 rows of 7168: 105 us, with twice
// as many workgroups 118).
static RowTeams norm_grad_teams(const semmoe_config* cfg) {
  RowTeams g(cfg->dtype == SEMMOE_BF16, cfg->d, 1024);
  g.teams = g.tr > 256 ? 1 : 512 / g.tr;
  return g;
}

static size_t norm_groups(const semmoe_config* cfg) {
  const RowTeams g = norm_grad_teams(cfg);
  const int rows = cdiv(cfg->T, g.teams), most = g.tr > 512 ? kNormGradGroups / 2 : kNormGradGroups;
  return rows < most ? rows : most;
}

}  // namespace semmoe

using namespace semmoe;

extern "C" int32_t semmoe_block_norm(const semmoe_config* cfg, void* stream, const semmoe_norm_shape* n, const void* R, const void* Y,
                                     const void* w_post, const void* gate, const void* w_pre, void* H, void* X, void* Xq,
                                     float* x_scale) {
  const int32_t st = n ? check_norm(cfg, n, {n->ld_r, n->ld_y, n->ld_h, n->ld_x, n->ld_gate}) : SEMMOE_EINVAL;
  if (st != SEMMOE_OK) return st;
  if ((!R && !Y) || (!Y && (w_post || gate)) || (!H && !X && !Xq)) return SEMMOE_EINVAL;
  if ((!w_pre && (X || Xq)) || (w_pre && !X && !Xq) || !Xq != !x_scale) return SEMMOE_EINVAL;
  for (const void* p : {R, Y, w_post, gate, w_pre, static_cast<const void*>(H), static_cast<const void*>(X), static_cast<const void*>(Xq)})
    if (!aligned16(p)) return SEMMOE_EINVAL;
  if (cfg->T == 0) return SEMMOE_OK;
  const bool bf = cfg->dtype == SEMMOE_BF16;
  const RowTeams g(bf, cfg->d);
  NormArgs a{};
  a.n_rows = cfg->T; a.d = cfg->d; a.tr = g.tr;
  a.res_scale = n->res_scale; a.eps_post = n->eps_post; a.eps_pre = n->eps_pre;
  a.R = R; a.Y = Y; a.w_post = w_post; a.gate = gate; a.w_pre = w_pre;
  a.H = H; a.X = X; a.Xq = static_cast<uint8_t*>(Xq); a.x_scale = x_scale;
  const int64_t d = cfg->d;
  a.ld_r = n->ld_r ? n->ld_r : d; a.ld_y = n->ld_y ? n->ld_y : d; a.ld_h = n->ld_h ? n->ld_h : d; a.ld_x = n->ld_x ? n->ld_x : d;
  a.ld_gate = n->gate_rows ? (n->ld_gate ? n->ld_gate : d) : 0;
  const dim3 block(g.tr * g.teams);
  hipStream_t s = static_cast<hipStream_t>(stream);
  const int per = rows_a_launch(g.teams, block.x);
  for (int row = 0; row < cfg->T; row += per) {
    const dim3 grid(cdiv(a.n_rows < per ? a.n_rows : per, g.teams));
    if (bf) {
      if (g.np == 1) hipLaunchKernelGGL((block_norm_kernel<true, 1>), grid, block, 0, s, a);
      else if (g.np == 2) hipLaunchKernelGGL((block_norm_kernel<true, 2>), grid, block, 0, s, a);
      else hipLaunchKernelGGL((block_norm_kernel<true, 4>), grid, block, 0, s, a);
    } else {
      if (g.np == 1) hipLaunchKernelGGL((block_norm_kernel<false, 1>), grid, block, 0, s, a);
      else if (g.np == 2) hipLaunchKernelGGL((block_norm_kernel<false, 2>), grid, block, 0, s, a);
      else hipLaunchKernelGGL((block_norm_kernel<false, 4>), grid, block, 0, s, a);
    }
    SEMMOE_LAUNCH_CHECK();
    a.n_rows -= per;
    auto rest = [&](const void* p, int64_t ld) { return p ? static_cast<const char*>(p) + size_t(per) * ld * (bf ? 2 : 4) : nullptr; };
    a.R = rest(a.R, a.ld_r); a.Y = rest(a.Y, a.ld_y); a.gate = rest(a.gate, a.ld_gate);
    a.H = const_cast<char*>(rest(a.H, a.ld_h)); a.X = const_cast<char*>(rest(a.X, a.ld_x));
    if (a.Xq) { a.Xq += size_t(per) * a.d; a.x_scale += per; }
  }
  return SEMMOE_OK;
}

extern "C" int32_t semmoe_block_norm_grad_workspace_bytes(const semmoe_config* cfg, size_t* bytes_out) {
  const semmoe_norm_shape n{};
  const int32_t st = check_norm(cfg, &n, {});
  if (st != SEMMOE_OK || !bytes_out) return st != SEMMOE_OK ? st : SEMMOE_EINVAL;
  *bytes_out = 3 * norm_groups(cfg) * cfg->d * 4 + 256;
  return SEMMOE_OK;
}

extern "C" int32_t semmoe_block_norm_grad(const semmoe_config* cfg, void* stream, const semmoe_norm_shape* n, const void* dH,
                                          const void* dX, const void* H, const void* Y, const void* w_post, const void* gate,
                                          const void* w_pre, void* dR, void* dY, void* dgate, void* dw_post, void* dw_pre, void* ws,
                                          size_t ws_bytes) {
  const int32_t st = n ? check_norm(cfg, n, {n->ld_h, n->ld_y, n->ld_gate, n->ld_dh, n->ld_dx, n->ld_dr, n->ld_dy, n->ld_dgate})
                       : SEMMOE_EINVAL;
  if (st != SEMMOE_OK) return st;
  if ((!dH && !dX) || !dX != !w_pre || (dX && !H) || (!Y && (w_post || gate || dY))) return SEMMOE_EINVAL;
  if ((dgate && !gate) || (dw_post && !w_post) || (dw_pre && !w_pre)) return SEMMOE_EINVAL;
  if (!dR && !dY && !dgate && !dw_post && !dw_pre) return SEMMOE_EINVAL;
  for (const void* p : {dH, dX, H, Y, w_post, gate, w_pre, static_cast<const void*>(dR), static_cast<const void*>(dY),
                        static_cast<const void*>(dgate), static_cast<const void*>(dw_post), static_cast<const void*>(dw_pre)})
    if (!aligned16(p)) return SEMMOE_EINVAL;
  const bool columns = dw_post || dw_pre || (dgate && !n->gate_rows);
  const size_t groups = norm_groups(cfg);
  float* sums = nullptr;
  if (columns) {
    Carver c(ws, ws_bytes);
    sums = c.take<float>(3 * groups * cfg->d);
    if (!c.ok) return SEMMOE_EWORKSPACE;
  }
  if (cfg->T == 0 && !columns) return SEMMOE_OK;
  const RowTeams g = norm_grad_teams(cfg);
  NormArgs a{};
  a.n_rows = cfg->T; a.d = cfg->d; a.tr = g.tr;
  a.res_scale = n->res_scale; a.eps_post = n->eps_post; a.eps_pre = n->eps_pre;
  a.Y = Y; a.w_post = w_post; a.gate = gate; a.w_pre = w_pre; a.H = const_cast<void*>(H);
  a.dH = dH; a.dX = dX; a.dR = dR; a.dY = dY; a.dgate = dgate; a.sums = sums;
  const int64_t d = cfg->d;
  auto ld = [&](int64_t v) { return v ? v : d; };
  a.ld_h = ld(n->ld_h); a.ld_y = ld(n->ld_y); a.ld_dh = ld(n->ld_dh); a.ld_dx = ld(n->ld_dx); a.ld_dr = ld(n->ld_dr);
  a.ld_dy = ld(n->ld_dy); a.ld_dgate = ld(n->ld_dgate);
  a.ld_gate = n->gate_rows ? ld(n->ld_gate) : 0;
  const bool bf = cfg->dtype == SEMMOE_BF16;
  hipStream_t s = static_cast<hipStream_t>(stream);
  if (cfg->T > 0) {
    const dim3 grid(groups), block(g.tr * g.teams);
    const size_t lds = 256 + (columns && g.teams > 1 ? size_t(g.tr) * g.teams * (bf ? 32 : 16) : 0);
#define SEMMOE_NORM_GRAD(BF_, NP_)                                                                             \
  do {                                                                                                         \
    if (a.gate && n->gate_rows) hipLaunchKernelGGL((block_norm_grad_kernel<BF_, NP_, true>), grid, block, lds, s, a); \
    else hipLaunchKernelGGL((block_norm_grad_kernel<BF_, NP_, false>), grid, block, lds, s, a);                \
  } while (0)
    if (bf) {
      if (g.np == 1) SEMMOE_NORM_GRAD(true, 1);
      else SEMMOE_NORM_GRAD(true, 2);
    } else {
      if (g.np == 1) SEMMOE_NORM_GRAD(false, 1);
      else if (g.np == 2) SEMMOE_NORM_GRAD(false, 2);
      else SEMMOE_NORM_GRAD(false, 4);
    }
#undef SEMMOE_NORM_GRAD
    SEMMOE_LAUNCH_CHECK();
  }
  if (columns) {
    const dim3 grid(cdiv(cfg->d, 64), 3);
    void* const dg = n->gate_rows ? nullptr : dgate;
    if (bf) hipLaunchKernelGGL(norm_sums_kernel<true>, grid, dim3(256), 0, s, sums, int(groups), cfg->d, dw_post, dw_pre, dg);
    else hipLaunchKernelGGL(norm_sums_kernel<false>, grid, dim3(256), 0, s, sums, int(groups), cfg->d, dw_post, dw_pre, dg);
    SEMMOE_LAUNCH_CHECK();
  }
  return SEMMOE_OK;
}
