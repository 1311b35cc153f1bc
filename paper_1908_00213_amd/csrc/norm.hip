// chn_layer_norm_fwd / _bwd, chn_residual_norm_fwd / _bwd: normalisation of rows, by itself or of residual + dropout(x).
//
//   forward   s = residual + dropout(x), rounded to the stream's type        (residual_norm; layer_norm: s is x)
//             mean = sum s / C    rstd = 1 / sqrt(sum (s - mean)^2 / C + eps)    y = (s - mean) rstd gamma + beta
//   backward  h = (s - mean) rstd    g = dy gamma    dn = rstd (g - sum g / C - h sum(g h) / C)
//             layer_norm: dx = dn;   residual_norm: dresidual = dn + ds, dx = dropout(dn + ds) with the forward's mask
//             dgamma = sum over rows of dy h      dbeta = sum over rows of dy
//
// All sums and statistics are fp32; the mean is corrected by the mean of what is left after its subtraction, so that rows whose mean
// is far larger than their spread keep their digits.  So do their gradients where the caller keeps the mean in two parts, the rounded one
// and what its rounding left (`mean` (N,2)): a mean of 1e4 spreads, rounded, costs dgamma 2.5e-4 of its largest element, one of 1e5 1.7e-3.
//
// Bound by memory: every element is read once and written once.  A row is held in the registers of 4 to 1024 lanes between the
// passes that its statistics need (rows.h); only rows that no block can hold are read again.
#include "philox.h"
#include "rows.h"

#include <type_traits>

namespace chn {
namespace {

struct NormArgs {
  int64_t N, C;
  int64_t px, pr, ps, py;            // row pitches in elements
  float eps;
  const float *gamma, *beta;
  float *mean, *rstd;
  int mean_parts;                    // of each row's mean: 1, or 2 with what its rounding left
  bool lines;                        // every row of every output begins a line of the cache
  DropArgs drop;
};

// Groups of up to sixteen lanes store rows a few hundred bytes at a time: past the usual order of replacement only if those are whole lines
// (forward, fp32 / bf16, us: 134217 x 250 67 / 31 so, 45 / 24 otherwise; 262144 x 128 40 / 21 so, 42 / 22 otherwise).
template <int G, typename T, int E>
__device__ __forceinline__ void put_unit(const Unit<T, E> &u, T *p, bool lines) {
  if (G >= 32 || lines) {
    u.store_nt(p);
  } else {
    asm volatile("");                                    // (without these two the compiler joins the branches into one ordinary store)
    u.store(p);
    asm volatile("");
  }
}

// A product that is rounded by itself: fused into the subtractions that follow, it would be another number there than in the mean that is kept.
__device__ __forceinline__ float times_rounded(float a, float b) {
#pragma clang fp contract(off)
  return a * b;
}

// The mean of a row, m0 + m1.
__device__ __forceinline__ void put_mean(const NormArgs &a, int64_t row, float m0, float m1) {
  if (!a.mean) return;
  const float mean = m0 + m1;
  if (a.mean_parts == 1) {
    a.mean[row] = mean;
  } else {                                               // (what the sum lost, whichever of the two is larger)
    const float of_m1 = mean - m0;
    a.mean[row * 2] = mean;
    a.mean[row * 2 + 1] = (m0 - (mean - of_m1)) + (m1 - of_m1);
  }
}

// The word of one column, for the elements behind the last whole unit.
__device__ __forceinline__ uint32_t word_of(const DropState &d, uint32_t c, uint32_t row) {
  const Philox4 w = d.words(c >> 2, row);
  return (c & 2) ? ((c & 1) ? w.w[3] : w.w[2]) : ((c & 1) ? w.w[1] : w.w[0]);
}

// v[0 .. E) dropped out, columns from c0 (a multiple of four) on
template <int E>
__device__ __forceinline__ void drop_unit(const DropState &d, uint32_t c0, uint32_t row, float (&v)[E]) {
#pragma unroll
  for (int b = 0; b < E / 4; ++b) {
    const Philox4 w = d.words((c0 >> 2) + b, row);
#pragma unroll
    for (int j = 0; j < 4; ++j) v[b * 4 + j] = d.apply(v[b * 4 + j], w.w[j]);
  }
}

// One row by G lanes of KE elements each; groups of up to 64 lanes share a block of 256.  (Kernels that walk over rows with gamma and beta
// in registers are slower: 8192 x 4096 bf16 24.9 us with 2048 blocks, 22.1 with a block for each row.)  Results are stored past the
// caches' usual order of replacement, since nothing of them is read here again: 4480 x 650 fp32 6.1 -> 5.6 us, 1024 x 1000 with residual 5.3 -> 5.0.
template <typename TX, typename TY, typename TS, bool RES, int G, int KE>
__global__ __launch_bounds__(G > 64 ? G : 256) void norm_fwd_rows_kernel(const TX *x, const TS *residual, TS *s, TY *y, NormArgs a) {
  constexpr int E = unit_elements<TX, TY, TS>(), K = KE / E, GROUPS = (G > 64 ? G : 256) / G;
  static_assert(G >= E - 1, "a lane for each element behind the last whole unit");
  __shared__ float2 smem[G > 64 ? 2 * G / 64 : 1];
  const int C = (int)a.C, whole = C / E, left = C - whole * E;
  const float inv = 1.0f / (float)C;
  const int g = threadIdx.x % G;
  int64_t row = block_number() * GROUPS;
  if constexpr (G == 64) row += __builtin_amdgcn_readfirstlane(threadIdx.x / 64);
  else if constexpr (G < 64) row += threadIdx.x / G;
  if (row >= a.N) return;                                // (groups that share a block meet at no barrier)
  const int cl = whole * E + g;                          // (l: the element behind the last whole unit, in the first few lanes)
  const TX *xr = x + row * a.px;
  TY *yr = y + row * a.py;
  float v[K][E], vl = 0.0f;
  Unit<TX, E> xu[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    xu[k].zero();
    if (g + k * G < whole) xu[k].load(xr + (g + k * G) * E);
  }
  if (g < left) vl = Elem<TX>::load(xr + cl);
  if constexpr (RES) {
    const TS *rr = residual + row * a.pr;
    TS *sr = s + row * a.ps;
    Unit<TS, E> ru[K];
    float rl = 0.0f;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      ru[k].zero();
      if (g + k * G < whole) ru[k].load(rr + (g + k * G) * E);
    }
    if (g < left) rl = Elem<TS>::load(rr + cl);
    const DropState d(a.drop);
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t c0 = (uint32_t)(g + k * G) * E;
#pragma unroll
      for (int i = 0; i < E; ++i) v[k][i] = xu[k].get(i);
      if (a.drop.rng) drop_unit<E>(d, c0, (uint32_t)row, v[k]);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        ru[k].set(i, add_rounded(ru[k].get(i), v[k][i]));
        v[k][i] = ru[k].get(i);
      }
      if (g + k * G < whole) put_unit<G>(ru[k], sr + c0, a.lines);
    }
    if (g < left) {
      if (a.drop.rng) vl = d.apply(vl, word_of(d, (uint32_t)cl, (uint32_t)row));
      vl = as_stored<TS>(add_rounded(rl, vl));
      Elem<TS>::store(sr + cl, vl);
    }
  } else {
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < E; ++i) v[k][i] = xu[k].get(i);
  }
  float sum = vl;                                        // (lanes without elements hold zeros)
#pragma unroll
  for (int k = 0; k < K; ++k)
#pragma unroll
    for (int i = 0; i < E; ++i) sum += v[k][i];
  const float m0 = times_rounded(group_sum<G>(make_float2(sum, 0.0f), smem, 0).x, inv);
  float dev = 0.0f, sq = 0.0f;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const bool there = g + k * G < whole;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      v[k][i] = there ? v[k][i] - m0 : 0.0f;
      dev += v[k][i];
      sq = fmaf(v[k][i], v[k][i], sq);
    }
  }
  vl = g < left ? vl - m0 : 0.0f;
  dev += vl;
  sq = fmaf(vl, vl, sq);
  const float2 t = group_sum<G>(make_float2(dev, sq), smem, 1);
  const float m1 = t.x * inv;
  const float rstd = 1.0f / sqrtf(fmaxf(t.y * inv - m1 * m1, 0.0f) + a.eps);
  if (g == 0) {
    put_mean(a, row, m0, m1);
    if (a.rstd) a.rstd[row] = rstd;
  }
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int c0 = (g + k * G) * E;
    if (g + k * G < whole) {
      Unit<float, E> gm, bt;
      if (a.gamma) gm.load(a.gamma + c0);
      if (a.beta) bt.load(a.beta + c0);
      Unit<TY, E> yu;
#pragma unroll
      for (int i = 0; i < E; ++i) yu.set(i, fmaf((v[k][i] - m1) * rstd, a.gamma ? gm.get(i) : 1.0f, a.beta ? bt.get(i) : 0.0f));
      put_unit<G>(yu, yr + c0, a.lines);
    }
  }
  if (g < left) Elem<TY>::store(yr + cl, fmaf((vl - m1) * rstd, a.gamma ? a.gamma[cl] : 1.0f, a.beta ? a.beta[cl] : 0.0f));
}

// Rows longer than a block holds: three passes over the row, a block of 1024 each.  A thread reads the elements that it stored itself.
template <typename TX, typename TY, typename TS, bool RES>
__global__ __launch_bounds__(1024) void norm_fwd_wide_kernel(const TX *x, const TS *residual, TS *s, TY *y, NormArgs a) {
  constexpr int E = unit_elements<TX, TY, TS>();
  __shared__ float2 smem[32];
  const float inv = 1.0f / (float)a.C;
  const int64_t row = block_number(), whole = a.C / E;
  if (row >= a.N) return;
  const TX *xr = x + row * a.px;
  TY *yr = y + row * a.py;
  TS *sr = RES ? s + row * a.ps : nullptr;
  const int64_t cl = whole * E + threadIdx.x;
  const bool last = cl < a.C;
  const auto at = [&](int64_t u, float (&v)[E]) {
    if constexpr (RES) {
      Unit<TS, E> t;
      t.load(sr + u * E);
#pragma unroll
      for (int i = 0; i < E; ++i) v[i] = t.get(i);
    } else {
      Unit<TX, E> t;
      t.load(xr + u * E);
#pragma unroll
      for (int i = 0; i < E; ++i) v[i] = t.get(i);
    }
  };
  float sum = 0.0f, vl = last ? Elem<TX>::load(xr + cl) : 0.0f;
  if constexpr (RES) {
    const DropState d(a.drop);
    const TS *rr = residual + row * a.pr;
    for (int64_t u = threadIdx.x; u < whole; u += 1024) {
      Unit<TX, E> xu;
      Unit<TS, E> ru;
      xu.load(xr + u * E);
      ru.load(rr + u * E);
      float v[E];
#pragma unroll
      for (int i = 0; i < E; ++i) v[i] = xu.get(i);
      if (a.drop.rng) drop_unit<E>(d, (uint32_t)u * E, (uint32_t)row, v);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        ru.set(i, add_rounded(ru.get(i), v[i]));
        sum += ru.get(i);
      }
      ru.store(sr + u * E);
    }
    if (last) {
      if (a.drop.rng) vl = d.apply(vl, word_of(d, (uint32_t)cl, (uint32_t)row));
      vl = as_stored<TS>(add_rounded(Elem<TS>::load(rr + cl), vl));
      Elem<TS>::store(sr + cl, vl);
    }
  } else {
    for (int64_t u = threadIdx.x; u < whole; u += 1024) {
      float v[E];
      at(u, v);
#pragma unroll
      for (int i = 0; i < E; ++i) sum += v[i];
    }
  }
  const float m0 = times_rounded(group_sum<1024>(make_float2(sum + vl, 0.0f), smem, 0).x, inv);
  if (last) vl -= m0;
  float dev = vl, sq = vl * vl;
  for (int64_t u = threadIdx.x; u < whole; u += 1024) {
    float v[E];
    at(u, v);
#pragma unroll
    for (int i = 0; i < E; ++i) {
      const float t = v[i] - m0;
      dev += t;
      sq = fmaf(t, t, sq);
    }
  }
  const float2 t = group_sum<1024>(make_float2(dev, sq), smem, 1);
  const float m1 = t.x * inv;
  const float rstd = 1.0f / sqrtf(fmaxf(t.y * inv - m1 * m1, 0.0f) + a.eps);
  if (threadIdx.x == 0) {
    put_mean(a, row, m0, m1);
    if (a.rstd) a.rstd[row] = rstd;
  }
  for (int64_t u = threadIdx.x; u < whole; u += 1024) {
    float v[E];
    at(u, v);
    Unit<float, E> gm, bt;
    if (a.gamma) gm.load(a.gamma + u * E);
    if (a.beta) bt.load(a.beta + u * E);
    Unit<TY, E> yu;
#pragma unroll
    for (int i = 0; i < E; ++i) yu.set(i, fmaf(((v[i] - m0) - m1) * rstd, a.gamma ? gm.get(i) : 1.0f, a.beta ? bt.get(i) : 0.0f));
    yu.store(yr + u * E);
  }
  if (last) Elem<TY>::store(yr + cl, fmaf((vl - m1) * rstd, a.gamma ? a.gamma[cl] : 1.0f, a.beta ? a.beta[cl] : 0.0f));
}

struct NormBwdArgs {
  int64_t N, C;
  int64_t pdy, ps, pds, pdr, pdx;
  const float *gamma, *mean, *rstd;
  int mean_parts;
  float *dgamma, *dbeta;
  float *partial;                    // [strips][2][C] or NULL
  float *pg, *pb;                    // where the first block leaves its sums, the others `step` behind each other: strips, or the results where there is
  int64_t step;                      // one block; NULL: not wanted
  int64_t strips;                    // wide rows: as many, of neighbouring rows
  float2 *sums;                      // wide rows: [N][segments] sums of g and g h
  int segments;
  bool lines;
  DropArgs drop;
};

// A row's statistics as a backward pass is given them, on their way in one load and one register: of four neighbouring lanes the first brings the mean, the second
// its last part, the third rstd.  (With the fold, us by three loads / by one: 8192 x 4096 bf16 with residual 57.8 / 56.0, 30504 x 1100 bf16 51.3 / 49.8,
// 8192 x 4096 bf16 38.2 / 38.3, 4480 x 650 fp32 10.25 / 10.25.)
struct RowStats {
  float mine = 0.0f;
  __device__ __forceinline__ void load(const NormBwdArgs &a, int64_t row) {
    const int q = threadIdx.x & 3;
    const float *mean = a.mean + row * a.mean_parts + (q == 1 ? a.mean_parts - 1 : 0);
    mine = *(q == 2 ? a.rstd + row : mean);
  }
  // The number that lane q of four brought, for a row of G lanes: where a wave has no second row, in a scalar register.
  template <int G, int q>
  __device__ __forceinline__ float of() const {
    if constexpr (G >= 64) return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(mine), q));
    else return __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(mine), 0x55 * q, 0xf, 0xf, true));   // quad_perm q q q q
  }
};

// h(s) is (s - mean) rstd: the first subtraction is exact where the mean is far above the spread, and what the mean's rounding left goes in behind the
// product (0 where it is not given: the product's bits).
struct Normal {
  float mean, rstd, shift;
  template <int G>
  static __device__ __forceinline__ Normal of(const NormBwdArgs &a, const RowStats &r) {
    const float rstd = r.of<G, 2>();
    return Normal{r.of<G, 0>(), rstd, a.mean_parts == 2 ? -r.of<G, 1>() * rstd : 0.0f};
  }
  __device__ __forceinline__ float h(float s) const { return fmaf(s - mean, rstd, shift); }
};

// One pass: a group of G lanes walks over rows, KE columns a lane, adding dy h and dy of its columns up in registers; at the end the groups
// of a block join theirs and the block leaves one strip of partial sums.  The rows after this one are on their way while a row is worked on.
template <typename TX, typename TY, typename TS, bool RES, int G, int KE, int THREADS>
__global__ __launch_bounds__(THREADS) void norm_bwd_rows_kernel(const TY *dy, const TS *s, const TS *ds, TS *dres, TX *dx, NormBwdArgs a) {
  constexpr int E = unit_elements<TX, TY, TS>(), K = KE / E, GROUPS = THREADS / G;
  static_assert(G >= E - 1, "a lane for each element behind the last whole unit");
  constexpr int PARTS = G < 64 ? THREADS / 64 : GROUPS;   // sets of column sums that a block joins
  constexpr int SPAN = G * KE;
  __shared__ float2 smem[G > 64 ? 2 * THREADS / 64 : 1];
  __shared__ float joined[PARTS > 1 ? PARTS * 2 * SPAN : 1];
  const DropState d(a.drop);
  const int C = (int)a.C, whole = C / E, left = C - whole * E;
  const float inv = 1.0f / (float)C;
  const int g = threadIdx.x % G;
  const int64_t stride = (int64_t)gridDim.x * GROUPS;
  int64_t row = (int64_t)blockIdx.x * GROUPS;
  if constexpr (G >= 64) row += __builtin_amdgcn_readfirstlane(threadIdx.x / G);
  else row += threadIdx.x / G;
  const int cl = whole * E + g;
  // gamma: in registers where a wave has the row, in LDS where a block has it (the registers are worth more there)
  constexpr bool SHARED = G > 64;
  __shared__ __align__(16) float gs[SHARED ? G * KE + 8 : 1];
  float gm[SHARED ? 1 : K][E], gml = 1.0f;
  float ag[K][E] = {}, ab[K][E] = {}, agl = 0.0f, abl = 0.0f;
  if constexpr (SHARED) {
    for (int c = threadIdx.x; c < C; c += THREADS) gs[c] = a.gamma ? a.gamma[c] : 1.0f;
    __syncthreads();
    if (g < left) gml = gs[cl];
  } else {
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const int u = g + k * G;
      Unit<float, E> gu;
#pragma unroll
      for (int i = 0; i < E; ++i) gu.set(i, 1.0f);
      if (u < whole && a.gamma) gu.load(a.gamma + u * E);
#pragma unroll
      for (int i = 0; i < E; ++i) gm[k][i] = gu.get(i);
    }
    if (g < left && a.gamma) gml = a.gamma[cl];
  }
  Unit<TY, E> yu[K];
  Unit<TS, E> su[K], eu[K];
  float yl = 0.0f, sl = 0.0f, el = 0.0f;
  RowStats next;
#pragma unroll
  for (int k = 0; k < K; ++k) {
    yu[k].zero();
    su[k].zero();
    eu[k].zero();
  }
  const auto fetch = [&](int64_t r) __attribute__((always_inline)) {
    if (r >= a.N) return;
    next.load(a, r);
    const TY *yr = dy + r * a.pdy;
    const TS *sr = s + r * a.ps;
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (g + k * G < whole) {
        yu[k].load(yr + (g + k * G) * E);
        su[k].load(sr + (g + k * G) * E);
      }
    if (g < left) {
      yl = Elem<TY>::load(yr + cl);
      sl = Elem<TS>::load(sr + cl);
    }
    if constexpr (RES) {
      if (ds) {
        const TS *er = ds + r * a.pds;
#pragma unroll
        for (int k = 0; k < K; ++k)
          if (g + k * G < whole) eu[k].load(er + (g + k * G) * E);
        if (g < left) el = Elem<TS>::load(er + cl);
      }
    }
  };
  int turn = 0;
  fetch(row);
  // (the waves of a block that meet at barriers make the same number of turns)
  for (int64_t first = G > 64 ? (int64_t)blockIdx.x * GROUPS : row; first < a.N; first += stride, row += stride) {
    const bool there_row = row < a.N;
    float h[K][E], gv[K][E], ev[K][E];
    float hl = 0.0f, gl = 0.0f, evl = 0.0f;
    const Normal normal = Normal::of<G>(a, next);
    const float rs = normal.rstd;
    float sg = 0.0f, sgh = 0.0f;
    if (G <= 64 || there_row) {
#pragma unroll
      for (int k = 0; k < K; ++k) {
        const bool there = g + k * G < whole;
        float gk[E];
        if constexpr (SHARED) {
#pragma unroll
          for (int i = 0; i < E; i += 4) *reinterpret_cast<float4 *>(gk + i) = *reinterpret_cast<const float4 *>(gs + (g + k * G) * E + i);
        }
#pragma unroll
        for (int i = 0; i < E; ++i) {
          const float v = yu[k].get(i);
          h[k][i] = there ? normal.h(su[k].get(i)) : 0.0f;
          gv[k][i] = there ? v * (SHARED ? gk[i] : gm[SHARED ? 0 : k][i]) : 0.0f;
          ag[k][i] = fmaf(v, h[k][i], ag[k][i]);
          ab[k][i] += v;
          sg += gv[k][i];
          sgh = fmaf(gv[k][i], h[k][i], sgh);
          if constexpr (RES) ev[k][i] = eu[k].get(i);
        }
      }
      hl = g < left ? normal.h(sl) : 0.0f;
      gl = yl * gml;
      evl = el;
      agl = fmaf(yl, hl, agl);
      abl += yl;
      sg += gl;
      sgh = fmaf(gl, hl, sgh);
    }
    fetch(row + stride);
    const float2 t = group_sum<G>(make_float2(sg, sgh), smem + (G > 64 ? threadIdx.x / G * (2 * G / 64) : 0), turn);
    turn ^= 1;
    if (G > 64 && !there_row) break;                      // (the last turn)
    const float c1 = t.x * inv, c2 = t.y * inv;
#pragma unroll
    for (int k = 0; k < K; ++k) {
      const uint32_t c0 = (uint32_t)(g + k * G) * E;
      float o[E];
#pragma unroll
      for (int i = 0; i < E; ++i) {
        o[i] = rs * (gv[k][i] - c1 - h[k][i] * c2);
        if constexpr (RES) {
          if (ds) o[i] += ev[k][i];
        }
      }
      if constexpr (RES) {
        if (dres) {
          Unit<TS, E> out;
#pragma unroll
          for (int i = 0; i < E; ++i) out.set(i, o[i]);
          if (g + k * G < whole) put_unit<G>(out, dres + row * a.pdr + c0, a.lines);
        }
        if (dx && a.drop.rng) drop_unit<E>(d, c0, (uint32_t)row, o);
      }
      if (!RES || dx) {
        Unit<TX, E> out;
#pragma unroll
        for (int i = 0; i < E; ++i) out.set(i, o[i]);
        if (g + k * G < whole) put_unit<G>(out, dx + row * a.pdx + c0, a.lines);
      }
    }
    if (g < left) {
      float o = rs * (gl - c1 - hl * c2);
      if constexpr (RES) {
        if (ds) o += evl;
        if (dres) Elem<TS>::store(dres + row * a.pdr + cl, o);
        if (dx && a.drop.rng) o = d.apply(o, word_of(d, (uint32_t)cl, (uint32_t)row));
      }
      if (!RES || dx) Elem<TX>::store(dx + row * a.pdx + cl, o);
    }
  }
  if (!a.pg && !a.pb) return;
  float *pg = a.pg ? a.pg + (int64_t)blockIdx.x * a.step : nullptr, *pb = a.pb ? a.pb + (int64_t)blockIdx.x * a.step : nullptr;
  if constexpr (GROUPS == 1) {
#pragma unroll
    for (int k = 0; k < K; ++k)
      if (g + k * G < whole) {
        Unit<float, E> out;
#pragma unroll
        for (int i = 0; i < E; ++i) out.set(i, ag[k][i]);
        if (pg) out.store(pg + (g + k * G) * E);
#pragma unroll
        for (int i = 0; i < E; ++i) out.set(i, ab[k][i]);
        if (pb) out.store(pb + (g + k * G) * E);
      }
    if (g < left) {
      if (pg) pg[cl] = agl;
      if (pb) pb[cl] = abl;
    }
  } else {
    // groups smaller than a wave first join within it
    const auto join = [&](float v) -> float {
#pragma unroll
      for (int o = G; o < 64; o <<= 1) v += __shfl_xor(v, o, 64);
      return v;
    };
    const int part = threadIdx.x / (G < 64 ? 64 : G);
    const bool writes = G >= 64 || (threadIdx.x & 63) < G;
    float *mg = joined + part * SPAN, *mb = joined + (PARTS + part) * SPAN;
#pragma unroll
    for (int k = 0; k < K; ++k)
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const float vg = join(ag[k][i]), vb = join(ab[k][i]);
        if (writes) {
          mg[(g + k * G) * E + i] = vg;
          mb[(g + k * G) * E + i] = vb;
        }
      }
    const float vg = join(agl), vb = join(abl);
    const auto add_up = [&](int c, int at) {
      float sg = joined[at], sb = joined[PARTS * SPAN + at];
#pragma unroll
      for (int p = 1; p < PARTS; ++p) {
        sg += joined[p * SPAN + at];
        sb += joined[(PARTS + p) * SPAN + at];
      }
      if (pg) pg[c] = sg;
      if (pb) pb[c] = sb;
    };
    __syncthreads();
    for (int c = threadIdx.x; c < whole * E; c += THREADS) add_up(c, c);
    if (left > 0) {
      __syncthreads();
      if (writes && g < left) {
        mg[g] = vg;
        mb[g] = vb;
      }
      __syncthreads();
      if ((int)threadIdx.x < left) add_up(whole * E + (int)threadIdx.x, (int)threadIdx.x);
    }
  }
}


// Rows longer than a block holds with their column sums, in two launches.  First the rows' sums of g and g h: a block has a segment of a
// row, so that few rows still fill the chip.
template <typename TY, typename TS>
__global__ __launch_bounds__(256) void norm_bwd_sums_kernel(const TY *dy, const TS *s, NormBwdArgs a) {
  constexpr int E = unit_elements<TY, TS>();
  __shared__ float2 smem[8];
  const int64_t row = (int64_t)blockIdx.z * gridDim.x + blockIdx.x, units = (a.C + E - 1) / E, per = (units + a.segments - 1) / a.segments;
  if (row >= a.N) return;
  const int64_t u0 = blockIdx.y * per, u1 = u0 + per < units ? u0 + per : units;
  const TY *yr = dy + row * a.pdy;
  const TS *sr = s + row * a.ps;
  RowStats stats;
  stats.load(a, row);
  const Normal normal = Normal::of<64>(a, stats);
  float sg = 0.0f, sgh = 0.0f;
  for (int64_t u = u0 + threadIdx.x; u < u1; u += 256) {
    const int64_t c0 = u * E;
    if (c0 + E <= a.C) {
      Unit<TY, E> yu;
      Unit<TS, E> su;
      Unit<float, E> gm;
      yu.load(yr + c0);
      su.load(sr + c0);
      if (a.gamma) gm.load(a.gamma + c0);
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const float g = a.gamma ? yu.get(i) * gm.get(i) : yu.get(i);
        sg += g;
        sgh = fmaf(g, normal.h(su.get(i)), sgh);
      }
    } else {
      for (int64_t c = c0; c < a.C; ++c) {
        const float g = Elem<TY>::load(yr + c) * (a.gamma ? a.gamma[c] : 1.0f);
        sg += g;
        sgh = fmaf(g, normal.h(Elem<TS>::load(sr + c)), sgh);
      }
    }
  }
  const float2 t = group_sum<256>(make_float2(sg, sgh), smem, 0);
  if (threadIdx.x == 0) a.sums[row * a.segments + blockIdx.y] = t;
}

// Then the gradients: a thread has E columns and walks over the neighbouring rows of a strip, R of them in flight together; the column sums need no
// exchange.  What a row's elements have in common comes through LDS (4092 x 8200 bf16 79.1 us where every wave loads the statistics, 75.8).
template <typename TX, typename TY, typename TS, bool RES>
__global__ __launch_bounds__(256) void norm_bwd_wide_kernel(const TY *dy, const TS *s, const TS *ds, TS *dres, TX *dx, NormBwdArgs a) {
  constexpr int E = unit_elements<TX, TY, TS>(), R = 4;
  struct Row {
    float d1, d2, mean, rstd, shift;                     // means of g and g h; what h is made of
  };
  __shared__ Row rows[2][R];
  const int64_t c0 = ((int64_t)blockIdx.x * 256 + threadIdx.x) * E;
  const DropState d(a.drop);
  const float inv = 1.0f / (float)a.C;
  const int n = a.C - c0 < E ? (a.C > c0 ? (int)(a.C - c0) : 0) : E;   // columns of this thread
  const bool all = n == E;
  float gm[E], ag[E] = {}, ab[E] = {};
#pragma unroll
  for (int i = 0; i < E; ++i) gm[i] = a.gamma && i < n ? a.gamma[c0 + i] : 1.0f;
  const int64_t per = (a.N + a.strips - 1) / a.strips, r0 = blockIdx.y * per, r1 = r0 + per < a.N ? r0 + per : a.N;
  for (int64_t first = r0, turn = 0; first < r1; first += R, turn ^= 1) {
    Unit<TY, E> yu[R];
    Unit<TS, E> su[R], eu[R];
    RowStats stats;
    float2 part = make_float2(0.0f, 0.0f);               // sixteen lanes add up the segments of a row
    if (threadIdx.x < 16 * R) {
      const int64_t row = first + threadIdx.x / 16;
      stats.load(a, row < r1 ? row : r1 - 1);
      if (row < r1)
        for (int k = threadIdx.x % 16; k < a.segments; k += 16) {
          const float2 t = a.sums[row * a.segments + k];
          part.x += t.x;
          part.y += t.y;
        }
    }
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int64_t row = first + j < r1 ? first + j : r1 - 1;         // (the last one again, and not used)
      const TY *yr = dy + row * a.pdy + c0;
      const TS *sr = s + row * a.ps + c0, *er = RES && ds ? ds + row * a.pds + c0 : nullptr;
      if (all) {
        yu[j].load(yr);
        su[j].load(sr);
        if (RES && ds) eu[j].load(er);
      } else {
        yu[j].zero();
        su[j].zero();
        eu[j].zero();
#pragma unroll
        for (int i = 0; i < E; ++i)
          if (i < n) {
            yu[j].set(i, Elem<TY>::load(yr + i));
            su[j].set(i, Elem<TS>::load(sr + i));
            if (RES && ds) eu[j].set(i, Elem<TS>::load(er + i));
          }
      }
    }
    if (threadIdx.x < 16 * R) {
      part = make_float2(sum16(part.x), sum16(part.y));
      const Normal normal = Normal::of<16>(a, stats);
      if (threadIdx.x % 16 == 0) rows[turn][threadIdx.x / 16] = Row{part.x * inv, part.y * inv, normal.mean, normal.rstd, normal.shift};
    }
    __syncthreads();                                     // (the other half of `rows` was read before the barrier in between)
#pragma unroll
    for (int j = 0; j < R; ++j) {
      const int64_t row = first + j;
      if (row >= r1) break;
      const Row of = rows[turn][j];
      const Normal normal{of.mean, of.rstd, of.shift};
      float o[E];
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const float v = yu[j].get(i), h = normal.h(su[j].get(i));
        ag[i] = fmaf(v, h, ag[i]);
        ab[i] += v;
        o[i] = of.rstd * (v * gm[i] - of.d1 - h * of.d2);
        if (RES && ds) o[i] += eu[j].get(i);
      }
      const auto put = [&](auto *p) __attribute__((always_inline)) {
        using T = std::remove_pointer_t<decltype(p)>;
        if (all) {
          Unit<T, E> out;
#pragma unroll
          for (int i = 0; i < E; ++i) out.set(i, o[i]);
          out.store_nt(p);
        } else {
#pragma unroll
          for (int i = 0; i < E; ++i)
            if (i < n) Elem<T>::store(p + i, o[i]);
        }
      };
      if constexpr (RES) {
        if (dres) put(dres + row * a.pdr + c0);
        if (dx && a.drop.rng) drop_unit<E>(d, (uint32_t)c0, (uint32_t)row, o);
      }
      if (!RES || dx) put(dx + row * a.pdx + c0);
    }
  }
#pragma unroll
  for (int i = 0; i < E; ++i)
    if (i < n) {
      if (a.pg) a.pg[blockIdx.y * a.step + c0 + i] = ag[i];
      if (a.pb) a.pb[blockIdx.y * a.step + c0 + i] = ab[i];
    }
}

// The strips' sums, 2 C columns of them: a block has 1024 / SLICES columns, a thread every SLICES-th strip of one; the threads' sums are added
// sixteen at a time, the same way at every call.
template <int SLICES>
__global__ __launch_bounds__(1024) void norm_fold_kernel(const float *partial, int strips, int64_t C, float *dgamma, float *dbeta) {
  constexpr int COLS = 1024 / SLICES;
  __shared__ float part[SLICES][COLS + 1];
  const int col = threadIdx.x % COLS, slice = threadIdx.x / COLS;
  const int64_t c0 = block_number() * COLS, c = c0 + col;
  float v = 0.0f;
  if (c < 2 * C) {
#pragma unroll 4
    for (int k = slice; k < strips; k += SLICES) v += partial[k * 2 * C + c];
  }
  part[slice][col] = v;
  __syncthreads();
  if (threadIdx.x < COLS * 16) {
    const int cc = threadIdx.x >> 4, k = threadIdx.x & 15;
    float t = part[k][cc];
#pragma unroll
    for (int q = 1; q < SLICES / 16; ++q) t += part[k + 16 * q][cc];
    t = sum16(t);
    const int64_t o = c0 + cc;
    if (k == 0 && o < 2 * C) {
      if (o < C) {
        if (dgamma) dgamma[o] = t;
      } else if (dbeta) {
        dbeta[o - C] = t;
      }
    }
  }
}

chn_status check_vector(const chn_array *v, const char *name, int64_t n, bool is_output) {
  CHN_TRY(validate(v, name, is_output));
  if (v->dtype != CHN_F32) return fail(CHN_ERR_DTYPE, "norm: %s must be F32", name);
  if (v->ndim != 1 || v->shape[0] != n) return fail(CHN_ERR_SHAPE, "norm: %s must have shape (%lld,)", name, (long long)n);
  if (!is_contiguous(v)) return fail(CHN_ERR_STRIDE, "norm: %s must be contiguous", name);
  return CHN_OK;
}

// The rows' means: (n,), or (n,2) with what their rounding left.
chn_status check_mean(const chn_array *m, int64_t n, bool is_output, int *parts) {
  *parts = 1;
  if (!m || m->ndim != 2) return check_vector(m, "mean", n, is_output);
  CHN_TRY(validate(m, "mean", is_output));
  if (m->dtype != CHN_F32) return fail(CHN_ERR_DTYPE, "norm: mean must be F32");
  if (m->shape[0] != n || m->shape[1] != 2) return fail(CHN_ERR_SHAPE, "norm: mean must have shape (%lld,) or (%lld, 2)", (long long)n, (long long)n);
  if (!is_contiguous(m)) return fail(CHN_ERR_STRIDE, "norm: mean must be contiguous");
  *parts = 2;
  return CHN_OK;
}

// A matrix of rows: F32 or BF16, unit stride along the last axis; N < 0: its own shape is taken.
chn_status check_matrix(const chn_array *m, const char *name, bool is_output, int64_t *N, int64_t *C, int64_t *pitch) {
  CHN_TRY(validate(m, name, is_output));
  if (!is_float(m->dtype)) return fail(CHN_ERR_DTYPE, "norm: %s must be F32 or BF16", name);
  int64_t n, c;
  CHN_TRY(row_major_2d(m, name, &n, &c, pitch));
  if (*N >= 0 && (n != *N || c != *C)) return fail(CHN_ERR_SHAPE, "norm: %s must have shape (%lld, %lld)", name, (long long)*N, (long long)*C);
  *N = n;
  *C = c;
  if (n > 0 && c == 0) return fail(CHN_ERR_SHAPE, "norm: %s has rows without elements", name);
  if (n > 0x7fffffffLL || c > 0x7fffffffLL) return fail(CHN_ERR_SHAPE, "norm: %s has more than 2^31 - 1 rows or columns", name);
  return CHN_OK;
}

// Whether rows of a matrix (NULL: no matter) begin lines of 128 bytes.
bool at_lines(const chn_array *m, int64_t pitch) {
  return !m || (reinterpret_cast<uintptr_t>(m->data) | (uintptr_t)(pitch * dtype_size(m->dtype))) % 128 == 0;
}

const float *floats(const chn_array *v) { return v ? static_cast<const float *>(v->data) : nullptr; }
float *floats_out(const chn_array *v) { return v ? static_cast<float *>(v->data) : nullptr; }

template <typename TX, typename TY, typename TS, bool RES>
void launch_fwd(const TX *x, const TS *residual, TS *s, TY *y, const NormArgs &a, hipStream_t st) {
  constexpr int E = unit_elements<TX, TY, TS>();
  const int64_t held = a.C / E * E;                      // (the elements behind the last whole unit come on top)
  // As few lanes as hold the row, since the others have nothing in flight (us by these / by twice to four times as many: 524288 x 64 fp32 39 / 43, bf16
  // 25 / 39, 127100 x 264 bf16 28 / 43, 30504 x 1100 bf16 29 / 42, 8176 x 4104 bf16 29 / 52), but stores of at least a line at once (524288 x 64 fp32
  // with residual 82, by four lanes 126).
#define CHN_ROWS(G, KE)                                                                                                             \
  hipLaunchKernelGGL((norm_fwd_rows_kernel<TX, TY, TS, RES, G, KE>), grid_of((a.N + (G > 64 ? 1 : 256 / G) - 1) / (G > 64 ? 1 : 256 / G)),    \
                     dim3(G > 64 ? G : 256), 0, st, x, residual, s, y, a)
  if constexpr (E == 4)                                  // (four lanes have no room for up to seven elements behind the last unit)
    if (held <= 4 * 8) {
      CHN_ROWS(4, 8);
      return;
    }
  if (held <= 8 * 16) CHN_ROWS(8, 16);
  else if (held <= 16 * 16) CHN_ROWS(16, 16);
  else if (held <= 32 * 16) CHN_ROWS(32, 16);
  else if (held <= 64 * 16) CHN_ROWS(64, 16);
  else if (held <= 128 * 16) CHN_ROWS(128, 16);
  else if (held <= 256 * 16) CHN_ROWS(256, 16);
  else if (held <= 512 * 16) CHN_ROWS(512, 16);
  else if (held <= 1024 * 16) CHN_ROWS(1024, 16);
  else if (held <= 1024 * 32) CHN_ROWS(1024, 32);
  else hipLaunchKernelGGL((norm_fwd_wide_kernel<TX, TY, TS, RES>), grid_of(a.N), dim3(1024), 0, st, x, residual, s, y, a);
#undef CHN_ROWS
}

chn_status norm_fwd(const chn_array *x, const chn_array *residual, double ratio, const chn_array *rng, int64_t site, const chn_array *gamma,
                    const chn_array *beta, double eps, const chn_array *s, const chn_array *y, const chn_array *mean, const chn_array *rstd,
                    bool res, const char *what, hipStream_t st) {
  NormArgs a{};
  a.N = -1;
  CHN_TRY(check_matrix(x, "x", false, &a.N, &a.C, &a.px));
  if (res) {
    CHN_TRY(check_matrix(residual, "residual", false, &a.N, &a.C, &a.pr));
    CHN_TRY(check_matrix(s, "sum", true, &a.N, &a.C, &a.ps));
    if (residual->dtype != s->dtype) return fail(CHN_ERR_DTYPE, "%s: residual and sum must have one dtype", what);
  }
  CHN_TRY(check_matrix(y, "y", true, &a.N, &a.C, &a.py));
  if (res && x->dtype != y->dtype) return fail(CHN_ERR_DTYPE, "%s: x and y must have one dtype", what);
  if (gamma) CHN_TRY(check_vector(gamma, "gamma", a.C, false));
  if (beta) CHN_TRY(check_vector(beta, "beta", a.C, false));
  if (mean) CHN_TRY(check_mean(mean, a.N, true, &a.mean_parts));
  if (rstd) CHN_TRY(check_vector(rstd, "rstd", a.N, true));
  if (!(eps >= 0.0) || eps > 3.4e38) return fail(CHN_ERR_OP, "%s: eps %g must be finite and not negative", what, eps);
  CHN_TRY(check_drop(rng, ratio, site, a.N, a.C, what, &a.drop));
  if (a.N == 0) return CHN_OK;
  a.eps = (float)eps;
  a.lines = at_lines(s, a.ps) && at_lines(y, a.py);
  a.gamma = floats(gamma);
  a.beta = floats(beta);
  a.mean = floats_out(mean);
  a.rstd = floats_out(rstd);
  const bool x32 = x->dtype == CHN_F32, y32 = y->dtype == CHN_F32;
#define CHN_GO(TX, TY, TS, RES)                                                                                                      \
  launch_fwd<TX, TY, TS, RES>(static_cast<const TX *>(x->data), residual ? static_cast<const TS *>(residual->data) : nullptr,          \
                              s ? static_cast<TS *>(s->data) : nullptr, static_cast<TY *>(y->data), a, st)
  if (res) {
    const bool s32 = s->dtype == CHN_F32;
    if (x32 && s32) CHN_GO(float, float, float, true);
    else if (x32) CHN_GO(float, float, bf16_raw, true);
    else if (s32) CHN_GO(bf16_raw, bf16_raw, float, true);
    else CHN_GO(bf16_raw, bf16_raw, bf16_raw, true);
  } else {
    if (x32 && y32) CHN_GO(float, float, float, false);
    else if (x32) CHN_GO(float, bf16_raw, float, false);
    else if (y32) CHN_GO(bf16_raw, float, bf16_raw, false);
    else CHN_GO(bf16_raw, bf16_raw, bf16_raw, false);
  }
#undef CHN_GO
  return check_launch(what);
}

// What the backward pass leaves in its workspace: strips of column sums, and for rows longer than a block holds the rows' sums behind them.
constexpr int64_t kHeld = 1024 * 8;                      // elements of a row that a block holds
constexpr int64_t kStrips = 256;                         // one for each compute unit
int64_t strips_of(int64_t N, int64_t C) {
  if (C <= kHeld) return N < kStrips ? (N > 0 ? N : 1) : kStrips;
  // wide rows: at least four rows to a strip, so that their sums stay a fraction of what is read
  const int64_t n = (N + 3) / 4;
  return n < 64 ? (n > 0 ? n : 1) : 64;
}
int segments_of(int64_t N, int64_t C) {
  if (C <= kHeld) return 0;
  const int64_t want = N > 0 ? (1024 + N - 1) / N : 1, most = (C + 4095) / 4096;
  return (int)(want < most ? want : most);
}
size_t bwd_sums_bytes(int64_t N, int64_t C) { return ((size_t)(N * segments_of(N, C)) * sizeof(float2) + 255) / 256 * 256; }
size_t bwd_workspace(int64_t N, int64_t C) { return bwd_sums_bytes(N, C) + (size_t)(strips_of(N, C) * 2 * C) * sizeof(float); }

// Where n blocks leave their column sums.  (One block has no strips to fold: 8 x 64 fp32 6.7 -> 5.2 us, 8 x 1000 5.8 -> 4.0.)
void place_sums(NormBwdArgs &a, int64_t n) {
  a.pg = n == 1 ? a.dgamma : a.partial;
  a.pb = n == 1 ? a.dbeta : a.partial ? a.partial + a.C : nullptr;
  a.step = 2 * a.C;
}

template <typename TX, typename TY, typename TS, bool RES, int G, int KE, int THREADS>
int64_t launch_bwd_rows(const TY *dy, const TS *s, const TS *ds, TS *dres, TX *dx, NormBwdArgs &a, hipStream_t st) {
  const int64_t blocks = (a.N + THREADS / G - 1) / (THREADS / G), n = blocks > 0 && blocks < a.strips ? blocks : a.strips;   // (a strip of the workspace each)
  place_sums(a, n);
  hipLaunchKernelGGL((norm_bwd_rows_kernel<TX, TY, TS, RES, G, KE, THREADS>), dim3((unsigned)n), dim3(THREADS), 0, st, dy, s, ds, dres, dx, a);
  return n;
}

// Returns the number of strips it leaves.
template <typename TX, typename TY, typename TS, bool RES>
int64_t launch_bwd(const TY *dy, const TS *s, const TS *ds, TS *dres, TX *dx, NormBwdArgs &a, hipStream_t st) {
  constexpr int E = unit_elements<TX, TY, TS>();
#define CHN_ROWS(G, KE, THREADS) return launch_bwd_rows<TX, TY, TS, RES, G, KE, THREADS>(dy, s, ds, dres, dx, a, st)
  // As in the forward pass; blocks of 960 for what leaves much of 1024 idle (us / by the next larger group: 127100 x 264 bf16 45 / 68,
  // 30504 x 1100 50 / 63, 16320 x 2056 44 / 54); beyond 4096 a block for each row (6710 x 5000 fp32 69, 512 threads with sixteen elements 83).
  if constexpr (E == 4)
    if (a.C <= 4 * 8) CHN_ROWS(4, 8, 512);
  if (a.C <= 8 * 16) CHN_ROWS(8, 16, 512);
  if (a.C <= 16 * 16) CHN_ROWS(16, 16, 512);
  if (a.C <= 32 * 16) CHN_ROWS(32, 16, 512);
  if (a.C <= 64 * 16) CHN_ROWS(64, 16, 512);
  if (a.C <= 192 * 8) CHN_ROWS(192, 8, 960);
  if (a.C <= 256 * 8) CHN_ROWS(256, 8, 1024);
  if (a.C <= 320 * 8) CHN_ROWS(320, 8, 960);
  if (a.C <= 512 * 8) CHN_ROWS(512, 8, 1024);
  if (a.C <= kHeld) CHN_ROWS(1024, 8, 1024);
#undef CHN_ROWS
  place_sums(a, a.strips);
  if (a.N > 0)
    hipLaunchKernelGGL((norm_bwd_sums_kernel<TY, TS>), dim3(grid_of(a.N).x, (unsigned)a.segments, grid_of(a.N).y), dim3(256), 0, st, dy, s, a);
  hipLaunchKernelGGL((norm_bwd_wide_kernel<TX, TY, TS, RES>), dim3((unsigned)((a.C + 256 * E - 1) / (256 * E)), (unsigned)a.strips), dim3(256), 0, st,
                     dy, s, ds, dres, dx, a);
  return a.strips;
}

chn_status norm_bwd(const chn_array *dy, const chn_array *ds, const chn_array *s, const chn_array *mean, const chn_array *rstd, const chn_array *gamma,
                    double ratio, const chn_array *rng, int64_t site, const chn_array *dres, const chn_array *dx, const chn_array *dgamma,
                    const chn_array *dbeta, void *ws, size_t ws_bytes, bool res, const char *what, hipStream_t st) {
  NormBwdArgs a{};
  a.N = -1;
  CHN_TRY(check_matrix(s, res ? "sum" : "x", false, &a.N, &a.C, &a.ps));
  CHN_TRY(check_matrix(dy, "dy", false, &a.N, &a.C, &a.pdy));
  if (res) {
    if (ds) CHN_TRY(check_matrix(ds, "dsum", false, &a.N, &a.C, &a.pds));
    if (dres) CHN_TRY(check_matrix(dres, "dresidual", true, &a.N, &a.C, &a.pdr));
    if (dx) CHN_TRY(check_matrix(dx, "dx", true, &a.N, &a.C, &a.pdx));
    if (ds && ds->dtype != s->dtype) return fail(CHN_ERR_DTYPE, "%s: dsum must have sum's dtype", what);
    if (dres && dres->dtype != s->dtype) return fail(CHN_ERR_DTYPE, "%s: dresidual must have sum's dtype", what);
    if (dx && dx->dtype != dy->dtype) return fail(CHN_ERR_DTYPE, "%s: dx must have dy's dtype", what);
  } else {
    CHN_TRY(check_matrix(dx, "dx", true, &a.N, &a.C, &a.pdx));
    if (dx->dtype != s->dtype) return fail(CHN_ERR_DTYPE, "%s: dx must have x's dtype", what);
  }
  CHN_TRY(check_mean(mean, a.N, false, &a.mean_parts));
  CHN_TRY(check_vector(rstd, "rstd", a.N, false));
  if (gamma) CHN_TRY(check_vector(gamma, "gamma", a.C, false));
  if (dgamma) CHN_TRY(check_vector(dgamma, "dgamma", a.C, true));
  if (dbeta) CHN_TRY(check_vector(dbeta, "dbeta", a.C, true));
  CHN_TRY(check_drop(rng, ratio, site, a.N, a.C, what, &a.drop));
  if (a.C == 0) return CHN_OK;
  a.gamma = floats(gamma);
  a.mean = floats(mean);
  a.rstd = floats(rstd);
  a.lines = at_lines(dres, a.pdr) && at_lines(dx, a.pdx);
  a.strips = strips_of(a.N, a.C);
  const bool sums = dgamma || dbeta;
  a.segments = segments_of(a.N, a.C);
  if (!sums && (a.N == 0 || (!dx && !dres))) return CHN_OK;
  const size_t rows_bytes = bwd_sums_bytes(a.N, a.C);
  CHN_TRY(check_ws(ws, ws_bytes, sums ? bwd_workspace(a.N, a.C) : rows_bytes, what));
  a.sums = static_cast<float2 *>(ws);
  a.dgamma = floats_out(dgamma);
  a.dbeta = floats_out(dbeta);
  if (sums) a.partial = reinterpret_cast<float *>(static_cast<char *>(ws) + rows_bytes);
  const bool y32 = dy->dtype == CHN_F32, s32 = s->dtype == CHN_F32;
  int64_t strips = 0;
#define CHN_GO(TX, TY, TS, RES)                                                                                                     \
  strips = launch_bwd<TX, TY, TS, RES>(static_cast<const TY *>(dy->data), static_cast<const TS *>(s->data),                          \
                                       ds ? static_cast<const TS *>(ds->data) : nullptr, dres ? static_cast<TS *>(dres->data) : nullptr, \
                                       dx ? static_cast<TX *>(dx->data) : nullptr, a, st)
  if (res) {
    if (y32 && s32) CHN_GO(float, float, float, true);
    else if (y32) CHN_GO(float, float, bf16_raw, true);
    else if (s32) CHN_GO(bf16_raw, bf16_raw, float, true);
    else CHN_GO(bf16_raw, bf16_raw, bf16_raw, true);
  } else {
    if (y32 && s32) CHN_GO(float, float, float, false);
    else if (y32) CHN_GO(bf16_raw, float, bf16_raw, false);
    else if (s32) CHN_GO(float, bf16_raw, float, false);
    else CHN_GO(bf16_raw, bf16_raw, bf16_raw, false);
  }
#undef CHN_GO
  CHN_TRY(check_launch(what));
  if (a.partial && strips > 1) {
    // (64 columns a block for few strips, sixteen for many: 99 x 20011 with 25 strips 6.0 us with sixteen)
    if (strips <= 64)
      hipLaunchKernelGGL(norm_fold_kernel<16>, grid_of((2 * a.C + 63) / 64), dim3(1024), 0, st, a.partial, (int)strips, a.C, a.dgamma, a.dbeta);
    else
      hipLaunchKernelGGL(norm_fold_kernel<64>, grid_of((2 * a.C + 15) / 16), dim3(1024), 0, st, a.partial, (int)strips, a.C, a.dgamma, a.dbeta);
  }
  return check_launch(what);
}

}  // namespace
}  // namespace chn

extern "C" {

chn_status chn_layer_norm_fwd(const chn_array *x, const chn_array *gamma, const chn_array *beta, double eps, const chn_array *y,
                              const chn_array *mean, const chn_array *rstd, chn_stream stream) {
  return chn::norm_fwd(x, nullptr, 0.0, nullptr, 0, gamma, beta, eps, nullptr, y, mean, rstd, false, "layer_norm_fwd", chn::as_stream(stream));
}

size_t chn_layer_norm_bwd_workspace_bytes(const chn_array *x) {
  if (!x || x->ndim != 2 || x->shape[0] < 0 || x->shape[1] < 0) return 0;
  return chn::bwd_workspace(x->shape[0], x->shape[1]);
}

chn_status chn_layer_norm_bwd(const chn_array *dy, const chn_array *x, const chn_array *mean, const chn_array *rstd, const chn_array *gamma,
                              const chn_array *dx, const chn_array *dgamma, const chn_array *dbeta, void *ws, size_t ws_bytes, chn_stream stream) {
  return chn::norm_bwd(dy, nullptr, x, mean, rstd, gamma, 0.0, nullptr, 0, nullptr, dx, dgamma, dbeta, ws, ws_bytes, false, "layer_norm_bwd",
                       chn::as_stream(stream));
}

chn_status chn_residual_norm_fwd(const chn_array *x, const chn_array *residual, double ratio, const chn_array *rng, int64_t site,
                                 const chn_array *gamma, const chn_array *beta, double eps, const chn_array *sum, const chn_array *y,
                                 const chn_array *mean, const chn_array *rstd, chn_stream stream) {
  return chn::norm_fwd(x, residual, ratio, rng, site, gamma, beta, eps, sum, y, mean, rstd, true, "residual_norm_fwd", chn::as_stream(stream));
}

chn_status chn_residual_norm_bwd(const chn_array *dy, const chn_array *dsum, const chn_array *sum, const chn_array *mean, const chn_array *rstd,
                                 const chn_array *gamma, double ratio, const chn_array *rng, int64_t site, const chn_array *dresidual,
                                 const chn_array *dx, const chn_array *dgamma, const chn_array *dbeta, void *ws, size_t ws_bytes, chn_stream stream) {
  return chn::norm_bwd(dy, dsum, sum, mean, rstd, gamma, ratio, rng, site, dresidual, dx, dgamma, dbeta, ws, ws_bytes, true, "residual_norm_bwd",
                       chn::as_stream(stream));
}

}  // extern "C"
