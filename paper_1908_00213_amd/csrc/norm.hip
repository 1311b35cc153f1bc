// chn_layer_norm_fwd / _bwd, chn_residual_norm_fwd / _bwd: normalisation of rows, by itself or of residual + dropout(x).
//
//   forward   s = residual + dropout(x), rounded to the stream's type        (residual_norm; layer_norm: s is x)
//             mean = sum s / C    rstd = 1 / sqrt(sum (s - mean)^2 / C + eps)    y = (s - mean) rstd gamma + beta
//   backward  h = (s - mean) rstd    g = dy gamma    dn = rstd (g - sum g / C - h sum(g h) / C)
//             layer_norm: dx = dn;   residual_norm: dresidual = dn + ds, dx = dropout(dn + ds) with the forward's mask
//             dgamma = sum over rows of dy h      dbeta = sum over rows of dy
//
// All sums and statistics are fp32; the mean is corrected by the mean of what is left after its subtraction, so that rows whose mean
// is far larger than their spread keep their digits.
#include "philox.h"

namespace chn {
namespace {

struct NormArgs {
  int64_t N, C;
  int64_t px, pr, ps, py;            // row pitches in elements
  float eps;
  const float *gamma, *beta;
  float *mean, *rstd;
  DropArgs drop;
};

__device__ __forceinline__ float block_sum(float v, float *smem) {
  v = wave_sum(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) smem[threadIdx.x >> 6] = v;
  __syncthreads();
  return smem[0] + smem[1] + smem[2] + smem[3];
}

// TL: the layer's type (x and y); TS: the stream's (residual and s); RES: s = residual + dropout(x) is formed and stored first
template <typename TX, typename TY, typename TS, bool RES>
__global__ __launch_bounds__(256) void norm_fwd_kernel(const TX *x, const TS *residual, TS *s, TY *y, NormArgs a) {
  __shared__ float smem[4];
  const DropState d(a.drop);
  const float inv = 1.0f / (float)a.C;
  for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
    float sum = 0.0f;
    if constexpr (RES) {
      for (int64_t c0 = threadIdx.x * 4; c0 < a.C; c0 += 1024) {
        Philox4 w{{~0u, ~0u, ~0u, ~0u}};
        if (a.drop.rng) w = d.words((uint32_t)(c0 >> 2), (uint32_t)row);
        for (int j = 0; j < 4 && c0 + j < a.C; ++j) {
          const float v = add_rounded(Elem<TS>::load(residual + row * a.pr + c0 + j), d.apply(Elem<TX>::load(x + row * a.px + c0 + j), w.w[j]));
          Elem<TS>::store(s + row * a.ps + c0 + j, v);
        }
      }
    }
    const auto at = [&](int64_t c) -> float {
      if constexpr (RES) return Elem<TS>::load(s + row * a.ps + c);
      else return Elem<TX>::load(x + row * a.px + c);
    };
    // (a thread reads the elements that it stored itself)
    const auto each = [&](auto f) {
      for (int64_t c0 = threadIdx.x * 4; c0 < a.C; c0 += 1024)
        for (int j = 0; j < 4 && c0 + j < a.C; ++j) f(c0 + j);
    };
    each([&](int64_t c) { sum += at(c); });
    const float m0 = block_sum(sum, smem) * inv;
    float dev = 0.0f, sq = 0.0f;
    each([&](int64_t c) { const float t = at(c) - m0; dev += t; sq += t * t; });
    const float m1 = block_sum(dev, smem) * inv;
    const float var = fmaxf(block_sum(sq, smem) * inv - m1 * m1, 0.0f);
    const float rstd = 1.0f / sqrtf(var + a.eps);
    if (threadIdx.x == 0) {
      if (a.mean) a.mean[row] = m0 + m1;
      if (a.rstd) a.rstd[row] = rstd;
    }
    each([&](int64_t c) {
      const float h = ((at(c) - m0) - m1) * rstd;
      Elem<TY>::store(y + row * a.py + c, h * (a.gamma ? a.gamma[c] : 1.0f) + (a.beta ? a.beta[c] : 0.0f));
    });
  }
}

struct NormBwdArgs {
  int64_t N, C;
  int64_t pdy, ps, pds, pdr, pdx;
  const float *gamma, *mean, *rstd;
  float *partial;                    // [strips][2][C] or NULL
  int64_t strips;
  DropArgs drop;
};

// Column sums of dy h and dy over a strip of rows: strip k takes rows k, k + strips, ...
template <typename TY, typename TS>
__global__ __launch_bounds__(256) void norm_partial_kernel(const TY *dy, const TS *s, NormBwdArgs a) {
  const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (c >= a.C) return;
  float sg = 0.0f, sb = 0.0f;
  for (int64_t row = blockIdx.y; row < a.N; row += a.strips) {
    const float g = Elem<TY>::load(dy + row * a.pdy + c);
    sg += g * ((Elem<TS>::load(s + row * a.ps + c) - a.mean[row]) * a.rstd[row]);
    sb += g;
  }
  a.partial[(blockIdx.y * 2) * a.C + c] = sg;
  a.partial[(blockIdx.y * 2 + 1) * a.C + c] = sb;
}

// The strips' sums added in their order.
__global__ __launch_bounds__(256) void norm_fold_kernel(const float *partial, int64_t strips, int64_t C, float *dgamma, float *dbeta) {
  const int64_t c = (int64_t)blockIdx.x * 256 + threadIdx.x;
  if (c >= C) return;
  float sg = 0.0f, sb = 0.0f;
  for (int64_t k = 0; k < strips; ++k) {
    sg += partial[(k * 2) * C + c];
    sb += partial[(k * 2 + 1) * C + c];
  }
  if (dgamma) dgamma[c] = sg;
  if (dbeta) dbeta[c] = sb;
}

template <typename TX, typename TY, typename TS, bool RES>
__global__ __launch_bounds__(256) void norm_bwd_kernel(const TY *dy, const TS *s, const TS *ds, TS *dres, TX *dx, NormBwdArgs a) {
  __shared__ float smem[4];
  const DropState d(a.drop);
  const float inv = 1.0f / (float)a.C;
  for (int64_t row = blockIdx.x; row < a.N; row += gridDim.x) {
    const float mean = a.mean[row], rstd = a.rstd[row];
    float sg = 0.0f, sgh = 0.0f;
    for (int64_t c = threadIdx.x; c < a.C; c += 256) {
      const float g = Elem<TY>::load(dy + row * a.pdy + c) * (a.gamma ? a.gamma[c] : 1.0f);
      sg += g;
      sgh += g * ((Elem<TS>::load(s + row * a.ps + c) - mean) * rstd);
    }
    const float c1 = block_sum(sg, smem) * inv, c2 = block_sum(sgh, smem) * inv;
    for (int64_t c0 = threadIdx.x * 4; c0 < a.C; c0 += 1024) {
      Philox4 w{{~0u, ~0u, ~0u, ~0u}};
      if (RES && a.drop.rng && dx) w = d.words((uint32_t)(c0 >> 2), (uint32_t)row);
      for (int j = 0; j < 4 && c0 + j < a.C; ++j) {
        const int64_t c = c0 + j;
        const float g = Elem<TY>::load(dy + row * a.pdy + c) * (a.gamma ? a.gamma[c] : 1.0f);
        const float h = (Elem<TS>::load(s + row * a.ps + c) - mean) * rstd;
        float v = rstd * (g - c1 - h * c2);
        if constexpr (RES) {
          if (ds) v += Elem<TS>::load(ds + row * a.pds + c);
          if (dres) Elem<TS>::store(dres + row * a.pdr + c, v);
          if (dx) Elem<TX>::store(dx + row * a.pdx + c, d.apply(v, w.w[j]));
        } else {
          Elem<TX>::store(dx + row * a.pdx + c, v);
        }
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
  return CHN_OK;
}

const float *floats(const chn_array *v) { return v ? static_cast<const float *>(v->data) : nullptr; }
float *floats_out(const chn_array *v) { return v ? static_cast<float *>(v->data) : nullptr; }

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
  if (mean) CHN_TRY(check_vector(mean, "mean", a.N, true));
  if (rstd) CHN_TRY(check_vector(rstd, "rstd", a.N, true));
  if (!(eps >= 0.0) || eps > 3.4e38) return fail(CHN_ERR_OP, "%s: eps %g must be finite and not negative", what, eps);
  CHN_TRY(check_drop(rng, ratio, site, a.N, a.C, what, &a.drop));
  if (a.N == 0) return CHN_OK;
  a.eps = (float)eps;
  a.gamma = floats(gamma);
  a.beta = floats(beta);
  a.mean = floats_out(mean);
  a.rstd = floats_out(rstd);
  const dim3 grid((unsigned)(a.N < (1 << 20) ? a.N : (1 << 20)));
  const bool x32 = x->dtype == CHN_F32, y32 = y->dtype == CHN_F32;
#define CHN_GO(TX, TY, TS, RES)                                                                                                        \
  hipLaunchKernelGGL((norm_fwd_kernel<TX, TY, TS, RES>), grid, dim3(256), 0, st, static_cast<const TX *>(x->data),                      \
                     residual ? static_cast<const TS *>(residual->data) : nullptr, s ? static_cast<TS *>(s->data) : nullptr,            \
                     static_cast<TY *>(y->data), a)
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

int64_t strips_of(int64_t N) { return N < 64 ? (N > 0 ? N : 1) : 64; }

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
  CHN_TRY(check_vector(mean, "mean", a.N, false));
  CHN_TRY(check_vector(rstd, "rstd", a.N, false));
  if (gamma) CHN_TRY(check_vector(gamma, "gamma", a.C, false));
  if (dgamma) CHN_TRY(check_vector(dgamma, "dgamma", a.C, true));
  if (dbeta) CHN_TRY(check_vector(dbeta, "dbeta", a.C, true));
  CHN_TRY(check_drop(rng, ratio, site, a.N, a.C, what, &a.drop));
  if (a.C == 0) return CHN_OK;
  a.gamma = floats(gamma);
  a.mean = floats(mean);
  a.rstd = floats(rstd);
  a.strips = strips_of(a.N);
  if (dgamma || dbeta) {
    CHN_TRY(check_ws(ws, ws_bytes, (size_t)(a.strips * 2 * a.C * 4), what));
    a.partial = static_cast<float *>(ws);
  }
  const bool y32 = dy->dtype == CHN_F32, s32 = s->dtype == CHN_F32;
  const unsigned cb = (unsigned)((a.C + 255) / 256);
  if (a.partial) {
    const dim3 grid(cb, (unsigned)a.strips);
#define CHN_GO(TY, TS) \
  hipLaunchKernelGGL((norm_partial_kernel<TY, TS>), grid, dim3(256), 0, st, static_cast<const TY *>(dy->data), static_cast<const TS *>(s->data), a)
    if (y32 && s32) CHN_GO(float, float);
    else if (y32) CHN_GO(float, bf16_raw);
    else if (s32) CHN_GO(bf16_raw, float);
    else CHN_GO(bf16_raw, bf16_raw);
#undef CHN_GO
    hipLaunchKernelGGL(norm_fold_kernel, dim3(cb), dim3(256), 0, st, a.partial, a.strips, a.C, floats_out(dgamma), floats_out(dbeta));
    CHN_TRY(check_launch(what));
  }
  if (a.N == 0 || (!dx && !dres)) return CHN_OK;
  const dim3 grid((unsigned)(a.N < (1 << 20) ? a.N : (1 << 20)));
#define CHN_GO(TX, TY, TS, RES)                                                                                                      \
  hipLaunchKernelGGL((norm_bwd_kernel<TX, TY, TS, RES>), grid, dim3(256), 0, st, static_cast<const TY *>(dy->data),                   \
                     static_cast<const TS *>(s->data), ds ? static_cast<const TS *>(ds->data) : nullptr,                              \
                     dres ? static_cast<TS *>(dres->data) : nullptr, dx ? static_cast<TX *>(dx->data) : nullptr, a)
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
  return (size_t)(chn::strips_of(x->shape[0]) * 2 * x->shape[1] * 4);
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
