// chn_dropout, chn_rng_advance: dropout whose mask is drawn from a counter-based generator and never stored.
//
// y = (residual +) [word >= threshold] * x / (1 - ratio), the word of element (row, col) from philox.h.  Nothing is kept for the
// backward pass: the gradient of x is the same call on the gradient of y.
//
// The leading dimensions of the arrays are merged where all of them allow it; what is left are rows with a list of strides.
#include "philox.h"

namespace chn {
namespace {

constexpr int kMaxLead = CHN_MAX_NDIM - 1;

struct DropShape {
  int lead;                          // leading dimensions after merging, outermost first
  int64_t rows, cols, units;         // units: columns / 4, rounded up
  uint32_t n[kMaxLead];
  int64_t sx[kMaxLead], sr[kMaxLead], sy[kMaxLead];   // elements
  int64_t cx, cr, cy;                // strides along the last axis
};

// One thread per four columns: any strides.
template <typename TX, typename TY>
__global__ __launch_bounds__(256) void dropout_kernel(const TX *x, const TY *residual, TY *y, DropShape s, DropArgs a) {
  const DropState d(a);
  const int64_t total = s.rows * s.units;
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < total; i += (int64_t)gridDim.x * 256) {
    const int64_t row = i / s.units, unit = i - row * s.units;
    int64_t ox = 0, orr = 0, oy = 0;
    uint32_t left = (uint32_t)row;
    for (int k = s.lead - 1; k >= 0; --k) {
      const uint32_t q = left / s.n[k], at = left - q * s.n[k];
      left = q;
      ox += at * s.sx[k];
      orr += at * s.sr[k];
      oy += at * s.sy[k];
    }
    Philox4 w{{~0u, ~0u, ~0u, ~0u}};
    if (a.rng) w = d.words((uint32_t)unit, (uint32_t)row);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const int64_t c = unit * 4 + j;
      if (c >= s.cols) break;
      float v = d.apply(Elem<TX>::load(x + ox + c * s.cx), w.w[j]);
      if (residual) v = add_rounded(Elem<TY>::load(residual + orr + c * s.cr), v);
      Elem<TY>::store(y + oy + c * s.cy, v);
    }
  }
}

__global__ void rng_advance_kernel(int64_t *rng, int64_t steps) {
  if (threadIdx.x == 0) rng[1] = (int64_t)((uint64_t)rng[1] + (uint64_t)steps);
}

// The rows and strides of a call.  Without elements nothing is filled in.
chn_status plan(const chn_array *x, const chn_array *r, const chn_array *y, DropShape *s) {
  *s = DropShape{};
  const int nd = x->ndim;
  s->rows = 1;
  s->cols = nd ? x->shape[nd - 1] : 1;
  for (int k = 0; k + 1 < nd; ++k) s->rows *= x->shape[k];
  s->units = (s->cols + 3) / 4;
  if (s->rows > 0xffffffffLL) return fail(CHN_ERR_SHAPE, "dropout: more than 2^32 rows");
  if (s->rows == 0 || s->cols == 0) return CHN_OK;
  const int bx = dtype_size(x->dtype), by = dtype_size(y->dtype);
  const auto stride = [](const chn_array *a, int k, int b) { return a ? a->strides[k] / b : 0; };
  if (nd) {
    s->cx = stride(x, nd - 1, bx);
    s->cr = stride(r, nd - 1, by);
    s->cy = stride(y, nd - 1, by);
    if (s->cols == 1) s->cx = s->cr = s->cy = 1;             // (never stepped along)
  } else {
    s->cx = s->cr = s->cy = 1;
  }
  for (int k = 0; k + 1 < nd; ++k) {
    if (x->shape[k] == 1) continue;
    const int64_t n = x->shape[k], sx = stride(x, k, bx), sr = stride(r, k, by), sy = stride(y, k, by);
    const int p = s->lead - 1;
    if (p >= 0 && s->sx[p] == n * sx && s->sr[p] == n * sr && s->sy[p] == n * sy) {
      s->n[p] *= (uint32_t)n;
      s->sx[p] = sx;
      s->sr[p] = sr;
      s->sy[p] = sy;
    } else {
      s->n[s->lead] = (uint32_t)n;
      s->sx[s->lead] = sx;
      s->sr[s->lead] = sr;
      s->sy[s->lead] = sy;
      ++s->lead;
    }
  }
  return CHN_OK;
}

chn_status same_shape(const chn_array *a, const chn_array *x, const char *name) {
  if (a->ndim != x->ndim) return fail(CHN_ERR_SHAPE, "dropout: %s must have x's shape", name);
  for (int k = 0; k < x->ndim; ++k)
    if (a->shape[k] != x->shape[k]) return fail(CHN_ERR_SHAPE, "dropout: %s must have x's shape", name);
  return CHN_OK;
}

template <typename TX, typename TY>
void launch(const chn_array *x, const chn_array *r, const chn_array *y, const DropShape &s, const DropArgs &a, hipStream_t st) {
  const int64_t total = s.rows * s.units, want = (total + 255) / 256, most = 1 << 20;
  hipLaunchKernelGGL((dropout_kernel<TX, TY>), dim3((unsigned)(want < most ? want : most)), dim3(256), 0, st, static_cast<const TX *>(x->data),
                     r ? static_cast<const TY *>(r->data) : nullptr, static_cast<TY *>(y->data), s, a);
}

}  // namespace
}  // namespace chn

extern "C" {

chn_status chn_dropout(const chn_array *x, const chn_array *residual, double ratio, const chn_array *rng, int64_t site,
                       const chn_array *y, chn_stream stream) {
  using namespace chn;
  CHN_TRY(validate(x, "x", false));
  CHN_TRY(validate(y, "y", true));
  if (residual) CHN_TRY(validate(residual, "residual", false));
  if (!is_float(x->dtype) || !is_float(y->dtype)) return fail(CHN_ERR_DTYPE, "dropout: x and y must be F32 or BF16");
  if (residual && residual->dtype != y->dtype) return fail(CHN_ERR_DTYPE, "dropout: residual must have y's dtype");
  CHN_TRY(same_shape(y, x, "y"));
  if (residual) CHN_TRY(same_shape(residual, x, "residual"));
  DropShape s;
  CHN_TRY(plan(x, residual, y, &s));
  DropArgs a;
  CHN_TRY(check_drop(rng, ratio, site, s.rows, s.cols, "dropout", &a));
  if (s.rows == 0 || s.cols == 0) return CHN_OK;
  hipStream_t st = as_stream(stream);
  const bool x32 = x->dtype == CHN_F32, y32 = y->dtype == CHN_F32;
  if (x32 && y32) launch<float, float>(x, residual, y, s, a, st);
  else if (x32) launch<float, bf16_raw>(x, residual, y, s, a, st);
  else if (y32) launch<bf16_raw, float>(x, residual, y, s, a, st);
  else launch<bf16_raw, bf16_raw>(x, residual, y, s, a, st);
  return check_launch("dropout");
}

chn_status chn_rng_advance(const chn_array *rng, int64_t steps, chn_stream stream) {
  using namespace chn;
  CHN_TRY(validate(rng, "rng", true));
  if (rng->dtype != CHN_I64) return fail(CHN_ERR_DTYPE, "rng_advance: rng must be I64");
  if (rng->ndim != 1 || rng->shape[0] != 2) return fail(CHN_ERR_SHAPE, "rng_advance: rng must have shape (2,): seed and offset");
  if (!is_contiguous(rng)) return fail(CHN_ERR_STRIDE, "rng_advance: rng must be contiguous");
  hipLaunchKernelGGL(rng_advance_kernel, dim3(1), dim3(64), 0, as_stream(stream), static_cast<int64_t *>(rng->data), steps);
  return check_launch("rng_advance");
}

}  // extern "C"
