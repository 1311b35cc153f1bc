// chn_dropout, chn_rng_advance: dropout whose mask is drawn from a counter-based generator and never stored.
//
// y = (residual +) [word >= threshold] * x / (1 - ratio), the word of element (row, col) from philox.h.  Nothing is kept for the
// backward pass: the gradient of x is the same call on the gradient of y.
//
// Bound by memory: one read (two with a residual) and one write an element, 8192 x 4096 bf16 with residual 31 us, its gradient 23 (6.5 and
// 5.8 TB/s; without a mask 21).  The mask is what comes closest to costing time: with two instructions for a three-way exclusive or the gradient
// took 26.
//
// The leading dimensions of the arrays are merged where all of them allow it; what is left are rows with a list of strides.  Rows of unit stride with one pitch go
// in 16-byte pieces; the others element by element, four columns a thread behind a division for each dimension that is left.  4096 x 4096, us (a plain copy):
// fp32 / bf16 22 (24) / 13.5 (13); rows of a 3-d slice 30 (19) / 26 (12); a repeated row 15 (12) / 13 (8); every second column 43 (42) / 26 (43); transposed 83 (26) / 71 (13), where
// neighbouring threads read lines apart.  No model here drops out anything but rows of unit stride.
#include "philox.h"
#include "rows.h"

namespace chn {
namespace {

constexpr int kMaxLead = CHN_MAX_NDIM - 1;
// units a thread has in flight (us of dropout and its gradient with 1, 2 and 4: 8192 x 4096 bf16 54.8, 54.2, 55.7; 4480 x 650 fp32 11.0, 11.1, 12.1)
constexpr int kUnitsPerThread = 2;

struct DropShape {
  int lead;                          // leading dimensions after merging, outermost first
  int64_t rows, cols, units;         // units: columns / 4, rounded up
  uint32_t n[kMaxLead];
  int64_t sx[kMaxLead], sr[kMaxLead], sy[kMaxLead];   // elements
  int64_t cx, cr, cy;                // strides along the last axis
};

// Rows of unit stride: a thread takes units of E neighbouring columns, U of them at a time so that their loads are in flight together, at
// whatever element address they have; the last unit of a row that is not whole goes element by element.  `upr`: units of a row.
template <typename TX, typename TY, bool RES, int U>
__global__ __launch_bounds__(256) void dropout_rows_kernel(const TX *x, const TY *residual, TY *y, int64_t rows, int64_t cols, uint32_t upr,
                                                           int64_t px, int64_t pr, int64_t py, DropArgs a) {
  constexpr int E = unit_elements<TX, TY>();
  const DropState d(a);
  const int64_t total = rows * upr, first = ((int64_t)blockIdx.x * U) * 256 + threadIdx.x;
  Unit<TX, E> xu[U];
  Unit<TY, E> ru[U];
  int64_t row[U];
  uint32_t c0[U];
  int n[U];                                              // columns of the unit: E, fewer at a row's end, 0 behind the last row
#pragma unroll
  for (int u = 0; u < U; ++u) {
    const int64_t i = first + u * 256;
    if (total <= 0xffffffffLL) {
      row[u] = (uint32_t)i / upr;
    } else {
      row[u] = i / upr;
    }
    c0[u] = (uint32_t)(i - row[u] * upr);
    const int64_t left = cols - (int64_t)c0[u] * E;
    n[u] = i < total ? (left < E ? (int)left : E) : 0;
    if (n[u] == E) {
      xu[u].load(x + row[u] * px + (int64_t)c0[u] * E);
      if constexpr (RES) ru[u].load(residual + row[u] * pr + (int64_t)c0[u] * E);
    }
  }
#pragma unroll
  for (int u = 0; u < U; ++u) {
    if (n[u] == 0) continue;
    const int64_t c = (int64_t)c0[u] * E;
    Philox4 w[E / 4];
#pragma unroll
    for (int b = 0; b < E / 4; ++b) w[b] = a.rng ? d.words(c0[u] * (E / 4) + b, (uint32_t)row[u]) : Philox4{{~0u, ~0u, ~0u, ~0u}};
    if (n[u] == E) {
      Unit<TY, E> out;
#pragma unroll
      for (int i = 0; i < E; ++i) {
        float v = d.apply(xu[u].get(i), w[i / 4].w[i % 4]);
        if constexpr (RES) v = add_rounded(ru[u].get(i), v);
        out.set(i, v);
      }
      out.store_nt(y + row[u] * py + c);
    } else {
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (i < n[u]) {
          float v = d.apply(Elem<TX>::load(x + row[u] * px + c + i), w[i / 4].w[i % 4]);
          if constexpr (RES) v = add_rounded(Elem<TY>::load(residual + row[u] * pr + c + i), v);
          Elem<TY>::store(y + row[u] * py + c + i, v);
        }
    }
  }
}

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
  const TX *xp = static_cast<const TX *>(x->data);
  const TY *rp = r ? static_cast<const TY *>(r->data) : nullptr;
  TY *yp = static_cast<TY *>(y->data);
  constexpr int E = unit_elements<TX, TY>(), U = kUnitsPerThread;
  const int64_t upr = (s.cols + E - 1) / E, fast = (s.rows * upr + 256 * U - 1) / (256 * U);
  // (a launch takes fewer than 2^32 threads; a row shorter than a unit leaves most of a thread idle either way, and the general kernel takes four columns, not E)
  if (s.lead <= 1 && s.cx == 1 && s.cy == 1 && (!r || s.cr == 1) && s.cols >= E && fast < (1 << 24) && upr <= 0xffffffffLL / (E / 4)) {
    const int64_t px = s.lead ? s.sx[0] : 0, pr = s.lead ? s.sr[0] : 0, py = s.lead ? s.sy[0] : 0;
    if (r) hipLaunchKernelGGL((dropout_rows_kernel<TX, TY, true, U>), dim3((unsigned)fast), dim3(256), 0, st, xp, rp, yp, s.rows, s.cols, (uint32_t)upr, px, pr, py, a);
    else hipLaunchKernelGGL((dropout_rows_kernel<TX, TY, false, U>), dim3((unsigned)fast), dim3(256), 0, st, xp, rp, yp, s.rows, s.cols, (uint32_t)upr, px, pr, py, a);
    return;
  }
  const int64_t want = (s.rows * s.units + 255) / 256, most = 1 << 20;
  hipLaunchKernelGGL((dropout_kernel<TX, TY>), dim3((unsigned)(want < most ? want : most)), dim3(256), 0, st, xp, rp, yp, s, a);
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
