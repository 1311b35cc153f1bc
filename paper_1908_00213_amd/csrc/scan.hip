// chn_gated_scan_fwd / _bwd: a gated linear recurrence over time and its gradient.
#include "rows.h"

namespace chn {
namespace {

struct ScanArgs {
  const void *gate, *x, *dy;
  void *y, *dgate, *dx;
  const float *h0, *dh_last;
  float *h_last, *states, *dh0;
  const void *lengths;
  int64_t T, B, D;
  int64_t gt, gb, xt, xb, yt, yb, ht, hb;   // strides in elements: gate (dgate: ht, hb), x, y or dy
  int64_t ut, ub, p0, pl;                   // dx; rows of h0 or dh0, of h_last or dh_last
  int64_t len_stride;
  int len64;
};

// a and 1 - a of the sigmoid gate, both to about an ulp: exp(-|g|) from the hardware's 2^t, t in two parts, and a reciprocal with a Newton step.
__device__ __forceinline__ void gate_parts(float g, float &a, float &rest) {
  float m = fabsf(g);
  m = m > 200.0f ? 200.0f : m;               // (2^-288 is 0; NaN stays)
  const float t = m * -1.44269502f;
  const float lo = fmaf(m, -1.92596299e-8f, fmaf(m, -1.44269502f, -t));
  const float e0 = __builtin_amdgcn_exp2f(t);
  const float e = fmaf(e0, lo * 0.693147181f, e0);
  const float d = 1.0f + e;
  float r = __builtin_amdgcn_rcpf(d);
  r = fmaf(fmaf(-d, r, 1.0f), r, r);
  const float er = e * r;
  a = g >= 0.0f ? r : er;
  rest = g >= 0.0f ? er : r;
}

__device__ __forceinline__ int64_t sequence_end(const ScanArgs &s, int64_t b) {
  if (!s.lengths) return s.T;
  const int64_t n = s.len64 ? static_cast<const int64_t *>(s.lengths)[b * s.len_stride] : static_cast<const int32_t *>(s.lengths)[b * s.len_stride];
  return n < 0 ? 0 : n > s.T ? s.T : n;
}

template <typename TI, typename TO, bool SIGMOID>
__global__ __launch_bounds__(256) void scan_fwd_kernel(ScanArgs s) {
  const int64_t c = block_number() * 256 + threadIdx.x;
  if (c >= s.B * s.D) return;
  const int64_t b = c / s.D, d = c - b * s.D;
  const TI *g = static_cast<const TI *>(s.gate) + b * s.gb + d, *x = static_cast<const TI *>(s.x) + b * s.xb + d;
  TO *y = static_cast<TO *>(s.y) + b * s.yb + d;
  const int64_t end = sequence_end(s, b);
  float h = s.h0 ? s.h0[b * s.p0 + d] : 0.0f;
  for (int64_t t = 0; t < s.T; ++t) {
    if (s.states && t % CHN_SCAN_STRIDE == 0) s.states[t / CHN_SCAN_STRIDE * s.B * s.D + c] = h;
    float out = 0.0f;
    if (t < end) {
      float a = Elem<TI>::load(g + t * s.gt), u = Elem<TI>::load(x + t * s.xt);
      if constexpr (SIGMOID) {
        float rest;
        gate_parts(a, a, rest);
        u *= rest;
      }
      out = h = fmaf(a, h, u);
    }
    Elem<TO>::store(y + t * s.yt, out);
  }
  if (s.h_last) s.h_last[b * s.pl + d] = h;
}

template <typename TI, typename TO, bool SIGMOID>
__global__ __launch_bounds__(256) void scan_bwd_kernel(ScanArgs s) {
  const int64_t c = block_number() * 256 + threadIdx.x;
  if (c >= s.B * s.D) return;
  const int64_t b = c / s.D, d = c - b * s.D;
  const TI *g = static_cast<const TI *>(s.gate) + b * s.gb + d, *x = static_cast<const TI *>(s.x) + b * s.xb + d;
  const TO *dy = static_cast<const TO *>(s.dy) + b * s.yb + d;
  TI *dg = static_cast<TI *>(s.dgate) + b * s.hb + d, *dx = static_cast<TI *>(s.dx) + b * s.ub + d;
  const int64_t end = sequence_end(s, b);
  float G = s.dh_last ? s.dh_last[b * s.pl + d] : 0.0f;
  for (int64_t k = (s.T + CHN_SCAN_STRIDE - 1) / CHN_SCAN_STRIDE - 1; k >= 0; --k) {
    float h = s.states[k * s.B * s.D + c], before[CHN_SCAN_STRIDE], av[CHN_SCAN_STRIDE], rv[CHN_SCAN_STRIDE], xv[CHN_SCAN_STRIDE];
#pragma unroll
    for (int i = 0; i < CHN_SCAN_STRIDE; ++i) {
      const int64_t t = k * CHN_SCAN_STRIDE + i;
      before[i] = h;
      av[i] = rv[i] = xv[i] = 0.0f;
      if (t < end) {
        av[i] = Elem<TI>::load(g + t * s.gt);
        xv[i] = Elem<TI>::load(x + t * s.xt);
        rv[i] = 1.0f;
        if constexpr (SIGMOID) gate_parts(av[i], av[i], rv[i]);
        h = fmaf(av[i], h, rv[i] * xv[i]);
      }
    }
#pragma unroll
    for (int i = CHN_SCAN_STRIDE - 1; i >= 0; --i) {
      const int64_t t = k * CHN_SCAN_STRIDE + i;
      if (t >= s.T) continue;
      float vg = 0.0f, vx = 0.0f;
      if (t < end) {
        G += Elem<TO>::load(dy + t * s.yt);
        vx = rv[i] * G;
        vg = SIGMOID ? vx * av[i] * (before[i] - xv[i]) : before[i] * G;
        G *= av[i];
      }
      Elem<TI>::store(dg + t * s.ht, vg);
      Elem<TI>::store(dx + t * s.ut, vx);
    }
  }
  if (s.dh0) s.dh0[b * s.p0 + d] = G;
}

// (T,B,D) with unit inner stride; the strides of the others in elements.
chn_status steps_of(const chn_array *a, const char *name, bool is_output, int64_t T, int64_t B, int64_t D, int64_t *st, int64_t *sb) {
  CHN_TRY(validate(a, name, is_output));
  if (!is_float(a->dtype)) return fail(CHN_ERR_DTYPE, "gated_scan: %s must be F32 or BF16", name);
  if (a->ndim != 3) return fail(CHN_ERR_NDIM, "gated_scan: %s must have 3 dimensions, got %d", name, a->ndim);
  if (a->shape[0] != T || a->shape[1] != B || a->shape[2] != D)
    return fail(CHN_ERR_SHAPE, "gated_scan: %s must have shape (%lld,%lld,%lld)", name, (long long)T, (long long)B, (long long)D);
  const int isz = dtype_size(a->dtype);
  if (D > 1 && a->strides[2] != isz) return fail(CHN_ERR_STRIDE, "gated_scan: the last axis of %s must have unit stride", name);
  *st = T > 1 ? a->strides[0] / isz : 0;
  *sb = B > 1 ? a->strides[1] / isz : 0;
  if (is_output && T * B * D > 0) {          // rows that do not run into each other, whichever axis is the outer one
    const int64_t inner_b = (B - 1) * *sb + D, inner_t = (T - 1) * *st + D;
    const bool ok = (B == 1 || *sb >= D) && (T == 1 || *st >= inner_b);
    const bool ok2 = (T == 1 || *st >= D) && (B == 1 || *sb >= inner_t);
    if (!ok && !ok2) return fail(CHN_ERR_STRIDE, "gated_scan: the rows of %s overlap", name);
  }
  return CHN_OK;
}

chn_status state_of(const chn_array *a, const char *name, bool is_output, int64_t B, int64_t D, int64_t *pitch) {
  int64_t n, d;
  *pitch = D;
  if (!a) return CHN_OK;
  CHN_TRY(validate(a, name, is_output));
  if (a->dtype != CHN_F32) return fail(CHN_ERR_DTYPE, "gated_scan: %s must be F32", name);
  CHN_TRY(row_major_2d(a, name, &n, &d, pitch));
  if (n != B || d != D) return fail(CHN_ERR_SHAPE, "gated_scan: %s must have shape (%lld,%lld)", name, (long long)B, (long long)D);
  return CHN_OK;
}

// What both directions check first: sizes, types, lengths and states.
chn_status common_args(int kind, const chn_array *gate, const chn_array *x, const chn_array *lengths, const chn_array *states, bool states_out, ScanArgs *s) {
  if (kind != CHN_SCAN_SIGMOID && kind != CHN_SCAN_DECAY) return fail(CHN_ERR_OP, "gated_scan: unknown kind %d", kind);
  CHN_TRY(validate(gate, "gate", false));
  if (gate->ndim != 3) return fail(CHN_ERR_NDIM, "gated_scan: gate must have 3 dimensions, got %d", gate->ndim);
  s->T = gate->shape[0]; s->B = gate->shape[1]; s->D = gate->shape[2];
  if (s->T > 0x7fffffff || s->B > 0x7fffffff || s->D > 0x7fffffff || s->B * s->D > (1ll << 40))
    return fail(CHN_ERR_SHAPE, "gated_scan: sizes of (%lld,%lld,%lld)", (long long)s->T, (long long)s->B, (long long)s->D);
  CHN_TRY(steps_of(gate, "gate", false, s->T, s->B, s->D, &s->gt, &s->gb));
  CHN_TRY(steps_of(x, "x", false, s->T, s->B, s->D, &s->xt, &s->xb));
  if (x->dtype != gate->dtype) return fail(CHN_ERR_DTYPE, "gated_scan: gate and x must have one dtype");
  s->gate = gate->data; s->x = x->data;
  if (lengths) {
    CHN_TRY(validate(lengths, "lengths", false));
    if (!is_index(lengths->dtype)) return fail(CHN_ERR_DTYPE, "gated_scan: lengths must be I32 or I64");
    if (lengths->ndim != 1 || lengths->shape[0] != s->B) return fail(CHN_ERR_SHAPE, "gated_scan: lengths must have shape (%lld,)", (long long)s->B);
    s->lengths = lengths->data;
    s->len64 = lengths->dtype == CHN_I64;
    s->len_stride = s->B > 1 ? lengths->strides[0] / dtype_size(lengths->dtype) : 0;
  }
  if (states) {
    CHN_TRY(validate(states, "states", states_out));
    if (states->dtype != CHN_F32) return fail(CHN_ERR_DTYPE, "gated_scan: states must be F32");
    if (states->ndim != 3 || states->shape[0] != chn_gated_scan_states(s->T) || states->shape[1] != s->B || states->shape[2] != s->D || !is_contiguous(states))
      return fail(CHN_ERR_SHAPE, "gated_scan: states must be contiguous, of shape (%lld,%lld,%lld)", (long long)chn_gated_scan_states(s->T), (long long)s->B,
                  (long long)s->D);
    s->states = static_cast<float *>(states->data);
  }
  return CHN_OK;
}

}  // namespace
}  // namespace chn

extern "C" {

int64_t chn_gated_scan_states(int64_t steps) { return steps <= 0 ? 0 : (steps - 1) / CHN_SCAN_STRIDE + 1; }

size_t chn_gated_scan_workspace_bytes(const chn_array *gate) { return 0; }

chn_status chn_gated_scan_fwd(int kind, const chn_array *gate, const chn_array *x, const chn_array *h0, const chn_array *lengths, const chn_array *y,
                              const chn_array *h_last, const chn_array *states, void *ws, size_t ws_bytes, chn_stream stream) {
  using namespace chn;
  ScanArgs s = {};
  CHN_TRY(common_args(kind, gate, x, lengths, states, true, &s));
  CHN_TRY(steps_of(y, "y", true, s.T, s.B, s.D, &s.yt, &s.yb));
  CHN_TRY(state_of(h0, "h0", false, s.B, s.D, &s.p0));
  CHN_TRY(state_of(h_last, "h_last", true, s.B, s.D, &s.pl));
  CHN_TRY(check_ws(ws, ws_bytes, chn_gated_scan_workspace_bytes(gate), "gated_scan_fwd"));
  if (s.B * s.D == 0) return CHN_OK;
  s.y = y->data;
  if (h0) s.h0 = static_cast<const float *>(h0->data);
  if (h_last) s.h_last = static_cast<float *>(h_last->data);
  const dim3 grid = grid_of((s.B * s.D + 255) / 256);
  hipStream_t st = as_stream(stream);
#define CHN_GO(TI, TO)                                                                                                                     \
  do {                                                                                                                                     \
    if (kind == CHN_SCAN_SIGMOID) hipLaunchKernelGGL((scan_fwd_kernel<TI, TO, true>), grid, dim3(256), 0, st, s);                          \
    else hipLaunchKernelGGL((scan_fwd_kernel<TI, TO, false>), grid, dim3(256), 0, st, s);                                                  \
  } while (0)
  if (gate->dtype == CHN_F32) { if (y->dtype == CHN_F32) CHN_GO(float, float); else CHN_GO(float, bf16_raw); }
  else { if (y->dtype == CHN_F32) CHN_GO(bf16_raw, float); else CHN_GO(bf16_raw, bf16_raw); }
#undef CHN_GO
  return check_launch("gated_scan_fwd");
}

chn_status chn_gated_scan_bwd(int kind, const chn_array *gate, const chn_array *x, const chn_array *states, const chn_array *lengths, const chn_array *dy,
                              const chn_array *dh_last, const chn_array *dgate, const chn_array *dx, const chn_array *dh0, void *ws, size_t ws_bytes,
                              chn_stream stream) {
  using namespace chn;
  ScanArgs s = {};
  if (!states) return fail(CHN_ERR_NULL, "gated_scan_bwd: states is NULL");
  CHN_TRY(common_args(kind, gate, x, lengths, states, false, &s));
  CHN_TRY(steps_of(dy, "dy", false, s.T, s.B, s.D, &s.yt, &s.yb));
  CHN_TRY(steps_of(dgate, "dgate", true, s.T, s.B, s.D, &s.ht, &s.hb));
  CHN_TRY(steps_of(dx, "dx", true, s.T, s.B, s.D, &s.ut, &s.ub));
  if (dgate->dtype != gate->dtype || dx->dtype != gate->dtype) return fail(CHN_ERR_DTYPE, "gated_scan_bwd: dgate and dx must have the dtype of gate");
  CHN_TRY(state_of(dh_last, "dh_last", false, s.B, s.D, &s.pl));
  CHN_TRY(state_of(dh0, "dh0", true, s.B, s.D, &s.p0));
  CHN_TRY(check_ws(ws, ws_bytes, chn_gated_scan_workspace_bytes(gate), "gated_scan_bwd"));
  if (s.B * s.D == 0) return CHN_OK;
  s.dy = dy->data; s.dgate = dgate->data; s.dx = dx->data;
  if (dh_last) s.dh_last = static_cast<const float *>(dh_last->data);
  if (dh0) s.dh0 = static_cast<float *>(dh0->data);
  const dim3 grid = grid_of((s.B * s.D + 255) / 256);
  hipStream_t st = as_stream(stream);
#define CHN_GO(TI, TO)                                                                                                                     \
  do {                                                                                                                                     \
    if (kind == CHN_SCAN_SIGMOID) hipLaunchKernelGGL((scan_bwd_kernel<TI, TO, true>), grid, dim3(256), 0, st, s);                          \
    else hipLaunchKernelGGL((scan_bwd_kernel<TI, TO, false>), grid, dim3(256), 0, st, s);                                                  \
  } while (0)
  if (gate->dtype == CHN_F32) { if (dy->dtype == CHN_F32) CHN_GO(float, float); else CHN_GO(float, bf16_raw); }
  else { if (dy->dtype == CHN_F32) CHN_GO(bf16_raw, float); else CHN_GO(bf16_raw, bf16_raw); }
#undef CHN_GO
  return check_launch("gated_scan_bwd");
}

}  // extern "C"
