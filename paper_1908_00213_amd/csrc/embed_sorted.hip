// chn_embed_scaled_fwd / chn_embed_sorted_bwd: the lookup with its scale, and the table's gradient.
#include "rows.h"

namespace chn {
namespace {

template <typename L>
__device__ __forceinline__ int64_t id_at(const L *ids, int64_t n, int64_t stride, int64_t V) {
  const int64_t id = (int64_t)ids[n * stride];
  return (uint64_t)id < (uint64_t)V ? id : V;            // an id outside the table is never used as an offset
}

// A wave for each row, in units at whatever address the rows have; what is left of a row behind its last whole unit goes element by element.
template <typename TI, typename TO, typename L>
__global__ __launch_bounds__(256) void embed_scaled_kernel(const TI *table, int64_t tp, int64_t V, const L *ids, int64_t is, int64_t N, int64_t D, float scale,
                                                           TO *out, int64_t op) {
  constexpr int E = unit_elements<TI, TO>();
  const int lane = threadIdx.x & 63;
  const int64_t n = block_number() * 4 + (threadIdx.x >> 6);
  if (n >= N) return;
  const int64_t id = id_at(ids, n, is, V);
  const TI *src = table + id * tp;
  TO *dst = out + n * op;
  const bool none = id == V;
  for (int64_t d = (int64_t)lane * E; d < D; d += 64 * E) {
    if (d + E <= D) {
      Unit<TI, E> u;
      Unit<TO, E> o;
      if (none) {
        o.zero();
      } else {
        u.load(src + d);
#pragma unroll
        for (int e = 0; e < E; ++e) o.set(e, u.get(e) * scale);
      }
      o.store(dst + d);
    } else {
      for (int64_t e = d; e < D; ++e) Elem<TO>::store(dst + e, none ? 0.0f : Elem<TI>::load(src + e) * scale);
    }
  }
}

// A block for each row of the table, which looks for its token in the whole list.
template <typename T, typename L>
__global__ __launch_bounds__(256) void embed_rows_kernel(const L *ids, int64_t is, int64_t N, const T *dout, int64_t dp, int64_t D, float scale, float *dtable,
                                                         int64_t tp, int64_t V, int accumulate) {
  const int64_t v = block_number();
  if (v >= V) return;
  for (int64_t d = threadIdx.x; d < D; d += 256) {
    float sum = 0.0f;
    for (int64_t n = 0; n < N; ++n)
      if ((int64_t)ids[n * is] == v) sum += Elem<T>::load(dout + n * dp + d);
    float *p = dtable + v * tp + d;
    *p = accumulate ? fmaf(scale, sum, *p) : scale * sum;
  }
}

chn_status ids_of(const chn_array *ids, int64_t *N, int64_t *stride) {
  CHN_TRY(validate(ids, "ids", false));
  if (!is_index(ids->dtype)) return fail(CHN_ERR_DTYPE, "embed: ids must be I32 or I64");
  if (ids->ndim != 1) return fail(CHN_ERR_NDIM, "embed: ids must have 1 dimension, got %d", ids->ndim);
  *N = ids->shape[0];
  *stride = *N > 1 ? ids->strides[0] / dtype_size(ids->dtype) : 0;
  if (*N > 0x7fffffff) return fail(CHN_ERR_SHAPE, "embed: %lld ids", (long long)*N);
  return CHN_OK;
}

}  // namespace
}  // namespace chn

extern "C" {

chn_status chn_embed_scaled_fwd(const chn_array *table, const chn_array *ids, double scale, const chn_array *out, chn_stream stream) {
  using namespace chn;
  int64_t N, is, V, D, tp, on, od, op;
  CHN_TRY(ids_of(ids, &N, &is));
  CHN_TRY(validate(table, "table", false));
  CHN_TRY(validate(out, "out", true));
  if (!is_float(table->dtype) || !is_float(out->dtype)) return fail(CHN_ERR_DTYPE, "embed: table and out must be F32 or BF16");
  CHN_TRY(row_major_2d(table, "table", &V, &D, &tp));
  CHN_TRY(row_major_2d(out, "out", &on, &od, &op));
  if (on != N || od != D) return fail(CHN_ERR_SHAPE, "embed: out must have shape (%lld,%lld)", (long long)N, (long long)D);
  if (V > 0x7fffffff) return fail(CHN_ERR_SHAPE, "embed: a table of %lld rows", (long long)V);
  if (N == 0 || D == 0) return CHN_OK;
  const dim3 grid = grid_of((N + 3) / 4);
  hipStream_t st = as_stream(stream);
#define CHN_GO(TI, TO)                                                                                                                               \
  do {                                                                                                                                               \
    if (ids->dtype == CHN_I32)                                                                                                                       \
      hipLaunchKernelGGL((embed_scaled_kernel<TI, TO, int32_t>), grid, dim3(256), 0, st, static_cast<const TI *>(table->data), tp, V,                \
                         static_cast<const int32_t *>(ids->data), is, N, D, (float)scale, static_cast<TO *>(out->data), op);                         \
    else                                                                                                                                             \
      hipLaunchKernelGGL((embed_scaled_kernel<TI, TO, int64_t>), grid, dim3(256), 0, st, static_cast<const TI *>(table->data), tp, V,                \
                         static_cast<const int64_t *>(ids->data), is, N, D, (float)scale, static_cast<TO *>(out->data), op);                         \
  } while (0)
  if (table->dtype == CHN_F32) { if (out->dtype == CHN_F32) CHN_GO(float, float); else CHN_GO(float, bf16_raw); }
  else { if (out->dtype == CHN_F32) CHN_GO(bf16_raw, float); else CHN_GO(bf16_raw, bf16_raw); }
#undef CHN_GO
  return check_launch("embed_scaled_fwd");
}

size_t chn_embed_sorted_workspace_bytes(const chn_array *ids, const chn_array *dtable) { return 0; }

chn_status chn_embed_sorted_bwd(const chn_array *ids, const chn_array *dout, double scale, const chn_array *dtable, int accumulate, void *ws,
                                size_t ws_bytes, chn_stream stream) {
  using namespace chn;
  int64_t N, is, V, D, tp, dn, dd, dp;
  CHN_TRY(ids_of(ids, &N, &is));
  CHN_TRY(validate(dout, "dout", false));
  CHN_TRY(validate(dtable, "dtable", true));
  if (!is_float(dout->dtype)) return fail(CHN_ERR_DTYPE, "embed: dout must be F32 or BF16");
  if (dtable->dtype != CHN_F32) return fail(CHN_ERR_DTYPE, "embed: dtable must be F32");
  CHN_TRY(row_major_2d(dtable, "dtable", &V, &D, &tp));
  CHN_TRY(row_major_2d(dout, "dout", &dn, &dd, &dp));
  if (dn != N || dd != D) return fail(CHN_ERR_SHAPE, "embed: dout must have shape (%lld,%lld)", (long long)N, (long long)D);
  if (V > 0x7fffffff) return fail(CHN_ERR_SHAPE, "embed: a table of %lld rows", (long long)V);
  CHN_TRY(check_ws(ws, ws_bytes, chn_embed_sorted_workspace_bytes(ids, dtable), "embed_sorted_bwd"));
  if (V == 0 || D == 0) return CHN_OK;
  const dim3 grid = grid_of(V);
  hipStream_t st = as_stream(stream);
#define CHN_GO(T, L)                                                                                                                             \
  hipLaunchKernelGGL((embed_rows_kernel<T, L>), grid, dim3(256), 0, st, static_cast<const L *>(ids->data), is, N, static_cast<const T *>(dout->data), dp, D, \
                     (float)scale, static_cast<float *>(dtable->data), tp, V, accumulate)
  if (ids->dtype == CHN_I32) { if (dout->dtype == CHN_F32) CHN_GO(float, int32_t); else CHN_GO(bf16_raw, int32_t); }
  else { if (dout->dtype == CHN_F32) CHN_GO(float, int64_t); else CHN_GO(bf16_raw, int64_t); }
#undef CHN_GO
  return check_launch("embed_sorted_bwd");
}

}  // extern "C"
