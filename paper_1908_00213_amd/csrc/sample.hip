// chn_sample: one token for each row of logits, filtered by temperature, top-k, top-p and min-p, drawn by a given number.
//
// Weights are whole numbers: w(z) = round(2^shift exp((z - max z) / temperature)), the exponential in 64 bits, so that every sum is exact,
// whatever the order in which it is taken; the token is the first whose running sum (in the vocabulary's order, over the tokens that
// the filters keep) exceeds u times the whole sum.  The filters come down to one border in the order of descending logits: every token
// with a larger key is kept, and of those with the border's key the first few by index.
#include "common.h"

namespace chn {
namespace {

struct SampleArgs {
  int64_t N, pitch;
  int V, shift;
  const float *u, *temperature, *top_p, *min_p;
  int64_t su, st, sp, sm, sk;        // strides in elements
  const void *top_k;
  int k64;
  void *out;
  int out64;
};

// Monotone in the logit, -0 and 0 alike.  0: not a token that can be drawn (-inf, NaN).
__device__ __forceinline__ uint32_t key_of(float z) {
  if (!(z > -INFINITY)) return 0;
  const uint32_t b = __float_as_uint(z + 0.0f);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}

__device__ __forceinline__ uint64_t wave_sum_u64(uint64_t v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor((unsigned long long)v, o, 64);
  return v;
}

constexpr int kThreads = 1024, kWaves = kThreads / 64;

// Sum over the block, the same in every thread.
__device__ __forceinline__ uint64_t block_sum_u64(uint64_t v, uint64_t *smem) {
  v = wave_sum_u64(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) smem[threadIdx.x >> 6] = v;
  __syncthreads();
  uint64_t s = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) s += smem[w];
  return s;
}

// Sum over the threads before this one.
__device__ __forceinline__ uint64_t block_before_u64(uint64_t v, uint64_t *smem) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  uint64_t s = v;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint64_t other = __shfl_up((unsigned long long)s, o, 64);
    if (lane >= o) s += other;
  }
  __syncthreads();
  if (lane == 63) smem[wave] = s;
  __syncthreads();
  uint64_t before = s - v;
  for (int w = 0; w < wave; ++w) before += smem[w];
  return before;
}

__device__ __forceinline__ float block_max(float v, float *smem) {
  v = wave_max(v);
  __syncthreads();
  if ((threadIdx.x & 63) == 0) smem[threadIdx.x >> 6] = v;
  __syncthreads();
  float m = smem[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) m = fmaxf(m, smem[w]);
  return m;
}

// A thread owns a run of neighbouring tokens.
template <typename T>
__global__ __launch_bounds__(kThreads) void sample_kernel(const T *logits, SampleArgs a) {
  __shared__ float smax[kWaves];
  __shared__ uint64_t sum[kWaves];
  __shared__ int found;
  const int64_t row = blockIdx.x;
  const T *z = logits + row * a.pitch;
  const int per = (a.V + kThreads - 1) / kThreads;
  const int lo = min(a.V, (int)threadIdx.x * per), hi = min(a.V, lo + per);
  const auto put = [&](int64_t token) {
    if (a.out64) static_cast<int64_t *>(a.out)[row] = token;
    else static_cast<int32_t *>(a.out)[row] = (int32_t)token;
  };
  float m = -INFINITY;
  for (int i = lo; i < hi; ++i) m = fmaxf(m, Elem<T>::load(z + i));
  const float best = block_max(m, smax);
  if (best == -INFINITY) {                               // nothing to choose from
    if (threadIdx.x == 0) put(-1);
    return;
  }
  const uint32_t top = key_of(best);
  const float t = a.temperature ? a.temperature[row * a.st] : 1.0f;
  // the first token among those with this key, if it lies in this thread's run: `nth` counts them from 0
  const auto nth_with_key = [&](uint32_t key, int64_t nth) -> int {
    uint64_t mine = 0;
    for (int i = lo; i < hi; ++i) mine += key_of(Elem<T>::load(z + i)) == key;
    int64_t before = (int64_t)block_before_u64(mine, sum);
    if (threadIdx.x == 0) found = a.V;
    __syncthreads();
    if (before <= nth && nth < before + (int64_t)mine)
      for (int i = lo; i < hi; ++i)
        if (key_of(Elem<T>::load(z + i)) == key && before++ == nth) { found = i; break; }
    __syncthreads();
    return found;
  };
  if (!(t > 0.0f)) {
    const int i = nth_with_key(top, 0);
    if (threadIdx.x == 0) put(i);
    return;
  }
  const float m0 = a.min_p ? a.min_p[row * a.sm] : 0.0f, minp = m0 > 0.0f ? fminf(m0, 1.0f) : 0.0f;
  const double one = (double)(1ull << a.shift);
  const auto exponential = [&](float v) -> double { return v == best ? 1.0 : exp(((double)v - (double)best) / (double)t); };
  const auto weight = [&](double e) -> uint64_t { return (uint64_t)rint(e * one); };
  uint32_t border = 1;                                    // keys above it are kept,
  int64_t ties = INT64_MAX;                               // and so many of the tokens that have it
  const auto count_from = [&](uint32_t key) -> uint64_t {
    uint64_t n = 0;
    for (int i = lo; i < hi; ++i) n += key_of(Elem<T>::load(z + i)) >= key;
    return block_sum_u64(n, sum);
  };
  int64_t k = 0;
  if (a.top_k) k = a.k64 ? static_cast<const int64_t *>(a.top_k)[row * a.sk] : static_cast<const int32_t *>(a.top_k)[row * a.sk];
  if (k > 0 && (uint64_t)k < count_from(1)) {
    uint32_t b = 0;                                       // the largest key that at least k tokens reach
    for (int bit = 31; bit >= 0; --bit)
      if (count_from(b | (1u << bit)) >= (uint64_t)k) b |= 1u << bit;
    border = b;
    ties = k - (int64_t)(b == 0xffffffffu ? 0 : count_from(b + 1));
  }
  const float p = a.top_p ? a.top_p[row * a.sp] : 1.0f;
  if (p < 1.0f) {
    // sum over keys from `key` on, of what top-k keeps (key >= border)
    const auto sum_from = [&](uint32_t key) -> uint64_t {
      uint64_t s = 0;
      for (int i = lo; i < hi; ++i) {
        const float v = Elem<T>::load(z + i);
        const uint32_t q = key_of(v);
        if (q > border && q >= key) s += weight(exponential(v));
      }
      uint64_t all = block_sum_u64(s, sum);
      if (border >= key && ties != INT64_MAX) {
        const uint32_t bits = (border & 0x80000000u) ? border & 0x7fffffffu : ~border;
        all += (uint64_t)ties * weight(exponential(__uint_as_float(bits)));
      }
      return all;
    };
    const uint64_t whole = sum_from(1);
    uint64_t target = p > 0.0f ? (uint64_t)ceil((double)p * (double)whole) : 1;
    if (target < 1) target = 1;
    uint32_t b = 0;                                       // the largest key from which on the sum reaches the target
    for (int bit = 31; bit >= 0; --bit)
      if (sum_from(b | (1u << bit)) >= target) b |= 1u << bit;
    const uint64_t above = b == 0xffffffffu ? 0 : sum_from(b + 1);
    const uint32_t bits = (b & 0x80000000u) ? b & 0x7fffffffu : ~b;
    const uint64_t w = weight(exponential(__uint_as_float(bits)));
    const int64_t need = (int64_t)((target - above + w - 1) / w);
    ties = b == border ? min(ties, need) : need;
    border = b;
  }
  const int last = ties == INT64_MAX ? a.V : nth_with_key(border, ties - 1);
  // exp of a token that is kept, 0 of one that is not
  const auto kept = [&](int i) -> double {
    const float v = Elem<T>::load(z + i);
    const uint32_t q = key_of(v);
    if (q < border || q == 0 || (q == border && i > last)) return 0.0;
    const double e = exponential(v);
    return e >= (double)minp ? e : 0.0;
  };
  const float u = a.u[row * a.su];
  if (!(u > 0.0f) || u >= 1.0f) {                         // the ends of the range: the first and the last token, however light
    if (threadIdx.x == 0) found = u >= 1.0f ? -1 : a.V;
    __syncthreads();
    for (int i = lo; i < hi; ++i)
      if (kept(i) > 0.0) {
        if (u >= 1.0f) atomicMax(&found, i);
        else { atomicMin(&found, i); break; }
      }
    __syncthreads();
    if (threadIdx.x == 0) put(found);
    return;
  }
  uint64_t mine = 0;
  for (int i = lo; i < hi; ++i) mine += weight(kept(i));
  const uint64_t whole = block_sum_u64(mine, sum);
  uint64_t before = block_before_u64(mine, sum);
  const uint64_t target = (uint64_t)((double)u * (double)whole);   // below `whole`: u is at most 1 - 2^-24
  if (before <= target && target < before + mine)
    for (int i = lo; i < hi; ++i) {
      before += weight(kept(i));
      if (before > target) { put(i); break; }
    }
}

chn_status check_row_parameter(const chn_array *v, const char *name, int64_t n, int64_t *stride) {
  CHN_TRY(validate(v, name, false));
  if (v->ndim != 1 || v->shape[0] != n) return fail(CHN_ERR_SHAPE, "sample: %s must have shape (%lld,)", name, (long long)n);
  *stride = n > 1 ? v->strides[0] / dtype_size(v->dtype) : 1;
  return CHN_OK;
}

chn_status check_row_float(const chn_array *v, const char *name, int64_t n, const float **data, int64_t *stride) {
  if (!v) return CHN_OK;
  CHN_TRY(check_row_parameter(v, name, n, stride));
  if (v->dtype != CHN_F32) return fail(CHN_ERR_DTYPE, "sample: %s must be F32", name);
  *data = static_cast<const float *>(v->data);
  return CHN_OK;
}

}  // namespace
}  // namespace chn

extern "C" {

size_t chn_sample_workspace_bytes(const chn_array *logits) {
  (void)logits;
  return 0;
}

chn_status chn_sample(const chn_array *logits, const chn_array *u, const chn_array *temperature, const chn_array *top_k, const chn_array *top_p,
                      const chn_array *min_p, const chn_array *out, void *ws, size_t ws_bytes, chn_stream stream) {
  using namespace chn;
  SampleArgs a{};
  CHN_TRY(validate(logits, "logits", false));
  if (!is_float(logits->dtype)) return fail(CHN_ERR_DTYPE, "sample: logits must be F32 or BF16");
  int64_t V;
  CHN_TRY(row_major_2d(logits, "logits", &a.N, &V, &a.pitch));
  if (!u) return fail(CHN_ERR_NULL, "sample: u is NULL");
  CHN_TRY(check_row_float(u, "u", a.N, &a.u, &a.su));
  CHN_TRY(check_row_float(temperature, "temperature", a.N, &a.temperature, &a.st));
  CHN_TRY(check_row_float(top_p, "top_p", a.N, &a.top_p, &a.sp));
  CHN_TRY(check_row_float(min_p, "min_p", a.N, &a.min_p, &a.sm));
  if (top_k) {
    CHN_TRY(check_row_parameter(top_k, "top_k", a.N, &a.sk));
    if (!is_index(top_k->dtype)) return fail(CHN_ERR_DTYPE, "sample: top_k must be I32 or I64");
    a.top_k = top_k->data;
    a.k64 = top_k->dtype == CHN_I64;
  }
  CHN_TRY(validate(out, "out", true));
  if (!is_index(out->dtype)) return fail(CHN_ERR_DTYPE, "sample: out must be I32 or I64");
  if (out->ndim != 1 || out->shape[0] != a.N) return fail(CHN_ERR_SHAPE, "sample: out must have shape (%lld,)", (long long)a.N);
  if (!is_contiguous(out)) return fail(CHN_ERR_STRIDE, "sample: out must be contiguous");
  if (a.N > 0 && V == 0) return fail(CHN_ERR_SHAPE, "sample: no tokens");
  if (V > (1LL << 30) || a.N > 0x7fffffffLL) return fail(CHN_ERR_SHAPE, "sample: more than 2^30 tokens or 2^31 - 1 rows");
  if (a.N == 0) return CHN_OK;
  a.V = (int)V;
  // the sum of V weights of at most 2^shift fits 63 bits; 46 bits leave nothing to tell the draw from the exact one's
  a.shift = 46;
  while (a.shift > 0 && (V >> (63 - a.shift)) > 0) --a.shift;
  a.out = out->data;
  a.out64 = out->dtype == CHN_I64;
  (void)ws;
  (void)ws_bytes;
  hipStream_t st = as_stream(stream);
  if (logits->dtype == CHN_F32)
    hipLaunchKernelGGL((sample_kernel<float>), dim3((unsigned)a.N), dim3(kThreads), 0, st, static_cast<const float *>(logits->data), a);
  else
    hipLaunchKernelGGL((sample_kernel<bf16_raw>), dim3((unsigned)a.N), dim3(kThreads), 0, st, static_cast<const bf16_raw *>(logits->data), a);
  return check_launch("sample");
}

}  // extern "C"
