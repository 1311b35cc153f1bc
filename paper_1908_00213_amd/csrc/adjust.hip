// chn_logits_adjust: what a row's text, its caller and its grammar say about its logits, in one pass over them.
//
// A block owns a piece of one row.  It counts the piece's tokens in LDS while it looks through the row's whole list (a 32-bit word for a token: how
// often it stands behind the prompt, whether the prompt has it, whether it has a bias), then walks over the piece once: a read and a write for each logit.
// Whole numbers are counted, so the order in which the list is seen does not show.  The few tokens with biases are left out by that walk: the threads
// that hold the list's entries write them, each token by the thread with its first entry, which adds up the others in the list's order.
//
// Bound by memory where the launch fills the chip: 256 x 131072 fp32 with lists of up to 8192 tokens, 300 biases and masks 68 us (4.1 TB/s), without any of them 40 (a plain copy 37,
// part of it in the last-level cache).  A block's chain of waits is what costs beside that, so the logits, the masks and the list's first part are fetched before anything is
// counted, and four blocks of 512 threads with 16 logits each share a compute unit (two with 32 each: 80).  Biases of one id that stands twice were 40 us more while every
// thread looked through the whole list for its id: they are put in order in LDS first.
#include "rows.h"

namespace chn {
namespace {

constexpr int kThreads = 512;                // of a block, at most
constexpr int kHeld = 16;                    // logits that a thread of a large launch holds
constexpr int kListed = 512;                  // biases of a piece that are put in order in LDS
constexpr uint32_t kSeen = 0x80000000u, kBiased = 0x40000000u, kCount = 0x3fffffffu;

struct AdjustArgs {
  const void *z;
  void *out;
  const void *tokens, *lengths, *prompt, *bias_ids;
  const float *repetition, *frequency, *presence, *bias;
  const int32_t *allowed;
  int64_t N, V, L, M, pz, po, pt, ts, pi, pb, pa;  // sizes, pitches, the step from token to token
  int64_t sl, sp, sr, sf, ss;                   // strides of lengths, prompt, repetition, frequency, presence
  int64_t tiles, tile;                          // pieces of a row, tokens of a piece
  int len64, prompt64;
};

__device__ __forceinline__ int cut(const void *p, int is64, int64_t at, int L) {
  const int64_t n = is64 ? static_cast<const int64_t *>(p)[at] : static_cast<const int32_t *>(p)[at];
  return n < 0 ? 0 : n > L ? L : (int)n;
}

struct Penalties {
  float repetition, up, divisor, inverse, frequency, presence;   // divisor: up times the repetition, so that its reciprocal is in fp32's range
  bool rep;
  // (without frequency or presence: zeros, which change nothing but the sign of a zero)
  __device__ __forceinline__ float apply(float z, uint32_t word) const {
    const uint32_t c = word & kCount;
    if (rep) {
      const float y = z * up, q = y * inverse, d = fmaf(fmaf(-q, divisor, y), inverse, q);   // z / repetition, its rounding made good
      const float less = z > 0.0f ? (d == d ? d : q) : z * repetition;
      z = word & (kSeen | kCount) ? less : z;
    }
    return c ? fmaf(-frequency, (float)c, z) - presence : z;
  }
};

// A token's place in the piece, `len` and above where it lies outside: ids are below 2^31, whatever wraps lies above.
__device__ __forceinline__ uint32_t place(int32_t id, int64_t v0) { return (uint32_t)id - (uint32_t)v0; }
__device__ __forceinline__ uint32_t place(int64_t id, int64_t v0) {
  const uint64_t at = (uint64_t)id - (uint64_t)v0;
  return at > 0xffffffffull ? ~0u : (uint32_t)at;
}

// f(i, values[i]) for the indexes [0, n) that belong to the thread, eight loads in flight.  `v` holds the first eight already.
constexpr int kAhead = 8;
template <typename ID>
__device__ __forceinline__ void ahead(const ID *values, int64_t stride, int n, ID (&v)[kAhead], int from) {
  const int step = blockDim.x;
#pragma unroll
  for (int k = 0; k < kAhead; ++k) v[k] = values[min(from + k * step, n - 1) * stride];
}
template <typename ID, typename F>
__device__ __forceinline__ void each(const ID *values, int64_t stride, int n, ID (&v)[kAhead], F f) {
  const int step = blockDim.x;
  for (int i = threadIdx.x; i < n; i += kAhead * step) {
    if (i >= kAhead * step) ahead(values, stride, n, v, i);
#pragma unroll
    for (int k = 0; k < kAhead; ++k)
      if (i + k * step < n) f(i + k * step, v[k]);
  }
}

// K: units of a thread, which are on their way while the list is looked through.
template <typename TI, typename TO, typename ID, int K>
__global__ __launch_bounds__(kThreads, 8) void adjust_kernel(AdjustArgs a) {
  extern __shared__ uint32_t words[];
  __shared__ int twice, listed;
  __shared__ uint32_t place_of[kListed];               // the list's entries in this piece, in its order, where an id stands more than once
  __shared__ float bias_of[kListed];
  constexpr int E = unit_elements<TI, TO>();
  const int64_t n = block_number() / a.tiles, v0 = (block_number() - n * a.tiles) * a.tile;
  if (n >= a.N) return;                                // (the grid's last line may be longer than its blocks)
  const int len = (int)min(a.tile, a.V - v0), step = (int)blockDim.x * E;
  const TI *z = static_cast<const TI *>(a.z) + n * a.pz + v0;
  TO *out = static_cast<TO *>(a.out) + n * a.po + v0;
  const int32_t *allowed = a.allowed ? a.allowed + n * a.pa : nullptr;
  const bool lists = a.tokens || a.bias;
  Unit<TI, E> u[K];
  uint32_t bits[K];
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int i = (int)threadIdx.x * E + k * step;
    if (i + E <= len) u[k].load(z + i);
    bits[k] = allowed && i < len ? (uint32_t)allowed[(v0 + i) >> 5] >> ((v0 + i) & 31) : ~0u;
  }
  Penalties p;
  p.rep = a.repetition != nullptr;
  p.repetition = p.rep ? a.repetition[n * a.sr] : 1.0f;
  p.up = fabsf(p.repetition) < 0x1p-100f ? 0x1p40f : 1.0f;   // (a logit that this takes out of the range has an infinite quotient)
  p.divisor = p.repetition * p.up;
  p.inverse = 1.0f / p.divisor;
  p.frequency = a.frequency ? a.frequency[n * a.sf] : 0.0f;
  p.presence = a.presence ? a.presence[n * a.ss] : 0.0f;
  const ID *tokens = static_cast<const ID *>(a.tokens) + n * a.pt, *named = static_cast<const ID *>(a.bias_ids) + n * a.pi;
  ID name = -1;                                        // of the thread's first bias
  if (lists) {
    // (the barriers wait for every load: the list's first part is fetched together with the logits)
    ID first[kAhead];
    int end = 0, mine = 0;
    if (a.tokens) {
      ahead(tokens, a.ts, (int)a.L, first, threadIdx.x);
      end = a.lengths ? cut(a.lengths, a.len64, n * a.sl, (int)a.L) : (int)a.L;
      mine = a.prompt ? cut(a.prompt, a.prompt64, n * a.sp, (int)a.L) : 0;
    }
    if (a.bias && (int)threadIdx.x < (int)a.M) name = named[threadIdx.x];
    for (int i = (int)threadIdx.x * 4; i < len; i += (int)blockDim.x * 4) *reinterpret_cast<uint4 *>(words + i) = make_uint4(0, 0, 0, 0);
    if (threadIdx.x == 0) twice = 0;
    __syncthreads();
    each(tokens, a.ts, end, first, [&](int i, ID id) {
      const uint32_t at = place(id, v0);
      if (at < (uint32_t)len) {
        if (i >= mine) atomicAdd(&words[at], 1u);
        else atomicOr(&words[at], kSeen);
      }
    });
    if (a.bias) {
      for (int i = threadIdx.x; i < (int)a.M; i += blockDim.x) {
        const uint32_t at = place(i < (int)blockDim.x ? name : named[i], v0);
        if (at < (uint32_t)len && (atomicOr(&words[at], kBiased) & kBiased)) twice = 1;
      }
    }
    __syncthreads();
    if (a.bias && twice) {
      if (threadIdx.x < 64) {
        int count = 0;
        for (int i0 = 0; i0 < (int)a.M; i0 += 64) {
          const int i = i0 + (int)threadIdx.x;
          const uint32_t at = i < (int)a.M ? place(named[i], v0) : ~0u;
          const bool in = at < (uint32_t)len;
          const unsigned long long m = __ballot(in);
          const int to = count + __popcll(m & ((1ull << threadIdx.x) - 1));
          if (in && to < kListed) {
            place_of[to] = at;
            bias_of[to] = a.bias[n * a.pb + i];
          }
          count += __popcll(m);
        }
        if (threadIdx.x == 0) listed = count;
      }
      __syncthreads();
    }
  }
#pragma unroll
  for (int k = 0; k < K; ++k) {
    const int i = (int)threadIdx.x * E + k * step;
    if (i + E <= len) {
      uint32_t w[E], any = 0;
      Unit<TO, E> o;
#pragma unroll
      for (int e = 0; e < E; e += 4) {
        const uint4 q = lists ? *reinterpret_cast<const uint4 *>(words + i + e) : make_uint4(0, 0, 0, 0);
        w[e] = q.x; w[e + 1] = q.y; w[e + 2] = q.z; w[e + 3] = q.w;
        any |= q.x | q.y | q.z | q.w;
      }
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const float v = p.apply(u[k].get(e), w[e]);
        o.set(e, bits[k] >> e & 1 ? v : -INFINITY);
      }
      if (any & kBiased) {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (!(w[e] & kBiased)) Elem<TO>::store(out + i + e, o.get(e));
      } else {
        o.store(out + i);
      }
    } else {
      for (int e = 0; e < len - i; ++e) {
        const uint32_t w = lists ? words[i + e] : 0u;
        const float v = p.apply(Elem<TI>::load(z + i + e), w);
        if (!(w & kBiased)) Elem<TO>::store(out + i + e, bits[k] >> e & 1 ? v : -INFINITY);
      }
    }
  }
  if (a.bias) {
    const float *b = a.bias + n * a.pb;
    auto add = [&](uint32_t at, float sum) {
      const float v = p.apply(Elem<TI>::load(z + at), words[at]) + sum;
      Elem<TO>::store(out + at, !allowed || ((uint32_t)allowed[(v0 + at) >> 5] >> ((v0 + at) & 31) & 1) ? v : -INFINITY);
    };
    if (twice && listed <= kListed) {
      // (the thread with an id's first entry adds up those behind it, in their order)
      for (int i = threadIdx.x; i < listed; i += blockDim.x) {
        const uint32_t at = place_of[i];
        float sum = bias_of[i];
        bool first = true;
        for (int j = 0; j < listed; ++j)
          if (j != i && place_of[j] == at) {
            first = first && j > i;
            sum += bias_of[j];
          }
        if (first) add(at, sum);
      }
    } else {
      for (int i = threadIdx.x; i < (int)a.M; i += blockDim.x) {
        const ID id = i < (int)blockDim.x ? name : named[i];
        const uint32_t at = place(id, v0);
        if (at >= (uint32_t)len) continue;
        float sum = b[i];
        bool first = true;
        for (int j = 0; twice && j < (int)a.M; ++j)
          if (j != i && named[j] == id) {
            first = first && j > i;
            sum += b[j];
          }
        if (first) add(at, sum);
      }
    }
  }
}

chn_status row_param(const chn_array *p, const char *name, bool index, int64_t N, int64_t *stride) {
  *stride = 0;
  if (!p) return CHN_OK;
  CHN_TRY(validate(p, name, false));
  if (index ? !is_index(p->dtype) : p->dtype != CHN_F32) return fail(CHN_ERR_DTYPE, "logits_adjust: %s must be %s", name, index ? "I32 or I64" : "F32");
  if (p->ndim != 1 || p->shape[0] != N) return fail(CHN_ERR_SHAPE, "logits_adjust: %s must have shape (%lld,)", name, (long long)N);
  *stride = N > 1 ? p->strides[0] / dtype_size(p->dtype) : 0;
  return CHN_OK;
}

// A list for each row: (N,n), any pitch, 0 for one list for all; unit inner stride, or any where `step` takes it.
chn_status row_list(const chn_array *p, const char *name, int64_t N, int64_t *n, int64_t *pitch, int64_t *step = nullptr) {
  CHN_TRY(validate(p, name, false));
  if (p->ndim != 2) return fail(CHN_ERR_NDIM, "logits_adjust: %s must have 2 dimensions, got %d", name, p->ndim);
  if (p->shape[0] != N) return fail(CHN_ERR_SHAPE, "logits_adjust: %s must have %lld rows", name, (long long)N);
  const int isz = dtype_size(p->dtype);
  if (step) *step = p->shape[1] > 1 ? p->strides[1] / isz : 0;
  else if (p->shape[1] > 1 && p->strides[1] != isz) return fail(CHN_ERR_STRIDE, "logits_adjust: the last axis of %s must have unit stride", name);
  *n = p->shape[1];
  *pitch = N > 1 ? p->strides[0] / isz : 0;
  return CHN_OK;
}

}  // namespace
}  // namespace chn

extern "C" {

chn_status chn_logits_adjust(const chn_array *logits, const chn_array *tokens, const chn_array *lengths, const chn_array *prompt,
                             const chn_array *repetition, const chn_array *frequency, const chn_array *presence, const chn_array *bias_ids,
                             const chn_array *bias, const chn_array *allowed, const chn_array *out, chn_stream stream) {
  using namespace chn;
  AdjustArgs a = {};
  int64_t on, ov, words;
  CHN_TRY(validate(logits, "logits", false));
  CHN_TRY(validate(out, "out", true));
  if (!is_float(logits->dtype) || !is_float(out->dtype)) return fail(CHN_ERR_DTYPE, "logits_adjust: logits and out must be F32 or BF16");
  CHN_TRY(row_major_2d(logits, "logits", &a.N, &a.V, &a.pz));
  CHN_TRY(row_major_2d(out, "out", &on, &ov, &a.po));
  const int64_t N = a.N;
  if (on != N || ov != a.V) return fail(CHN_ERR_SHAPE, "logits_adjust: out must have shape (%lld,%lld)", (long long)N, (long long)a.V);
  if (a.V > 0x7fffffff || N > 0x7fffffff) return fail(CHN_ERR_SHAPE, "logits_adjust: (%lld,%lld) logits", (long long)N, (long long)a.V);
  if (!bias != !bias_ids) return fail(CHN_ERR_NULL, "logits_adjust: bias and bias_ids come together");
  CHN_TRY(row_param(lengths, "lengths", true, N, &a.sl));
  CHN_TRY(row_param(prompt, "prompt", true, N, &a.sp));
  CHN_TRY(row_param(repetition, "repetition", false, N, &a.sr));
  CHN_TRY(row_param(frequency, "frequency", false, N, &a.sf));
  CHN_TRY(row_param(presence, "presence", false, N, &a.ss));
  bool id64 = true;
  if (tokens) {
    CHN_TRY(row_list(tokens, "tokens", N, &a.L, &a.pt, &a.ts));
    if (!is_index(tokens->dtype)) return fail(CHN_ERR_DTYPE, "logits_adjust: tokens must be I32 or I64");
    if (a.L >= 1 << 30) return fail(CHN_ERR_SHAPE, "logits_adjust: lists of %lld tokens", (long long)a.L);
    id64 = tokens->dtype == CHN_I64;
  }
  if (bias) {
    int64_t m;
    CHN_TRY(row_list(bias_ids, "bias_ids", N, &a.M, &a.pi));
    CHN_TRY(row_list(bias, "bias", N, &m, &a.pb));
    if (!is_index(bias_ids->dtype)) return fail(CHN_ERR_DTYPE, "logits_adjust: bias_ids must be I32 or I64");
    if (bias->dtype != CHN_F32) return fail(CHN_ERR_DTYPE, "logits_adjust: bias must be F32");
    if (a.M >= 1 << 30) return fail(CHN_ERR_SHAPE, "logits_adjust: lists of %lld biases", (long long)a.M);
    if (m != a.M) return fail(CHN_ERR_SHAPE, "logits_adjust: %lld biases for %lld ids", (long long)m, (long long)a.M);
    if (tokens && (bias_ids->dtype == CHN_I64) != id64) return fail(CHN_ERR_DTYPE, "logits_adjust: tokens and bias_ids must have one dtype");
    id64 = bias_ids->dtype == CHN_I64;
  }
  if (allowed) {
    CHN_TRY(row_list(allowed, "allowed", N, &words, &a.pa));
    if (allowed->dtype != CHN_I32) return fail(CHN_ERR_DTYPE, "logits_adjust: allowed must be I32");
    if (words != (a.V + 31) / 32) return fail(CHN_ERR_SHAPE, "logits_adjust: allowed must have shape (%lld,%lld)", (long long)N, (long long)((a.V + 31) / 32));
    a.allowed = static_cast<const int32_t *>(allowed->data);
  }
  if (N == 0 || a.V == 0) return CHN_OK;
  a.z = logits->data; a.out = out->data;
  if (tokens && a.L > 0) a.tokens = tokens->data;
  if (lengths) { a.lengths = lengths->data; a.len64 = lengths->dtype == CHN_I64; }
  if (prompt) { a.prompt = prompt->data; a.prompt64 = prompt->dtype == CHN_I64; }
  if (a.tokens) {
    if (repetition) a.repetition = static_cast<const float *>(repetition->data);
    if (frequency) a.frequency = static_cast<const float *>(frequency->data);
    if (presence) a.presence = static_cast<const float *>(presence->data);
  }
  if (bias && a.M > 0) { a.bias = static_cast<const float *>(bias->data); a.bias_ids = bias_ids->data; }
  const int E = logits->dtype == CHN_F32 && out->dtype == CHN_F32 ? 4 : 8;
// From 2^21 logits on in rows of two large pieces and more a thread holds kHeld logits, below one unit (us: 16 x 131072 with lists of 8192 tokens 9.4 / 13.4, 64 x 32768 8.4 / 9.8,
  // 128 x 65536 18.7 / 25.0, 256 x 32768 22.4 / 37.7; 8 x 131072 7.7 / 6.7, 1 x 131072 7.1 / 5.3, and of rows that leave a large piece mostly empty 256 x 10000 14.3 / 11.1): the
  // list is looked through once for a piece.
  const bool large = a.V * N >= 1 << 21 && a.V >= 2 * kThreads * kHeld;
  const int threads = large ? kThreads : 256;
  a.tile = threads * (large ? kHeld : E);
  a.tiles = (a.V + a.tile - 1) / a.tile;
  const size_t lds = a.tokens || a.bias ? (size_t)(a.tile < (a.V + 3) / 4 * 4 ? a.tile : (a.V + 3) / 4 * 4) * 4 : 0;
  hipStream_t st = as_stream(stream);
  const dim3 grid = grid_of(N * a.tiles), block(threads);
#define CHN_GO(TI, TO, H)                                                                                                         \
  do {                                                                                                                            \
    if (id64 && large) hipLaunchKernelGGL((adjust_kernel<TI, TO, int64_t, H>), grid, block, lds, st, a);                          \
    else if (id64) hipLaunchKernelGGL((adjust_kernel<TI, TO, int64_t, 1>), grid, block, lds, st, a);                              \
    else if (large) hipLaunchKernelGGL((adjust_kernel<TI, TO, int32_t, H>), grid, block, lds, st, a);                             \
    else hipLaunchKernelGGL((adjust_kernel<TI, TO, int32_t, 1>), grid, block, lds, st, a);                                        \
  } while (0)
  if (logits->dtype == CHN_F32) { if (out->dtype == CHN_F32) CHN_GO(float, float, kHeld / 4); else CHN_GO(float, bf16_raw, kHeld / 8); }
  else { if (out->dtype == CHN_F32) CHN_GO(bf16_raw, float, kHeld / 8); else CHN_GO(bf16_raw, bf16_raw, kHeld / 8); }
#undef CHN_GO
  return check_launch("logits_adjust");
}

}  // extern "C"
