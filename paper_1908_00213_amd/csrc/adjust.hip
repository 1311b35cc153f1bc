// chn_logits_adjust: what a row's text, its caller and its grammar say about its logits, in one pass over them.
//
// A block owns a piece of one row.  It counts the piece's tokens in LDS while it looks through the row's whole list (a 32-bit word for a token: how
// often it stands behind the prompt, whether the prompt has it, whether it has a bias), then walks over the piece once: a read and a write for each logit.
// Whole numbers are counted, so the order in which the list is seen does not show.  The few tokens with biases are left out by that walk: the threads
// that hold the list's entries write them, each token by the thread with its first entry, which adds up the others in the list's order.
#include "rows.h"

namespace chn {
namespace {

constexpr uint32_t kSeen = 0x80000000u, kBiased = 0x40000000u, kCount = 0x3fffffffu;

struct AdjustArgs {
  const void *z;
  void *out;
  const void *tokens, *lengths, *prompt, *bias_ids;
  const float *repetition, *frequency, *presence, *bias;
  const int32_t *allowed;
  int64_t N, V, L, M, pz, po, pt, pi, pb, pa;      // sizes, pitches
  int64_t sl, sp, sr, sf, ss;                   // strides of lengths, prompt, repetition, frequency, presence
  int64_t tiles, tile;                          // pieces of a row, tokens of a piece
  int len64, prompt64;
};

__device__ __forceinline__ int64_t cut(const void *p, int is64, int64_t at, int64_t L) {
  const int64_t n = is64 ? static_cast<const int64_t *>(p)[at] : static_cast<const int32_t *>(p)[at];
  return n < 0 ? 0 : n > L ? L : n;
}

struct Penalties {
  float repetition, frequency, presence;
  bool rep, freq, pres;
  __device__ __forceinline__ float apply(float z, uint32_t word) const {
    const uint32_t c = word & kCount;
    if (rep && (word & (kSeen | kCount))) z = z > 0.0f ? z / repetition : z * repetition;
    if (freq) z = fmaf(-frequency, (float)c, z);
    if (pres && c) z -= presence;
    return z;
  }
};

template <typename TI, typename TO, typename ID>
__global__ __launch_bounds__(256) void adjust_kernel(AdjustArgs a) {
  extern __shared__ uint32_t words[];
  __shared__ int twice;
  constexpr int E = unit_elements<TI, TO>();
  const int64_t n = block_number() / a.tiles, v0 = (block_number() - n * a.tiles) * a.tile;
  if (n >= a.N) return;                                // (the grid's last line may be longer than its blocks)
  const int len = (int)min(a.tile, a.V - v0);
  const TI *z = static_cast<const TI *>(a.z) + n * a.pz + v0;
  TO *out = static_cast<TO *>(a.out) + n * a.po + v0;
  const bool lists = a.tokens || a.bias;
  if (lists) {
    for (int i = threadIdx.x; i < len; i += 256) words[i] = 0;
    if (threadIdx.x == 0) twice = 0;
    __syncthreads();
    if (a.tokens) {
      const ID *t = static_cast<const ID *>(a.tokens) + n * a.pt;
      const int64_t end = a.lengths ? cut(a.lengths, a.len64, n * a.sl, a.L) : a.L, mine = a.prompt ? cut(a.prompt, a.prompt64, n * a.sp, a.L) : 0;
      for (int64_t i = threadIdx.x; i < end; i += 256) {
        const int64_t at = (int64_t)t[i] - v0;
        if ((uint64_t)at < (uint64_t)len) {
          if (i >= mine) atomicAdd(&words[at], 1u);
          else atomicOr(&words[at], kSeen);
        }
      }
    }
    if (a.bias) {
      const ID *t = static_cast<const ID *>(a.bias_ids) + n * a.pi;
      for (int64_t i = threadIdx.x; i < a.M; i += 256) {
        const int64_t at = (int64_t)t[i] - v0;
        if ((uint64_t)at < (uint64_t)len && (atomicOr(&words[at], kBiased) & kBiased)) twice = 1;
      }
    }
    __syncthreads();
  }
  Penalties p;
  p.rep = a.repetition != nullptr; p.freq = a.frequency != nullptr; p.pres = a.presence != nullptr;
  p.repetition = p.rep ? a.repetition[n * a.sr] : 1.0f;
  p.frequency = p.freq ? a.frequency[n * a.sf] : 0.0f;
  p.presence = p.pres ? a.presence[n * a.ss] : 0.0f;
  const int32_t *allowed = a.allowed ? a.allowed + n * a.pa : nullptr;
  for (int i = (int)threadIdx.x * E; i < len; i += 256 * E) {
    const uint32_t bits = allowed ? (uint32_t)allowed[(v0 + i) >> 5] >> ((v0 + i) & 31) : ~0u;
    if (i + E <= len) {
      Unit<TI, E> u;
      Unit<TO, E> o;
      u.load(z + i);
      uint32_t any = 0;
#pragma unroll
      for (int e = 0; e < E; ++e) {
        const uint32_t w = lists ? words[i + e] : 0u;
        any |= w;
        float v = u.get(e);
        if (w) v = p.apply(v, w);
        o.set(e, bits >> e & 1 ? v : -INFINITY);
      }
      if (any & kBiased) {
#pragma unroll
        for (int e = 0; e < E; ++e)
          if (!(words[i + e] & kBiased)) Elem<TO>::store(out + i + e, o.get(e));
      } else {
        o.store(out + i);
      }
    } else {
      for (int e = 0; e < len - i; ++e) {
        const uint32_t w = lists ? words[i + e] : 0u;
        float v = Elem<TI>::load(z + i + e);
        if (w) v = p.apply(v, w);
        if (!(w & kBiased)) Elem<TO>::store(out + i + e, bits >> e & 1 ? v : -INFINITY);
      }
    }
  }
  if (a.bias) {
    const ID *t = static_cast<const ID *>(a.bias_ids) + n * a.pi;
    const float *b = a.bias + n * a.pb;
    for (int64_t i = threadIdx.x; i < a.M; i += 256) {
      const int64_t id = (int64_t)t[i], at = id - v0;
      if ((uint64_t)at >= (uint64_t)len) continue;
      float sum = b[i];
      if (twice) {                                       // (the same id more than once, somewhere in this piece)
        sum = 0.0f;
        bool first = true;
        for (int64_t j = 0; j < a.M; ++j)
          if ((int64_t)t[j] == id) {
            first = first && j >= i;
            sum = j == i && first ? b[j] : sum + b[j];
          }
        if (!first) continue;
      }
      const float v = p.apply(Elem<TI>::load(z + at), words[at]) + sum;
      Elem<TO>::store(out + at, !allowed || ((uint32_t)allowed[id >> 5] >> (id & 31) & 1) ? v : -INFINITY);
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

// A list for each row: (N,n), unit inner stride, any pitch, 0 for one list for all.
chn_status row_list(const chn_array *p, const char *name, int64_t N, int64_t *n, int64_t *pitch) {
  CHN_TRY(validate(p, name, false));
  if (p->ndim != 2) return fail(CHN_ERR_NDIM, "logits_adjust: %s must have 2 dimensions, got %d", name, p->ndim);
  if (p->shape[0] != N) return fail(CHN_ERR_SHAPE, "logits_adjust: %s must have %lld rows", name, (long long)N);
  const int isz = dtype_size(p->dtype);
  if (p->shape[1] > 1 && p->strides[1] != isz) return fail(CHN_ERR_STRIDE, "logits_adjust: the last axis of %s must have unit stride", name);
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
    CHN_TRY(row_list(tokens, "tokens", N, &a.L, &a.pt));
    if (!is_index(tokens->dtype)) return fail(CHN_ERR_DTYPE, "logits_adjust: tokens must be I32 or I64");
    if (a.L >= (1 << 30)) return fail(CHN_ERR_SHAPE, "logits_adjust: lists of %lld tokens", (long long)a.L);
    id64 = tokens->dtype == CHN_I64;
  }
  if (bias) {
    int64_t m;
    CHN_TRY(row_list(bias_ids, "bias_ids", N, &a.M, &a.pi));
    CHN_TRY(row_list(bias, "bias", N, &m, &a.pb));
    if (!is_index(bias_ids->dtype)) return fail(CHN_ERR_DTYPE, "logits_adjust: bias_ids must be I32 or I64");
    if (bias->dtype != CHN_F32) return fail(CHN_ERR_DTYPE, "logits_adjust: bias must be F32");
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
  // Pieces of at most 8192 tokens (32 KiB of words: four blocks on a compute unit), shorter ones while the launch has fewer than 1024 blocks.
  int64_t tile = (a.V * N / 1024 + 1023) / 1024 * 1024;
  tile = tile < 1024 ? 1024 : tile > 8192 ? 8192 : tile;
  a.tile = tile;
  a.tiles = (a.V + tile - 1) / tile;
  const size_t lds = a.tokens || a.bias ? (size_t)tile * 4 : 0;
  hipStream_t st = as_stream(stream);
  const dim3 grid = grid_of(N * a.tiles);
#define CHN_GO(TI, TO)                                                                                                            \
  do {                                                                                                                            \
    if (id64) hipLaunchKernelGGL((adjust_kernel<TI, TO, int64_t>), grid, dim3(256), lds, st, a);                                  \
    else hipLaunchKernelGGL((adjust_kernel<TI, TO, int32_t>), grid, dim3(256), lds, st, a);                                       \
  } while (0)
  if (logits->dtype == CHN_F32) { if (out->dtype == CHN_F32) CHN_GO(float, float); else CHN_GO(float, bf16_raw); }
  else { if (out->dtype == CHN_F32) CHN_GO(bf16_raw, float); else CHN_GO(bf16_raw, bf16_raw); }
#undef CHN_GO
  return check_launch("logits_adjust");
}

}  // extern "C"
