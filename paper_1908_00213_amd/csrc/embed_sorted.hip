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

// ---- the ids in order -------------------------------------------------------------------------------------------
// (key, place) pairs are sorted by key, places of one key in their order: a radix sort from the low digits up, every pass of which keeps the order of
// equal digits.  Keys are ids, of ids outside the table V, which is sorted behind all of them and left out from there on.

constexpr int kMaxBits = 9, kBins = 1 << kMaxBits;           // of a digit
constexpr int kSortWaves = 16;

struct SortArgs {
  const void *ids;                   // pass 0 reads these
  const uint32_t *keys, *places;     // later ones these
  uint32_t *keys_out, *places_out;
  uint32_t *counts;                  // (blocks, bins)
  uint32_t *ends;                    // (V), which the first launch clears
  int64_t stride, V;
  uint32_t N, share;                 // pairs of a block
  int id64, shift, bits, blocks, first;
};

__device__ __forceinline__ uint32_t key_of(const SortArgs &s, bool first, const uint32_t *keys, uint32_t i) {
  if (!first) return keys[i];
  return (uint32_t)(s.id64 ? id_at(static_cast<const int64_t *>(s.ids), i, s.stride, s.V) : id_at(static_cast<const int32_t *>(s.ids), i, s.stride, s.V));
}

__device__ __forceinline__ void clear_ends(uint32_t *ends, int64_t V, int64_t block, int64_t blocks) {
  for (int64_t i = block * 1024 + threadIdx.x; i < V; i += blocks * 1024) ends[i] = 0;
}

// How often a block's share has each digit.
__global__ __launch_bounds__(1024) void embed_count_kernel(SortArgs s) {
  __shared__ uint32_t count[kBins];
  if (threadIdx.x < kBins) count[threadIdx.x] = 0;
  __syncthreads();
  const uint32_t lo = blockIdx.x * s.share, hi = min(lo + s.share, s.N), mask = (1u << s.bits) - 1;
  for (uint32_t i = lo + threadIdx.x; i < hi; i += 1024) atomicAdd(&count[key_of(s, s.first, s.keys, i) >> s.shift & mask], 1u);
  if (s.first) clear_ends(s.ends, s.V, blockIdx.x, gridDim.x);
  __syncthreads();
  if (threadIdx.x <= mask) s.counts[blockIdx.x * kBins + threadIdx.x] = count[threadIdx.x];
}

struct SortShared {
  uint32_t at[kSortWaves][kBins];    // where a wave's next pair of a digit goes
  uint32_t sums[kSortWaves];
};

// One pass over the block's share [lo, hi), split over the waves.  Before it: the same digit in the blocks before, smaller digits anywhere.
__device__ __forceinline__ void sort_pass(const SortArgs &s, SortShared &sh, bool first, const uint32_t *keys, const uint32_t *places, uint32_t *keys_out,
                                          uint32_t *places_out, uint32_t lo, uint32_t hi, int shift, const uint32_t *counts, int block, int blocks) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t mask = (1u << s.bits) - 1;
  for (int i = tid; i < kSortWaves * kBins; i += 1024) (&sh.at[0][0])[i] = 0;
  __syncthreads();
  const uint32_t part = ((hi - lo + kSortWaves - 1) / kSortWaves + 63) / 64 * 64;
  const uint32_t from = min(lo + wave * part, hi), to = min(from + part, hi);
  for (uint32_t i = from + lane; i < to; i += 64) atomicAdd(&sh.at[wave][key_of(s, first, keys, i) >> shift & mask], 1u);
  __syncthreads();
  uint32_t mine = 0, all = 0;
  if (tid < kBins) {
    if (blocks == 1) {
      for (int w = 0; w < kSortWaves; ++w) all += sh.at[w][tid];
    } else if (tid <= (int)mask) {
#pragma unroll 8
      for (int b = 0; b < blocks; ++b) {
        const uint32_t c = counts[b * kBins + tid];
        mine += b < block ? c : 0;
        all += c;
      }
    }
  }
  uint32_t run = all;                                        // running sums over the digits: in the wave, then over the waves
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t up = __shfl_up(run, o, 64);
    if (lane >= o) run += up;
  }
  if (lane == 63) sh.sums[wave] = run;
  __syncthreads();
  if (tid < kBins) {
    uint32_t base = run - all + mine;
    for (int w = 0; w < wave; ++w) base += sh.sums[w];
    for (int w = 0; w < kSortWaves; ++w) {
      const uint32_t c = sh.at[w][tid];
      sh.at[w][tid] = base;
      base += c;
    }
  }
  __syncthreads();
  for (uint32_t i0 = from; i0 < to; i0 += 64) {
    const uint32_t i = i0 + lane;
    const bool on = i < to;
    const uint32_t key = on ? key_of(s, first, keys, i) : 0, place = on && !first ? places[i] : i, digit = key >> shift & mask;
    unsigned long long same = __ballot(on);
    for (int b = 0; b < s.bits; ++b) {
      const bool bit = digit >> b & 1;
      const unsigned long long m = __ballot(bit);
      same &= bit ? m : ~m;
    }
    if (on) {
      const uint32_t rank = __popcll(same & ((1ull << lane) - 1)), to_ = sh.at[wave][digit] + rank;
      keys_out[to_] = key;
      places_out[to_] = place;
    }
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
    if (on && same >> lane == 1) sh.at[wave][digit] += __popcll(same);   // (the digit's last lane)
    __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
    __builtin_amdgcn_wave_barrier();
  }
}

__global__ __launch_bounds__(1024) void embed_sort_kernel(SortArgs s) {
  __shared__ SortShared sh;
  const uint32_t lo = min(blockIdx.x * s.share, s.N), hi = min(lo + s.share, s.N);
  sort_pass(s, sh, s.first, s.keys, s.places, s.keys_out, s.places_out, lo, hi, s.shift, s.counts, blockIdx.x, s.blocks);
}

// Few ids: one block makes all passes, the others clear.  `keys` and `places` are the memory between two passes; the last one ends in the outputs.
__global__ __launch_bounds__(1024) void embed_sort_few_kernel(SortArgs s, int passes, uint32_t *keys_between, uint32_t *places_between) {
  if (blockIdx.x > 0) {
    clear_ends(s.ends, s.V, blockIdx.x - 1, gridDim.x - 1);
    return;
  }
  __shared__ SortShared sh;
  const uint32_t *keys = nullptr, *places = nullptr;
  for (int p = 0; p < passes; ++p) {
    const bool out = (passes - 1 - p) % 2 == 0;
    uint32_t *ko = out ? s.keys_out : keys_between, *po = out ? s.places_out : places_between;
    sort_pass(s, sh, p == 0, keys, places, ko, po, 0, s.N, p * s.bits, nullptr, 0, 1);
    __threadfence_block();
    __syncthreads();
    keys = ko;
    places = po;
  }
}

// ---- the sums -----------------------------------------------------------------------------------------------------
constexpr int kPiece = 64;           // places of a piece: tokens with more of them than that are summed by pieces
constexpr int kTogether = 8;         // rows in flight

struct SumArgs {
  const uint32_t *keys, *places;
  uint32_t *starts, *ends;           // (V): a token's places in the sorted list; an end of 0 where it has none
  const void *dout;
  float *dtable, *partial;           // (pieces, 2, pitch): of a piece's first and of its last token, where they stand often
  int64_t dp, tp, pitch, V, D, chunks, pieces;
  float scale;
  uint32_t N;
  int accumulate;
};

__global__ __launch_bounds__(256) void embed_ranges_kernel(SumArgs s) {
  const uint32_t i = blockIdx.x * 256 + threadIdx.x;
  if (i >= s.N) return;
  const uint32_t k = s.keys[i];
  if (k >= s.V) return;
  if (i == 0 || s.keys[i - 1] != k) s.starts[k] = i;
  if (i == s.N - 1 || s.keys[i + 1] != k) s.ends[k] = i + 1;
}

// The sum of the rows at places [lo, hi) in a lane's columns, in their order.
template <typename T, int E>
__device__ __forceinline__ void sum_rows(const SumArgs &s, uint32_t lo, uint32_t hi, int64_t d, float (&sum)[E]) {
  const T *base = static_cast<const T *>(s.dout) + d;
#pragma unroll
  for (int e = 0; e < E; ++e) sum[e] = 0.0f;
  if (d >= s.D) return;
  if (d + E <= s.D) {
    for (uint32_t i = lo; i < hi; i += kTogether) {
      Unit<T, E> u[kTogether];
#pragma unroll
      for (int k = 0; k < kTogether; ++k) u[k].load(base + (int64_t)s.places[min(i + k, hi - 1)] * s.dp);
#pragma unroll
      for (int k = 0; k < kTogether; ++k)
        if (i + k < hi) {
#pragma unroll
          for (int e = 0; e < E; ++e) sum[e] += u[k].get(e);
        }
    }
  } else {
    for (uint32_t i = lo; i < hi; ++i) {
      const T *row = base + (int64_t)s.places[i] * s.dp;
#pragma unroll
      for (int e = 0; e < E; ++e)
        if (d + e < s.D) sum[e] += Elem<T>::load(row + e);
    }
  }
}

template <int E>
__device__ __forceinline__ void write_row(const SumArgs &s, int64_t v, int64_t d, const float (&sum)[E]) {
  float *p = s.dtable + v * s.tp + d;
  if (d + E <= s.D) {
    Unit<float, E> u;
    if (s.accumulate) u.load(p);
#pragma unroll
    for (int e = 0; e < E; ++e) u.set(e, s.accumulate ? fmaf(s.scale, sum[e], u.get(e)) : s.scale * sum[e]);
    u.store(p);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (d + e < s.D) p[e] = s.accumulate ? fmaf(s.scale, sum[e], p[e]) : s.scale * sum[e];
  }
}

__device__ __forceinline__ bool often(const SumArgs &s, uint32_t v) { return v < s.V && s.ends[v] - s.starts[v] > kPiece; }

// A wave for each (piece, chunk of columns), then for each (row of the table, chunk).
template <typename T>
__global__ __launch_bounds__(256) void embed_sum_kernel(SumArgs s) {
  constexpr int E = unit_elements<T>();
  const int lane = threadIdx.x & 63;
  int64_t job = block_number() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  float sum[E];
  if (job < s.pieces * s.chunks) {
    const int64_t piece = job / s.chunks, d = ((job - piece * s.chunks) * 64 + lane) * E;
    const uint32_t lo = (uint32_t)piece * kPiece, hi = min(lo + kPiece, s.N), f = s.keys[lo], l = s.keys[hi - 1];
    for (int side = 0; side < 2; ++side) {
      const uint32_t v = side ? l : f;
      if ((side && l == f) || !often(s, v)) continue;
      sum_rows<T, E>(s, side ? s.starts[v] : lo, side ? hi : min(hi, s.ends[v]), d, sum);
      if (d < s.D) {
        Unit<float, E> u;
#pragma unroll
        for (int e = 0; e < E; ++e) u.set(e, sum[e]);
        u.store(s.partial + (piece * 2 + side) * s.pitch + d);
      }
    }
    return;
  }
  job -= s.pieces * s.chunks;
  const int64_t v = job / s.chunks, d = ((job - v * s.chunks) * 64 + lane) * E;
  if (v >= s.V || d >= s.D) return;
  const uint32_t hi = s.ends[v];
  if (hi == 0) {
    if (s.accumulate) return;
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] = 0.0f;
  } else {
    const uint32_t lo = s.starts[v];
    if (hi - lo > kPiece) return;
    sum_rows<T, E>(s, lo, hi, d, sum);
  }
  write_row<E>(s, v, d, sum);
}

// The pieces of the token that stands often and begins in the block's piece, if there is one: sixteen waves take neighbouring shares of them.
template <int E>
__global__ __launch_bounds__(1024) void embed_join_kernel(SumArgs s) {
  __shared__ float parts[kSortWaves][E][64];
  const int64_t job = block_number(), piece = job / s.chunks;
  if (piece >= s.pieces) return;
  const uint32_t lo = (uint32_t)piece * kPiece, hi = min(lo + kPiece, s.N), v = s.keys[hi - 1];
  if (!often(s, v) || s.starts[v] < lo) return;
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t d = ((job - piece * s.chunks) * 64 + lane) * E;
  const int64_t last = (s.ends[v] - 1) / kPiece, share = (last - piece + kSortWaves) / kSortWaves;
  const int64_t from = piece + wave * share, to = min(from + share, last + 1);
  float sum[E];
#pragma unroll
  for (int e = 0; e < E; ++e) sum[e] = 0.0f;
  if (d < s.D) {
    for (int64_t i = from; i < to; i += kTogether) {
      Unit<float, E> u[kTogether];
#pragma unroll
      for (int k = 0; k < kTogether; ++k) {
        const int64_t p = min(i + k, to - 1);
        u[k].load(s.partial + (p * 2 + (p == piece && s.starts[v] != lo)) * s.pitch + d);   // (of the first piece the last token, of the others the first)
      }
#pragma unroll
      for (int k = 0; k < kTogether; ++k)
        if (i + k < to) {
#pragma unroll
          for (int e = 0; e < E; ++e) sum[e] += u[k].get(e);
        }
    }
  }
#pragma unroll
  for (int e = 0; e < E; ++e) parts[wave][e][lane] = sum[e];
  __syncthreads();
  if (wave > 0 || d >= s.D) return;
#pragma unroll
  for (int e = 0; e < E; ++e)
    for (int w = 1; w < kSortWaves; ++w) sum[e] += parts[w][e][lane];
  write_row<E>(s, v, d, sum);
}

// The workspace, in the order in which its parts lie.
struct Layout {
  int bits, passes, blocks;
  uint32_t share;
  int64_t pieces, pitch;
  size_t keys, between, places, places_between, counts, starts, ends, partial, bytes;
  Layout(int64_t N, int64_t V, int64_t D) {
    int whole = 1;
    while (whole < 32 && (V >> whole)) ++whole;              // keys are 0 .. V
    passes = (whole + kMaxBits - 1) / kMaxBits;
    bits = (whole + passes - 1) / passes;
    blocks = (int)(N <= kFew ? 1 : N / 2048 < 64 ? N / 2048 : 64);
    share = (uint32_t)((N + blocks - 1) / blocks);
    pieces = (N + kPiece - 1) / kPiece;
    pitch = (D + 7) / 8 * 8;
    size_t at = 0;
    auto put = [&](size_t n) { const size_t here = at; at += (n + 255) / 256 * 256; return here; };
    keys = put(4 * (size_t)N);
    places = put(4 * (size_t)N);
    between = put(passes > 1 ? 4 * (size_t)N : 0);
    places_between = put(passes > 1 ? 4 * (size_t)N : 0);
    counts = put(blocks > 1 ? 4 * (size_t)blocks * kBins : 0);
    starts = put(4 * (size_t)V);
    ends = put(4 * (size_t)V);
    partial = put(8 * (size_t)pieces * pitch);
    bytes = at;
  }
  static constexpr int64_t kFew = 8192;
};

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

size_t chn_embed_sorted_workspace_bytes(const chn_array *ids, const chn_array *dtable) {
  using namespace chn;
  if (!ids || !dtable || ids->ndim != 1 || dtable->ndim != 2) return 0;
  const int64_t N = ids->shape[0], V = dtable->shape[0], D = dtable->shape[1];
  if (N < 0 || V <= 0 || D <= 0 || N > 0x7fffffff || V > 0x7fffffff) return 0;
  return Layout(N, V, D).bytes;
}

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
  const Layout z(N, V, D);
  char *w = static_cast<char *>(ws);
  hipStream_t st = as_stream(stream);
  auto words = [&](size_t at) { return reinterpret_cast<uint32_t *>(w + at); };
  SortArgs o = {};
  o.ids = ids->data; o.stride = is; o.id64 = ids->dtype == CHN_I64;
  o.V = V; o.N = (uint32_t)N; o.share = z.share; o.bits = z.bits; o.blocks = z.blocks;
  o.counts = words(z.counts); o.ends = words(z.ends);
  o.keys_out = words(z.keys); o.places_out = words(z.places);
  if (z.blocks == 1) {
    const int64_t clearing = (V + 4095) / 4096;
    hipLaunchKernelGGL(embed_sort_few_kernel, dim3(1 + (unsigned)(clearing < 256 ? clearing : 256)), dim3(1024), 0, st, o, z.passes, words(z.between),
                       words(z.places_between));
    CHN_TRY(check_launch("embed_sorted_bwd"));
  } else {
    for (int p = 0; p < z.passes; ++p) {
      const bool last = (z.passes - 1 - p) % 2 == 0;         // the last pass ends in `keys`
      o.first = p == 0;
      o.shift = p * z.bits;
      o.keys = words(last ? z.between : z.keys); o.places = words(last ? z.places_between : z.places);
      o.keys_out = words(last ? z.keys : z.between); o.places_out = words(last ? z.places : z.places_between);
      hipLaunchKernelGGL(embed_count_kernel, dim3(z.blocks), dim3(1024), 0, st, o);
      CHN_TRY(check_launch("embed_sorted_bwd"));
      hipLaunchKernelGGL(embed_sort_kernel, dim3(z.blocks), dim3(1024), 0, st, o);
      CHN_TRY(check_launch("embed_sorted_bwd"));
    }
  }
  const int E = dout->dtype == CHN_F32 ? 4 : 8;
  SumArgs s = {};
  s.keys = words(z.keys); s.places = words(z.places); s.starts = words(z.starts); s.ends = words(z.ends);
  s.dout = dout->data; s.dtable = static_cast<float *>(dtable->data); s.partial = reinterpret_cast<float *>(w + z.partial);
  s.dp = dp; s.tp = tp; s.pitch = z.pitch; s.V = V; s.D = D; s.chunks = (D + 64 * E - 1) / (64 * E); s.pieces = z.pieces;
  s.scale = (float)scale; s.N = (uint32_t)N; s.accumulate = accumulate;
  if (N > 0) {
    hipLaunchKernelGGL(embed_ranges_kernel, dim3((unsigned)((N + 255) / 256)), dim3(256), 0, st, s);
    CHN_TRY(check_launch("embed_sorted_bwd"));
  }
  const dim3 grid = grid_of(((z.pieces + V) * s.chunks + 3) / 4);
  if (dout->dtype == CHN_F32) hipLaunchKernelGGL((embed_sum_kernel<float>), grid, dim3(256), 0, st, s);
  else hipLaunchKernelGGL((embed_sum_kernel<bf16_raw>), grid, dim3(256), 0, st, s);
  CHN_TRY(check_launch("embed_sorted_bwd"));
  if (N <= kPiece) return CHN_OK;                            // (no token stands more often)
  if (dout->dtype == CHN_F32) hipLaunchKernelGGL((embed_join_kernel<4>), grid_of(z.pieces * s.chunks), dim3(1024), 0, st, s);
  else hipLaunchKernelGGL((embed_join_kernel<8>), grid_of(z.pieces * s.chunks), dim3(1024), 0, st, s);
  return check_launch("embed_sorted_bwd");
}

}  // extern "C"
