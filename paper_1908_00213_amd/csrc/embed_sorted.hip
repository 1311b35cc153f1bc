// chn_embed_scaled_fwd / chn_embed_sorted_bwd: the lookup with its scale, and the table's gradient.
//
// The gradient sums rows of dout by token.  The ids are sorted (which keeps a token's places in the order of n), and then
//   - a wave for a row of the table (several rows of a large table, 64 units of columns) adds up the rows of its token, or writes zeros;
//   - tokens with more than 64 places are summed by pieces of 64 places of the sorted list, and these sums joined in a launch of its own: a word that is every tenth of a
//     text would otherwise be one wave's work.
// Every order is fixed by the ids alone.  Up to 256 ids are not sorted: every wave looks for its rows' tokens among them (1 x 650 into 10000 rows 21 -> 9 us, 128 ids 21 -> 9;
// 512 ids 18 with the sort, 25 without).
//
// Bound by memory for a large table: 65536 x 1024 bf16 into 131072 rows 30 us for the lookup (4.5 TB/s of its output), 155 for the gradient, of which clearing 537 MB takes 104 (5.2 TB/s)
// while a few blocks sort beside it, and sums 40.  Cleared by the launch that sums, it was 31 us for the sort alone and 146 for the sums.  Stores past the caches: what
// follows does not wait for their lines to leave (the lookup 41 us and the sums 58 with ordinary stores).  Small cases are launches: 4480 x 650 into 10000 rows 13 (one block sorts), 13 and 5 traced.
#include "rows.h"

namespace chn {
namespace {

template <typename L>
__device__ __forceinline__ int64_t id_at(const L *ids, int64_t n, int64_t stride, int64_t V) {
  const int64_t id = (int64_t)ids[n * stride];
  return (uint64_t)id < (uint64_t)V ? id : V;            // an id outside the table is never used as an offset
}

// Units of a row, whichever rows they belong to, one after the other: a thread has kUnits of them, whose ids and then whose units are on their way
// together, at whatever address they have.  What is left of a row behind its last whole unit goes element by element.
constexpr int kUnits = 4;

template <typename TI, typename TO, typename L, bool PAST>
__global__ __launch_bounds__(256) void embed_scaled_kernel(const TI *table, int64_t tp, int64_t V, const L *ids, int64_t is, int64_t N, int64_t D, uint32_t upr, float scale,
                                                           TO *out, int64_t op) {
  constexpr int E = unit_elements<TI, TO>();
  const int64_t total = N * upr, first = (block_number() * 4 + (threadIdx.x >> 6)) * (64 * kUnits) + (threadIdx.x & 63);
  int64_t n[kUnits], id[kUnits];
  uint32_t c[kUnits];
#pragma unroll
  for (int k = 0; k < kUnits; ++k) {
    const int64_t i = min(first + k * 64, total - 1);
    n[k] = total <= 0xffffffffll ? (int64_t)((uint32_t)i / upr) : i / upr;
    c[k] = (uint32_t)(i - n[k] * upr);
    id[k] = id_at(ids, n[k], is, V);
  }
  Unit<TI, E> u[kUnits];
#pragma unroll
  for (int k = 0; k < kUnits; ++k) {
    const int64_t d = (int64_t)c[k] * E;
    if (id[k] == V) u[k].zero();
    else if (d + E <= D) u[k].load(table + id[k] * tp + d);
  }
#pragma unroll
  for (int k = 0; k < kUnits; ++k) {
    if (first + k * 64 >= total) break;
    const int64_t d = (int64_t)c[k] * E;
    TO *dst = out + n[k] * op + d;
    if (d + E <= D) {
      Unit<TO, E> o;
#pragma unroll
      for (int e = 0; e < E; ++e) o.set(e, id[k] == V ? 0.0f : u[k].get(e) * scale);
      if constexpr (PAST) o.store_nt(dst);
      else o.store(dst);
    } else {
      for (int e = 0; e < D - d; ++e) Elem<TO>::store(dst + e, id[k] == V ? 0.0f : Elem<TI>::load(table + id[k] * tp + d + e) * scale);
    }
  }
}

// ---- the ids in order -------------------------------------------------------------------------------------------
// (key, place) pairs are sorted by key, places of one key in their order: a radix sort from the low digits up, every pass of which keeps the order of
// equal digits.  Keys are ids, of ids outside the table V, which is sorted behind all of them and left out from there on.

constexpr int kMaxBits = 9, kBins = 1 << kMaxBits;           // of a digit
constexpr int kSortWaves = 16;
constexpr int kFew = 8192;                                    // ids that one block sorts

struct SortArgs {
  const void *ids;                   // pass 0 reads these
  const uint32_t *keys, *places;     // later ones these
  uint32_t *keys_out, *places_out;
  uint32_t *counts;                  // (blocks, bins)
  uint32_t *starts, *ends;           // (V)
  int64_t stride, V;
  uint32_t N, share;                 // pairs of a block
  int id64, shift, bits, blocks, first, only;
  float *dtable;                     // of this launch's blocks behind the sort's: rows [row, row_end) of the table become zeros
  int64_t tp, D, row, row_end;
};

// Sorting keeps a few blocks busy; the others meanwhile clear a table most rows of which will stay empty.
__device__ __forceinline__ bool fills(const SortArgs &s) {
  if ((int)blockIdx.x < s.blocks) return false;
  const int lane = threadIdx.x & 63;
  const int64_t waves = (int64_t)(gridDim.x - s.blocks) * kSortWaves;
  const chn_u32x4 none = {0, 0, 0, 0};
  for (int64_t v = s.row + ((int64_t)blockIdx.x - s.blocks) * kSortWaves + (threadIdx.x >> 6); v < s.row_end; v += waves) {
    float *p = s.dtable + v * s.tp;
    for (int64_t d = lane * 4; d < s.D; d += 256) {
      if (d + 4 <= s.D) {
        __builtin_nontemporal_store(none, reinterpret_cast<chn_u32x4_any *>(p + d));
      } else {
        for (int64_t e = d; e < s.D; ++e) p[e] = 0.0f;
      }
    }
  }
  return true;
}

__device__ __forceinline__ uint32_t key_of(const SortArgs &s, bool first, const uint32_t *keys, uint32_t i) {
  if (!first) return keys[i];
  return (uint32_t)(s.id64 ? id_at(static_cast<const int64_t *>(s.ids), i, s.stride, s.V) : id_at(static_cast<const int32_t *>(s.ids), i, s.stride, s.V));
}

// How often a block's share has each digit.
__global__ __launch_bounds__(1024) void embed_count_kernel(SortArgs s) {
  __shared__ uint32_t count[kBins];
  if (fills(s)) return;
  if (threadIdx.x < kBins) count[threadIdx.x] = 0;
  __syncthreads();
  const uint32_t lo = blockIdx.x * s.share, hi = min(lo + s.share, s.N), mask = (1u << s.bits) - 1;
  for (uint32_t i = lo + threadIdx.x; i < hi; i += 1024) atomicAdd(&count[key_of(s, s.first, s.keys, i) >> s.shift & mask], 1u);
  __syncthreads();
  if (threadIdx.x <= mask) s.counts[blockIdx.x * kBins + threadIdx.x] = count[threadIdx.x];
}

struct SortShared {
  uint32_t at[kSortWaves][kBins];    // where a wave's next pair of a digit goes
  uint32_t sums[kSortWaves];
};

// The lanes whose digit is this lane's.
__device__ __forceinline__ unsigned long long equals(bool on, uint32_t digit, int bits) {
  const unsigned long long all = __ballot(on);
  uint32_t low = (uint32_t)all, high = (uint32_t)(all >> 32);
  for (int b = 0; b < bits; ++b) {
    const int bit = (int)(digit << (31 - b)) >> 31;          // all ones where it is set
    const unsigned long long m = __ballot(bit);
    low &= ~((uint32_t)m ^ bit);
    high &= ~((uint32_t)(m >> 32) ^ bit);
  }
  return (unsigned long long)high << 32 | low;
}

// What the wave's lanes have written to LDS is what its lanes read from here on.
__device__ __forceinline__ void wave_order() {
  __builtin_amdgcn_fence(__ATOMIC_ACQ_REL, "wavefront");
  __builtin_amdgcn_wave_barrier();
}

// From the number of a digit's pairs in each wave to the place of its first one there.  count(d, before, all): how many pairs of digit d the blocks
// before this one have, and how many there are.
template <typename F>
__device__ __forceinline__ void bases(SortShared &sh, F count) {
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  uint32_t mine = 0, all = 0;
  if (tid < kBins) count(tid, mine, all);
  uint32_t run = all;                                        // running sums over the digits: in the wave, then over the waves
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const uint32_t up = __shfl_up(run, o, 64);
    if (lane >= o) run += up;
  }
  if (lane == 63) sh.sums[wave] = run;
  __syncthreads();
  if (tid < kBins) {
    uint32_t base = run - all + mine, c[kSortWaves];
    for (int w = 0; w < wave; ++w) base += sh.sums[w];
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) c[w] = sh.at[w][tid];
#pragma unroll
    for (int w = 0; w < kSortWaves; ++w) {
      sh.at[w][tid] = base;
      base += c[w];
    }
  }
  __syncthreads();
}

// One pass over the block's share, split over the waves.
__global__ __launch_bounds__(1024) void embed_sort_kernel(SortArgs s) {
  __shared__ SortShared sh;
  if (fills(s)) return;
  const uint32_t lo = min(blockIdx.x * s.share, s.N), hi = min(lo + s.share, s.N);
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t mask = (1u << s.bits) - 1;
  for (int i = tid; i < kSortWaves * kBins; i += 1024) (&sh.at[0][0])[i] = 0;
  __syncthreads();
  const uint32_t part = ((hi - lo + kSortWaves - 1) / kSortWaves + 63) / 64 * 64;
  const uint32_t from = min(lo + wave * part, hi), to = min(from + part, hi);
  for (uint32_t i = from + lane; i < to; i += 64) atomicAdd(&sh.at[wave][key_of(s, s.first, s.keys, i) >> s.shift & mask], 1u);
  __syncthreads();
  uint32_t total = 0;                                        // of the thread's digit
  bases(sh, [&](int d, uint32_t &mine, uint32_t &all) {
    if (d > (int)mask) return;
#pragma unroll 8
    for (int b = 0; b < s.blocks; ++b) {
      const uint32_t c = s.counts[b * kBins + d];
      mine += b < (int)blockIdx.x ? c : 0;
      all += c;
    }
    total = all;
  });
  if (s.only && blockIdx.x == 0 && tid < s.V) {              // (one pass: digits are tokens, and this block's wave 0 has their first places)
    s.starts[tid] = sh.at[0][tid];
    s.ends[tid] = sh.at[0][tid] + total;
  }
  __syncthreads();
  for (uint32_t i0 = from; i0 < to; i0 += 64) {
    const uint32_t i = i0 + lane;
    const bool on = i < to;
    const uint32_t key = on ? key_of(s, s.first, s.keys, i) : 0, place = on && !s.first ? s.places[i] : i, digit = key >> s.shift & mask;
    const unsigned long long same = equals(on, digit, s.bits);
    if (on) {
      const uint32_t to_ = sh.at[wave][digit] + __popcll(same & ((1ull << lane) - 1));
      s.keys_out[to_] = key;
      s.places_out[to_] = place;
    }
    wave_order();
    if (on && same >> lane == 1) sh.at[wave][digit] += __popcll(same);   // (the digit's last lane)
    wave_order();
  }
}

// Few ids: one block makes all passes, its pairs in registers while a pass counts, in LDS in between, and says where each token's places begin and end.
__global__ __launch_bounds__(1024) void embed_sort_few_kernel(SortArgs s, int passes) {
  __shared__ SortShared sh;
  __shared__ uint2 pairs[kFew];
  static_assert(kFew % 1024 == 0, "pairs of a thread");
  constexpr int M = kFew / 1024;
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t mask = (1u << s.bits) - 1, part = ((s.N + kSortWaves - 1) / kSortWaves + 63) / 64 * 64;
  const uint32_t from = min(wave * part, s.N), to = min(from + part, s.N);
  uint32_t key[M], place[M], at[M];
#pragma unroll
  for (int m = 0; m < M; ++m) {
    place[m] = from + m * 64 + lane;
    key[m] = place[m] < to ? key_of(s, true, nullptr, place[m]) : 0;
  }
  for (int p = 0; p < passes; ++p) {
    const int shift = p * s.bits;
    for (int i = tid; i < kSortWaves * kBins; i += 1024) (&sh.at[0][0])[i] = 0;
    __syncthreads();
    // where a pair goes among the wave's own of its digit; behind that the digit's number in the wave
#pragma unroll
    for (int m = 0; m < M; ++m) {
      if (from + m * 64 >= to) break;
      const bool on = from + m * 64 + lane < to;
      const uint32_t digit = key[m] >> shift & mask;
      const unsigned long long same = equals(on, digit, s.bits);
      at[m] = on ? sh.at[wave][digit] + __popcll(same & ((1ull << lane) - 1)) : 0;
      wave_order();
      if (on && same >> lane == 1) sh.at[wave][digit] += __popcll(same);
      wave_order();
    }
    __syncthreads();
    bases(sh, [&](int d, uint32_t &mine, uint32_t &all) {
      mine = all = 0;
#pragma unroll
      for (int w = 0; w < kSortWaves; ++w) all += sh.at[w][d];
    });
#pragma unroll
    for (int m = 0; m < M; ++m)
      if (from + m * 64 + lane < to) pairs[sh.at[wave][key[m] >> shift & mask] + at[m]] = make_uint2(key[m], place[m]);
    __syncthreads();
#pragma unroll
    for (int m = 0; m < M; ++m) {
      const uint32_t i = from + m * 64 + lane;
      if (i < to) {
        key[m] = pairs[i].x;
        place[m] = pairs[i].y;
      }
    }
  }
#pragma unroll
  for (int m = 0; m < M; ++m) {
    const uint32_t i = from + m * 64 + lane;
    if (i < to) {
      s.keys_out[i] = key[m];
      s.places_out[i] = place[m];
      if (key[m] < s.V) {
        if (i == 0 || pairs[i - 1].x != key[m]) s.starts[key[m]] = i;
        if (i == s.N - 1 || pairs[i + 1].x != key[m]) s.ends[key[m]] = i + 1;
      }
    }
  }
}

// ---- the sums -----------------------------------------------------------------------------------------------------
constexpr int kPiece = 64;           // places of a piece: tokens with more of them than that are summed by pieces
constexpr int kTogether = 16;        // rows in flight

struct SumArgs {
  const uint32_t *keys, *places;
  uint32_t *starts, *ends;           // (V): a token's places in the sorted list, anything where it has none
  const void *dout;
  float *dtable, *partial;           // (pieces, 2, pitch): of a piece's first and of its last token, where they stand often
  int64_t dp, tp, pitch, V, D, chunks, pieces;
  float scale;
  uint32_t N;
  int accumulate, leave, rows;       // whether rows without a token stay as they are; rows of the table for a wave
};

__global__ __launch_bounds__(256) void embed_ranges_kernel(SumArgs s) {
  const uint32_t i = blockIdx.x * 256 + threadIdx.x;
  if (i >= s.N) return;
  const uint32_t k = s.keys[i];
  if (k >= s.V) return;
  if (i == 0 || s.keys[i - 1] != k) s.starts[k] = i;
  if (i == s.N - 1 || s.keys[i + 1] != k) s.ends[k] = i + 1;
}

template <typename T, int E, int M, typename F>
__device__ __forceinline__ void add_rows(F row, int i, int n, int64_t at, float (&sum)[E]) {
  Unit<T, E> u[M];
#pragma unroll
  for (int k = 0; k < M; ++k) u[k].load(row(min(i + k, n - 1)) + at);
#pragma unroll
  for (int k = 0; k < M; ++k)
    if (i + k < n) {
#pragma unroll
      for (int e = 0; e < E; ++e) sum[e] += u[k].get(e);
    }
}

// Adds n rows, 64 of them at most, to a lane's columns, in the order in which the lanes hold their numbers.  A lane behind the last whole unit of a row adds the row's last
// E columns; `own_columns` moves the sums to where the lane's own ones begin.
template <typename T, int E>
__device__ __forceinline__ void add_places(const SumArgs &s, uint32_t place, int n, int64_t d, float (&sum)[E]) {
  auto row = [&](int i) { return static_cast<const T *>(s.dout) + (int64_t)(uint32_t)__builtin_amdgcn_readlane((int)place, i) * s.dp; };
  if (s.D >= E) {
    const int64_t at = min(d, s.D - E);
    int i = 0;
    for (; n - i > kTogether / 2; i += kTogether) add_rows<T, E, kTogether>(row, i, n, at, sum);
    for (; i < n; i += kTogether / 4) add_rows<T, E, kTogether / 4>(row, i, n, at, sum);
  } else {
    for (int i = 0; i < n; ++i) {
      const T *r = row(i);
#pragma unroll
      for (int e = 0; e < E; ++e) sum[e] += d + e < s.D ? Elem<T>::load(r + d + e) : 0.0f;
    }
  }
}
template <int E>
__device__ __forceinline__ void own_columns(const SumArgs &s, int64_t d, float (&sum)[E]) {
  const int off = s.D >= E ? (int)min(d - min(d, s.D - E), (int64_t)E) : 0;
  if (__any(off > 0)) {
    float moved[E];
#pragma unroll
    for (int e = 0; e < E; ++e) {
      moved[e] = 0.0f;
#pragma unroll
      for (int f = e; f < E; ++f) moved[e] = f == e + off ? sum[f] : moved[e];
    }
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] = moved[e];
  }
}

// The sum of the rows at places [lo, hi) of the sorted list, 64 at most: each lane fetches one, and from there on only rows are waited for.
template <typename T, int E>
__device__ __forceinline__ void sum_rows(const SumArgs &s, uint32_t lo, uint32_t hi, int64_t d, float (&sum)[E]) {
  const int n = __builtin_amdgcn_readfirstlane((int)(hi - lo));
#pragma unroll
  for (int e = 0; e < E; ++e) sum[e] = 0.0f;
  add_places<T, E>(s, s.places[min(lo + (threadIdx.x & 63), hi - 1)], n, d, sum);
  own_columns<E>(s, d, sum);
}

template <int E>
__device__ __forceinline__ void write_row(const SumArgs &s, int64_t v, int64_t d, const float (&sum)[E]) {
  float *p = s.dtable + v * s.tp + d;
  if (d + E <= s.D) {
    Unit<float, E> u;
    if (s.accumulate) u.load(p);
#pragma unroll
    for (int e = 0; e < E; ++e) u.set(e, s.accumulate ? fmaf(s.scale, sum[e], u.get(e)) : s.scale * sum[e]);
    u.store_nt(p);
  } else {
#pragma unroll
    for (int e = 0; e < E; ++e)
      if (d + e < s.D) p[e] = s.accumulate ? fmaf(s.scale, sum[e], p[e]) : s.scale * sum[e];
  }
}

// A chunk of a row of zeros, neighbouring lanes next to each other.
template <int E>
__device__ __forceinline__ void zero_row(const SumArgs &s, int64_t v, int64_t d0) {
  float *p = s.dtable + v * s.tp;
  const chn_u32x4 none = {0, 0, 0, 0};
#pragma unroll
  for (int j = 0; j < E / 4; ++j) {
    const int64_t d = d0 + j * 256 + (threadIdx.x & 63) * 4;
    if (d + 4 <= s.D) {
      __builtin_nontemporal_store(none, reinterpret_cast<chn_u32x4_any *>(p + d));
    } else {
      for (int64_t e = d; e < s.D; ++e) p[e] = 0.0f;
    }
  }
}

// of a token that is in the list
__device__ __forceinline__ bool often(const SumArgs &s, uint32_t v) { return v < s.V && s.ends[v] - s.starts[v] > kPiece; }

// A wave for each (piece, chunk of columns), then for every few rows of the table and each chunk.
template <typename T>
__global__ __launch_bounds__(256) void embed_sum_kernel(SumArgs s) {
  constexpr int E = unit_elements<T>();
  const int lane = threadIdx.x & 63;
  int64_t job = block_number() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  float sum[E];
  if (job < s.pieces * s.chunks) {
    const int64_t piece = job / s.chunks, d = ((job - piece * s.chunks) * 64 + lane) * E;
    const uint32_t lo = (uint32_t)piece * kPiece, hi = min(lo + kPiece, s.N), f = s.keys[lo], l = s.keys[hi - 1];
    const uint32_t fv = f < s.V ? f : 0, lv = l < s.V ? l : 0;
    const uint32_t f0 = s.starts[fv], f1 = s.ends[fv], l0 = s.starts[lv], l1 = s.ends[lv];
    for (int side = 0; side < 2; ++side) {
      if (side ? l == f || l >= s.V || l1 - l0 <= kPiece : f >= s.V || f1 - f0 <= kPiece) continue;
      sum_rows<T, E>(s, side ? l0 : lo, side ? hi : min(hi, f1), d, sum);
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
  const int64_t rows = job / s.chunks, v0 = rows * s.rows, d = ((job - rows * s.chunks) * 64 + lane) * E;
  if (v0 >= s.V) return;
  const int n = (int)min((int64_t)s.rows, s.V - v0);
  // A token is in the list where the list says so: at the place that is noted for it, whatever an earlier call may have left there.
  uint32_t lo = 0, count = 0;
  if (lane < n) {
    lo = s.starts[v0 + lane];
    const uint32_t end = s.ends[v0 + lane];
    if (lo < s.N && s.keys[lo] == v0 + lane) count = end - lo;
  }
  for (int r = 0; r < n; ++r) {
    const uint32_t from = __builtin_amdgcn_readlane(lo, r), c = __builtin_amdgcn_readlane(count, r);
    if (c > kPiece || (c == 0 && s.leave)) continue;
    if (c > 0) {
      sum_rows<T, E>(s, from, from + c, d, sum);
      if (d < s.D) write_row<E>(s, v0 + r, d, sum);
    } else {
      zero_row<E>(s, v0 + r, d - lane * E);
    }
  }
}

// Few ids: nothing is sorted.  A wave looks through them for its rows' tokens, 64 at a time, and adds the rows that it finds there to the sum.
constexpr int kDirect = 256;

template <typename T, typename L>
__global__ __launch_bounds__(256) void embed_direct_kernel(SumArgs s, const L *ids, int64_t stride) {
  constexpr int E = unit_elements<T>(), M = kDirect / 64;
  const int lane = threadIdx.x & 63;
  const int64_t job = block_number() * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), rows = job / s.chunks, v0 = rows * s.rows;
  const int64_t d = ((job - rows * s.chunks) * 64 + lane) * E;
  if (v0 >= s.V) return;
  const int n = (int)min((int64_t)s.rows, s.V - v0), N = (int)s.N;
  uint32_t id[M];                                            // of ids outside the table V and above, which no row has
#pragma unroll
  for (int m = 0; m < M; ++m) {
    id[m] = ~0u;
    if (m * 64 < N) {
      const int i = m * 64 + lane;
      const int64_t v = id_at(ids, min(i, N - 1), stride, s.V);
      id[m] = i < N ? (uint32_t)v : ~0u;
    }
  }
  for (int r = 0; r < n; ++r) {
    unsigned long long found[M], any = 0;                    // the places of the row's token
#pragma unroll
    for (int m = 0; m < M; ++m) {
      found[m] = __ballot(id[m] == (uint32_t)(v0 + r));
      any |= found[m];
    }
    if (!any) {
      if (!s.accumulate) zero_row<E>(s, v0 + r, d - lane * E);
      continue;
    }
    float sum[E];
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] = 0.0f;
#pragma unroll
    for (int m = 0; m < M; ++m) {
      if (!found[m]) continue;
      // in their order, one to a lane
      const int count = __popcll(found[m]);
      int place = 0;
      for (int k = 0; k < count; ++k, found[m] &= found[m] - 1) place = lane == k ? m * 64 + (int)__builtin_ctzll(found[m]) : place;
      add_places<T, E>(s, (uint32_t)place, count, d, sum);
    }
    own_columns<E>(s, d, sum);
    if (d < s.D) write_row<E>(s, v0 + r, d, sum);
  }
}

// A block looks at kLooked pieces for tokens that stand often and begin in one of them, and adds up their pieces: its waves take neighbouring shares.
constexpr int kLooked = 4, kJoinWaves = 8;

template <int E>
__global__ __launch_bounds__(64 * kJoinWaves) void embed_join_kernel(SumArgs s) {
  __shared__ float parts[kJoinWaves][E][64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t job = block_number(), group = job / s.chunks, d = ((job - group * s.chunks) * 64 + lane) * E;
  bool found = false;
  if (lane < kLooked && group * kLooked + lane < s.pieces) {
    const uint32_t lo = (uint32_t)(group * kLooked + lane) * kPiece, hi = min(lo + kPiece, s.N), v = s.keys[hi - 1];
    found = often(s, v) && s.starts[v] >= lo;
  }
  for (unsigned long long left = __ballot(found); left; left &= left - 1) {
    const int64_t piece = group * kLooked + __builtin_ctzll(left);
    const uint32_t lo = (uint32_t)piece * kPiece, v = s.keys[min(lo + kPiece, s.N) - 1];
    const int64_t last = (s.ends[v] - 1) / kPiece, share = (last - piece + kJoinWaves) / kJoinWaves;
    const int64_t from = piece + wave * share, to = min(from + share, last + 1);
    const int side = s.starts[v] != lo;                      // of its first piece the token is the last one, of the others the first
    float sum[E];
#pragma unroll
    for (int e = 0; e < E; ++e) sum[e] = 0.0f;
    if (d < s.D) {
      for (int64_t i = from; i < to; i += 8) {
        Unit<float, E> u[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int64_t p = min(i + k, to - 1);
          u[k].load(s.partial + (p * 2 + (p == piece ? side : 0)) * s.pitch + d);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (i + k < to) {
#pragma unroll
            for (int e = 0; e < E; ++e) sum[e] += u[k].get(e);
          }
      }
    }
#pragma unroll
    for (int e = 0; e < E; ++e) parts[wave][e][lane] = sum[e];
    __syncthreads();
    if (wave == 0 && d < s.D) {
#pragma unroll
      for (int e = 0; e < E; ++e)
        for (int w = 1; w < kJoinWaves; ++w) sum[e] += parts[w][e][lane];
      write_row<E>(s, v, d, sum);
    }
    __syncthreads();
  }
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
    blocks = (int)(N <= kFew ? 1 : N < 2 * 2048 ? 2 : N / 2048 < 64 ? N / 2048 : 64);   // (one block: its kernel takes no more than kFew)
    share = (uint32_t)((N + blocks - 1) / blocks);
    pieces = (N + kPiece - 1) / kPiece;
    pitch = (D + 7) / 8 * 8;
    size_t at = 0;
    auto put = [&](size_t n) { const size_t here = at; at += (n + 255) / 256 * 256; return here; };
    keys = put(4 * (size_t)N);
    places = put(4 * (size_t)N);
    between = put(blocks > 1 && passes > 1 ? 4 * (size_t)N : 0);
    places_between = put(blocks > 1 && passes > 1 ? 4 * (size_t)N : 0);
    counts = put(blocks > 1 ? 4 * (size_t)blocks * kBins : 0);
    starts = put(4 * (size_t)V);
    ends = put(4 * (size_t)V);
    partial = put(8 * (size_t)pieces * pitch);
    bytes = at;
  }
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
  const int E = table->dtype == CHN_F32 && out->dtype == CHN_F32 ? 4 : 8;
  const int64_t upr = (D + E - 1) / E;
  if (upr > 0x7fffffff) return fail(CHN_ERR_SHAPE, "embed: rows of %lld elements", (long long)D);
  const dim3 grid = grid_of((N * upr + 256 * kUnits - 1) / (256 * kUnits));
  hipStream_t st = as_stream(stream);
  // whole lines go past the caches (65536 rows of 2048 bytes into them 41 us, past them 31; 100003 rows of 1332 bytes 27 and 34)
  const int64_t osz = dtype_size(out->dtype);
  const bool past = D * osz % 128 == 0 && op * osz % 128 == 0 && reinterpret_cast<uintptr_t>(out->data) % 128 == 0;
#define CHN_LAUNCH(TI, TO, L, P)                                                                                                                     \
  hipLaunchKernelGGL((embed_scaled_kernel<TI, TO, L, P>), grid, dim3(256), 0, st, static_cast<const TI *>(table->data), tp, V,                       \
                     static_cast<const L *>(ids->data), is, N, D, (uint32_t)upr, (float)scale, static_cast<TO *>(out->data), op)
#define CHN_GO(TI, TO)                                                                                                                               \
  do {                                                                                                                                               \
    if (ids->dtype == CHN_I32) { if (past) CHN_LAUNCH(TI, TO, int32_t, true); else CHN_LAUNCH(TI, TO, int32_t, false); }                             \
    else { if (past) CHN_LAUNCH(TI, TO, int64_t, true); else CHN_LAUNCH(TI, TO, int64_t, false); }                                                   \
  } while (0)
  if (table->dtype == CHN_F32) { if (out->dtype == CHN_F32) CHN_GO(float, float); else CHN_GO(float, bf16_raw); }
  else { if (out->dtype == CHN_F32) CHN_GO(bf16_raw, float); else CHN_GO(bf16_raw, bf16_raw); }
#undef CHN_GO
#undef CHN_LAUNCH
  return check_launch("embed_scaled_fwd");
}

size_t chn_embed_sorted_workspace_bytes(const chn_array *ids, const chn_array *dtable) {
  using namespace chn;
  if (!ids || !dtable || ids->ndim != 1 || dtable->ndim != 2) return 0;
  const int64_t N = ids->shape[0], V = dtable->shape[0], D = dtable->shape[1];
  if (V <= 0 || D <= 0 || N > 0x7fffffff || V > 0x7fffffff) return 0;
  return N <= kDirect ? 0 : Layout(N, V, D).bytes;
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
  const int E = dout->dtype == CHN_F32 ? 4 : 8;
  SumArgs s = {};
  s.dout = dout->data; s.dtable = static_cast<float *>(dtable->data);
  s.dp = dp; s.tp = tp; s.V = V; s.D = D; s.chunks = (D + 64 * E - 1) / (64 * E);
  s.scale = (float)scale; s.N = (uint32_t)N; s.accumulate = accumulate;
  const int64_t each = V * s.chunks / 8192;                  // (about as many waves as run at once: with one row each, 4480 x 650 into 10000 rows 16.5 us, 12.7 like this)
  s.rows = (int)(each < 1 ? 1 : each > 16 ? 16 : each);
  const int64_t row_jobs = (V + s.rows - 1) / s.rows * s.chunks;
  hipStream_t st = as_stream(stream);
  if (N <= kDirect) {
#define CHN_GO(T, L) hipLaunchKernelGGL((embed_direct_kernel<T, L>), grid_of((row_jobs + 3) / 4), dim3(256), 0, st, s, static_cast<const L *>(ids->data), is)
    if (ids->dtype == CHN_I32) { if (dout->dtype == CHN_F32) CHN_GO(float, int32_t); else CHN_GO(bf16_raw, int32_t); }
    else { if (dout->dtype == CHN_F32) CHN_GO(float, int64_t); else CHN_GO(bf16_raw, int64_t); }
#undef CHN_GO
    return check_launch("embed_sorted_bwd");
  }
  const Layout z(N, V, D);
  char *w = static_cast<char *>(ws);
  auto words = [&](size_t at) { return reinterpret_cast<uint32_t *>(w + at); };
  SortArgs o = {};
  o.ids = ids->data; o.stride = is; o.id64 = ids->dtype == CHN_I64;
  o.V = V; o.N = (uint32_t)N; o.share = z.share; o.bits = z.bits; o.blocks = z.blocks;
  o.counts = words(z.counts); o.starts = words(z.starts); o.ends = words(z.ends);
  o.keys_out = words(z.keys); o.places_out = words(z.places);
  // Clearing beside the sort against clearing by the sums, us with tokens as frequent as words are (and evenly drawn), in graphs of ten calls.
  // bfloat16 dout, N <= V / 2: 16384 x 1024 into 131072 130 / 141 (132 / 150), 32768 x 1024 into 65536 87 / 97 (97 / 105), 65536 x 1024 into 131072 155 / 164 (181 / 184), 65536 x 512 into
  // 131072 87 / 101 (96 / 106), 65536 x 4096 into 131072 590 / 611 (710 / 593); at N = V 32768 x 1024 66 / 67 (71 / 66), 65536 x 1024 102 / 107 (121 / 114).
  // fp32 dout, whose sums write zeros in narrower pieces: 10000 x 650 into 100000 98 / 114 (98 / 110), 8500 x 1024 into 68000 82 / 86 (82 / 84), 16384 x 512 into 131072 75 / 80 (77 / 78); beyond each
  // of its three limits 32768 x 512 into 131072 81 / 83 (85 / 80) and 65536 x 512 into 131072 96 / 91 (101 / 84), 65536 x 128 into 524288 99 / 89 (101 / 88), 16384 x 1024 into 131072 138 / 131 (143 / 130)
  // and 65536 x 1024 into 200000 246 / 217 (269 / 191).
  const bool mostly_zeros = dout->dtype == CHN_BF16 ? N <= V / 2 : N <= V / 8 && N <= 1 << 15 && V * D < 1 << 27;
  const bool filled = z.blocks > 1 && !accumulate && mostly_zeros;
  o.dtable = static_cast<float *>(dtable->data); o.tp = tp; o.D = D;
  if (z.blocks == 1) {
    hipLaunchKernelGGL(embed_sort_few_kernel, dim3(1), dim3(1024), 0, st, o, z.passes);
    CHN_TRY(check_launch("embed_sorted_bwd"));
  } else {
    for (int p = 0; p < z.passes; ++p) {
      const bool last = (z.passes - 1 - p) % 2 == 0;         // the last pass ends in `keys`
      o.first = p == 0;
      o.only = z.passes == 1;
      o.shift = p * z.bits;
      o.keys = words(last ? z.between : z.keys); o.places = words(last ? z.places_between : z.places);
      o.keys_out = words(last ? z.keys : z.between); o.places_out = words(last ? z.places : z.places_between);
      for (int half = 0; half < 2; ++half) {
        if (filled) {
          const int64_t k = p * 2 + half, parts = z.passes * 2;
          o.row = V * k / parts;
          o.row_end = V * (k + 1) / parts;
        }
        const dim3 grid(z.blocks + (filled ? 512 : 0));
        if (half == 0) hipLaunchKernelGGL(embed_count_kernel, grid, dim3(1024), 0, st, o);
        else hipLaunchKernelGGL(embed_sort_kernel, grid, dim3(1024), 0, st, o);
        CHN_TRY(check_launch("embed_sorted_bwd"));
      }
    }
  }
  s.keys = words(z.keys); s.places = words(z.places); s.starts = words(z.starts); s.ends = words(z.ends);
  s.partial = reinterpret_cast<float *>(w + z.partial); s.pitch = z.pitch; s.pieces = z.pieces;
  s.leave = accumulate || filled;
  if (z.blocks > 1 && z.passes > 1) {
    hipLaunchKernelGGL(embed_ranges_kernel, dim3((unsigned)((N + 255) / 256)), dim3(256), 0, st, s);
    CHN_TRY(check_launch("embed_sorted_bwd"));
  }
  const dim3 grid = grid_of((z.pieces * s.chunks + row_jobs + 3) / 4);
  if (dout->dtype == CHN_F32) hipLaunchKernelGGL((embed_sum_kernel<float>), grid, dim3(256), 0, st, s);
  else hipLaunchKernelGGL((embed_sum_kernel<bf16_raw>), grid, dim3(256), 0, st, s);
  CHN_TRY(check_launch("embed_sorted_bwd"));
  if (dout->dtype == CHN_F32) hipLaunchKernelGGL((embed_join_kernel<4>), grid_of((z.pieces + kLooked - 1) / kLooked * s.chunks), dim3(64 * kJoinWaves), 0, st, s);
  else hipLaunchKernelGGL((embed_join_kernel<8>), grid_of((z.pieces + kLooked - 1) / kLooked * s.chunks), dim3(64 * kJoinWaves), 0, st, s);
  return check_launch("embed_sorted_bwd");
}

}  // extern "C"
