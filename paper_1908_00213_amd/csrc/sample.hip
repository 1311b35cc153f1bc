// chn_sample: one token for each row of logits, filtered by temperature, top-k, top-p and min-p, drawn by a given number.
//
// Weights are whole numbers: w(z) = round(2^shift exp((z - max z) / temperature)), the exponential in 64 bits, so that every sum is exact,
// whatever the order in which it is taken; the token is the first whose running sum (in the vocabulary's order, over the tokens that
// the filters keep) exceeds u times the whole sum.
//
// The order by which the filters choose -- descending logits, equals by index -- is that of one 64-bit number for each token (`Rank`), so a filter is a
// border: the tokens from some number on are kept.  A border is found without sorting the row: sums (top-p) or counts (top-k) in 2048 bins of
// equal width in the logit, the bin that the border lies in, and the few tokens of that bin in their exact order.  Where top-k
// leaves only a few tokens anyway, these are gathered first and the rest of the row is never looked at again: the k-th largest of
// the maxima of parts of the row is a bound that at least k tokens reach.
//
// A row is the work of one block of 1024 threads, of a wave up to 256 tokens.  Few long rows are cut in chunks, in four launches that exchange through the workspace:
// maxima of all parts; bins, candidates or sums; the bin of the border and the sums above it; the draw (see the rule at chunks_of).
#include "common.h"
#include "rows.h"

namespace chn {
namespace {

typedef unsigned long long u64;
constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBins = 2048;          // two for each thread
constexpr int kFewBins = 256;        // for a bound: coarser, and read by every wave
constexpr int kSmall = 1024;         // tokens that are ordered by comparing each with each
constexpr int kHeldUnits = 4;         // of a row that a thread keeps in registers
constexpr int kMaxChunks = 32, kMaxParts = 4096, kLeastParts = 1024;

// What the launches over chunks leave for each other, of one row.
struct RowSpace {
  u64 bins[kBins];                   // sums by bin
  u64 list[kSmall];                  // tokens of the border's bin
  u64 sums[kMaxChunks];              // kept weights of each chunk
  float maxima[kMaxParts];           // of parts; the tokens behind the last unit count to the last part
  float minima[kMaxParts];
  int count, pad[63];
};

struct SampleArgs {
  int64_t N, pitch;
  int V, shift;
  const float *u, *temperature, *top_p, *min_p;
  int64_t su, st, sp, sm, sk;        // strides in elements
  const void *top_k;
  int k64;
  void *out;
  int out64;
  RowSpace *space;
  int chunks, chunk_units;           // chunks are multiples of 64 units
  int parts, part_bits;              // parts of a row, and the units of one: 2^2 to 2^6
  int most_k;                        // of a top-k that the parts' maxima narrow to few tokens
};

// Monotone in the logit, -0 and 0 alike.  0: not a token that can be drawn (-inf, NaN).
__device__ __forceinline__ uint32_t key_of(float z) {
  if (!(z > -INFINITY)) return 0;
  const uint32_t b = __float_as_uint(z + 0.0f);
  return (b & 0x80000000u) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float logit_of(uint32_t key) { return __uint_as_float((key & 0x80000000u) ? key & 0x7fffffffu : ~key); }

// A token's place in the order of the filters: larger comes first.  0: cannot be drawn.
typedef u64 Rank;
__device__ __forceinline__ Rank rank_of(float z, uint32_t index) {
  const uint32_t k = key_of(z);
  return k ? (u64)k << 32 | (0xffffffffu - index) : 0;
}
__device__ __forceinline__ uint32_t index_of(Rank r) { return 0xffffffffu - (uint32_t)r; }

// 2^(-j / 32)
__constant__ const double kPowers[32] = {
    0x1.0000000000000p+0, 0x1.f50765b6e4540p-1, 0x1.ea4afa2a490dap-1, 0x1.dfc97337b9b5fp-1, 0x1.d5818dcfba487p-1, 0x1.cb720dcef9069p-1,
    0x1.c199bdd85529cp-1, 0x1.b7f76f2fb5e47p-1, 0x1.ae89f995ad3adp-1, 0x1.a5503b23e255dp-1, 0x1.9c49182a3f090p-1, 0x1.93737b0cdc5e5p-1,
    0x1.8ace5422aa0dbp-1, 0x1.82589994cce13p-1, 0x1.7a11473eb0187p-1, 0x1.71f75e8ec5f74p-1, 0x1.6a09e667f3bcdp-1, 0x1.6247eb03a5585p-1,
    0x1.5ab07dd485429p-1, 0x1.5342b569d4f82p-1, 0x1.4bfdad5362a27p-1, 0x1.44e086061892dp-1, 0x1.3dea64c123422p-1, 0x1.371a7373aa9cbp-1,
    0x1.306fe0a31b715p-1, 0x1.29e9df51fdee1p-1, 0x1.2387a6e756238p-1, 0x1.1d4873168b9aap-1, 0x1.172b83c7d517bp-1, 0x1.11301d0125b51p-1,
    0x1.0b5586cf9890fp-1, 0x1.059b0d3158574p-1};

struct Shared {
  u64 bins[kBins];
  u64 sorted[kSmall];                // the small set in descending order
  u64 weight[kSmall];
  u64 list[kSmall];                  // the small set as it was gathered
  u64 waves[kWaves];
  double powers[32];                 // kPowers: 64 banks' worth, no two lanes meet in one unless they read the same number
  float fmax[kWaves], fmin[kWaves], fleast[kWaves];
  u64 result, above;
  int count, slot;
};

// exp((z - best) / t) and the weight it stands for.
//
// exp = 2^(-y / 32), y = 32 (best - z) / (t ln 2): with n the whole number next to y, 2^((n - y) / 32) by a polynomial of degree four through the Chebyshev
// nodes (relative error below 2e-13), the low five bits of n by a table and the others taken off the exponent.  To tell a token from its
// neighbour by the same u takes an error of about a token's share of the sum, which is 1e-6 of it at the least.
struct Weights {
  float best;
  double c;                          // 32 / (t ln 2)
  double magic;                      // adding it leaves a whole number of 2^-shift in the low bits
  const double *powers;
  __device__ __forceinline__ Weights(float best_, float t, int shift, const Shared &sh) : Weights(best_, t, shift, sh.powers) {}
  __device__ __forceinline__ Weights(float best_, float t, int shift, const double *powers_) : best(best_), powers(powers_) {
    c = 46.166241308446828384 / (double)t;
    magic = __longlong_as_double((long long)(1023 + 52 - shift) << 52);
  }
  __device__ __forceinline__ double distance(float z) const { return ((double)best - (double)z) * c; }
  // For every number below `best` and best itself.
  __device__ __forceinline__ double exponential(float z) const {
    if (z == best) return 1.0;
    return exp2(distance(z) * -0.03125);
  }
  // From here on weights are not zero, and what lies above is near enough for `near`.  (Sixty octaves below the largest logit, rounded to a
  // number of its kind; the lowest finite one at the least.)
  __device__ __forceinline__ float zero(float t) const { return fmaxf((float)((double)best - 41.6 * (double)t), -3.4028234663852886e38f); }
  // For logits whose distance is below 32 * 1000; any number for others.  y + 1.5 2^52 has the whole number next to y in its low word: no
  // rounding, conversion or ldexp.
  __device__ __forceinline__ double near(float z) const {
    const double dz = (double)best - (double)z, rough = fma(dz, c, 0x1.8p52), n = rough - 0x1.8p52, r = fma(-dz, c, n);
    const int m = __double2loint(rough);
    double q = fma(0x1.3b2b07bdf358dp-27, r, 0x1.c6b13c3465457p-20);
    q = fma(q, r, 0x1.ebfbdff82240ap-13);
    q = fma(q, r, 0x1.62e42fef8dc67p-6);
    const double p = powers[m & 31], e = fma(p, q * r, p);
    return __hiloint2double(__double2hiint(e) - ((m & ~31) << 15), __double2loint(e));
  }
  __device__ __forceinline__ u64 of(double e) const { return (u64)__double_as_longlong(e + magic) & 0xfffffffffffffull; }
};

// Tokens that are kept: logits above `z`, and of those equal to it the ones before index `end`.
struct Limit {
  float z;
  uint32_t end;
  __device__ __forceinline__ bool keeps(float v, uint32_t i) const { return v > z || (v == z && i < end); }
  __device__ __forceinline__ void not_below(float least) {
    if (least > z) {
      z = least;
      end = 0xffffffffu;
    }
  }
};

// Whether a token's exponential is at least m: by e, which may be of `near`, unless that is too close to tell.  So min-p has one border on every path.  (By
// `least_logit` 128 x 10000 with top-k and min-p 11.1 us, so 10.4.)
__device__ __forceinline__ bool reaches(const Weights &wt, float z, double e, float m) {
  return fabs(e - (double)m) < 1e-12 * (double)m ? wt.exponential(z) >= (double)m : e >= (double)m;
}

// The smallest logit whose exponential is at least m, 0 < m <= 1: near the logarithm's, 64 of them tried at once, or by search, 64 at a time.
__device__ __forceinline__ float least_logit(const Weights &wt, float t, float m) {
  const uint32_t lane = threadIdx.x & 63, low = 0x00800000u, high = key_of(wt.best);   // (from the lowest finite number on)
  const uint32_t guess = key_of(fmaxf((float)((double)wt.best + (double)t * (double)logf(m)), -3.4028234663852886e38f));
  uint32_t a = guess - low > 31 ? guess - 31 : low, b = high;
  const uint32_t mine = b - a < lane ? b : a + lane;
  const u64 hit = __ballot(wt.exponential(logit_of(mine)) >= (double)m);
  const int first = __ffsll((long long)hit) - 1;
  if (first > 0) return logit_of(b - a < (uint32_t)first ? b : a + first);
  a = low;
  while (a < b) {
    const uint32_t step = (b - a + 63) / 64, at = b - a < lane * (u64)step ? b : a + lane * step;
    const int f = __ffsll((long long)__ballot(wt.exponential(logit_of(at)) >= (double)m)) - 1;    // the first lane for which it holds
    if (f == 0) {
      b = a;
    } else if (f < 0) {
      a += 63 * step + 1;
    } else {
      const uint32_t to = b - a < f * (u64)step ? b : a + f * step;
      a += (f - 1) * step + 1;
      b = to;
    }
  }
  return logit_of(b);
}

// v of the lane that CTRL names, 0 where there is none (or where a row of sixteen lanes is not in ROWS)
template <int CTRL, int ROWS>
__device__ __forceinline__ u64 dpp_u64(u64 v) {
  const uint32_t lo = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)v, CTRL, ROWS, 0xf, false);
  const uint32_t hi = (uint32_t)__builtin_amdgcn_update_dpp(0, (int)(uint32_t)(v >> 32), CTRL, ROWS, 0xf, false);
  return (u64)hi << 32 | lo;
}
__device__ __forceinline__ u64 lane_u64(u64 v, int lane) {
  return (u64)(uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)(v >> 32), lane) << 32 | (uint32_t)__builtin_amdgcn_readlane((int)(uint32_t)v, lane);
}
// Sum over the lanes up to this one, exchanged inside the registers: within rows of sixteen lanes, then each row's last lane to the
// next row, then the first half's to the second.  (By shuffles through LDS twelve of these in a draw took 4 us more.)
__device__ __forceinline__ u64 wave_upto_u64(u64 v) {
  v += dpp_u64<0x111, 0xf>(v);    // row_shr 1, 2, 4, 8
  v += dpp_u64<0x112, 0xf>(v);
  v += dpp_u64<0x114, 0xf>(v);
  v += dpp_u64<0x118, 0xf>(v);
  v += dpp_u64<0x142, 0xa>(v);    // row_bcast 15 into rows 1 and 3
  v += dpp_u64<0x143, 0xc>(v);    // row_bcast 31 into rows 2 and 3
  return v;
}
__device__ __forceinline__ u64 wave_sum_u64(u64 v) { return lane_u64(wave_upto_u64(v), 63); }

// Sum over the threads before this one; *all: over all of them.
__device__ __forceinline__ u64 block_before_u64(u64 v, Shared &sh, u64 *all) {
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const u64 upto = wave_upto_u64(v);
  __syncthreads();
  if (lane == 63) sh.waves[wave] = upto;
  __syncthreads();
  // every wave sums the sixteen waves' up by itself, in a row of its lanes
  u64 w = sh.waves[lane & 15];
  w += dpp_u64<0x111, 0xf>(w);
  w += dpp_u64<0x112, 0xf>(w);
  w += dpp_u64<0x114, 0xf>(w);
  w += dpp_u64<0x118, 0xf>(w);
  const u64 sum = lane_u64(w, 15);
  u64 before = upto - v;
  if (wave > 0) before += lane_u64(w, wave - 1);
  *all = sum;
  return before;
}

// What a block walks over: a row or a chunk of it.  Every wave has a stretch of neighbouring tokens, in units of whole 16-byte pieces; the
// last wave has those behind the row's last whole unit too, where they belong to the block.
template <typename T>
struct Span {
  static constexpr int E = unit_elements<T>();
  const T *z;
  int V, whole, from, to;            // units of the block
  bool tail;
  int per, first, end;               // units of a wave; this wave's
  // (to_ > whole: to the end of the row)
  __device__ __forceinline__ Span(const T *z_, int V_, int from_, int to_) : z(z_), V(V_), whole(V_ / E) {
    from = min(from_, whole);
    to = max(from, min(to_, whole));
    tail = to_ > whole;
    per = (to - from + kWaves - 1) / kWaves;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    first = min(to, from + wave * per);
    end = min(to, first + per);
  }
  // U units are on their way while one is worked on, four tokens at a time: work on more of them mixed up by the compiler takes more registers
  // than there are.
  template <int U, typename F>
  __device__ __forceinline__ void stretch(int u0, int u1, F f) const {
    Unit<T, E> t[U];
    int u = u0 + (int)(threadIdx.x & 63);
#pragma unroll
    for (int j = 0; j < U; ++j)
      if (u + 64 * j < u1) t[j].load(z + (u + 64 * j) * E);
    for (; u - (int)(threadIdx.x & 63) < u1; u += 64 * U) {
#pragma unroll
      for (int j = 0; j < U; ++j) {
        const int at = u + 64 * j;
        __builtin_amdgcn_sched_barrier(0);
        if (at < u1) {
          const Unit<T, E> now = t[j];
          if (at + 64 * U < u1) t[j].load(z + (at + 64 * U) * E);
#pragma unroll
          for (int i = 0; i < E; ++i) {
            if (i == 4) __builtin_amdgcn_sched_barrier(0);
            f(now.get(i), (uint32_t)(at * E + i));
          }
        }
      }
    }
  }
  // f(unit, index of its first token) for every unit of the block
  template <int U = 4, typename F>
  __device__ __forceinline__ void units(F f) const {
    Unit<T, E> t[U];
    int u = first + (int)(threadIdx.x & 63);
#pragma unroll
    for (int j = 0; j < U; ++j)
      if (u + 64 * j < end) t[j].load(z + (u + 64 * j) * E);
    for (; u - (int)(threadIdx.x & 63) < end; u += 64 * U) {
#pragma unroll
      for (int j = 0; j < U; ++j) {
        const int at = u + 64 * j;
        if (at < end) {
          const Unit<T, E> now = t[j];
          if (at + 64 * U < end) t[j].load(z + (at + 64 * U) * E);
          f(now, (uint32_t)(at * E));
        }
      }
    }
  }
  template <typename F>
  __device__ __forceinline__ void behind(F f) const {
    const int i = whole * E + (int)(threadIdx.x & 63);
    if (tail && (threadIdx.x >> 6) == kWaves - 1 && i < V) f(Elem<T>::load(z + i), (uint32_t)i);
  }
  // f(logit, index) for every token of the block, by some thread
  template <int U = 4, typename F>
  __device__ __forceinline__ void each(F f) const {
    stretch<U>(first, end, f);
    behind(f);
  }
};

// Bins of equal width below the largest logit.
template <int N = kBins>
struct Bins {
  float best, scale;
  __device__ __forceinline__ Bins(float best_, float width) : best(best_), scale((float)N / width) {
    if (!(scale < INFINITY)) scale = 0.0f;               // (all in the first bin)
  }
  __device__ __forceinline__ int of(float z) const { return z == best ? 0 : (int)fminf((best - z) * scale, (float)(N - 1)); }   // (NaN: the last)
};

// The bin in which the sum over bins, from the first on, reaches the target (at least 1 and at most the whole sum); the sum before it in
// sh.above.
__device__ __forceinline__ int crossing_bin(Shared &sh, u64 target) {
  const u64 a = sh.bins[2 * threadIdx.x], b = sh.bins[2 * threadIdx.x + 1];
  u64 all;
  const u64 before = block_before_u64(a + b, sh, &all);
  if (before < target && target <= before + a + b) {
    const bool second = target > before + a;
    sh.result = 2 * threadIdx.x + (second ? 1 : 0);
    sh.above = second ? before + a : before;
  }
  __syncthreads();
  return (int)sh.result;
}
__device__ __forceinline__ void clear_bins(Shared &sh) {
  __syncthreads();
  sh.bins[2 * threadIdx.x] = 0;
  sh.bins[2 * threadIdx.x + 1] = 0;
  if (threadIdx.x == 0) sh.count = 0;
  __syncthreads();
}
// Adds w to a bin.  Lanes that all bring the same `tag`, which says bin and weight (equal logits, say), add once together.
__device__ __forceinline__ void add_to_bin(Shared &sh, int bin, uint32_t tag, u64 w) {
  const u64 active = __ballot(1);
  const uint32_t head = __builtin_amdgcn_readfirstlane(tag);
  if (__ballot(tag != head) == 0) {
    const int leader = __ffsll((long long)active) - 1;
    if ((int)(threadIdx.x & 63) == leader) atomicAdd(&sh.bins[bin], w * (u64)__popcll(active));
  } else {
    atomicAdd(&sh.bins[bin], w);
  }
}

__device__ __forceinline__ void gather(Shared &sh, Rank r) {
  const int at = atomicAdd(&sh.count, 1);
  if (at < kSmall) sh.list[at] = r;
}

// Those of a unit's tokens for which `take`: a place for all of a lane's at once, so that the waves wait for the counter once a unit.
template <int E, typename FU, typename F>
__device__ __forceinline__ void gather_unit(Shared &sh, FU logit, uint32_t first, F take) {
  uint32_t hits = 0;
#pragma unroll
  for (int i = 0; i < E; ++i) hits |= take(logit(i)) ? 1u << i : 0u;
  if (hits == 0) return;
  int at = atomicAdd(&sh.count, __popc(hits));
#pragma unroll
  for (int i = 0; i < E; ++i)
    if (hits >> i & 1) {
      if (at < kSmall) sh.list[at] = rank_of(logit(i), first + i);
      ++at;
    }
}

// sh.list[0 .. M) into sh.sorted, descending, with every token's place found by comparing it with all the others; P threads share a token.
__device__ __forceinline__ void sort_small(Shared &sh, int M) {
  int size = 1;
  while (size < M) size <<= 1;
  const int parts = min(64, kThreads / size), me = (int)threadIdx.x / parts, part = (int)threadIdx.x % parts;
  const Rank mine = me < M ? sh.list[me] : 0;
  int place = 0;
  if (me < M)
#pragma unroll 4
    for (int j = part; j < M; j += parts) place += sh.list[j] > mine;
  for (int o = 1; o < parts; o <<= 1) place += __shfl_xor(place, o, 64);
  if (me < M && part == 0) sh.sorted[place] = mine;
  __syncthreads();
}

// The rank in sh.list[0 .. M), none below the border, from which on the sum of W reaches the target; `before`: the sum over the tokens above all of these.
template <typename FW>
__device__ __forceinline__ Rank border_in_list(Shared &sh, int M, u64 before, u64 target, FW W) {
  sort_small(sh, M);
  const Rank r = (int)threadIdx.x < M ? sh.sorted[threadIdx.x] : 0;
  const u64 w = r ? W(logit_of((uint32_t)(r >> 32))) : 0;
  u64 all;
  const u64 upto = before + block_before_u64(w, sh, &all);
  if (r && upto < target && target <= upto + w) sh.result = r;
  __syncthreads();
  return sh.result;
}

// The token of a span at which the running sum of W, which is `start` before the span, passes point(its sum over the span): the wave in whose
// stretch that is, the sixteenth of this stretch, the token.
template <int U, typename T, typename FT, typename FW, typename FP>
__device__ __forceinline__ void locate(const Span<T> &span, Shared &sh, u64 start, FT point, FW W, FP put) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  u64 sum = 0, all;
  span.template each<U>([&](float z, uint32_t i) { sum += W(z, i); });
  sum = wave_sum_u64(sum);
  u64 before = start + block_before_u64(lane == 0 ? sum : 0, sh, &all);
  const u64 target = point(all);
  if (lane == 0 && before <= target && target < before + sum) {
    sh.slot = wave;
    sh.result = before;
  }
  __syncthreads();
  const int s0 = min(span.to, span.from + sh.slot * span.per), s1 = min(span.to, s0 + span.per);
  const bool tail = span.tail && sh.slot == kWaves - 1;
  const u64 from = sh.result;
  const int sub = (s1 - s0 + kWaves - 1) / kWaves, t0 = min(s1, s0 + wave * sub), t1 = min(s1, t0 + sub);
  sum = 0;
  span.template stretch<1>(t0, t1, [&](float z, uint32_t i) { sum += W(z, i); });
  if (tail) span.behind([&](float z, uint32_t i) { sum += W(z, i); });
  sum = wave_sum_u64(sum);
  before = from + block_before_u64(lane == 0 ? sum : 0, sh, &all);
  before = lane_u64(before, 0);
  if (!(before <= target && target < before + sum)) return;
  // one wave: its units in order, 64 at a time, then the tokens behind the last unit
  constexpr int E = Span<T>::E;
  for (int u0 = t0; u0 < t1; u0 += 64) {
    const int unit = u0 + lane;
    u64 w[E], own = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      w[i] = unit < t1 ? W(Elem<T>::load(span.z + unit * E + i), (uint32_t)(unit * E + i)) : 0;
      own += w[i];
    }
    const u64 upto = wave_upto_u64(own);
    u64 at = before + upto - own;
    if (at <= target && target < at + own) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        if (at <= target && target < at + w[i]) put(unit * E + i);
        at += w[i];
      }
    }
    before += lane_u64(upto, 63);
  }
  if (tail && wave == kWaves - 1) {
    const int i = span.whole * E + lane;
    const u64 w = i < span.V ? W(Elem<T>::load(span.z + i), (uint32_t)i) : 0;
    const u64 at = before + wave_upto_u64(w) - w;
    if (at <= target && target < at + w) put(i);
  }
}

// The largest of the threads' first numbers and the smallest of their second and third ones, in all threads.
__device__ __forceinline__ void extremes(Shared &sh, float &top, float &low, float &least) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  top = max64(top);
  low = -max64(-low);
  least = -max64(-least);
  if (lane == 0) {
    sh.fmax[wave] = top;
    sh.fmin[wave] = low;
    sh.fleast[wave] = least;
  }
  __syncthreads();
  static_assert(kWaves == 16, "a row of lanes");
  top = max16(sh.fmax[lane & 15]);
  low = -max16(-sh.fmin[lane & 15]);
  least = -max16(-sh.fleast[lane & 15]);
}

// The rank from which on the sum of W over the row's tokens of at least `border` reaches the target.  W(logit): a token's share.
template <typename R, typename FW>
__device__ __forceinline__ Rank find_border(const R &row, Shared &sh, const Bins<> &bins, Rank border, u64 target, FW W) {
  // (sh.bins holds the sums by bin)
  const int bin = crossing_bin(sh, target);
  const u64 before = sh.above;
  __syncthreads();
  float high = -INFINITY, low = INFINITY, none = INFINITY;
  row.each([&](float z, uint32_t i) {
    if (bins.of(z) != bin) return;
    const Rank r = rank_of(z, i);
    if (r == 0 || r < border) return;
    gather(sh, r);
    high = fmaxf(high, z);
    low = fminf(low, z);
  });
  __syncthreads();
  const int M = sh.count;
  if (M <= kSmall) return border_in_list(sh, M, before, target, W);
  extremes(sh, high, low, none);
  if (high == low) {                                     // all equal: so many of them, the first by index
    const u64 w = W(high), nth = (target - before + w - 1) / w - 1;
    locate<1>(row, sh, 0, [=](u64) { return nth; }, [&](float z, uint32_t i) -> u64 { return z == high && rank_of(z, i) >= border; },
              [&](int64_t i) { sh.above = rank_of(high, (uint32_t)i); });
    __syncthreads();
    return sh.above;
  }
  // More than that in one bin (many nearly equal logits): the rank's bits, eleven at a time, over the tokens that share the bits found so far.
  Rank found = 0;
  u64 sum = before;
  // (the logit's 32 in three turns, the index's in three)
  for (int low = 53; ; low = low == 53 ? 42 : low == 42 ? 32 : low == 32 ? 21 : low == 21 ? 10 : 0) {
    const int width = low == 32 || low == 0 ? 10 : 11, high = low + width;
    clear_bins(sh);
    row.template each<2>([&](float z, uint32_t i) {
      if (bins.of(z) != bin) return;
      const Rank r = rank_of(z, i);
      if (r == 0 || r < border || (high < 64 && (r >> high) != (found >> high))) return;
      // (descending: the first bin has the largest ranks; in the bits of the index all logits are equal, above them equal logits have one bin)
      const int at = (1 << width) - 1 - (int)((r >> low) & ((1u << width) - 1));
      add_to_bin(sh, at, low < 32 ? (uint32_t)at : __float_as_uint(z), W(z));
    });
    __syncthreads();
    const int at = crossing_bin(sh, target - sum);
    sum += sh.above;
    found |= (u64)((1 << width) - 1 - at) << low;
    __syncthreads();
    if (low == 0) break;
  }
  return found;
}

// The same for a row whose units the threads hold, U each at most: the waves' running sums unit by unit, then the token.
template <int U, typename T, int E, typename FT, typename FW, typename FP>
__device__ __forceinline__ void locate_held(const Span<T> &row, Shared &sh, const Unit<T, E> (&held)[U], FT point, FW W, FP put) {
  const int lane = threadIdx.x & 63;
  u64 own[U], upto[U], sum = 0, all, behind = 0;
  const int u0 = row.first + lane, last = row.whole * E + lane;
#pragma unroll
  for (int j = 0; j < U; ++j) {
    own[j] = 0;
    if (u0 + 64 * j < row.end) {
#pragma unroll
      for (int i = 0; i < E; ++i) own[j] += W(held[j].get(i), (uint32_t)((u0 + 64 * j) * E + i));
    }
  }
  row.behind([&](float z, uint32_t i) { behind = W(z, i); });
#pragma unroll
  for (int j = 0; j < U; ++j) {
    upto[j] = sum + wave_upto_u64(own[j]);
    sum = lane_u64(upto[j], 63);
  }
  const u64 upto_behind = sum + wave_upto_u64(behind);
  sum = lane_u64(upto_behind, 63);
  const u64 before = lane_u64(block_before_u64(lane == 0 ? sum : 0, sh, &all), 0), target = point(all);
  if (!(before <= target && target < before + sum)) return;
#pragma unroll
  for (int j = 0; j < U; ++j) {
    u64 at = before + upto[j] - own[j];
    if (at <= target && target < at + own[j]) {
#pragma unroll
      for (int i = 0; i < E; ++i) {
        const u64 w = W(held[j].get(i), (uint32_t)((u0 + 64 * j) * E + i));
        if (at <= target && target < at + w) put((u0 + 64 * j) * E + i);
        at += w;
      }
    }
  }
  const u64 at = before + upto_behind - behind;
  if (at <= target && target < at + behind) put(last);
}

// What bins of weights have to cover: 33 temperatures below the largest logit weights are zero, and below the smallest (which is -inf where
// tokens are masked) there is nothing.
__device__ __forceinline__ float width_of(const Weights &wt, float t, float least) { return fminf(33.0f * t, wt.best - least); }

// What the caller asks of a row.
struct Asked {
  float t, u, p, minp;
  int64_t k;
  __device__ __forceinline__ Asked(const SampleArgs &a, int64_t n) {
    t = a.temperature ? a.temperature[n * a.st] : 1.0f;
    u = a.u[n * a.su];
    p = a.top_p ? a.top_p[n * a.sp] : 1.0f;
    const float m = a.min_p ? a.min_p[n * a.sm] : 0.0f;
    minp = m > 0.0f ? fminf(m, 1.0f) : 0.0f;
    k = 0;
    if (a.top_k) k = a.k64 ? static_cast<const int64_t *>(a.top_k)[n * a.sk] : static_cast<const int32_t *>(a.top_k)[n * a.sk];
  }
  __device__ __forceinline__ bool greedy() const { return !(t > 0.0f); }
  __device__ __forceinline__ bool inside() const { return u > 0.0f && u < 1.0f; }
  // up to where the weights of the kept tokens have to sum, of `all`
  __device__ __forceinline__ u64 share(u64 all) const {
    const u64 target = p > 0.0f ? (u64)ceil((double)p * (double)all) : 1;
    return target < 1 ? 1 : target;
  }
  __device__ __forceinline__ u64 point(u64 all) const { return (u64)((double)u * (double)all); }   // below `all`: u is at most 1 - 2^-24
};

struct Put {
  const SampleArgs &a;
  int64_t n;
  __device__ __forceinline__ void operator()(int64_t token) const {
    if (a.out64) static_cast<int64_t *>(a.out)[n] = token;
    else static_cast<int32_t *>(a.out)[n] = (int32_t)token;
  }
};

// A logit such that at least those in bins up to `last` are not below it.
template <int N>
__device__ __forceinline__ float bound_of(const Bins<N> &few, int last) {
  // the smallest key of these bins, by search: 64 at a time
  uint32_t a = 0x00800000u, b = key_of(few.best);
  while (a < b) {
    const uint32_t step = (b - a + 63) / 64, lane = threadIdx.x & 63, at = b - a < lane * (u64)step ? b : a + lane * step;
    const int f = __ffsll((long long)__ballot(few.of(logit_of(at)) <= last)) - 1;
    if (f == 0) {
      b = a;
    } else if (f < 0) {
      a += 63 * step + 1;
    } else {
      const uint32_t to = b - a < f * (u64)step ? b : a + f * step;
      a += (f - 1) * step + 1;
      b = to;
    }
  }
  return logit_of(b);
}

// The last bin of those that hold the k largest of the values that the threads add, -1 if there are fewer than k: 256 bins of counts, which
// every wave reads and sums by itself, so that one barrier is enough.  sh.bins has to be clear, and is not afterwards.
template <typename F>
__device__ __forceinline__ int bin_of_kth(Shared &sh, int64_t k, F add) {
  uint32_t *counts = reinterpret_cast<uint32_t *>(sh.bins);
  add([&](int bin) { atomicAdd(&counts[bin], 1u); });
  __syncthreads();
  const int lane = threadIdx.x & 63;
  static_assert(kFewBins == 256, "four for each lane");
  const uint4 c = *reinterpret_cast<const uint4 *>(counts + 4 * lane);
  const u64 upto = wave_upto_u64((u64)(c.x + c.y + c.z + c.w));
  const u64 enough = __ballot(upto >= (u64)k);
  if (enough == 0) return -1;
  const int l = __ffsll((long long)enough) - 1;
  const uint32_t x = __builtin_amdgcn_readlane(c.x, l), y = __builtin_amdgcn_readlane(c.y, l), z = __builtin_amdgcn_readlane(c.z, l),
                 w = __builtin_amdgcn_readlane(c.w, l);
  const uint32_t need = (uint32_t)((u64)k - (lane_u64(upto, l) - (x + y + z + w)));
  return 4 * l + (need <= x ? 0 : need <= x + y ? 1 : need <= x + y + z ? 2 : 3);
}

// The draw from sh.list[0 .. M): every token that top-k (with top-p and min-p) can keep.
__device__ __forceinline__ void draw_small(Shared &sh, int M, const Asked &q, const Weights &wt, int V, const Put &put) {
  sort_small(sh, M);
  const Rank r = (int)threadIdx.x < M && !(q.k > 0 && (int64_t)threadIdx.x >= q.k) ? sh.sorted[threadIdx.x] : 0;
  const float v = logit_of((uint32_t)(r >> 32));
  double e = r != 0 && v >= wt.zero(q.t) ? wt.near(v) : 0.0;
  const u64 w = wt.of(e);
  if (!q.inside()) e = r == 0 ? 0.0 : wt.exponential(v);   // (the ends ask for the lightest; top-p sums the same weights there)
  bool kept = r != 0;
  if (q.p < 1.0f) {
    u64 all;
    const u64 before = block_before_u64(w, sh, &all);
    kept = kept && (before < q.share(all) || threadIdx.x == 0);
  }
  kept = kept && reaches(wt, v, e, q.minp);
  if (q.inside()) {
    u64 all;
    block_before_u64(kept ? w : 0, sh, &all);
    const u64 target = q.point(all);
    if ((int)threadIdx.x < M) {
      sh.list[threadIdx.x] = r;
      sh.weight[threadIdx.x] = kept ? w : 0;
    }
    __syncthreads();
    // running sums in the order of indices, by comparing each with each
    int size = 1;
    while (size < M) size <<= 1;
    const int parts = min(64, kThreads / size), me = (int)threadIdx.x / parts, part = (int)threadIdx.x % parts;
    const uint32_t index = me < M ? index_of(sh.list[me]) : 0;
    u64 before = 0;
    if (me < M)
#pragma unroll 4
      for (int j = part; j < M; j += parts) before += index_of(sh.list[j]) < index ? sh.weight[j] : 0;
    for (int o = 1; o < parts; o <<= 1) before += __shfl_xor(before, o, 64);
    if (me < M && part == 0 && before <= target && target < before + sh.weight[me]) put(index);
  } else {                                               // the ends of the range: the first and the last token, however light
    if (threadIdx.x == 0) sh.slot = q.u >= 1.0f ? -1 : V;
    __syncthreads();
    if (kept && e > 0.0) {
      if (q.u >= 1.0f) atomicMax(&sh.slot, (int)index_of(r));
      else atomicMin(&sh.slot, (int)index_of(r));
    }
    __syncthreads();
    if (threadIdx.x == 0) put(sh.slot);
  }
}

// The draw from a whole row whose largest logit is known, in passes over it; `finish` makes the draw once it is known what is kept.
template <typename T, typename FF>
__device__ __forceinline__ void draw_whole(const Span<T> &row, Shared &sh, const Asked &q, const Weights &wt, float least, const Put &put,
                                           FF finish) {
  const float best = wt.best;
  if (best == INFINITY) {                                // equal weights for the tokens that have it, none for the others
    u64 m = 0, all;
    row.template each<1>([&](float z, uint32_t) { m += z == INFINITY; });
    block_before_u64(m, sh, &all);
    if (q.k > 0 && (u64)q.k < all) all = (u64)q.k;
    if (q.p < 1.0f) all = q.share(all);
    const u64 target = !(q.u > 0.0f) ? 0 : q.u >= 1.0f ? all - 1 : q.point(all);
    locate<1>(row, sh, 0, [=](u64) { return target; }, [](float z, uint32_t) -> u64 { return z == INFINITY; }, put);
    return;
  }
  Rank border = 1;
  // first the border of top-k, counting tokens, then that of top-p among what is left, adding weights (one piece of code)
#pragma unroll 1
  for (int by_weight = 0; by_weight < 2; ++by_weight) {
    float width;                                         // of what the bins cover
    if (by_weight) {
      if (!(q.p < 1.0f)) break;
      width = width_of(wt, q.t, least);
    } else {
      if (q.k <= 0) continue;
      u64 have = 0, all;
      float none = -INFINITY, lowest = INFINITY;
      row.template each<1>([&](float z, uint32_t) {
        if (z > -INFINITY) {
          lowest = fminf(lowest, z);
          ++have;
        }
      });
      block_before_u64(have, sh, &all);
      if ((u64)q.k >= all) continue;
      extremes(sh, none, none, lowest);
      width = best - lowest;
    }
    const Bins<> bins(best, width);
    const float zero = by_weight ? wt.zero(q.t) : -INFINITY;
    const auto share = [&](float z) -> u64 { return by_weight ? (z >= zero ? wt.of(wt.near(z)) : 0) : 1; };
    clear_bins(sh);
    row.each([&](float z, uint32_t i) {
      if (z > -INFINITY && (border <= 1 || rank_of(z, i) >= border)) add_to_bin(sh, bins.of(z), __float_as_uint(z), share(z));
    });
    __syncthreads();
    u64 target = (u64)q.k;
    if (by_weight) {
      u64 all;
      block_before_u64(sh.bins[2 * threadIdx.x] + sh.bins[2 * threadIdx.x + 1], sh, &all);
      target = q.share(all);
      __syncthreads();
    }
    border = find_border(row, sh, bins, border, target, share);
    __syncthreads();
  }
  Limit limit = border <= 1 ? Limit{-INFINITY, 0} : Limit{logit_of((uint32_t)(border >> 32)), index_of(border) + 1};
  if (q.minp > 0.0f) limit.not_below(least_logit(wt, q.t, q.minp));
  if (!q.inside()) {                                     // the ends of the range: the first and the last token, however light
    __syncthreads();
    if (threadIdx.x == 0) sh.slot = q.u >= 1.0f ? -1 : row.V;
    __syncthreads();
    row.template each<1>([&](float z, uint32_t i) {
      if (limit.keeps(z, i) && wt.exponential(z) > 0.0) {
        if (q.u >= 1.0f) atomicMax(&sh.slot, (int)i);
        else atomicMin(&sh.slot, (int)i);
      }
    });
    __syncthreads();
    if (threadIdx.x == 0) put(sh.slot);
    return;
  }
  limit.not_below(wt.zero(q.t));
  const auto W = [&](float z, uint32_t i) -> u64 { return wt.of(limit.keeps(z, i) ? wt.near(z) : 0.0); };
  finish(W);
}

// What a kernel begins with; the next barrier makes it everybody's.
__device__ __forceinline__ void begin(Shared &sh) {
  if (threadIdx.x < 32) sh.powers[threadIdx.x] = kPowers[threadIdx.x];
  sh.bins[2 * threadIdx.x] = 0;
  sh.bins[2 * threadIdx.x + 1] = 0;
  if (threadIdx.x == 0) sh.count = 0;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_kernel(const T *logits, SampleArgs a) {
  __shared__ Shared sh;
  const int64_t n = block_number();
  if (n >= a.N) return;
  const Asked q(a, n);                                   // (first, so that its loads are under way with the row's)
  begin(sh);
  const Span<T> row(logits + n * a.pitch, a.V, 0, a.V);
  const int lane = threadIdx.x & 63;
  const Put put{a, n};
  // the largest logit, the threads' own, and the smallest of those; the units of rows of up to four a thread stay in registers
  constexpr int E = Span<T>::E, U = kHeldUnits;
  Unit<T, E> held[U];
  const bool holds = row.per <= 64 * U;
  float mine = -INFINITY, least = INFINITY;
  const auto look = [&](float z) {
    mine = fmaxf(mine, z);
    least = fminf(least, z);                             // (-inf where a token is masked: what it is for does without)
  };
  if (holds) {
#pragma unroll
    for (int j = 0; j < U; ++j) {
      held[j].zero();
      if (row.first + lane + 64 * j < row.end) held[j].load(row.z + (row.first + lane + 64 * j) * E);
    }
#pragma unroll
    for (int j = 0; j < U; ++j)
      if (row.first + lane + 64 * j < row.end) {
#pragma unroll
        for (int i = 0; i < E; ++i) look(held[j].get(i));
      }
    row.behind([&](float z, uint32_t) { look(z); });
  } else {
    row.each([&](float z, uint32_t) { look(z); });
  }
  float best = mine, low = mine > -INFINITY ? mine : INFINITY;
  extremes(sh, best, low, least);
  if (best == -INFINITY) {                               // nothing to choose from
    if (threadIdx.x == 0) put(-1);
    return;
  }
  if (q.greedy()) {
    if (threadIdx.x == 0) sh.slot = a.V;
    __syncthreads();
    if (mine == best)                                    // (the others have nothing to find)
      row.template each<1>([&](float z, uint32_t i) {
        if (z == best) atomicMin(&sh.slot, (int)i);
      });
    __syncthreads();
    if (threadIdx.x == 0) put(sh.slot);
    return;
  }
  const Weights wt(best, q.t, a.shift, sh);
  // a row that comes down to a few tokens by top-k: all of them from a bound on.  (Not by min-p, which asks for no order: 128 x 10000 fp32 44 us so, 9.5 with
  // the whole row's weights; 64 x 50000 91 / 23, 128 x 300 8.9 / 8.1)
  int M = kSmall + 1;
  if (best < INFINITY && q.k > 0 && q.k <= kThreads) {
    const Bins<kFewBins> few(best, best - low);
    const int last = bin_of_kth(sh, q.k, [&](auto add) {
      if (mine > -INFINITY) add(few.of(mine));
    });
    if (last >= 0) {
      const auto take = [&](float z) { return z > -INFINITY && few.of(z) <= last; };
      if (few.of(mine) <= last) {                        // (the others hold none)
        if (holds) {
#pragma unroll
          for (int j = 0; j < U; ++j)
            if (row.first + lane + 64 * j < row.end)
              gather_unit<E>(sh, [&](int i) { return held[j].get(i); }, (uint32_t)((row.first + lane + 64 * j) * E), take);
        } else {
          row.units([&](const Unit<T, E> &t, uint32_t first) { gather_unit<E>(sh, [&](int i) { return t.get(i); }, first, take); });
        }
        row.behind([&](float z, uint32_t i) {
          if (take(z)) gather(sh, rank_of(z, i));
        });
      }
      __syncthreads();
      M = sh.count;
    }
  }
  if (M <= kSmall) draw_small(sh, M, q, wt, a.V, put);
  else draw_whole(row, sh, q, wt, least, put, [&](auto W) __attribute__((always_inline)) {
    const auto point = [&](u64 all) { return q.point(all); };
    if (holds) locate_held(row, sh, held, point, W, put);
    else locate<4>(row, sh, 0, point, W, put);
  });
}

// ---- short rows -----------------------------------------------------------------------------------------------------
// Up to 256 tokens: a wave has a row, a lane four neighbouring tokens of it in registers.  A token's place in the order of the filters is the
// number of those before it, counted by comparing it with all.  No barriers, and four rows to a block.  Measured in us, a block of 1024 for each row / so
// (fp32; top-k, top-p, none, and all filters mixed):
//   8 x 64 14 13 8 20 / 5 6 3 6        4096 x 64 200 187 105 269 / 9 10 4 10    27 x 141 9 13 8 13 / 7 8 3 8
//   128 x 256 9 13 8 14 / 11 11 3 11   4096 x 256 108 187 105 176 / 23 23 5 23
// Comparing grows with the square: blocks that order up to 512 tokens by it, without bins, take 19 at 8 x 300 where bins take 8 to 13.
constexpr int kShort = 256;

struct alignas(16) ShortShared {
  double powers[32];
  uint32_t keys[kShort];
  u64 weight[kShort];                // by place
};

// What a wave wrote to LDS is there for all of its lanes.
__device__ __forceinline__ void wave_sync() {
  __builtin_amdgcn_fence(__ATOMIC_RELEASE, "wavefront");
  __builtin_amdgcn_wave_barrier();
  __builtin_amdgcn_fence(__ATOMIC_ACQUIRE, "wavefront");
}

template <typename T>
__global__ __launch_bounds__(256) void sample_short_kernel(const T *logits, SampleArgs a) {
  __shared__ ShortShared all_waves[4];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int64_t n = block_number() * 4 + wave;
  if (n >= a.N) return;
  ShortShared &sh = all_waves[wave];
  const Asked q(a, n);
  const Put put{a, n};
  const T *row = logits + n * a.pitch;
  float z[4], best = -INFINITY;
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    z[j] = lane * 4 + j < a.V ? Elem<T>::load(row + lane * 4 + j) : -INFINITY;
    best = fmaxf(best, z[j]);
  }
  if (lane < 32) sh.powers[lane] = kPowers[lane];
  best = max64(best);
  // the first or the last token of those that the lanes name (at least one of the wave's)
  const auto put_end = [&](const bool (&these)[4], bool last) {
    const u64 any = __ballot(these[0] || these[1] || these[2] || these[3]);
    const int l = last ? 63 - __clzll((long long)any) : __ffsll((long long)any) - 1;
    if (lane != l) return;
    int at = 0;
#pragma unroll
    for (int j = 0; j < 4; ++j) at = these[last ? j : 3 - j] ? (last ? j : 3 - j) : at;
    put(l * 4 + at);
  };
  // the token at which the running sum of w in the order of indices passes point(whole sum)
  const auto put_at = [&](const u64 (&w)[4], auto point) {
    const u64 own = w[0] + w[1] + w[2] + w[3], upto = wave_upto_u64(own), target = point(lane_u64(upto, 63));
    u64 at = upto - own;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (at <= target && target < at + w[j]) put(lane * 4 + j);
      at += w[j];
    }
  };
  if (best == -INFINITY) {                               // nothing to choose from
    if (lane == 0) put(-1);
    return;
  }
  bool kept[4];
  if (q.greedy()) {
#pragma unroll
    for (int j = 0; j < 4; ++j) kept[j] = z[j] == best;
    put_end(kept, false);
    return;
  }
  u64 w[4];
  if (best == INFINITY) {                                // equal weights for the tokens that have it, none for the others
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = z[j] == INFINITY;
    put_at(w, [&](u64 all) {
      if (q.k > 0 && (u64)q.k < all) all = (u64)q.k;
      if (q.p < 1.0f) all = q.share(all);
      return !(q.u > 0.0f) ? 0 : q.u >= 1.0f ? all - 1 : q.point(all);
    });
    return;
  }
  wave_sync();
  const Weights wt(best, q.t, a.shift, sh.powers);
  const float zero = wt.zero(q.t);
  double e[4];
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    kept[j] = z[j] > -INFINITY;
    e[j] = kept[j] && z[j] >= zero ? wt.near(z[j]) : 0.0;
    w[j] = wt.of(e[j]);
  }
  if (!q.inside()) {                                     // (the ends ask for the lightest; top-p sums the same weights there)
#pragma unroll
    for (int j = 0; j < 4; ++j) e[j] = kept[j] ? wt.exponential(z[j]) : 0.0;
  }
  if (q.k > 0 || q.p < 1.0f) {
    uint32_t key[4], place[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      key[j] = key_of(z[j]);
      place[j] = 0;
      sh.keys[lane * 4 + j] = key[j];
      sh.weight[lane * 4 + j] = 0;
    }
    wave_sync();
    const int lanes = (a.V + 3) / 4;
#pragma unroll 4
    for (int l = 0; l < lanes; ++l) {                    // an equal one of an earlier lane comes before, of a later lane behind
      const uint4 c = *reinterpret_cast<const uint4 *>(sh.keys + 4 * l);
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const uint32_t above = key[j] - (l < lane ? 1 : 0);
        place[j] += (c.x > above) + (c.y > above) + (c.z > above) + (c.w > above);
      }
    }
#pragma unroll
    for (int j = 1; j < 4; ++j)
#pragma unroll
      for (int i = 0; i < j; ++i) place[j] += key[i] == key[j];
    if (q.k > 0) {
#pragma unroll
      for (int j = 0; j < 4; ++j) kept[j] = kept[j] && (int64_t)place[j] < q.k;
    }
    if (q.p < 1.0f) {
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (kept[j]) sh.weight[place[j]] = w[j];
      wave_sync();
      u64 by_place[4], own = 0;
#pragma unroll
      for (int j = 0; j < 4; ++j) own += by_place[j] = sh.weight[lane * 4 + j];
      const u64 upto = wave_upto_u64(own), target = q.share(lane_u64(upto, 63));
      u64 before = upto - own;
      int last = 0;                                      // places that are kept: a few from the first on
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        last += __popcll(__ballot(before < target));
        before += by_place[j];
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) kept[j] = kept[j] && (int)place[j] < max(last, 1);
    }
  }
#pragma unroll
  for (int j = 0; j < 4; ++j) kept[j] = kept[j] && reaches(wt, z[j], e[j], q.minp);
  if (q.inside()) {
#pragma unroll
    for (int j = 0; j < 4; ++j) w[j] = kept[j] ? w[j] : 0;
    put_at(w, [&](u64 all) { return q.point(all); });
  } else {
#pragma unroll
    for (int j = 0; j < 4; ++j) kept[j] = kept[j] && e[j] > 0.0;
    put_end(kept, q.u >= 1.0f);
  }
}

// ---- rows in chunks -------------------------------------------------------------------------------------------------
// The code of these kernels runs once through, from a cold instruction cache: loops work on one or two units at a time, not on four.
template <typename T>
__device__ __forceinline__ Span<T> chunk_of(const T *logits, const SampleArgs &a, int64_t n, int chunk) {
  return Span<T>(logits + n * a.pitch, a.V, chunk * a.chunk_units, chunk + 1 == a.chunks ? a.V : (chunk + 1) * a.chunk_units);
}

// The largest over the PART lanes of a part, in all of these lanes.
template <int PART>
__device__ __forceinline__ float max_part(float v) {
  if constexpr (PART == 64) return max64(v);
  v = dpp_max<0x4E>(dpp_max<0xB1>(v));
  if constexpr (PART >= 8) v = dpp_max<0x141>(v);
  if constexpr (PART >= 16) v = dpp_max<0x140>(v);
  if constexpr (PART >= 32) {
    const auto row = [&](int r) { return __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 16 * r)); };
    v = (threadIdx.x & 63) < 32 ? fmaxf(row(0), row(1)) : fmaxf(row(2), row(3));
  }
  return v;
}

// Launch 1: the maxima and minima of all parts; what later launches add to is cleared.
template <typename T, int PART>
__global__ __launch_bounds__(kThreads) void sample_maxima_kernel(const T *logits, SampleArgs a) {
  constexpr int E = Span<T>::E, U = 4;
  const int64_t n = blockIdx.y;
  const int chunk = blockIdx.x, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  RowSpace &space = a.space[n];
  if (chunk == 0) {
    space.bins[2 * threadIdx.x] = 0;
    space.bins[2 * threadIdx.x + 1] = 0;
    if (threadIdx.x == 0) space.count = 0;
  }
  const T *z = logits + n * a.pitch;
  const int whole = a.V / E, u0 = chunk * a.chunk_units, u1 = min(whole, u0 + a.chunk_units);
  for (int first = u0 + wave * 64; first < u1; first += kWaves * 64 * U) {
    Unit<T, E> t[U];
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int u = first + j * kWaves * 64 + lane;
      if (first + j * kWaves * 64 < u1 && u < whole) t[j].load(z + u * E);
    }
#pragma unroll
    for (int j = 0; j < U; ++j) {
      const int base = first + j * kWaves * 64, u = base + lane;
      if (base >= u1) break;
      float m = -INFINITY, l = INFINITY;
      const auto look = [&](float v) {
        m = fmaxf(m, v);
        l = fminf(l, v);
      };
      if (u < whole) {
#pragma unroll
        for (int i = 0; i < E; ++i) look(t[j].get(i));
      }
      const int at = base / PART + lane / PART;
      if (base + 64 >= whole && at == a.parts - 1)       // the tokens behind the last unit, by the lanes of the last part
#pragma unroll
        for (int i = whole * E + lane % PART, k = 0; k < E - 1; i += PART, k += PART)
          if (i < a.V) look(Elem<T>::load(z + i));
      m = max_part<PART>(m);
      l = -max_part<PART>(-l);
      if (lane % PART == 0 && at < a.parts) {
        space.maxima[at] = m;
        space.minima[at] = l;
      }
    }
  }
}

// How a row is drawn from, the same in all launches that follow.
enum Way { kNothing, kGreedy, kFew, kSums, kPlain, kWhole };
struct Plan {
  Way way;
  float best, low, least;            // largest and smallest of the parts' maxima, smallest of their minima
};

__device__ __forceinline__ Plan plan_row(Shared &sh, const SampleArgs &a, const RowSpace &space, const Asked &q) {
  begin(sh);
  float top = -INFINITY, down = INFINITY, least = INFINITY;
  for (int p = threadIdx.x; p < a.parts; p += kThreads) {
    const float m = space.maxima[p];
    top = fmaxf(top, m);
    if (m > -INFINITY) down = fminf(down, m);
    least = fminf(least, space.minima[p]);
  }
  Plan plan{kNothing, top, down, least};
  extremes(sh, plan.best, plan.low, plan.least);
  if (plan.best == -INFINITY) return plan;
  plan.way = q.greedy() ? kGreedy : plan.best < INFINITY ? (q.k > 0 ? kFew : !q.inside() ? kWhole : q.p < 1.0f ? kSums : kPlain) : kWhole;
  return plan;
}

// Launch 2: sums by bin where top-p asks for them, otherwise the chunk's sum.
template <typename T>
__global__ __launch_bounds__(kThreads) void sample_bins_kernel(const T *logits, SampleArgs a) {
  __shared__ Shared sh;
  const int64_t n = blockIdx.y;
  const Asked q(a, n);
  if (q.greedy() || q.k > 0) return;
  const int chunk = blockIdx.x;
  RowSpace &space = a.space[n];
  const Plan plan = plan_row(sh, a, space, q);
  if (plan.way != kSums && plan.way != kPlain) return;
  const Span<T> span = chunk_of(logits, a, n, chunk);
  const Weights wt(plan.best, q.t, a.shift, sh);
  float least = wt.zero(q.t);
  if (plan.way == kSums) {
    const Bins<> bins(plan.best, width_of(wt, q.t, plan.least));
    span.template each<8 / Span<T>::E>([&](float z, uint32_t) {
      if (z >= least) add_to_bin(sh, bins.of(z), __float_as_uint(z), wt.of(wt.near(z)));
    });
    __syncthreads();
    for (int b = threadIdx.x; b < kBins; b += kThreads)
      if (sh.bins[b]) atomicAdd(&space.bins[b], sh.bins[b]);
  } else {
    if (q.minp > 0.0f) least = fmaxf(least, least_logit(wt, q.t, q.minp));
    u64 sum = 0, all;
    span.template each<8 / Span<T>::E>([&](float z, uint32_t) { sum += wt.of(z >= least ? wt.near(z) : 0.0); });
    block_before_u64(sum, sh, &all);
    if (threadIdx.x == 0) space.sums[chunk] = all;
  }
}

// The bin of top-p's border; the sum before it in sh.above, the target in *target.
__device__ __forceinline__ int border_bin(Shared &sh, const RowSpace &space, const Asked &q, u64 *target) {
  sh.bins[2 * threadIdx.x] = space.bins[2 * threadIdx.x];
  sh.bins[2 * threadIdx.x + 1] = space.bins[2 * threadIdx.x + 1];
  u64 all;
  block_before_u64(sh.bins[2 * threadIdx.x] + sh.bins[2 * threadIdx.x + 1], sh, &all);
  *target = q.share(all);
  return crossing_bin(sh, *target);
}

// Launch 3, rows with top-p alone: the tokens of the border's bin, and the chunk's sum over the tokens above it that min-p keeps.
template <typename T>
__global__ __launch_bounds__(kThreads) void sample_border_kernel(const T *logits, SampleArgs a) {
  __shared__ Shared sh;
  const int64_t n = blockIdx.y;
  const Asked q(a, n);
  if (q.k > 0 || !(q.p < 1.0f) || !q.inside() || q.greedy()) return;
  const int chunk = blockIdx.x;
  RowSpace &space = a.space[n];
  const Plan plan = plan_row(sh, a, space, q);
  if (plan.way != kSums) return;
  const Span<T> span = chunk_of(logits, a, n, chunk);
  const Weights wt(plan.best, q.t, a.shift, sh);
  const Bins<> bins(plan.best, width_of(wt, q.t, plan.least));
  u64 target, all, sum = 0;
  const int bin = border_bin(sh, space, q, &target);
  float least = wt.zero(q.t);
  if (q.minp > 0.0f) least = fmaxf(least, least_logit(wt, q.t, q.minp));
  span.template each<8 / Span<T>::E>([&](float z, uint32_t i) {
    const int b = bins.of(z);
    if (b == bin && z > -INFINITY) {
      const int at = atomicAdd(&space.count, 1);
      if (at < kSmall) space.list[at] = rank_of(z, i);
    }
    if (b < bin && z >= least) sum += wt.of(wt.near(z));
  });
  block_before_u64(sum, sh, &all);
  if (threadIdx.x == 0) space.sums[chunk] = all;
}

// f(logit, index) for every token of the parts whose maxima are at least `least`, by some thread.
template <typename T, typename F>
__device__ __forceinline__ void parts_from(Shared &sh, const T *z, const SampleArgs &a, const RowSpace &space, float least, F f) {
  constexpr int E = Span<T>::E;
  int *hits = reinterpret_cast<int *>(sh.weight);        // (room for 2048)
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), whole = a.V / E;
  for (int base = 0; base < a.parts; base += 2 * kSmall) {
    __syncthreads();
    if (threadIdx.x == 0) sh.slot = 0;
    __syncthreads();
    for (int p = base + threadIdx.x; p < min(a.parts, base + 2 * kSmall); p += kThreads)
      if (space.maxima[p] >= least) hits[atomicAdd(&sh.slot, 1)] = p;
    __syncthreads();
    const int n = sh.slot, per = 64 >> a.part_bits;       // parts that a wave looks at together
    for (int h = wave * per; h < n; h += 2 * kWaves * per) {
      Unit<T, E> t[2];
      int u[2];
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        const int at = h + j * kWaves * per + (lane >> a.part_bits);
        u[j] = at < n ? (hits[at] << a.part_bits) + (lane & ((1 << a.part_bits) - 1)) : whole;
        if (u[j] < whole) t[j].load(z + u[j] * E);
      }
#pragma unroll
      for (int j = 0; j < 2; ++j)
        if (u[j] < whole) {
#pragma unroll
          for (int i = 0; i < E; ++i) f(t[j].get(i), (uint32_t)(u[j] * E + i));
        }
    }
  }
  // the tokens behind the last unit
  const int i = whole * E + (int)threadIdx.x;
  if (i < a.V) f(Elem<T>::load(z + i), (uint32_t)i);
  __syncthreads();
}

// Launch 4: a block for each row.
template <typename T>
__global__ __launch_bounds__(kThreads) void sample_draw_kernel(const T *logits, SampleArgs a) {
  __shared__ Shared sh;
  const int64_t n = blockIdx.x;
  const Put put{a, n};
  const RowSpace &space = a.space[n];
  const Asked q(a, n);
  const Plan plan = plan_row(sh, a, space, q);
  const T *z = logits + n * a.pitch;
  if (plan.way == kNothing) {
    if (threadIdx.x == 0) put(-1);
    return;
  }
  if (plan.way == kGreedy) {
    if (threadIdx.x == 0) sh.count = a.V;
    parts_from(sh, z, a, space, plan.best, [&](float v, uint32_t i) {
      if (v == plan.best) atomicMin(&sh.count, (int)i);
    });
    if (threadIdx.x == 0) put(sh.count);
    return;
  }
  const Weights wt(plan.best, q.t, a.shift, sh);
  bool whole = plan.way == kWhole;
  if (plan.way == kFew) {
    // the k-th largest of the parts' maxima is a bound (to the width of a bin)
    const Bins<kFewBins> few(plan.best, plan.best - plan.low);
    const int last = q.k > a.most_k ? -1 : bin_of_kth(sh, q.k, [&](auto add) {
      for (int p = threadIdx.x; p < a.parts; p += kThreads) {
        const float m = space.maxima[p];
        if (m > -INFINITY) add(few.of(m));
      }
    });
    whole = last < 0;
    if (!whole) {
      const float bound = bound_of(few, last);
      if (threadIdx.x == 0) sh.count = 0;
      parts_from(sh, z, a, space, bound, [&](float v, uint32_t i) {
        if (v >= bound) gather(sh, rank_of(v, i));
      });
      const int M = sh.count;
      if (M <= kSmall) {
        draw_small(sh, M, q, wt, a.V, put);
        return;
      }
      whole = true;
    }
  } else if (plan.way == kSums) {
    whole = space.count > kSmall;
  }
  if (whole) {
    const Span<T> row(z, a.V, 0, a.V);
    draw_whole(row, sh, q, wt, plan.least, put, [&](auto W) __attribute__((always_inline)) { locate<4>(row, sh, 0, [&](u64 all) { return q.point(all); }, W, put); });
    return;
  }
  Limit limit{-INFINITY, 0};
  const float zero = wt.zero(q.t);
  float least = zero;
  if (q.minp > 0.0f) least = fmaxf(least, least_logit(wt, q.t, q.minp));
  u64 sum = (int)threadIdx.x < a.chunks ? space.sums[threadIdx.x] : 0;
  if (plan.way == kSums) {
    const int M = space.count;
    if ((int)threadIdx.x < M) sh.list[threadIdx.x] = space.list[threadIdx.x];
    u64 target;
    border_bin(sh, space, q, &target);
    const u64 before = sh.above;
    __syncthreads();
    const Rank border = border_in_list(sh, M, before, target, [&](float v) -> u64 { return v >= zero ? wt.of(wt.near(v)) : 0; });
    limit = Limit{logit_of((uint32_t)(border >> 32)), index_of(border) + 1};
    // the kept tokens of the border's bin belong to their chunks' sums
    clear_bins(sh);
    if ((int)threadIdx.x < M && sh.list[threadIdx.x] >= border) {
      const Rank r = sh.list[threadIdx.x];
      const float v = logit_of((uint32_t)(r >> 32));
      const int unit = (int)(index_of(r) / Span<T>::E);
      if (v >= least) atomicAdd(&sh.bins[min(a.chunks - 1, unit / a.chunk_units)], wt.of(wt.near(v)));
    }
    __syncthreads();
    if ((int)threadIdx.x < a.chunks) sum += sh.bins[threadIdx.x];
  }
  limit.not_below(least);
  u64 all;
  const u64 before = block_before_u64(sum, sh, &all);
  const u64 target = q.point(all);
  if (before <= target && target < before + sum) {
    sh.slot = threadIdx.x;
    sh.result = before;
  }
  __syncthreads();
  const int chunk = sh.slot;
  const u64 from = sh.result;
  __syncthreads();
  locate<8 / Span<T>::E>(chunk_of(logits, a, n, chunk), sh, from, [=](u64) { return target; },
                         [&](float v, uint32_t i) -> u64 { return wt.of(limit.keeps(v, i) ? wt.near(v) : 0.0); }, put);
}

// Chunks that a row is cut in; 1: a block has it whole.  `unit`: tokens of a unit.  Measured in us, whole rows / chunks (rows of each with parameters of its own: top-k, top-p,
// none, min-p, and top-k in half of the rows with top-p and min-p in all; several batches in turn):
//   fp32   1 x 32768   13 34 16 13 15 / 14 26 15 15 16     32 x 32768  15 34 17 16 33 / 15 30 17 17 29      64 x 50257   20 50 25 23 46 / 18 51 27 25 41
//          1 x 65536   18 55 25 18 19 / 14 26 15 15 17     64 x 65536  22 58 28 25 53 / 19 52 26 26 42      1 x 131072   27 100 44 29 29 / 14 30 15 15 17
//          128 x 131072  38 115 56 47 101 / 31 105 52 49 80     256 x 131072  52 140 74 68 121 / 51 153 88 79 121      256 x 262144  86 252 126 109 218 / 82 245 140 125 178
//   bf16   1 x 32768   12 31 14 10 13 / 14 29 18 16 17     1 x 36000   14 39 19 14 15 / 14 29 17 16 17      32 x 44000   17 45 22 19 42 / 16 40 22 20 38
//          64 x 50257  20 55 26 24 50 / 18 52 27 25 41     64 x 65536  19 56 26 23 51 / 18 60 30 27 45      128 x 131072  32 103 47 38 92 / 25 100 47 43 74
//          256 x 131072  35 112 53 46 100 / 32 133 66 56 103     256 x 262144  63 224 104 87 193 / 53 220 112 88 151
// So chunks win where blocks of whole rows leave compute units idle and a block cannot hold the row in its registers, and in large batches with top-k, or whose rows
// ask for different things and keep the launch waiting; with top-p alone, min-p alone or no filter they lose up to a quarter there, which this rule, that knows
// the sizes only, takes into the bargain.
int chunks_of(int64_t N, int64_t V, int unit) {
  if (V < 32768 || V / unit <= kHeldUnits * kThreads || V < (V < 131072 ? 768 : 512) * N || V > (int64_t)kMaxParts * 64 * 4) return 1;   // (a unit has four elements at the least)
  int64_t n = V / 4096;                                  // a unit or two for each thread
  const int64_t most = (2048 + N - 1) / N;               // and about eight blocks for each compute unit
  if (n > most) n = most;
  return n > kMaxChunks ? kMaxChunks : (int)n;
}

int unit_of(const chn_array *logits) { return logits->dtype == CHN_F32 ? Span<float>::E : Span<bf16_raw>::E; }

chn_status check_row_parameter(const chn_array *v, const char *name, int64_t n, int64_t *stride) {
  CHN_TRY(validate(v, name, false));
  if (v->ndim != 1 || v->shape[0] != n) return fail(CHN_ERR_SHAPE, "sample: %s must have shape (%lld,)", name, (long long)n);
  *stride = n > 1 ? v->strides[0] / dtype_size(v->dtype) : 1;
  return CHN_OK;
}

template <typename T>
void launch(const chn_array *logits, SampleArgs &a, hipStream_t st) {
  const T *z = static_cast<const T *>(logits->data);
  const dim3 threads(kThreads);
  if (a.V <= kShort) {
    hipLaunchKernelGGL((sample_short_kernel<T>), grid_of((a.N + 3) / 4), dim3(256), 0, st, z, a);
    return;
  }
  if (a.chunks == 1) {
    hipLaunchKernelGGL((sample_kernel<T>), grid_of(a.N), threads, 0, st, z, a);
    return;
  }
  const int units = a.V / Span<T>::E;
  // The k-th largest of the parts' maxima bounds a top-k, so as many parts as a block that has the whole row has threads: the two ways narrow the same k.
  // (With parts of 64 units a bfloat16 row of 50257 tokens had 99 of them, and a top-k of 100 went through the row in passes: 40 us, so 15.)
  const auto parts = [&](int bits) { return (units + (1 << bits) - 1) >> bits; };
  a.part_bits = 6;
  while (a.part_bits > 2 && parts(a.part_bits) < kLeastParts) --a.part_bits;
  a.parts = parts(a.part_bits);
  // Tokens in no order: P ln(P / (P - k)) of them reach the k-th largest of the maxima of P parts.  Beyond kSmall of them, and a bound is no
  // finer than its bin, gathering is for nothing (1 x 131072 bf16 with a top-k of 1000: 92 us with it, 73).
  a.most_k = (int)(a.parts * (1.0 - exp(-0.75 * kSmall / a.parts)));
  const int blocks = (units + 63) / 64;
  a.chunk_units = (blocks + a.chunks - 1) / a.chunks * 64;
  a.chunks = (blocks * 64 + a.chunk_units - 1) / a.chunk_units;   // (none without a unit)
  const dim3 grid((unsigned)a.chunks, (unsigned)a.N);
#define CHN_MAXIMA(BITS) \
  if (a.part_bits == BITS) hipLaunchKernelGGL((sample_maxima_kernel<T, 1 << BITS>), grid, threads, 0, st, z, a)
  CHN_MAXIMA(2);
  CHN_MAXIMA(3);
  CHN_MAXIMA(4);
  CHN_MAXIMA(5);
  CHN_MAXIMA(6);
#undef CHN_MAXIMA
  hipLaunchKernelGGL((sample_bins_kernel<T>), grid, threads, 0, st, z, a);
  if (a.top_p) hipLaunchKernelGGL((sample_border_kernel<T>), grid, threads, 0, st, z, a);
  hipLaunchKernelGGL((sample_draw_kernel<T>), dim3((unsigned)a.N), threads, 0, st, z, a);
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
  if (!logits || logits->ndim != 2 || logits->shape[0] <= 0 || logits->shape[1] <= 0) return 0;
  return chn::chunks_of(logits->shape[0], logits->shape[1], chn::unit_of(logits)) > 1 ? (size_t)logits->shape[0] * sizeof(chn::RowSpace) : 0;
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
  // the sum of V weights of at most 2^shift is at most 2^63; 46 bits leave nothing to tell the draw from the exact one's
  a.shift = 46;
  while ((V - 1) >> (63 - a.shift) > 0) --a.shift;
  a.out = out->data;
  a.out64 = out->dtype == CHN_I64;
  hipStream_t st = as_stream(stream);
  const size_t need = chn_sample_workspace_bytes(logits);
  a.chunks = need > 0 && ws && ws_bytes >= need && reinterpret_cast<uintptr_t>(ws) % 256 == 0 ? chunks_of(a.N, V, unit_of(logits)) : 1;
  a.space = static_cast<RowSpace *>(ws);
  if (logits->dtype == CHN_F32) launch<float>(logits, a, st);
  else launch<bf16_raw>(logits, a, st);
  return check_launch("sample");
}

}  // extern "C"
