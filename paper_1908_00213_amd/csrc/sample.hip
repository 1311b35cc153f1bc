// chn_sample: one token for each row of logits, filtered by temperature, top-k, top-p and min-p, drawn by a given number.
//
// Weights are whole numbers: w(z) = round(2^shift exp((z - max z) / temperature)), the exponential in 64 bits, so that every sum is exact,
// whatever the order in which it is taken; the token is the first whose running sum (in the vocabulary's order, over the tokens that
// the filters keep) exceeds u times the whole sum.
//
// The order by which the filters choose -- descending logits, equals by index -- is that of one 64-bit number for each token (`Rank`), so a filter is a
// border: the tokens from some number on are kept.  A border is found without sorting the row: sums (top-p) or counts (top-k) in 2048 bins of
// equal width in the logit, the bin that the border lies in, and the few tokens of that bin in their exact order.  Where top-k or
// min-p leaves only a few tokens anyway, these are gathered first and the rest of the row is never looked at again: the k-th largest of
// the threads' maxima is a bound that at least k tokens reach.
#include "common.h"
#include "rows.h"

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

typedef unsigned long long u64;
constexpr int kThreads = 1024, kWaves = kThreads / 64;
constexpr int kBins = 2048;          // two for each thread
constexpr int kSmall = 1024;         // tokens that are ordered by comparing each with each

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

// exp((z - best) / t) and the weight it stands for.
struct Weights {
  float best;
  double c, magic;
  __device__ __forceinline__ Weights(float best_, float t, int shift) : best(best_) {
    c = 1.4426950408889634074 / (double)t;
    magic = __longlong_as_double((long long)(1023 + 52 - shift) << 52);   // adding it leaves a whole number of 2^-shift in the low bits
  }
  // 2^-y, y = (best - z) c: 2^f, |f| <= 1/2, by a polynomial through the Chebyshev nodes of degree nine (relative error below 4e-14) and
  // the exponent.  To tell a token from its neighbour by the same u takes an error of about a token's share, which is 1e-6 at the least.
  __device__ __forceinline__ double exponential(float z) const {
    if (z == best) return 1.0;
    const double y = fmin(((double)best - (double)z) * c, 1100.0);        // (infinities and NaN: 1100)
    const double n = rint(y), f = n - y;
    double p = 0x1.b63880a30e9ffp-24;
    p = fma(p, f, 0x1.63d136366db24p-20);
    p = fma(p, f, 0x1.ffcb9515a8016p-17);
    p = fma(p, f, 0x1.4308ac85aa947p-13);
    p = fma(p, f, 0x1.5d87fe86fe88ep-10);
    p = fma(p, f, 0x1.3b2ab7181b755p-7);
    p = fma(p, f, 0x1.c6b08d7047e52p-5);
    p = fma(p, f, 0x1.ebfbdff823cedp-3);
    p = fma(p, f, 0x1.62e42fefa39efp-1);
    return ldexp(fma(p, f, 1.0), -(int)n);
  }
  __device__ __forceinline__ u64 of(double e) const { return (u64)(__double_as_longlong(e + magic) - __double_as_longlong(magic)); }
};

__device__ __forceinline__ u64 wave_sum_u64(u64 v) {
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) v += __shfl_xor(v, o, 64);
  return v;
}
// Sum over the lanes up to this one.
__device__ __forceinline__ u64 wave_upto_u64(u64 v) {
  const int lane = threadIdx.x & 63;
#pragma unroll
  for (int o = 1; o < 64; o <<= 1) {
    const u64 other = __shfl_up(v, o, 64);
    if (lane >= o) v += other;
  }
  return v;
}

struct Shared {
  u64 bins[kBins];
  u64 sorted[kSmall];                // the small set in descending order
  u64 weight[kSmall];
  u64 list[kSmall];                  // the small set as it was gathered
  u64 waves[kWaves];
  float fmax[kWaves], fmin[kWaves];
  u64 result, above;
  int count, slot;
};

// Sum over the threads before this one; *all: over all of them.
__device__ __forceinline__ u64 block_before_u64(u64 v, Shared &sh, u64 *all) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const u64 upto = wave_upto_u64(v);
  __syncthreads();
  if (lane == 63) sh.waves[wave] = upto;
  __syncthreads();
  u64 before = upto - v, sum = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    if (w < wave) before += sh.waves[w];
    sum += sh.waves[w];
  }
  *all = sum;
  return before;
}

// A row as the block walks over it: every wave has a stretch of neighbouring tokens, in units of whole 16-byte pieces; the last wave has those
// behind the last whole unit too.
template <typename T>
struct Row {
  static constexpr int E = unit_elements<T>();
  const T *z;
  int V, whole, first, end;          // units of this wave
  __device__ __forceinline__ Row(const T *z_, int V_) : z(z_), V(V_) {
    whole = V / E;
    const int per = (whole + kWaves - 1) / kWaves, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    first = min(whole, wave * per);
    end = min(whole, first + per);
  }
  // U units are loaded together
  template <int U = 8 / E, typename F>
  __device__ __forceinline__ void stretch(int from, int to, F f) const {
    for (int u = from + (threadIdx.x & 63); u < to; u += 64 * U) {
      Unit<T, E> t[U];
#pragma unroll
      for (int j = 0; j < U; ++j)
        if (u + 64 * j < to) t[j].load(z + (u + 64 * j) * E);
#pragma unroll
      for (int j = 0; j < U; ++j)
        if (u + 64 * j < to) {
#pragma unroll
          for (int i = 0; i < E; ++i) f(t[j].get(i), (uint32_t)((u + 64 * j) * E + i));
        }
    }
  }
  template <typename F>
  __device__ __forceinline__ void behind(F f) const {
    const int i = whole * E + (int)(threadIdx.x & 63);
    if ((threadIdx.x >> 6) == kWaves - 1 && i < V) f(Elem<T>::load(z + i), (uint32_t)i);
  }
  // f(logit, index) for every token of the row, by some thread
  template <int U = 8 / E, typename F>
  __device__ __forceinline__ void each(F f) const {
    stretch<U>(first, end, f);
    behind(f);
  }
};

// Bins of equal width below the largest logit.
struct Bins {
  float best, scale;
  __device__ __forceinline__ int of(float z) const { return z == best ? 0 : (int)fminf((best - z) * scale, (float)(kBins - 1)); }   // (NaN: the last)
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
// Adds w to a bin.  Lanes that all bring the same logit (a row of equals) add once together.
__device__ __forceinline__ void add_to_bin(Shared &sh, int bin, float z, u64 w) {
  const u64 active = __ballot(1);
  const uint32_t head = __builtin_amdgcn_readfirstlane(__float_as_uint(z));
  if (__ballot(__float_as_uint(z) != head) == 0) {
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

// sh.list[0 .. M) into sh.sorted, descending, with every token's place found by comparing it with all the others; P threads share a token.
__device__ __forceinline__ void sort_small(Shared &sh, int M) {
  int size = 1;
  while (size < M) size <<= 1;
  const int parts = min(64, kThreads / size), me = (int)threadIdx.x / parts, part = (int)threadIdx.x % parts;
  const Rank mine = me < M ? sh.list[me] : 0;
  int place = 0;
  if (me < M)
    for (int j = part; j < M; j += parts) place += sh.list[j] > mine;
  for (int o = 1; o < parts; o <<= 1) place += __shfl_xor(place, o, 64);
  if (me < M && part == 0) sh.sorted[place] = mine;
  __syncthreads();
}

// The rank from which on the sum of W over the row's tokens of at least `border` reaches the target, and the sum before it in sh.above.
// W(logit): a token's share.
template <typename R, typename FW>
__device__ Rank find_border(const R &row, Shared &sh, const Bins &bins, Rank border, u64 target, FW W) {
  // (sh.bins holds the sums by bin)
  const int bin = crossing_bin(sh, target);
  const u64 before = sh.above;
  __syncthreads();
  row.each([&](float z, uint32_t i) {
    if (bins.of(z) != bin) return;
    const Rank r = rank_of(z, i);
    if (r != 0 && r >= border) gather(sh, r);
  });
  __syncthreads();
  const int M = sh.count;
  if (M <= kSmall) {
    sort_small(sh, M);
    const Rank r = (int)threadIdx.x < M ? sh.sorted[threadIdx.x] : 0;
    const u64 w = r ? W(logit_of((uint32_t)(r >> 32))) : 0;
    u64 all;
    const u64 upto = before + block_before_u64(w, sh, &all);
    if (r && upto < target && target <= upto + w) {
      sh.result = r;
      sh.above = upto;
    }
    __syncthreads();
    return sh.result;
  }
  // More than that in one bin (many equal logits): the rank's bits, eleven at a time, over the tokens that share the bits found so far.
  Rank found = 0;
  u64 sum = before;
  for (int low = 53; ; low = low > 11 ? low - 11 : 0) {
    const int width = low == 0 ? 9 : 11, high = low + width;
    clear_bins(sh);
    row.each([&](float z, uint32_t i) {
      if (bins.of(z) != bin) return;
      const Rank r = rank_of(z, i);
      if (r == 0 || r < border || (high < 64 && (r >> high) != (found >> high))) return;
      // (descending: the first bin has the largest ranks)
      const int at = (1 << width) - 1 - (int)((r >> low) & ((1u << width) - 1));
      if (low >= 32) add_to_bin(sh, at, z, W(z));        // (bits of the logit alone)
      else atomicAdd(&sh.bins[at], W(z));
    });
    __syncthreads();
    const int at = crossing_bin(sh, target - sum);
    sum += sh.above;
    found |= (u64)((1 << width) - 1 - at) << low;
    __syncthreads();
    if (low == 0) break;
  }
  if (threadIdx.x == 0) sh.above = sum;
  __syncthreads();
  return found;
}

template <typename T>
__global__ __launch_bounds__(kThreads) void sample_kernel(const T *logits, SampleArgs a) {
  __shared__ Shared sh;
  const int64_t n = blockIdx.x;
  const Row<T> row(logits + n * a.pitch, a.V);
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const auto put = [&](int64_t token) {
    if (a.out64) static_cast<int64_t *>(a.out)[n] = token;
    else static_cast<int32_t *>(a.out)[n] = (int32_t)token;
  };
  // the largest logit, the threads' own, and the smallest of those
  float mine = -INFINITY;
  row.template each<4>([&](float z, uint32_t) { mine = fmaxf(mine, z); });
  const float wmax = wave_max(mine), wmin = -wave_max(mine > -INFINITY ? -mine : -INFINITY);
  if (lane == 0) {
    sh.fmax[wave] = wmax;
    sh.fmin[wave] = wmin;
  }
  clear_bins(sh);
  float best = sh.fmax[0], low = sh.fmin[0];
#pragma unroll
  for (int w = 1; w < kWaves; ++w) {
    best = fmaxf(best, sh.fmax[w]);
    low = fminf(low, sh.fmin[w]);
  }
  if (best == -INFINITY) {                               // nothing to choose from
    if (threadIdx.x == 0) put(-1);
    return;
  }
  const float t = a.temperature ? a.temperature[n * a.st] : 1.0f;
  const float u = a.u[n * a.su];
  int64_t k = 0;
  if (a.top_k) k = a.k64 ? static_cast<const int64_t *>(a.top_k)[n * a.sk] : static_cast<const int32_t *>(a.top_k)[n * a.sk];
  const float p = a.top_p ? a.top_p[n * a.sp] : 1.0f;
  const float m0 = a.min_p ? a.min_p[n * a.sm] : 0.0f, minp = m0 > 0.0f ? fminf(m0, 1.0f) : 0.0f;
  const bool greedy = !(t > 0.0f);
  const Weights wt(best, greedy ? 1.0f : t, a.shift);
  if (greedy) {
    if (threadIdx.x == 0) sh.slot = a.V;
    __syncthreads();
    row.each([&](float z, uint32_t i) {
      if (z == best) atomicMin(&sh.slot, (int)i);
    });
    __syncthreads();
    if (threadIdx.x == 0) put(sh.slot);
    return;
  }
  // ---- a row that comes down to a few tokens: all of them from a bound on
  int M = kSmall + 1;
  Bins few{best, 0.0f};
  int last = -1;                                         // tokens in bins up to this one are the few
  if (k > 0 && k <= kThreads) {
    few.scale = (float)kBins / (best - low);             // (infinite or NaN where all maxima are equal: they fall in the first bin)
    if (!(few.scale < INFINITY)) few.scale = 0.0f;
    if (mine > -INFINITY) atomicAdd(&sh.bins[few.of(mine)], 1ull);
    __syncthreads();
    const u64 x = sh.bins[2 * threadIdx.x], y = sh.bins[2 * threadIdx.x + 1];
    u64 all;
    const u64 before = block_before_u64(x + y, sh, &all);
    if (threadIdx.x == 0) sh.slot = -1;
    __syncthreads();
    if (before < (u64)k && (u64)k <= before + x + y) sh.slot = 2 * threadIdx.x + ((u64)k > before + x ? 1 : 0);
    __syncthreads();
    last = sh.slot;                                      // (-1: fewer threads than k hold a token)
  }
  if (last >= 0) {
    row.each([&](float z, uint32_t i) {
      if (z > -INFINITY && few.of(z) <= last) gather(sh, rank_of(z, i));
    });
    __syncthreads();
    M = sh.count;
  } else if (k <= 0 && !(p < 1.0f) && minp > 0.0f) {
    row.each([&](float z, uint32_t i) {
      if (wt.exponential(z) >= (double)minp) gather(sh, rank_of(z, i));
    });
    __syncthreads();
    M = sh.count;
  }
  if (M <= kSmall) {
    sort_small(sh, M);
    const Rank r = (int)threadIdx.x < M && !(k > 0 && (int64_t)threadIdx.x >= k) ? sh.sorted[threadIdx.x] : 0;
    const double e = r ? wt.exponential(logit_of((uint32_t)(r >> 32))) : 0.0;
    const u64 w = wt.of(e);
    bool kept = r != 0;
    if (p < 1.0f) {
      u64 all;
      const u64 before = block_before_u64(w, sh, &all);
      const u64 target = p > 0.0f ? (u64)ceil((double)p * (double)all) : 1;
      kept = kept && (before < target || threadIdx.x == 0);
    }
    kept = kept && e >= (double)minp;
    if (u > 0.0f && u < 1.0f) {
      u64 all;
      block_before_u64(kept ? w : 0, sh, &all);
      const u64 target = (u64)((double)u * (double)all);
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
        for (int j = part; j < M; j += parts)
          if (index_of(sh.list[j]) < index) before += sh.weight[j];
      for (int o = 1; o < parts; o <<= 1) before += __shfl_xor(before, o, 64);
      if (me < M && part == 0 && before <= target && target < before + sh.weight[me]) put(index);
    } else {
      if (threadIdx.x == 0) sh.slot = u >= 1.0f ? -1 : a.V;
      __syncthreads();
      if (kept && e > 0.0) {
        if (u >= 1.0f) atomicMax(&sh.slot, (int)index_of(r));
        else atomicMin(&sh.slot, (int)index_of(r));
      }
      __syncthreads();
      if (threadIdx.x == 0) put(sh.slot);
    }
    return;
  }
  // ---- the whole row
  Rank border = 1;
  if (k > 0) {
    float least = INFINITY;
    int have = 0;
    row.each([&](float z, uint32_t) {
      if (z > -INFINITY) {
        least = fminf(least, z);
        ++have;
      }
    });
    u64 all;
    block_before_u64((u64)have, sh, &all);
    if ((u64)k < all) {
      least = -wave_max(-least);
      if (lane == 0) sh.fmin[wave] = least;
      clear_bins(sh);
#pragma unroll
      for (int w = 0; w < kWaves; ++w) least = fminf(least, sh.fmin[w]);
      Bins bins{best, (float)kBins / (best - least)};
      if (!(bins.scale < INFINITY)) bins.scale = 0.0f;
      row.each([&](float z, uint32_t) {
        if (z > -INFINITY) add_to_bin(sh, bins.of(z), z, 1);
      });
      __syncthreads();
      border = find_border(row, sh, bins, 1, (u64)k, [](float) -> u64 { return 1; });
    }
  }
  if (p < 1.0f) {
    // (from 33 temperatures below the largest logit on, weights are zero)
    Bins bins{best, (float)kBins / (33.0f * t)};
    if (!(bins.scale < INFINITY)) bins.scale = 0.0f;
    clear_bins(sh);
    row.each([&](float z, uint32_t i) {
      if (z > -INFINITY && (border <= 1 || rank_of(z, i) >= border)) add_to_bin(sh, bins.of(z), z, wt.of(wt.exponential(z)));
    });
    __syncthreads();
    u64 all;
    block_before_u64(sh.bins[2 * threadIdx.x] + sh.bins[2 * threadIdx.x + 1], sh, &all);
    u64 target = p > 0.0f ? (u64)ceil((double)p * (double)all) : 1;
    if (target < 1) target = 1;
    __syncthreads();
    border = find_border(row, sh, bins, border, target, [&](float z) -> u64 { return wt.of(wt.exponential(z)); });
  }
  const auto kept = [&](float z, uint32_t i) -> double {
    const Rank r = rank_of(z, i);
    if (r == 0 || r < border) return 0.0;
    const double e = wt.exponential(z);
    return e >= (double)minp ? e : 0.0;
  };
  if (!(u > 0.0f) || u >= 1.0f) {                        // the ends of the range: the first and the last token, however light
    __syncthreads();
    if (threadIdx.x == 0) sh.slot = u >= 1.0f ? -1 : a.V;
    __syncthreads();
    row.each([&](float z, uint32_t i) {
      if (kept(z, i) > 0.0) {
        if (u >= 1.0f) atomicMax(&sh.slot, (int)i);
        else atomicMin(&sh.slot, (int)i);
      }
    });
    __syncthreads();
    if (threadIdx.x == 0) put(sh.slot);
    return;
  }
  // the wave in whose stretch the running sum passes the target, then the sixteenth of that stretch, then the token
  u64 sum = 0;
  row.each([&](float z, uint32_t i) { sum += wt.of(kept(z, i)); });
  sum = wave_sum_u64(sum);
  u64 all;
  u64 before = block_before_u64(lane == 0 ? sum : 0, sh, &all);
  const u64 target = (u64)((double)u * (double)all);     // below `all`: u is at most 1 - 2^-24
  if (lane == 0 && before <= target && target < before + sum) {
    sh.slot = wave;
    sh.result = before;
  }
  __syncthreads();
  const int per = (row.whole + kWaves - 1) / kWaves, s0 = min(row.whole, sh.slot * per), s1 = min(row.whole, s0 + per);
  const bool tail = sh.slot == kWaves - 1;
  const u64 start = sh.result;
  const int sub = (s1 - s0 + kWaves - 1) / kWaves, t0 = min(s1, s0 + wave * sub), t1 = min(s1, t0 + sub);
  sum = 0;
  row.stretch(t0, t1, [&](float z, uint32_t i) { sum += wt.of(kept(z, i)); });
  if (tail) row.behind([&](float z, uint32_t i) { sum += wt.of(kept(z, i)); });
  sum = wave_sum_u64(sum);
  before = start + block_before_u64(lane == 0 ? sum : 0, sh, &all);
  before = __shfl(before, 0, 64);
  if (!(before <= target && target < before + sum)) return;
  // one wave: its units in order, 64 at a time, then the tokens behind the last unit
  constexpr int E = Row<T>::E;
  for (int u0 = t0; u0 < t1; u0 += 64) {
    const int unit = u0 + lane;
    u64 w[E], own = 0;
#pragma unroll
    for (int i = 0; i < E; ++i) {
      w[i] = unit < t1 ? wt.of(kept(Elem<T>::load(row.z + unit * E + i), (uint32_t)(unit * E + i))) : 0;
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
    before += __shfl(upto, 63, 64);
  }
  if (tail && wave == kWaves - 1) {
    const int i = row.whole * E + lane;
    const u64 w = i < a.V ? wt.of(kept(Elem<T>::load(row.z + i), (uint32_t)i)) : 0;
    const u64 at = before + wave_upto_u64(w) - w;
    if (at <= target && target < at + w) put(i);
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
