// chn_gated_scan_fwd / _bwd: a gated linear recurrence over time and its gradient.
//
// A step maps the state affinely, h -> a h + u, and so does any run of steps: its effect is a pair (product of the decays, state from zero), and effects of
// neighbouring runs join into one, (a, u) then (a', u') being (a' a, a' u + u').  A lane has one column (two of bfloat16 arrays) and walks through 16 steps that lie
// in its registers; the eight waves of a block take neighbouring sixteens, a piece of 128 steps, and join their effects in LDS.  Then each wave knows its first
// state and goes through its steps once more, out of registers.  Every element is read once and written once.  Backwards it is the same, from the last step on: the
// gradient C that flows into a step from the next one goes on as a (dy + C); the states are computed again from one in sixteen that the forward pass keeps (1/16 of
// 4 bytes an element; kept for every step they would cost 4).
//
// Pieces of one tile (64 lanes) are joined in two ways, which give a state its value in a fixed order each:
//   - from kTiles tiles on a block walks through its tile's pieces, the state staying in its registers;
//   - otherwise pieces are blocks of their own.  Each makes its effect known in device memory and joins those of the pieces before it in its group of 16 to the state at
//     the group's start, which the last piece of the group before has made known.  A word is its own sign that it is there (a pattern that no value has, written
//     before by a small launch), so nothing has to be ordered but a word's own arrival.  Pieces are drawn by tickets, so a block waits only for blocks that already run, and
//     every wait is bounded: what has not come after kPolls looks counts as NaN.
//
// Bound by memory, and in the second way by how long a block holds its registers (a third of which it waits: 1.4 us for the ticket, 3.4 to 4.6 for its loads, 3 to 4 for the others'
// words, 1.6 for its stores).  2048 x 8 x 4096 bf16 100 us forward, 157 backward (4.0 and 4.3 TB/s), 65536 x 1 x 1024 105 and 144; without the waiting it would be 92 and 78 forward.
// Of groups of 8, 16, 32 and 64 pieces, pieces of 64, 128 and 256 steps and two or three blocks on a compute unit none was faster than these by more than 3 %, pieces of 64 a quarter
// slower; tiles dealt out over the XCDs, with tickets for each: 777 x 5 x 1001 43.5 -> 40.8, 65536 x 1 x 1024 245 -> 284 (a stripe of every row for an XCD, few channels of its L2).  The walk against single pieces, both directions, us: 200 x 128 x 650 fp32 136 / 147, 256 x 64 x 2048 bf16 113 / 119, 512 x 32 x 2048 112 / 122 (512 tiles); with
// 256 tiles 132 / 125 (1024 x 16 x 2048) and 262 / 248 (2048 x 8 x 4096): one block on a compute unit.  Results past the caches: 255 -> 249 for 2048 x 8 x 4096, 262 -> 249 for 65536 x 1 x 1024.
#include "rows.h"

#include <initializer_list>
#include <type_traits>

namespace chn {
namespace {

constexpr int kSteps = CHN_SCAN_STRIDE;        // steps of a wave
constexpr int kWaves = 8;                      // waves of a block, at most
constexpr int kPiece = kSteps * kWaves;        // steps of a block
constexpr int kEach = 2;                       // pieces before its own that a wave joins
constexpr int kGroup = kEach * kWaves;         // pieces of a group
constexpr int kTiles = 512;                    // two blocks for each of 256 compute units
constexpr int kPolls = 1 << 20;                // (a second: what is waited for is under way already)

struct ScanArgs {
  const void *gate, *x, *dy;
  void *y, *dgate, *dx;
  const float *h0, *dh_last;
  float *h_last, *states, *dh0;
  const void *lengths;
  int64_t T, B, D;
  int64_t gt, gb, xt, xb, yt, yb, ht, hb;   // strides in elements: gate, x, y or dy, dgate
  int64_t ut, ub, p0, pl;                   // dx; rows of h0 or dh0, of h_last or dh_last
  int64_t len_stride;
  int len64;
  // the launch
  int chained;                              // whether a block has one piece and hears of the state from the others, or all pieces of its tile
  int64_t subs, pieces, upr, tiles;         // waves' shares of the steps, blocks' shares; units of V columns in a row, blocks next to each other
  unsigned long long *effects;              // (piece, B, D): what a piece does to the state, the product of the decays and the state from zero
  unsigned *starts;                         // (group, B, D): the state before a group of pieces
  unsigned *ticket;
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

template <int V> using Vals = float __attribute__((ext_vector_type(V)));

// V neighbouring values as they lie in memory, at any element address.
template <typename T, int V> struct Few;
template <> struct Few<float, 1> {
  float r;
  __device__ __forceinline__ void load(const float *p) { r = *p; }
  __device__ __forceinline__ float get(int) const { return r; }
  static __device__ __forceinline__ void store(float *p, Vals<1> v) { __builtin_nontemporal_store(v[0], p); }
};
template <> struct Few<bf16_raw, 1> {
  uint32_t r;
  __device__ __forceinline__ void load(const bf16_raw *p) { r = *p; }
  __device__ __forceinline__ float get(int) const { return __uint_as_float(r << 16); }
  static __device__ __forceinline__ void store(bf16_raw *p, Vals<1> v) { *p = f32_to_bf16(v[0]); }
};
typedef uint32_t u32_any __attribute__((aligned(2)));
typedef float f32x2_any __attribute__((ext_vector_type(2), aligned(4)));
template <> struct Few<bf16_raw, 2> {
  uint32_t r;
  __device__ __forceinline__ void load(const bf16_raw *p) { r = *reinterpret_cast<const u32_any *>(p); }
  __device__ __forceinline__ float get(int i) const { return __uint_as_float(i ? r & 0xffff0000u : r << 16); }
  static __device__ __forceinline__ void store(bf16_raw *p, Vals<2> v) {
    __builtin_nontemporal_store((uint32_t)f32_to_bf16(v[0]) | (uint32_t)f32_to_bf16(v[1]) << 16, reinterpret_cast<u32_any *>(p));
  }
};
template <> struct Few<float, 2> {
  f32x2_any r;
  __device__ __forceinline__ void load(const float *p) { r = *reinterpret_cast<const f32x2_any *>(p); }
  __device__ __forceinline__ float get(int i) const { return r[i]; }
  static __device__ __forceinline__ void store(float *p, Vals<2> v) { *reinterpret_cast<f32x2_any *>(p) = f32x2_any{v[0], v[1]}; }
};

// Where a lane works: V columns of one sequence.  The last unit of a row of odd length begins one column early and stores its last column alone.
// A wave's rows are addressed from that of its first lane: a pointer for the wave and 32 bits for a lane, whose reach the host has looked at.
template <int V>
struct Place {
  int b, d, end;                                             // (each below 2^31)
  int b0;                                                    // of the first lane
  bool live, whole;
  __device__ __forceinline__ Place(const ScanArgs &s, int64_t tile) {
    const int64_t u = tile * 64 + (threadIdx.x & 63), row = u / s.upr, j = u - row * s.upr;
    live = row < s.B && j * V < s.D;
    b = (int)min(row, s.B - 1);
    b0 = __builtin_amdgcn_readfirstlane(b);
    whole = j * V + V <= s.D;
    d = (int)(whole ? j * V : s.D - V);
    end = (int)sequence_end(s, b);
  }
  template <typename T>
  __device__ __forceinline__ unsigned offset(int64_t sb) const { return (unsigned)(((b - b0) * sb + d) * (int64_t)sizeof(T)); }
  __device__ __forceinline__ bool owns(int v) const { return live && (whole || v == V - 1); }
  template <typename T>
  __device__ __forceinline__ void store(T *p, Vals<V> v) const {
    if (live) {
      if (whole) Few<T, V>::store(p, v);
      else Elem<T>::store(p + V - 1, v[V - 1]);
    }
  }
};

template <typename T>
__device__ __forceinline__ T *moved(T *p, unsigned bytes) {
  return reinterpret_cast<T *>(reinterpret_cast<char *>(const_cast<std::remove_const_t<T> *>(p)) + (uint64_t)bytes);
}

// (never all bits set, which is the sign of a word that is not there yet: a is finite or kBehind)
__device__ __forceinline__ unsigned long long together(unsigned a, float u) { return (unsigned long long)__float_as_uint(u) << 32 | a; }

// One effect after another.
__device__ __forceinline__ float2 after(float2 e, float2 f) { return make_float2(f.x * e.x, fmaf(f.x, e.y, f.y)); }

// Whether an effect says what it does to every state: a product of decays beyond fp32's range does not, not even to a state of zero.  Effects and states joined to
// such a one are infinite or NaN too, so it is enough to look at the last.
__device__ __forceinline__ bool says(float2 e) { return __builtin_isfinite(e.x + e.y); }

// In the place of a product (a NaN that no other effect is given): the word's other half is the state behind the piece, known once the state before it was.
constexpr unsigned kBehind = 0x7fc00001u;
__device__ __forceinline__ float through(unsigned long long word, float h) {
  const float u = __uint_as_float((unsigned)(word >> 32));
  return (unsigned)word == kBehind ? u : fmaf(__uint_as_float((unsigned)word), h, u);
}

template <int V>
struct Shared {
  float2 mine[2][kWaves][V][64];                             // what each wave does to the state; pieces take turns, so that one barrier is enough
  float2 theirs[kWaves][V][64];                              // what the pieces before this one do, two at a time
  float start[V][64];
  unsigned ticket;
};

// The state (forward: h, backward: the gradient that flows into a step from the next one) that a wave begins with, from what the waves do to it.
// An effect is an affine map: state -> a state + u.  `first`: the state that the walk begins with.  Waves, pieces and groups are joined in one fixed
// order, so results do not depend on which block runs when.  A piece waits for those before it in its group and for the group's start; all
// of them have drawn their tickets before, so their blocks run already and wait for nothing behind them.
// Joined effects hold products of up to 2048 decays, a walk from wave to wave none of more than 16.  Where such a product leaves fp32's range, pieces are gone through one
// after the other here too: one whose own effect says nothing makes known the state behind it as soon as it knows the one before it.  (Asking whether that is so is 1 % of 65536 x 1 x 1024.)
template <int V, bool CHAINED>
__device__ __forceinline__ void begin_with(const ScanArgs &s, Shared<V> &sh, const Place<V> &at, int64_t piece, int waves, Vals<V> a, Vals<V> u, Vals<V> &first,
                                           Vals<V> &state) {
  float2 (*mine)[V][64] = sh.mine[piece & 1];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
#pragma unroll
  for (int v = 0; v < V; ++v) {
    float f = first[v];
    asm volatile("" : "+v"(f));                              // (has been read when the others hear of this piece: its memory may be where the walk's last state goes)
    mine[wave][v][lane] = make_float2(a[v], u[v]);
    state[v] = f;
  }
  __syncthreads();
  if constexpr (CHAINED) {
    const int64_t group = piece / kGroup;
    const int before = (int)(piece - group * kGroup);
    const int64_t row = s.B * s.D, column = (int64_t)at.b * s.D + at.d;
    bool late = false;                                       // whether one of the wave's effects says nothing
    auto effect = [&](int v) {                               // of this piece
      float2 e = mine[0][v][lane];
      for (int w = 1; w < waves; ++w) e = after(e, mine[w][v][lane]);
      return e;
    };
    auto one_by_one = [&](int v, float h) {                  // the state behind the pieces before this one in its group
      const unsigned long long *p = s.effects + group * kGroup * row + column + v;
      for (int k = 0; k < before; ++k) h = through(__hip_atomic_load(p + k * row, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT), h);
      return h;
    };
    auto own_waves = [&](int v, float h) {                   // and then behind this one
      for (int w = 0; w < waves; ++w) h = fmaf(mine[w][v][lane].x, h, mine[w][v][lane].y);
      return h;
    };
    if (wave == 0 && before < kGroup - 1 && piece < s.pieces - 1) {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float2 e = effect(v);
        late |= !says(e);
        if (at.owns(v) && says(e)) __hip_atomic_store(s.effects + piece * row + column + v, together(__float_as_uint(e.x), e.y), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      }
      late = __any(late);
    }
    if (kEach * wave < before) {
      const int n = min(before - kEach * wave, kEach);
      const int64_t p = (group * kGroup + kEach * wave) * row + column;
      unsigned long long e[kEach][V];
      bool missing = true;
      for (int polls = 0; polls < kPolls && missing; ++polls) {
        missing = false;
#pragma unroll
        for (int k = 0; k < kEach; ++k)
#pragma unroll
          for (int v = 0; v < V; ++v) e[k][v] = __hip_atomic_load(s.effects + p + min(k, n - 1) * row + v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
        for (int k = 0; k < kEach; ++k)
#pragma unroll
          for (int v = 0; v < V; ++v) missing |= e[k][v] == ~0ull;
        missing = __any(missing);
      }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        // (one that never came is NaN, all of its bits set)
        float2 all = make_float2(1.0f, 0.0f);
#pragma unroll
        for (int k = 0; k < kEach; ++k)
          if (k < n) all = after(all, make_float2(__uint_as_float((unsigned)e[k][v]), __uint_as_float((unsigned)(e[k][v] >> 32))));
        sh.theirs[wave][v][lane] = all;
      }
    }
    if (before > 0) __syncthreads();
    const bool ends = before == kGroup - 1 && piece < s.pieces - 1;   // the group ends here and another one follows
    if (wave == kWaves - 1 && (group > 0 || ends)) {
      // What the pieces before this one do, and this one too, is joined before the group's start is waited for: from group to group it is one
      // load, one product and one store.
      float2 until[V], past[V];
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float2 e = make_float2(1.0f, 0.0f);
        for (int w = 0; kEach * w < before; ++w) e = after(e, sh.theirs[w][v][lane]);
        until[v] = e;
        if (ends)
          for (int w = 0; w < waves; ++w) e = after(e, mine[w][v][lane]);
        past[v] = e;
      }
      bool mute = false;
#pragma unroll
      for (int v = 0; v < V; ++v) mute |= !says(past[v]);
      mute = __any(mute);
      unsigned e[V];
#pragma unroll
      for (int v = 0; v < V; ++v) e[v] = __float_as_uint(state[v]);
      if (group > 0) {
        const int64_t p = group * row + column;
        bool missing = true;
        for (int polls = 0; polls < kPolls && missing; ++polls) {
          missing = false;
#pragma unroll
          for (int v = 0; v < V; ++v) e[v] = __hip_atomic_load(s.starts + p + v, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
#pragma unroll
          for (int v = 0; v < V; ++v) missing |= e[v] == ~0u;
          missing = __any(missing);
        }
      }
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float start = __uint_as_float(e[v]);
        float next = fmaf(past[v].x, start, past[v].y), here = fmaf(until[v].x, start, until[v].y);
        if (mute) {
          const float there = one_by_one(v, start), behind = own_waves(v, there);
          if (!says(past[v])) {                              // (every column by itself, whatever its neighbours hold)
            here = there;
            next = behind;
          }
        }
        const unsigned bits = __float_as_uint(next);
        if (ends && at.owns(v))
          __hip_atomic_store(s.starts + (group + 1) * row + column + v, bits == ~0u ? 0x7fc00000u : bits, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
        sh.start[v][lane] = here;
      }
    }
    if (group > 0) {
      __syncthreads();
#pragma unroll
      for (int v = 0; v < V; ++v) state[v] = sh.start[v][lane];
    } else {
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float h = state[v];
        for (int w = 0; kEach * w < before; ++w) h = fmaf(sh.theirs[w][v][lane].x, h, sh.theirs[w][v][lane].y);
        const bool mute = !__builtin_isfinite(h);
        if (__any(mute)) {
          const float there = one_by_one(v, state[v]);
          h = mute ? there : h;
        }
        state[v] = h;
      }
    }
    if (late) {
#pragma unroll
      for (int v = 0; v < V; ++v)
        if (at.owns(v) && !says(effect(v)))
          __hip_atomic_store(s.effects + piece * row + column + v, together(kBehind, own_waves(v, state[v])), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    }
  }
#pragma unroll
  for (int v = 0; v < V; ++v) {
    float h = state[v];
    for (int w = 0; w < wave; ++w) h = fmaf(mine[w][v][lane].x, h, mine[w][v][lane].y);
    state[v] = h;
    if constexpr (!CHAINED) {                                // (what the next piece begins with)
      for (int w = wave; w < waves; ++w) h = fmaf(mine[w][v][lane].x, h, mine[w][v][lane].y);
      first[v] = h;
    }
  }
}

// The block's tile and pieces: one piece, those of all tiles being drawn in the order of the walk, or all of the tile's, one after the other.  False for the
// blocks that the grid's last line has beyond the jobs.
template <int V, bool CHAINED>
__device__ __forceinline__ bool next_job(const ScanArgs &s, Shared<V> &sh, int64_t &piece, int64_t &end, int64_t &tile) {
  if constexpr (CHAINED) {
    if (threadIdx.x == 0) sh.ticket = __hip_atomic_fetch_add(s.ticket, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __syncthreads();
    const int64_t job = __builtin_amdgcn_readfirstlane((int)sh.ticket);   // (fewer than 2^31 jobs and blocks)
    piece = job / s.tiles;
    tile = job - piece * s.tiles;
    end = piece + 1;
    return piece < s.pieces;
  } else {
    piece = 0;
    tile = block_number();
    end = s.pieces;
    return tile < s.tiles;
  }
}

template <typename TI, typename TO, int V, bool SIGMOID, bool CHAINED>
__global__ __launch_bounds__(64 * kWaves, 4) void scan_fwd_kernel(ScanArgs s) {
  __shared__ Shared<V> sh;
  int64_t piece, end, tile;
  if (!next_job<V, CHAINED>(s, sh, piece, end, tile)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const Place<V> at(s, tile);
  const TI *g = static_cast<const TI *>(s.gate) + at.b0 * s.gb, *x = static_cast<const TI *>(s.x) + at.b0 * s.xb;
  const unsigned go = at.template offset<TI>(s.gb), xo = at.template offset<TI>(s.xb);
  const unsigned yo = at.template offset<TO>(s.yb);
  Vals<V> first;
#pragma unroll
  for (int v = 0; v < V; ++v) first[v] = s.h0 ? s.h0[at.b * s.p0 + at.d + v] : 0.0f;
  do {                                                       // (pieces of the tile, one where they are chained)
    const int64_t sub = piece * kWaves + wave, t0 = sub * kSteps;
    Few<TI, V> gr[kSteps], xr[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int64_t t = min(t0 + i, s.T - 1);
      gr[i].load(moved(g + t * s.gt, go));
      xr[i].load(moved(x + t * s.xt, xo));
    }
    __builtin_amdgcn_sched_barrier(0);                         // (all loads first)
    const int n = (int)min(max(at.end - t0, (int64_t)0), (int64_t)kSteps), nt = (int)min(s.T - t0, (int64_t)kSteps);
    Vals<V> h, A, U, a[kSteps], u[kSteps];
#pragma unroll
    for (int v = 0; v < V; ++v) {
      A[v] = 1.0f;
      U[v] = 0.0f;
    }
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const bool on = i < n;
      if (i % 2 == 0) __builtin_amdgcn_sched_barrier(0);       // (two steps at a time: more of them at once take registers that two blocks do not have)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float av = gr[i].get(v), uv = xr[i].get(v);
        if constexpr (SIGMOID) {
          float rest;
          gate_parts(av, av, rest);
          uv *= rest;
        }
        a[i][v] = on ? av : 1.0f;
        u[i][v] = on ? uv : 0.0f;
        A[v] *= a[i][v];
        U[v] = fmaf(a[i][v], U[v], u[i][v]);
      }
    }
    begin_with<V, CHAINED>(s, sh, at, piece, waves, A, U, first, h);
    if (t0 >= s.T) return;                                   // (behind the last step, so in the last piece)
    if (s.states) at.store(s.states + (sub * s.B + at.b) * s.D + at.d, h);
    TO *y = static_cast<TO *>(s.y) + at.b0 * s.yb + t0 * s.yt;
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      if (i >= nt) continue;
      Vals<V> out;
#pragma unroll
      for (int v = 0; v < V; ++v) {
        h[v] = fmaf(a[i][v], h[v], u[i][v]);
        out[v] = i < n ? h[v] : 0.0f;
      }
      at.store(moved(y + i * s.yt, yo), out);
    }
    if (s.h_last && t0 + kSteps >= s.T) at.store(s.h_last + at.b * s.pl + at.d, h);
  } while (!CHAINED && ++piece < end);
}

// Backwards: the wave whose steps are the last ones begins.  The state before each step is computed again from the one that the forward pass kept.  Of a
// step stay two numbers and dy: the smaller of a and 1 - a (with its sign saying which one it is: the other one is 1 minus it, to half a step),
// and what dgate has G multiplied with.
template <typename TI, typename TO, int V, bool SIGMOID, bool CHAINED>
__global__ __launch_bounds__(64 * kWaves, 4) void scan_bwd_kernel(ScanArgs s) {
  __shared__ Shared<V> sh;
  int64_t piece, end, tile;
  if (!next_job<V, CHAINED>(s, sh, piece, end, tile)) return;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6;
  const Place<V> at(s, tile);
  const TI *g = static_cast<const TI *>(s.gate) + at.b0 * s.gb, *x = static_cast<const TI *>(s.x) + at.b0 * s.xb;
  const TO *dy = static_cast<const TO *>(s.dy) + at.b0 * s.yb;
  const unsigned go = at.template offset<TI>(s.gb), xo = at.template offset<TI>(s.xb), yo = at.template offset<TO>(s.yb);
  Vals<V> first;
#pragma unroll
  for (int v = 0; v < V; ++v) first[v] = s.dh_last ? s.dh_last[at.b * s.pl + at.d + v] : 0.0f;
  do {                                                       // (pieces of the tile, one where they are chained)
    const int64_t walk = piece * kWaves + wave, sub = s.subs - 1 - walk, t0 = max(sub, (int64_t)0) * kSteps;
    const bool any = sub >= 0;                                 // (the last block's last waves may have no steps)
    Few<TI, V> gr[kSteps], xr[kSteps];
    Few<TO, V> yr[kSteps];
    Vals<V> h, A, U, part[kSteps], coef[kSteps];
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const int64_t t = min(t0 + i, s.T - 1);
      gr[i].load(moved(g + t * s.gt, go));
      xr[i].load(moved(x + t * s.xt, xo));
      yr[i].load(moved(dy + t * s.yt, yo));
    }
    const int n = any ? (int)min(max(at.end - t0, (int64_t)0), (int64_t)kSteps) : 0, nt = (int)min(s.T - t0, (int64_t)kSteps);
#pragma unroll
    for (int v = 0; v < V; ++v) {
      h[v] = s.states[((t0 / kSteps) * s.B + at.b) * s.D + at.d + v];
    }
    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
    for (int i = 0; i < kSteps; ++i) {
      const bool on = i < n;
      if (i % 2 == 0) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float xv = xr[i].get(v);
        float a = gr[i].get(v);
        if constexpr (SIGMOID) {
          float rest;
          const bool upper = a >= 0.0f;
          gate_parts(a, a, rest);
          float c = on ? (h[v] - xv) * (a * rest) : 0.0f;
          asm volatile("" : "+v"(c));                          // (worked out here: where it is used it would keep four numbers alive until then)
          coef[i][v] = c;
          part[i][v] = on ? (upper ? -rest : a) : -0.0f;
          h[v] = fmaf(a, h[v], rest * xv);
        } else {
          float c = on ? h[v] : 0.0f, q = on ? a : 1.0f;
          asm volatile("" : "+v"(c), "+v"(q));
          coef[i][v] = c;
          part[i][v] = q;
          h[v] = fmaf(a, h[v], xv);
        }
      }
    }
    auto decay = [](float q) {
      return !SIGMOID ? q : __float_as_int(q) < 0 ? 1.0f + q : q;
    };
#pragma unroll
    for (int v = 0; v < V; ++v) {
      A[v] = 1.0f;
      U[v] = 0.0f;
    }
#pragma unroll
    for (int i = kSteps - 1; i >= 0; --i) {
      if (i % 2) __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int v = 0; v < V; ++v) {
        const float a = decay(part[i][v]), d = i < n ? yr[i].get(v) : 0.0f;
        A[v] *= a;
        U[v] = a * (U[v] + d);
      }
    }
    __builtin_amdgcn_sched_barrier(0);
    Vals<V> G;
    begin_with<V, CHAINED>(s, sh, at, piece, waves, A, U, first, G);
    if (!any) return;                                        // (before the first step, so in the last piece)
    TI *dg = static_cast<TI *>(s.dgate) + at.b0 * s.hb + t0 * s.ht, *dx = static_cast<TI *>(s.dx) + at.b0 * s.ub + t0 * s.ut;
    const unsigned dgo = at.template offset<TI>(s.hb), dxo = at.template offset<TI>(s.ub);
#pragma unroll
    for (int i = kSteps - 1; i >= 0; --i) {
      if (i >= nt) continue;
      const bool on = i < n;
      Vals<V> vg, vx;
      if constexpr (sizeof(TO) == 2) asm volatile("" : "+v"(yr[i].r));   // (taken apart again, not kept apart)
#pragma unroll
      for (int v = 0; v < V; ++v) {
        float q = part[i][v];
        asm volatile("" : "+v"(q));                            // (what is worked out from it is neither kept from above nor begun early, in registers that are not there)
        const float a = decay(q);
        if (on) G[v] += yr[i].get(v);
        vg[v] = on ? coef[i][v] * G[v] : 0.0f;
        const float rest = !SIGMOID ? 1.0f : __float_as_int(q) < 0 ? -q : 1.0f - q;
        vx[v] = on ? rest * G[v] : 0.0f;
        G[v] *= a;
      }
      at.store(moved(dg + i * s.ht, dgo), vg);
      at.store(moved(dx + i * s.ut, dxo), vx);
    }
    if (s.dh0 && sub == 0) at.store(s.dh0 + at.b * s.p0 + at.d, G);
  } while (!CHAINED && ++piece < end);
}

// Nothing is there yet, no ticket drawn.
__global__ __launch_bounds__(256) void scan_clear_kernel(chn_u32x4 *words, int64_t n, unsigned *ticket) {
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n; i += (int64_t)gridDim.x * 256) words[i] = chn_u32x4{~0u, ~0u, ~0u, ~0u};
  if (blockIdx.x == 0 && threadIdx.x == 0) *ticket = 0;
}

// Without steps the state stays.
__global__ __launch_bounds__(256) void scan_keep_kernel(const float *from, int64_t pf, float *to, int64_t pt, int64_t B, int64_t D) {
  const int64_t c = block_number() * 256 + threadIdx.x;
  if (c >= B * D) return;
  const int64_t b = c / D, d = c - b * D;
  to[b * pt + d] = from ? from[b * pf + d] : 0.0f;
}

// Columns of a lane: what fills four bytes.  (Backward, fp32 gradients of bfloat16 arrays would take more registers than two blocks have.)
int columns(int dtype, int dy, int64_t D) { return dtype == CHN_BF16 && dy == CHN_BF16 && D > 1 ? 2 : 1; }

// `apart`: every row of units begins with a wave of its own, so that a wave's lanes lie in one sequence.
struct Sizes {
  int64_t subs, pieces, upr, tiles, jobs;
  size_t effects, starts, bytes;
  Sizes(int64_t T, int64_t B, int64_t D, int V, bool apart) {
    subs = (T + kSteps - 1) / kSteps;
    pieces = (subs + kWaves - 1) / kWaves;
    upr = (D + V - 1) / V;
    if (apart) upr = (upr + 63) / 64 * 64;
    tiles = (B * upr + 63) / 64;
    jobs = pieces * tiles;
    effects = ((size_t)pieces * B * D * 8 + 15) / 16 * 16;
    starts = ((size_t)((pieces + kGroup - 1) / kGroup) * B * D * 4 + 15) / 16 * 16;
    bytes = pieces > 1 ? 256 + effects + starts : 0;
  }
};

// Whether the rows of a wave's lanes lie further apart than 32 bits reach.
bool far_apart(int64_t B, int64_t D, int V, std::initializer_list<int64_t> strides) {
  const int64_t upr = (D + V - 1) / V, rows = (63 + upr - 1) / upr < B - 1 ? (63 + upr - 1) / upr : B - 1;
  for (int64_t sb : strides)
    if (rows > 0 && sb > ((1ll << 30) - D) / rows) return true;      // elements of four bytes at most
  return false;
}

// The launch that both directions share: clears the workspace where pieces wait for each other.
chn_status lay_out(const Sizes &z, void *ws, hipStream_t st, ScanArgs *s, dim3 *grid, dim3 *block) {
  s->subs = z.subs; s->pieces = z.pieces; s->upr = z.upr; s->tiles = z.tiles;
  s->chained = z.pieces > 1 && z.tiles < kTiles;
  *grid = grid_of(s->chained ? z.jobs : z.tiles);
  *block = dim3(64 * (unsigned)(z.subs < kWaves ? z.subs : kWaves));
  if (s->chained) {
    char *p = static_cast<char *>(ws);
    s->ticket = reinterpret_cast<unsigned *>(p);
    s->effects = reinterpret_cast<unsigned long long *>(p + 256);
    s->starts = reinterpret_cast<unsigned *>(p + 256 + z.effects);
    const int64_t n = (int64_t)(z.effects + z.starts) / 16;
    const int64_t blocks = (n + 1023) / 1024;
    hipLaunchKernelGGL(scan_clear_kernel, dim3((unsigned)(blocks < 2048 ? blocks : 2048)), dim3(256), 0, st, reinterpret_cast<chn_u32x4 *>(p + 256), n, s->ticket);
    return check_launch("gated_scan");
  }
  return CHN_OK;
}

chn_status keep(const float *from, int64_t pf, float *to, int64_t pt, int64_t B, int64_t D, hipStream_t st) {
  if (!to) return CHN_OK;
  hipLaunchKernelGGL(scan_keep_kernel, grid_of((B * D + 255) / 256), dim3(256), 0, st, from, pf, to, pt, B, D);
  return check_launch("gated_scan");
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
  if (s->T > 0x7fffffff || s->B > 0x7fffffff || s->D >= (1 << 30) || s->B * s->D > (1ll << 40))
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

size_t chn_gated_scan_workspace_bytes(const chn_array *gate) {
  using namespace chn;
  if (!gate || gate->ndim != 3 || !is_float(gate->dtype)) return 0;
  for (int k = 0; k < 3; ++k)
    if (gate->shape[k] <= 0 || gate->shape[k] > 0x7fffffff) return 0;
  const Sizes z(gate->shape[0], gate->shape[1], gate->shape[2], columns(gate->dtype, CHN_BF16, gate->shape[2]), false);
  return z.tiles < kTiles ? z.bytes : 0;                     // (fewer columns for a lane, or rows apart, make more tiles)
}

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
  hipStream_t st = as_stream(stream);
  if (s.T == 0) return keep(s.h0, s.p0, s.h_last, s.pl, s.B, s.D, st);
  const int V = columns(gate->dtype, CHN_BF16, s.D);
  const Sizes z(s.T, s.B, s.D, V, far_apart(s.B, s.D, V, {s.gb, s.xb, s.yb}));
  if (z.jobs > 0x7fffffffll) return fail(CHN_ERR_SHAPE, "gated_scan: %lld pieces of work", (long long)z.jobs);
  dim3 grid, block;
  CHN_TRY(lay_out(z, ws, st, &s, &grid, &block));
#define CHN_GO(TI, TO, V_)                                                                                                      \
  do {                                                                                                                          \
    if (kind == CHN_SCAN_SIGMOID && s.chained) hipLaunchKernelGGL((scan_fwd_kernel<TI, TO, V_, true, true>), grid, block, 0, st, s);   \
    else if (kind == CHN_SCAN_SIGMOID) hipLaunchKernelGGL((scan_fwd_kernel<TI, TO, V_, true, false>), grid, block, 0, st, s);          \
    else if (s.chained) hipLaunchKernelGGL((scan_fwd_kernel<TI, TO, V_, false, true>), grid, block, 0, st, s);                         \
    else hipLaunchKernelGGL((scan_fwd_kernel<TI, TO, V_, false, false>), grid, block, 0, st, s);                                       \
  } while (0)
  if (gate->dtype == CHN_F32) { if (y->dtype == CHN_F32) CHN_GO(float, float, 1); else CHN_GO(float, bf16_raw, 1); }
  else if (V == 2) { if (y->dtype == CHN_F32) CHN_GO(bf16_raw, float, 2); else CHN_GO(bf16_raw, bf16_raw, 2); }
  else { if (y->dtype == CHN_F32) CHN_GO(bf16_raw, float, 1); else CHN_GO(bf16_raw, bf16_raw, 1); }
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
  hipStream_t st = as_stream(stream);
  if (s.T == 0) return keep(s.dh_last, s.pl, s.dh0, s.p0, s.B, s.D, st);
  const int V = columns(gate->dtype, dy->dtype, s.D);
  const Sizes z(s.T, s.B, s.D, V, far_apart(s.B, s.D, V, {s.gb, s.xb, s.yb, s.hb, s.ub}));
  if (z.jobs > 0x7fffffffll) return fail(CHN_ERR_SHAPE, "gated_scan: %lld pieces of work", (long long)z.jobs);
  dim3 grid, block;
  CHN_TRY(lay_out(z, ws, st, &s, &grid, &block));
#define CHN_GO(TI, TO, V_)                                                                                                      \
  do {                                                                                                                          \
    if (kind == CHN_SCAN_SIGMOID && s.chained) hipLaunchKernelGGL((scan_bwd_kernel<TI, TO, V_, true, true>), grid, block, 0, st, s);   \
    else if (kind == CHN_SCAN_SIGMOID) hipLaunchKernelGGL((scan_bwd_kernel<TI, TO, V_, true, false>), grid, block, 0, st, s);          \
    else if (s.chained) hipLaunchKernelGGL((scan_bwd_kernel<TI, TO, V_, false, true>), grid, block, 0, st, s);                         \
    else hipLaunchKernelGGL((scan_bwd_kernel<TI, TO, V_, false, false>), grid, block, 0, st, s);                                       \
  } while (0)
  if (gate->dtype == CHN_F32) { if (dy->dtype == CHN_F32) CHN_GO(float, float, 1); else CHN_GO(float, bf16_raw, 1); }
  else if (V == 2) CHN_GO(bf16_raw, bf16_raw, 2);
  else { if (dy->dtype == CHN_F32) CHN_GO(bf16_raw, float, 1); else CHN_GO(bf16_raw, bf16_raw, 1); }
#undef CHN_GO
  return check_launch("gated_scan_bwd");
}

}  // extern "C"
