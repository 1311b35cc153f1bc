// Rows held in registers by groups of lanes: what the row kernels share.
//
// A row of C elements is cut in units of E neighbouring elements (whole 16-byte pieces of every type that takes part); lane g of the
// G that own the row holds units g, g + G, ..., K of them at most, and one of the C % E elements behind the last whole unit if there are
// any.  Every access is a whole 16-byte piece at whatever element address the row has (load16_any), save for those last few.
#pragma once

#include "common.h"

namespace chn {
#if defined(__HIPCC__)

// A grid of n blocks of up to 1024 threads each: a launch takes fewer than 2^32 threads along a dimension, so rows of blocks beyond 2^20.
inline dim3 grid_of(int64_t n) {
  const int64_t x = n < (1 << 20) ? n : (1 << 20);
  return dim3((unsigned)x, (unsigned)((n + x - 1) / x));
}
__device__ __forceinline__ int64_t block_number() { return (int64_t)blockIdx.y * gridDim.x + blockIdx.x; }

// elements of a unit: as many as the narrowest type has in 16 bytes
template <typename... T>
constexpr int unit_elements() {
  int e = 4;
  ((e = sizeof(T) == 2 ? 8 : e), ...);
  return e;
}

// A unit as it lies in memory.
template <typename T, int E>
struct Unit {
  Vec16<T> q[E / Vec16<T>::N];
  __device__ __forceinline__ void load(const T *p) {
#pragma unroll
    for (int i = 0; i < E / Vec16<T>::N; ++i) q[i] = load16_any(p + i * Vec16<T>::N);
  }
  __device__ __forceinline__ void store_nt(T *p) const {
#pragma unroll
    for (int i = 0; i < E / Vec16<T>::N; ++i) store16_any_nt(p + i * Vec16<T>::N, q[i]);
  }
  __device__ __forceinline__ void store(T *p) const {
#pragma unroll
    for (int i = 0; i < E / Vec16<T>::N; ++i) store16_any(p + i * Vec16<T>::N, q[i]);
  }
  __device__ __forceinline__ float get(int i) const { return q[i / Vec16<T>::N].get(i % Vec16<T>::N); }
  __device__ __forceinline__ void set(int i, float v) { q[i / Vec16<T>::N].set(i % Vec16<T>::N, v); }
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < E; ++i) set(i, 0.0f);
  }
};

// The value an fp32 number has once it is stored as T.
template <typename T>
__device__ __forceinline__ float as_stored(float v) {
  if constexpr (sizeof(T) == 2) return bf16_to_f32(f32_to_bf16(v));
  else return v;
}

// v + the value of another lane: lanes exchange inside their registers, without a trip through LDS
template <int CTRL>
__device__ __forceinline__ float dpp_add(float v) {
  return v + __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true));
}

// Sum over G = 4, 8, 16 (a row of the wave) or 32 neighbouring lanes, in all of them.
template <int G>
__device__ __forceinline__ float sum_lanes(float v) {
  v = dpp_add<0xB1>(v);                          // quad_perm 1 0 3 2
  v = dpp_add<0x4E>(v);                          // quad_perm 2 3 0 1
  if constexpr (G >= 8) v = dpp_add<0x141>(v);   // row_half_mirror
  if constexpr (G >= 16) v = dpp_add<0x140>(v);  // row_mirror
  if constexpr (G >= 32) v += __shfl_xor(v, 16, 64);
  return v;
}
__device__ __forceinline__ float sum16(float v) { return sum_lanes<16>(v); }

// Sum over the wave, uniform: the four rows' sums added in their order.
__device__ __forceinline__ float sum64(float v) {
  v = sum16(v);
  const float a = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 0)), b = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 16));
  const float c = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 32)), d = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 48));
  return (a + b) + (c + d);
}

template <int CTRL>
__device__ __forceinline__ float dpp_max(float v) {
  return fmaxf(v, __int_as_float(__builtin_amdgcn_update_dpp(0, __float_as_int(v), CTRL, 0xf, 0xf, true)));
}
__device__ __forceinline__ float max16(float v) { return dpp_max<0x140>(dpp_max<0x141>(dpp_max<0x4E>(dpp_max<0xB1>(v)))); }   // of a row of lanes
// The largest over the wave, uniform.
__device__ __forceinline__ float max64(float v) {
  v = max16(v);
  const float a = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 0)), b = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 16));
  const float c = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 32)), d = __int_as_float(__builtin_amdgcn_readlane(__float_as_int(v), 48));
  return fmaxf(fmaxf(a, b), fmaxf(c, d));
}

// Sums of two values over the G lanes of a row, in all of them.  smem: the group's 2 x G / 64 pairs for G > 64; `turn` alternates from call to
// call, so that one barrier is enough: what is overwritten was read before the barrier of the call in between.
template <int G>
__device__ __forceinline__ float2 group_sum(float2 v, float2 *smem, int turn) {
  if constexpr (G < 64) {
    return make_float2(sum_lanes<G>(v.x), sum_lanes<G>(v.y));
  } else {
    v = make_float2(sum64(v.x), sum64(v.y));
    if constexpr (G > 64) {
      constexpr int W = G / 64;
      float2 *p = smem + turn * W;
      if ((threadIdx.x & 63) == 0) p[threadIdx.x % G / 64] = v;
      __syncthreads();
      if constexpr (W == 16) {                           // a read by each lane, and a sum inside the registers
        const float2 s = p[threadIdx.x & 15];
        return make_float2(sum16(s.x), sum16(s.y));
      }
      float2 s = p[0];
#pragma unroll
      for (int w = 1; w < W; ++w) {
        s.x += p[w].x;
        s.y += p[w].y;
      }
      return s;
    }
    return v;
  }
}

#endif
}  // namespace chn
