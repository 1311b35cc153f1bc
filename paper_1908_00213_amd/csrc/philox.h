// The mask of a dropout call, from a counter instead of a state: Philox-4x32 of Salmon, Moraes, Dror, Shaw, "Parallel random
// numbers: as easy as 1, 2, 3" (SC'11), with seven rounds, the least that the paper finds to pass all of its statistical tests.
// Element (row, col) of an array takes word col % 4 of the block with counter (col / 4, row, offset, site) and the seed as key, so
// any kernel that holds any part of any row draws the same mask, forward or backward, and none is ever stored.
// Seven rounds and not the ten that the paper takes for a margin: a round costs two 32 x 32 -> 64 bit products, which run at a
// quarter of the rate.
#pragma once

#include "common.h"

namespace chn {

// A dropout as the kernels see it.  keep iff word >= threshold; a kept value is multiplied by scale.
struct DropArgs {
  const int64_t *rng;    // [0] seed, [1] offset (its low 32 bits count); device memory, NULL: nothing is dropped
  uint32_t site;
  uint32_t threshold;
  float scale;
};

#if defined(__HIPCC__)
struct Philox4 {
  uint32_t w[4];
};

// a ^ b ^ c in one instruction (the table of the three bits' exclusive or)
__device__ __forceinline__ uint32_t xor3(uint32_t a, uint32_t b, uint32_t c) { return __builtin_amdgcn_bitop3_b32(a, b, c, 0x96); }

__device__ __forceinline__ Philox4 philox7(uint32_t c0, uint32_t c1, uint32_t c2, uint32_t c3, uint32_t k0, uint32_t k1) {
#pragma unroll
  for (int r = 0; r < 7; ++r) {
    const uint64_t p0 = (uint64_t)0xD2511F53u * c0, p1 = (uint64_t)0xCD9E8D57u * c2;
    c0 = xor3((uint32_t)(p1 >> 32), c1, k0);
    c2 = xor3((uint32_t)(p0 >> 32), c3, k1);
    c1 = (uint32_t)p1;
    c3 = (uint32_t)p0;
    k0 += 0x9E3779B9u;
    k1 += 0xBB67AE85u;
  }
  return Philox4{{c0, c1, c2, c3}};
}

// What a kernel reads from the generator once, uniform over the grid.
struct DropState {
  uint32_t k0, k1, offset, site, threshold;
  float scale;
  __device__ __forceinline__ explicit DropState(const DropArgs &a) {
    const uint64_t seed = a.rng ? (uint64_t)a.rng[0] : 0;
    k0 = (uint32_t)seed;
    k1 = (uint32_t)(seed >> 32);
    offset = a.rng ? (uint32_t)a.rng[1] : 0;
    site = a.site;
    threshold = a.threshold;
    scale = a.scale;
  }
  // the words of columns 4 * block .. 4 * block + 3 of a row
  __device__ __forceinline__ Philox4 words(uint32_t block, uint32_t row) const { return philox7(block, row, offset, site, k0, k1); }
  // A dropped value is 0 whatever it was (an infinity or NaN too).
  __device__ __forceinline__ float apply(float x, uint32_t word) const { return word >= threshold ? x * scale : 0.0f; }
};

// residual + dropped value, each step rounded by itself: the sum of a residual stream has the same bits wherever it is formed
__device__ __forceinline__ float add_rounded(float a, float b) {
#pragma clang fp contract(off)
  return a + b;
}
#endif

inline chn_status check_drop(const chn_array *rng, double ratio, int64_t site, int64_t rows, int64_t cols, const char *what, DropArgs *a) {
  *a = DropArgs{nullptr, 0, 0, 1.0f};
  if (!(ratio >= 0.0 && ratio < 1.0)) return fail(CHN_ERR_OP, "%s: ratio %g outside [0, 1)", what, ratio);
  if (site < 0 || site > 0xffffffffLL) return fail(CHN_ERR_OP, "%s: site %lld outside 0 .. 2^32 - 1", what, (long long)site);
  if (ratio == 0.0) return CHN_OK;
  CHN_TRY(validate(rng, "rng", false));
  if (rng->dtype != CHN_I64) return fail(CHN_ERR_DTYPE, "%s: rng must be I64", what);
  if (rng->ndim != 1 || rng->shape[0] != 2) return fail(CHN_ERR_SHAPE, "%s: rng must have shape (2,): seed and offset", what);
  if (!is_contiguous(rng)) return fail(CHN_ERR_STRIDE, "%s: rng must be contiguous", what);
  if (rows > 0xffffffffLL || cols > (1LL << 34))
    return fail(CHN_ERR_SHAPE, "%s: %lld rows of %lld: the generator numbers up to 2^32 rows of 2^34", what, (long long)rows, (long long)cols);
  const double t = ratio * 4294967296.0 + 0.5;
  a->rng = static_cast<const int64_t *>(rng->data);
  a->site = (uint32_t)site;
  a->threshold = t >= 4294967295.0 ? 0xffffffffu : (uint32_t)t;
  a->scale = (float)(1.0 / (1.0 - ratio));
  return CHN_OK;
}

}  // namespace chn
