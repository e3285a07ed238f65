// One row's scale and the whole numbers of its elements (quant_q8.hip, gemm_q8.hip).
#pragma once
#include "lanes.h"

namespace lrb {
namespace {

// What a row's elements are.  bf16: the one quotient 127 |x| / max that lies on a half without being formed exactly is that of |x| = max / 2, 63.5 (254 |x| is an
// odd multiple of max only if that has the prime factor 127, where 127 / max is a power of two, or for this x), and every other one is off a half by at
// least 1/510 of a unit in the last place of x against max, 65 times the error of the product below; so 127 / max is rounded up, and 63.5 becomes
// 64, as it should.  fp32, also the rows between a layer's two products: quotients next to a half are settled, so that a row
// has the same integers whichever kernel quantises it.
enum class Rows { BF16, F32 };

template <Rows KIND>
struct Scale {
  uint32_t most;                           // bits of the largest magnitude
  float inv, scale;
  bool none, small;
  __device__ __forceinline__ explicit Scale(uint32_t m) : most(m) {
    const float a = __uint_as_float(m);
    none = m >= 0x7f800000u;
    scale = a / 127.f;
    small = !(scale > 0x1p-126f);
    inv = small ? 0x1p126f : 127.f / a;
    if (KIND == Rows::BF16 && !small && fmaf(inv, a, -127.f) < 0.f) inv = __uint_as_float(__float_as_uint(inv) + 1);
    if (small) scale = 0x1p-126f;
    if (none) scale = __builtin_nanf("");
  }
  // Four elements as bytes.  Adding 1.5 * 2^23 leaves the nearest whole number in the low bits.
  __device__ __forceinline__ uint32_t bytes(const float* x) const {
    constexpr float C = 12582912.f, NEAR = 0.5f - 0x1p-13f;
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; j++) w[j] = __float_as_uint(fmaf(x[j], inv, C));
    if constexpr (KIND == Rows::F32) {
      float off[4];
#pragma unroll
      for (int j = 0; j < 4; j++) off[j] = __builtin_fabsf(fmaf(x[j], inv, C - __uint_as_float(w[j])));
      if (fmaxf(fmaxf(off[0], off[1]), fmaxf(off[2], off[3])) > NEAR && !small) {
#pragma unroll
        for (int j = 0; j < 4; j++)
          if (off[j] > NEAR) w[j] = settled(x[j]);
      }
    }
    const uint32_t lo = __builtin_amdgcn_perm(w[1], w[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(w[3], w[2], 0x04000c0cu);
    return lo | hi;
  }
  // ... of a row without a scale zeros
  __device__ __forceinline__ uint32_t four(const float* x) const { return none ? 0u : bytes(x); }
  // An element next to k + 1/2: the sign of 127 |x| - (k + 1/2) max decides.  Both products have 32 bits at most; as a float and its error each they are
  // subtracted without rounding (the floats are neighbours, the errors have 8 bits and exponents within 8 of each other).
  __device__ __forceinline__ uint32_t settled(float x) const {
#pragma clang fp contract(off)
    const float a = __uint_as_float(most), f = a > 1.f ? 0x1p-8f : 0x1p32f;      // (neither overflow nor numbers below 2^-126)
    const float ax = __builtin_fabsf(x), k = __builtin_floorf(ax * inv), h = k + 0.5f;
    const float u = 127.f * (ax * f), p = h * (a * f);
    const float d = (u - p) + (fmaf(127.f, ax * f, -u) - fmaf(h, a * f, -p));
    const int r = (int)k, q = r + (d > 0.f || (d == 0.f && (r & 1)) ? 1 : 0);
    return (uint32_t)(x < 0.f ? -q : q);
  }
};

}  // namespace
}  // namespace lrb
