// One row's scale and the whole numbers of its elements (quant_q8.hip, gemm_q8.hip).
#pragma once
#include "lanes.h"

namespace lrb {
namespace {

// What a row's elements are.  Both round 127 x / max to the nearest whole number, ties to even, without forming the quotient.
// bf16: the one quotient 127 |x| / max that lies on a half without being formed exactly is that of |x| = max / 2, 63.5 (254 |x| is an
// odd multiple of max only if that has the prime factor 127, where 127 / max is a power of two, or for this x), and every other one is off a half by at
// least 1/510 of a unit in the last place of x against max, 65 times the error of the product below; so 127 / max is rounded up, and 63.5 becomes
// 64, as it should.  fp32, also the rows between a layer's two products, so that a row has the same integers whichever kernel quantises it: a product in 64 bits,
// off by less than 2^-45, rounded to a multiple of 2^-36 and then to a whole number.  254 |x| and odd multiples of max are multiples of 2^-8 of a unit in the last
// place of max where they are next to each other, so a quotient that is no half is off it by 2^-33 at least, and one that is comes out as it.
enum class Rows { BF16, F32 };

template <Rows KIND>
struct Scale {
  float inv, scale;
  double inv64;
  bool none;
  __device__ __forceinline__ explicit Scale(uint32_t most) {      // bits of the largest magnitude
    const float a = __uint_as_float(most);
    none = most >= 0x7f800000u;
    scale = a / 127.f;
    const bool small = !(scale > 0x1p-126f);
    if constexpr (KIND == Rows::BF16) {
      inv = small ? 0x1p126f : 127.f / a;
      if (!small && fmaf(inv, a, -127.f) < 0.f) inv = __uint_as_float(__float_as_uint(inv) + 1);
    } else {
      inv64 = small ? 0x1p126 : 127.0 / a;
    }
    if (small) scale = 0x1p-126f;
    if (none) scale = __builtin_nanf("");
  }
  // Four elements as bytes.  Adding 1.5 * 2^23 (2^52) leaves the nearest whole number in the low bits, 1.5 * 2^16 the nearest multiple of 2^-36.
  __device__ __forceinline__ uint32_t bytes(const float* x) const {
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 4; j++) {
      if constexpr (KIND == Rows::BF16) w[j] = __float_as_uint(fmaf(x[j], inv, 12582912.f));
      else w[j] = (uint32_t)__double2loint(fma((double)x[j], inv64, 98304.0) + (6755399441055744.0 - 98304.0));
    }
    const uint32_t lo = __builtin_amdgcn_perm(w[1], w[0], 0x0c0c0400u), hi = __builtin_amdgcn_perm(w[3], w[2], 0x04000c0cu);
    return lo | hi;
  }
  // ... of a row without a scale zeros
  __device__ __forceinline__ uint32_t four(const float* x) const { return none ? 0u : bytes(x); }
};

}  // namespace
}  // namespace lrb
