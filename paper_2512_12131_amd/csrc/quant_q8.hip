// Rows of activations or weights as 8-bit integers with one scale each: scale = max_j |x_j| / 127 (at least 2^-126), q_j the whole number next
// to 127 x_j / max_j |x_j|, ties to the even one.  A row that holds an infinity or a NaN has the scale NaN and zeros.
//
// The quotient is formed in 32 bits as a product with 127 / max, off by at most 127 * 2^-23 < 2^-16; where that leaves the nearest whole number open
// (2^-13 around a half; bf16 rows hold exact halves often: half of the largest value is 63.5) it is formed again in 64 bits, which hold it well enough to
// tell a tie.
//
// Bound: HBM, a row read once where it fits the registers of its lanes.
#include "common.h"

namespace lrb {
namespace {

constexpr int UNIT = 16;                   // elements of a lane at a time: 16 bytes of output

template <class T> struct Unit;
template <> struct Unit<uint16_t> {
  // n elements are there (a multiple of 8)
  __device__ static __forceinline__ void load(const uint16_t* p, int n, bool, float* f) {
    const uint4 zero = make_uint4(0, 0, 0, 0);
    const uint4 a = n > 0 ? *reinterpret_cast<const uint4*>(p) : zero, b = n > 8 ? *reinterpret_cast<const uint4*>(p + 8) : zero;
    unpack8(a, f);
    unpack8(b, f + 8);
  }
};
template <> struct Unit<float> {
  __device__ static __forceinline__ void load(const float* p, int n, bool vec, float* f) {
    if (vec && n >= UNIT) {
#pragma unroll
      for (int j = 0; j < UNIT; j += 4) *reinterpret_cast<float4*>(f + j) = *reinterpret_cast<const float4*>(p + j);
    } else {
#pragma unroll
      for (int j = 0; j < UNIT; j++) f[j] = j < n ? p[j] : 0.f;
    }
  }
};

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
    if (small) scale = 0x1p-126f;
    if (none) scale = __builtin_nanf("");
  }
  __device__ __forceinline__ int of(float x) const {
    const float t = x * inv, r = __builtin_rintf(t);
    int q = (int)r;
    if (__builtin_fabsf(t - r) > 0.5f - 0x1p-13f && !small)
      q = (int)__builtin_rint(127.0 * (double)x / (double)__uint_as_float(most));
    return none ? 0 : q;
  }
};

// TPR threads per row, NU units of 16 elements in a thread's registers; longer rows are read twice.
template <class T, int TPR, int NU>
__global__ __launch_bounds__(256) void quant_rows_kernel(const T* x, int64_t ldx, int8_t* q, int64_t ldq, float* scale, int64_t rows, int64_t n, int act, int vec) {
  constexpr int RPB = 256 / TPR;
  __shared__ uint32_t part[4];
  const int tid = threadIdx.x % TPR;
  const int64_t units = (n + UNIT - 1) / UNIT;
  for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < rows; r0 += (int64_t)gridDim.x * RPB) {
    const int64_t row = r0 + threadIdx.x / TPR;
    const bool in = row < rows;
    const T* px = x + row * ldx;
    float f[NU][UNIT];
    uint32_t most = 0;
    auto take = [&](int64_t u, float* v) {
      const int64_t left = n - u * UNIT;
      Unit<T>::load(px + u * UNIT, (int)(left < UNIT ? left : UNIT), vec != 0, v);
      if (act != LR_ACT_IDENTITY) {
#pragma unroll
        for (int j = 0; j < UNIT; j++) v[j] = act_f(v[j], act);
      }
    };
    auto look = [&](const float* v) {
#pragma unroll
      for (int j = 0; j < UNIT; j++) most = max(most, __float_as_uint(v[j]) & 0x7fffffffu);
    };
#pragma unroll
    for (int i = 0; i < NU; i++) {
      const int64_t u = tid + (int64_t)i * TPR;
      if (in && u < units) {
        take(u, f[i]);
        look(f[i]);
      }
    }
    for (int64_t u = tid + (int64_t)NU * TPR; in && u < units; u += TPR) {
      float v[UNIT];
      take(u, v);
      look(v);
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) most = max(most, (uint32_t)__shfl_xor((int)most, d));
    if constexpr (TPR == 256) {
      if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = most;
      __syncthreads();
      most = max(max(part[0], part[1]), max(part[2], part[3]));
      __syncthreads();
    }
    if (!in) continue;
    const Scale s(most);
    auto put = [&](int64_t u, const float* v) {
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; j++)
        w[j] = (uint32_t)(s.of(v[4 * j]) & 255) | (uint32_t)(s.of(v[4 * j + 1]) & 255) << 8 | (uint32_t)(s.of(v[4 * j + 2]) & 255) << 16 |
               (uint32_t)s.of(v[4 * j + 3]) << 24;
      *reinterpret_cast<uint4*>(q + row * ldq + u * UNIT) = make_uint4(w[0], w[1], w[2], w[3]);
    };
#pragma unroll
    for (int i = 0; i < NU; i++) {
      const int64_t u = tid + (int64_t)i * TPR;
      if (u < units) put(u, f[i]);
    }
    for (int64_t u = tid + (int64_t)NU * TPR; u < units; u += TPR) {
      float v[UNIT];
      take(u, v);
      put(u, v);
    }
    if (tid == 0) scale[row] = s.scale;
  }
}

template <class T>
hipError_t launch(const void* x, int64_t ldx, int8_t* q, int64_t ldq, float* scale, int64_t T_, int64_t n, int act, hipStream_t st) {
  const int vec = ((uintptr_t)x & 15) == 0 && ldx * sizeof(T) % 16 == 0;
  const bool narrow = n <= 1024;
  const int64_t rpb = narrow ? 4 : 1, blocks = (T_ + rpb - 1) / rpb;
  const dim3 grid((uint32_t)(blocks < (1 << 20) ? blocks : 1 << 20));
  if (narrow) hipLaunchKernelGGL((quant_rows_kernel<T, 64, 1>), grid, dim3(256), 0, st, (const T*)x, ldx, q, ldq, scale, T_, n, act, vec);
  else hipLaunchKernelGGL((quant_rows_kernel<T, 256, 2>), grid, dim3(256), 0, st, (const T*)x, ldx, q, ldq, scale, T_, n, act, vec);
  return hipGetLastError();
}

}  // namespace

hipError_t k_quant_rows(const void* x, int64_t ldx, int8_t* q, int64_t ldq, float* scale, int64_t T, int64_t n, int act, int dt, hipStream_t st) {
  if (T == 0) return hipSuccess;
  return dt == LR_BF16 ? launch<uint16_t>(x, ldx, q, ldq, scale, T, n, act, st) : launch<float>(x, ldx, q, ldq, scale, T, n, act, st);
}

}  // namespace lrb
