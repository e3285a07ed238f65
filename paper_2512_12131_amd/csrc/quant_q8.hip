// Rows of activations or weights as 8-bit integers with one scale each: scale = max_j |x_j| / 127 (at least 2^-126), q_j the whole number next
// to 127 x_j / max_j |x_j|, ties to the even one.  A row that holds an infinity or a NaN has the scale NaN and zeros.
//
// The quotient is not formed: quant_row.h says by which product the whole number is found.
//
// Bound: HBM, a row read once where it fits the registers of its lanes: 16384 x 4096 bf16 37 - 47 us (201 MB), 777 x 5461 fp32 in rows that start anywhere 8.0; few rows
// the way in and out of a launch, 16 x 4096 bf16 2.8.
#include "quant_row.h"

namespace lrb {
namespace {

constexpr int UNIT = 16;                   // elements of a lane at a time: 16 bytes of output
typedef float f32x4_anywhere __attribute__((ext_vector_type(4), aligned(4)));      // (fp32 rows may start at any element)

// 16 elements as they are stored, and as floats
template <class T> struct Unit;
template <> struct Unit<uint16_t> {
  uint4 v[2];
  // n of them are there (a multiple of 8)
  __device__ __forceinline__ void load(const uint16_t* p, int n) {
    v[0] = *reinterpret_cast<const uint4*>(p);
    v[1] = make_uint4(0, 0, 0, 0);
    if (n > 8) v[1] = *reinterpret_cast<const uint4*>(p + 8);
  }
  __device__ __forceinline__ void floats(float* f) const {
    unpack8(v[0], f);
    unpack8(v[1], f + 8);
  }
  __device__ __forceinline__ uint32_t most() const {      // bits of the largest magnitude, as a float
    uint32_t m = 0;
#pragma unroll
    for (int i = 0; i < 2; i++) {
      const uint32_t w[4] = {v[i].x, v[i].y, v[i].z, v[i].w};
#pragma unroll
      for (int j = 0; j < 4; j++) m = max(max(m, w[j] & 0x7fff0000u), (w[j] & 0x7fffu) << 16);
    }
    return m;
  }
};
template <> struct Unit<float> {
  float v[UNIT];
  __device__ __forceinline__ void load(const float* p, int n) {
    if (n >= UNIT) {
#pragma unroll
      for (int j = 0; j < UNIT; j += 4) {
        const f32x4_anywhere w = *reinterpret_cast<const f32x4_anywhere*>(p + j);
#pragma unroll
        for (int e = 0; e < 4; e++) v[j + e] = w[e];
      }
    } else {
#pragma unroll
      for (int j = 0; j < UNIT; j++) v[j] = j < n ? p[j] : 0.f;
    }
  }
  __device__ __forceinline__ void floats(float* f) const {
#pragma unroll
    for (int j = 0; j < UNIT; j++) f[j] = v[j];
  }
  __device__ __forceinline__ uint32_t most() const {
    uint32_t m = 0;
#pragma unroll
    for (int j = 0; j < UNIT; j++) m = max(m, __float_as_uint(v[j]) & 0x7fffffffu);
    return m;
  }
};

// TPR threads per row, NU units of 16 elements in a thread's registers; longer rows are read twice.  ACT (fp32): silu first.
template <class T, int TPR, int NU, bool ACT>
__global__ __launch_bounds__(256) void quant_rows_kernel(const T* x, int64_t ldx, int8_t* q, int64_t ldq, float* scale, int64_t rows, int64_t n) {
  constexpr int RPB = 256 / TPR;
  __shared__ uint32_t part[4];
  const int tid = threadIdx.x % TPR;
  const int64_t units = (n + UNIT - 1) / UNIT;
  for (int64_t r0 = (int64_t)blockIdx.x * RPB; r0 < rows; r0 += (int64_t)gridDim.x * RPB) {
    const int64_t row = r0 + threadIdx.x / TPR;
    const bool in = row < rows;
    const T* px = x + row * ldx;
    Unit<T> f[NU];
    uint32_t most = 0;
    auto take = [&](int64_t u, Unit<T>& v) {
      const int64_t left = n - u * UNIT;
      v.load(px + u * UNIT, (int)(left < UNIT ? left : UNIT));
    };
    auto act = [&](Unit<T>& v) {
      if constexpr (ACT) {
#pragma unroll
        for (int j = 0; j < UNIT; j++) v.v[j] = silu_f(v.v[j]);
      }
    };
#pragma unroll
    for (int i = 0; i < NU; i++) {
      const int64_t u = tid + (int64_t)i * TPR;
      if (in && u < units) take(u, f[i]);
    }
#pragma unroll
    for (int i = 0; i < NU; i++) {
      if (in && tid + (int64_t)i * TPR < units) {
        act(f[i]);
        most = max(most, f[i].most());
      }
    }
    for (int64_t u = tid + (int64_t)NU * TPR; in && u < units; u += TPR) {
      Unit<T> v;
      take(u, v);
      act(v);
      most = max(most, v.most());
    }
    most = wave_max(most);
    if constexpr (TPR == 256) {
      if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = most;
      __syncthreads();
      most = max(max(part[0], part[1]), max(part[2], part[3]));
      __syncthreads();
    }
    if (!in) continue;
    const Scale<sizeof(T) == 2 ? Rows::BF16 : Rows::F32> s(most);
    auto put = [&](int64_t u, const Unit<T>& v) {
      float e[UNIT];
      v.floats(e);
      uint32_t w[4];
#pragma unroll
      for (int j = 0; j < 4; j++) w[j] = s.four(e + 4 * j);
      *reinterpret_cast<uint4*>(q + row * ldq + u * UNIT) = make_uint4(w[0], w[1], w[2], w[3]);
    };
#pragma unroll
    for (int i = 0; i < NU; i++) {
      const int64_t u = tid + (int64_t)i * TPR;
      if (u < units) put(u, f[i]);
    }
    for (int64_t u = tid + (int64_t)NU * TPR; u < units; u += TPR) {
      Unit<T> v;
      take(u, v);
      act(v);
      put(u, v);
    }
    if (tid == 0) scale[row] = s.scale;
  }
}

template <class T, bool ACT>
hipError_t launch(const void* x, int64_t ldx, int8_t* q, int64_t ldq, float* scale, int64_t rows, int64_t n, hipStream_t st) {
  auto run = [&](auto kern, int64_t rpb) {
    const int64_t blocks = (rows + rpb - 1) / rpb;
    hipLaunchKernelGGL(kern, dim3((uint32_t)(blocks < (1 << 20) ? blocks : 1 << 20)), dim3(256), 0, st, (const T*)x, ldx, q, ldq, scale, rows, n);
    return hipGetLastError();
  };
  // us, one wavefront a row / four: 16384 x 1024 fp32 14.1 / 22.4, 16 x 4096 6.3 / 3.5, 16384 x 4096 79 / 53
  if (n <= 1024) return run(quant_rows_kernel<T, 64, 1, ACT>, 4);
  // us, 4096 / 12288 elements in registers: 16384 x 5460 fp32 81 / 87 (with 8192), 16384 x 11008 bf16 108 / 101, fp32 181 / 168, 4096 x 16384 bf16 48 / 39
  if (n <= 8192) return run(quant_rows_kernel<T, 256, 1, ACT>, 1);
  return run(quant_rows_kernel<T, 256, 3, ACT>, 1);
}

}  // namespace

hipError_t k_quant_rows(const void* x, int64_t ldx, int8_t* q, int64_t ldq, float* scale, int64_t T, int64_t n, int act, int dt, hipStream_t st) {
  if (T == 0) return hipSuccess;
  if (dt == LR_BF16) return act != LR_ACT_IDENTITY ? hipErrorInvalidValue : launch<uint16_t, false>(x, ldx, q, ldq, scale, T, n, st);
  return act == LR_ACT_SILU ? launch<float, true>(x, ldx, q, ldq, scale, T, n, st) : launch<float, false>(x, ldx, q, ldq, scale, T, n, st);
}

}  // namespace lrb
