// Products of 8-bit integers: C[m, n] = sa[m] sb[n] sum_k A[m, k] B[n, k], both operands k-contiguous in rows that start on 16 bytes, the sum
// exact in 32-bit integers, scaled in 32 bits (the row's scale first) and rounded once.
//
// Simple form: a wavefront per 32 x 32 tile, operands from global memory straight into the registers of v_mfma_i32_32x32x32_i8.  What lies
// in a row behind K is masked out of A's last operand, so that it may hold anything.
#include "common.h"

namespace lrb {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));

// bytes of a lane's 16 that lie below n
__device__ __forceinline__ i32x4 first_bytes(i32x4 v, int n) {
#pragma unroll
  for (int j = 0; j < 4; j++) {
    const int left = n - 4 * j;
    v[j] = left >= 4 ? v[j] : left <= 0 ? 0 : v[j] & ((1 << (8 * left)) - 1);
  }
  return v;
}

__global__ __launch_bounds__(64) void gemm_q8_simple_kernel(Q8Op op, int tiles_n) {
  const int lane = threadIdx.x;
  const int m0 = (int)(blockIdx.x / tiles_n) * 32, n0 = (int)(blockIdx.x % tiles_n) * 32;
  const int row = lane & 31, k0 = (lane >> 5) * 16;
  const bool ma = m0 + row < op.M, nb = n0 + row < op.N;
  const int8_t* a = op.A + (int64_t)(m0 + row) * op.lda;
  const int8_t* b = op.B + (int64_t)(n0 + row) * op.ldb;
  i32x16 acc = {};
  for (int k = k0; k < op.K + k0; k += 32) {
    const i32x4 zero = {0, 0, 0, 0};
    i32x4 fa = ma && k < op.K ? *reinterpret_cast<const i32x4*>(a + k) : zero;
    const i32x4 fb = nb && k < op.K ? *reinterpret_cast<const i32x4*>(b + k) : zero;
    fa = first_bytes(fa, op.K - k);
    acc = __builtin_amdgcn_mfma_i32_32x32x32_i8(fb, fa, acc, 0, 0, 0);
  }
  if (!ma) return;
  const float sa = op.sa[m0 + row];
#pragma unroll
  for (int g = 0; g < 4; g++)
#pragma unroll
    for (int r = 0; r < 4; r++) {
      const int n = n0 + 8 * g + 4 * (lane >> 5) + r;
      if (n >= op.N) continue;
      const float v = (float)acc[4 * g + r] * sa * op.sb[n];
      const int64_t at = (int64_t)(m0 + row) * op.ldc + n;
      if (op.dt == LR_BF16) ((uint16_t*)op.C)[at] = (uint16_t)f32_to_bf16_bits(v);
      else ((float*)op.C)[at] = v;
    }
}

}  // namespace

hipError_t gemm_q8(const Q8Op& op, hipStream_t st) {
  const int tiles_m = (op.M + 31) / 32, tiles_n = (op.N + 31) / 32;
  hipLaunchKernelGGL(gemm_q8_simple_kernel, dim3((uint32_t)tiles_m * tiles_n), dim3(64), 0, st, op, tiles_n);
  return hipGetLastError();
}

}  // namespace lrb
