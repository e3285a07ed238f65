// Attention of each sequence's new tokens over its pages of a key / value cache, heads of 128, bf16 in / fp32 softmax.
#include "common.h"

namespace lrb {
namespace {

constexpr int HD = 128;
constexpr float LOG2E = 1.4426950408889634f;

struct PagedArgs {
  KvCache c;
  const uint16_t* q;
  uint16_t* o;
  float* lse;
  int64_t ldq, ldo, T;
  int H, grp;
  float scale;
};

// The running maximum of a row that has seen no key: finite, so that no difference of two of them is undefined, and below any score whose
// product with the exponent's factor c is finite.
__device__ __forceinline__ float no_score(float c) { return -3.0e38f / fmaxf(c, 1.f); }

// One wavefront per (token, head): 16 lanes hold a row's 128 columns, four keys at a time, each quarter with its own running
// maximum and sum, joined at the end.
__global__ __launch_bounds__(256) void paged_simple_kernel(PagedArgs a) {
  const int lane = threadIdx.x & 63;
  const int64_t item = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 6);
  if (item >= a.T * a.H) return;
  const int64_t t = item / a.H;
  const int h = (int)(item % a.H), sub = lane & 15, quarter = lane >> 4;
  int before = 0;
  for (int i = 0; i < a.c.batch; i += 64) {
    const bool in = i + lane < a.c.batch;
    before += __popcll(__ballot(in && a.c.cu_q[in ? i + lane + 1 : 0] <= t));
  }
  if (before >= a.c.batch || a.c.cu_q[before] > t) return;
  const int64_t end = a.c.cu_q[before + 1] < a.T ? a.c.cu_q[before + 1] : a.T;
  int64_t keys = (int64_t)a.c.kv_len[before] - (end - t) + 1;
  keys = keys < a.c.capacity ? keys : a.c.capacity;
  const float c = a.scale * LOG2E;
  float qv[8], m = no_score(c), l = 0.f, acc[8] = {};
  unpack8(*reinterpret_cast<const uint4*>(a.q + t * a.ldq + h * HD + sub * 8), qv);
  for (int64_t j = quarter; j < keys; j += 4) {
    const int col = (int)a.c.by_page.div((uint32_t)j);
    const int page = a.c.page_table[before * a.c.table_ld + col];
    float kv[8] = {}, vv[8] = {};
    if ((uint32_t)page < (uint32_t)a.c.n_pages) {
      const int64_t at = page * a.c.page_stride + (j - (int64_t)col * a.c.page_size) * a.c.token_stride + h / a.grp * a.c.head_stride + sub * 8;
      unpack8(*reinterpret_cast<const uint4*>(a.c.k + at), kv);
      unpack8(*reinterpret_cast<const uint4*>(a.c.v + at), vv);
    }
    float s = 0.f;
#pragma unroll
    for (int i = 0; i < 8; i++) s = fmaf(qv[i], kv[i], s);
    for (int d = 1; d < 16; d <<= 1) s += __shfl_xor(s, d);
    const float mn = fmaxf(m, s), al = exp2f((m - mn) * c), p = exp2f((s - mn) * c);
    l = l * al + p;
#pragma unroll
    for (int i = 0; i < 8; i++) acc[i] = acc[i] * al + p * vv[i];
    m = mn;
  }
  for (int d = 16; d < 64; d <<= 1) {
    const float mo = __shfl_xor(m, d), lo = __shfl_xor(l, d), mn = fmaxf(m, mo);
    const float al = exp2f((m - mn) * c), bl = exp2f((mo - mn) * c);
    l = l * al + lo * bl;
#pragma unroll
    for (int i = 0; i < 8; i++) acc[i] = acc[i] * al + __shfl_xor(acc[i], d) * bl;
    m = mn;
  }
  if (quarter == 0) {
    const float inv = l > 0.f ? 1.f / l : 0.f;
#pragma unroll
    for (int i = 0; i < 8; i++) acc[i] *= inv;
    *reinterpret_cast<uint4*>(a.o + t * a.ldo + h * HD + sub * 8) = pack8(acc);
    if (sub == 0 && a.lse) a.lse[t * a.H + h] = l > 0.f ? m * a.scale + logf(l) : -INFINITY;
  }
}

}  // namespace

size_t attention_paged_ws_bytes(int64_t T, int H, int Hkv, int batch, int64_t capacity) { return 0; }

hipError_t attention_paged_bf16(const KvCache& c, const void* q, int64_t ldq, void* o, int64_t ldo, float* lse, int64_t T, int H, float scale,
                                void* ws, hipStream_t st) {
  PagedArgs a{c, (const uint16_t*)q, (uint16_t*)o, lse, ldq, ldo, T, H, H / c.n_kv_heads, scale};
  hipLaunchKernelGGL(paged_simple_kernel, dim3((unsigned)((T * H + 3) / 4)), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace lrb
