// The candidates of highest score over the beams of a prompt and the vocabulary: score[w] + logit[w, v] - log sum_u exp(logit[w, u]), the n
// largest for each prompt, ties to the lower beam, then the lower token.
//
// Scores are formed in 64 bits: candidates of different beams are compared through two such sums, and 32 bits would change the
// order of those that lie next to each other.
//
// First launch: a wavefront takes a run of one beam's logits.  Within a beam the order of the scores is that of the logits, so it keeps the
// n largest logits of the run, one per lane, and the sum of exponentials relative to the largest logit of its first piece.  Second launch:
// a workgroup per prompt adds up the beams' sums and merges their lists by score.
#include "common.h"

namespace lrb {
namespace {

__device__ __forceinline__ int lanes_in(uint64_t m) { return __popcll(m); }
__device__ __forceinline__ uint32_t lane_value(uint32_t v, int lane) { return (uint32_t)__builtin_amdgcn_readlane((int)v, lane); }
// the value of the lane before (lane 0: its own)
__device__ __forceinline__ uint32_t from_lane_before(uint32_t v) {
  return (uint32_t)__builtin_amdgcn_update_dpp((int)v, (int)v, 0x138, 0xf, 0xf, false);      // wave_shr:1
}

// Whole numbers in the order of floats (no NaN, no -0); all are above 0.
__device__ __forceinline__ uint32_t ordered(float f) {
  const uint32_t b = __float_as_uint(f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float unordered(uint32_t o) { return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o); }
__device__ __forceinline__ uint64_t ordered(double f) {
  const uint64_t b = (uint64_t)__double_as_longlong(f);
  return b >> 63 ? ~b : b | 0x8000000000000000ull;
}
__device__ __forceinline__ double unordered(uint64_t o) {
  return __longlong_as_double((long long)(o >> 63 ? o & 0x7fffffffffffffffull : ~o));
}

// exp(x) for x <= 700, within 1e-11 of it: 2^k exp(f) with x = k log 2 + f, |f| <= log(2) / 2, and the Taylor series of exp up to f^9 (the next
// term is (log(2) / 2)^10 / 10! = 7e-12).  -infinity gives 0, NaN gives NaN.
__device__ __forceinline__ double exp64(double x) {
  x = x < -1000.0 ? -1000.0 : x;
  const double k = __builtin_rint(x * 1.4426950408889634);
  const double f = fma(k, -0.6931471805599453, x);
  double p = 1.0 / 362880;
  p = fma(p, f, 1.0 / 40320);
  p = fma(p, f, 1.0 / 5040);
  p = fma(p, f, 1.0 / 720);
  p = fma(p, f, 1.0 / 120);
  p = fma(p, f, 1.0 / 24);
  p = fma(p, f, 1.0 / 6);
  p = fma(p, f, 0.5);
  p = fma(p, f, 1.0);
  p = fma(p, f, 1.0);
  return __builtin_ldexp(p, (int)k);
}

constexpr int SELECT_E = 32;                          // logits per lane and piece
constexpr int PIECE = 64 * SELECT_E;

// The n largest keys of a wavefront, lane i the i-th; 0: none.  Keys are unique.
struct Best {
  uint32_t hi = 0, lo = 0;
  __device__ __forceinline__ void insert(uint32_t h, uint32_t l, int lane) {      // (h and l the same in all lanes)
    const int at = lanes_in(__ballot(hi > h || (hi == h && lo > l)));
    const uint32_t ph = from_lane_before(hi), pl = from_lane_before(lo);
    if (lane == at) { hi = h; lo = l; }
    if (lane > at) { hi = ph; lo = pl; }
  }
};

// The largest value that at least n lanes reach (0: fewer have any).
__device__ __forceinline__ uint32_t nth_of_lanes(uint32_t v, int n) {
  uint32_t t = 0;
  for (int b = 31; b >= 0; b--) {
    const uint32_t u = t | (1u << b);
    if (lanes_in(__ballot(v >= u)) >= n) t = u;
  }
  return t;
}

template <class T> struct Vec;
template <> struct Vec<uint16_t> {
  static constexpr int N = 8;
  __device__ static __forceinline__ void load(const uint16_t* p, float* f) { unpack8(*reinterpret_cast<const uint4*>(p), f); }
  __device__ static __forceinline__ float one(const uint16_t* p) { return bf16_bits_to_f32(*p); }
};
template <> struct Vec<float> {
  static constexpr int N = 4;
  __device__ static __forceinline__ void load(const float* p, float* f) {
    const float4 q = *reinterpret_cast<const float4*>(p);
    f[0] = q.x; f[1] = q.y; f[2] = q.z; f[3] = q.w;
  }
  __device__ static __forceinline__ float one(const float* p) { return *p; }
};

template <class T>
__global__ __launch_bounds__(256) void beam_runs_kernel(BeamSelect s) {
  constexpr int N = Vec<T>::N, NV = SELECT_E / N;
  const int lane = threadIdx.x & 63;
  const int64_t item = (int64_t)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = (int)(item / s.parts), part = (int)(item % s.parts);
  if (row >= s.rows || (s.done && s.done[row] != 0)) return;
  const T* x = (const T*)s.logits + (int64_t)row * s.ld;
  // pieces start on 16 bytes; the first may reach before the row
  const int shift = (int)(((uintptr_t)x & 15) / sizeof(T));
  const int begin = part * s.run - shift, end = min(begin + s.run, s.V);
  Best best;
  float ref = -INFINITY;
  double sum = 0;
  bool bad = false;
  for (int p0 = begin; p0 < end; p0 += PIECE) {
    float f[SELECT_E];
#pragma unroll
    for (int v = 0; v < NV; v++) {
      const int i0 = p0 + (v * 64 + lane) * N;
      if (i0 >= 0 && i0 + N <= end) {
        Vec<T>::load(x + i0, f + v * N);
      } else {
#pragma unroll
        for (int j = 0; j < N; j++) f[v * N + j] = i0 + j >= 0 && i0 + j < end ? Vec<T>::one(x + i0 + j) : -INFINITY;
      }
    }
    float most = -INFINITY;
#pragma unroll
    for (int e = 0; e < SELECT_E; e++) {
      bad |= !(f[e] < INFINITY);
      f[e] += 0.f;                                     // (-0 becomes 0)
      most = fmaxf(most, f[e]);
    }
    // the exponentials refer to the largest logit of the first piece that has any, or of one that is far above it
    if (__ballot(most > ref + 500.f || (ref == -INFINITY && most > ref)) != 0) {
      float top = most;
#pragma unroll
      for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
      if (ref > -INFINITY) sum *= exp64((double)ref - top);
      ref = top;
    }
    if (ref > -INFINITY) {
#pragma unroll
      for (int e = 0; e < SELECT_E; e++) sum += exp64((double)f[e] - ref);
    }
    // Candidates: at least n lanes have one that reaches `floor`, or the list is full and ends with it.
    const uint32_t mine = most > -INFINITY ? ordered(most) : 0;
    uint32_t last_hi = lane_value(best.hi, s.n - 1), last_lo = lane_value(best.lo, s.n - 1);
    uint32_t floor = last_hi;
    if (floor == 0) floor = nth_of_lanes(mine, s.n);
    if (__ballot(mine != 0 && mine >= floor) == 0) continue;
#pragma unroll
    for (int e = 0; e < SELECT_E; e++) {
      const uint32_t hi = f[e] > -INFINITY ? ordered(f[e]) : 0;
      const uint32_t lo = ~(uint32_t)(p0 + ((e / N) * 64 + lane) * N + e % N);
      uint64_t m = __ballot(hi != 0 && hi >= floor && (hi > last_hi || (hi == last_hi && lo > last_lo)));
      while (m != 0) {
        const int from = __builtin_ctzll(m);
        best.insert(lane_value(hi, from), lane_value(lo, from), lane);
        last_hi = lane_value(best.hi, s.n - 1);
        last_lo = lane_value(best.lo, s.n - 1);
        m &= ~(1ull << from) & __ballot(hi > last_hi || (hi == last_hi && lo > last_lo));
      }
    }
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
  if (__ballot(bad) != 0) sum = __builtin_nan("");
  if (lane == 0) {
    s.part_ref[item] = ref;
    s.part_sum[item] = sum;
  }
  if (lane < s.n) s.part_key[item * s.n + lane] = make_uint2(best.hi, best.lo);
}

// Candidates by score, then by beam and token; one per lane, 0: none.
struct Scored {
  uint64_t score = 0;
  uint32_t at = 0;                                     // ~(beam of the prompt * 2^20 + token)
  __device__ __forceinline__ bool above(uint64_t s, uint32_t a) const { return score > s || (score == s && at > a); }
  __device__ __forceinline__ void insert(uint64_t s, uint32_t a, int lane) {
    const int to = lanes_in(__ballot(above(s, a)));
    const uint32_t sh = from_lane_before((uint32_t)(score >> 32)), sl = from_lane_before((uint32_t)score), pa = from_lane_before(at);
    if (lane == to) { score = s; at = a; }
    if (lane > to) { score = (uint64_t)sh << 32 | sl; at = pa; }
  }
};
__device__ __forceinline__ uint64_t lane_value64(uint64_t v, int lane) {
  return (uint64_t)lane_value((uint32_t)(v >> 32), lane) << 32 | lane_value((uint32_t)v, lane);
}

// One wavefront's candidates (one per lane) into its list.
__device__ __forceinline__ void merge(Scored& best, uint64_t score, uint32_t at, int n, int lane) {
  uint64_t last = lane_value64(best.score, n - 1);
  uint32_t last_at = lane_value(best.at, n - 1);
  const uint32_t floor = last == 0 ? nth_of_lanes((uint32_t)(score >> 32), n) : 0;      // (no full list yet)
  uint64_t m = __ballot(score != 0 && (uint32_t)(score >> 32) >= floor && (score > last || (score == last && at > last_at)));
  while (m != 0) {
    const int from = __builtin_ctzll(m);
    best.insert(lane_value64(score, from), lane_value(at, from), lane);
    last = lane_value64(best.score, n - 1);
    last_at = lane_value(best.at, n - 1);
    m &= ~(1ull << from) & __ballot(score > last || (score == last && at > last_at));
  }
}

__global__ __launch_bounds__(256) void beam_merge_kernel(BeamSelect s) {
  // a candidate's score is (logit - largest logit) - logarithm of the sum + score, in this order: the logits may be far from zero
  __shared__ double log_sum[BEAM_MOST];                // NaN: the beam offers nothing
  __shared__ float largest[BEAM_MOST];
  __shared__ uint64_t list_score[3 * 64];
  __shared__ uint32_t list_at[3 * 64];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int prompt = blockIdx.x, row0 = prompt * s.beams;
  for (int w = wave; w < s.beams; w += 4) {
    const int row = row0 + w;
    if (s.done && s.done[row] != 0) {                  // (its logits were not looked at)
      if (lane == 0) log_sum[w] = __builtin_nan("");
      continue;
    }
    const int64_t item = (int64_t)row * s.parts;
    float top = -INFINITY;
    for (int p = lane; p < s.parts; p += 64) top = fmaxf(top, s.part_ref[item + p]);
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
    double sum = 0;
    bool bad = false;
    for (int p = lane; p < s.parts; p += 64) {
      const double t = s.part_sum[item + p];
      bad |= !(t == t);
      if (s.part_ref[item + p] > -INFINITY) sum += t * exp64((double)s.part_ref[item + p] - top);
    }
#pragma unroll
    for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
    const float score = s.score[row];
    const bool none = __ballot(bad) != 0 || !(top > -INFINITY) || !(__builtin_fabsf(score) < INFINITY);
    if (lane == 0) {
      log_sum[w] = none ? __builtin_nan("") : log(sum);
      largest[w] = top;
    }
  }
  __syncthreads();
  Scored best;
  const int per = s.parts * s.n, total = s.beams * per;
  const uint2* keys = s.part_key + (int64_t)row0 * per;
  for (int k0 = wave * 64; k0 < total; k0 += 256) {
    const int k = k0 + lane, w = k / per;
    uint64_t score = 0;
    uint32_t at = 0;
    if (k < total && log_sum[w] == log_sum[w]) {
      const uint2 key = keys[k];
      if (key.x != 0) {
        score = ordered(((double)unordered(key.x) - largest[w] - log_sum[w]) + s.score[row0 + w] + 0.0);
        at = ~((uint32_t)w << 20 | ~key.y);
      }
    }
    merge(best, score, at, s.n, lane);
  }
  if (s.done && wave == 0) {                           // an ended beam goes on with one token, at its score
    const int w = lane;
    uint64_t score = 0;
    if (w < s.beams && s.done[row0 + w] != 0 && __builtin_fabsf(s.score[row0 + w]) < INFINITY) score = ordered((double)s.score[row0 + w] + 0.0);
    merge(best, score, ~((uint32_t)w << 20 | (uint32_t)s.done_token), s.n, lane);
  }
  if (wave > 0) {
    list_score[(wave - 1) * 64 + lane] = best.score;
    list_at[(wave - 1) * 64 + lane] = best.at;
  }
  __syncthreads();
  if (wave > 0) return;
  for (int l = 0; l < 3; l++) merge(best, lane < s.n ? list_score[l * 64 + lane] : 0, list_at[l * 64 + lane], s.n, lane);
  if (lane < s.n) {
    const int64_t o = (int64_t)prompt * s.n + lane;
    const bool some = best.score != 0;
    const uint32_t at = ~best.at;
    s.parent[o] = some ? row0 + (int)(at >> 20) : -1;
    s.token[o] = some ? (int)(at & 0xfffffu) : -1;
    s.score_out[o] = some ? (float)unordered(best.score) : -INFINITY;
  }
}

// Runs of at least a piece; as many as give every SIMD of the chip two wavefronts, where there is work for that.
int64_t parts_of(int64_t rows, int64_t V, int64_t* run) {
  const int64_t span = V + 7, pieces = (span + PIECE - 1) / PIECE;      // (a row may start up to 7 logits behind 16 bytes)
  int64_t parts = rows > 0 ? (2048 + rows - 1) / rows : 1;
  if (parts > pieces) parts = pieces;
  const int64_t per = (pieces + parts - 1) / parts;
  *run = per * PIECE;
  return (pieces + per - 1) / per;
}

}  // namespace

size_t beam_select_ws_bytes(int64_t rows, int64_t V, int64_t n) {
  int64_t run;
  const int64_t items = rows * parts_of(rows, V, &run);
  return (size_t)items * (sizeof(double) + (size_t)n * sizeof(uint2) + sizeof(float));
}
hipError_t k_beam_select(BeamSelect s, int dt, void* ws, hipStream_t st) {
  int64_t run;
  s.parts = (int)parts_of(s.rows, s.V, &run);
  s.run = (int)run;
  const int64_t items = (int64_t)s.rows * s.parts;
  s.part_sum = (double*)ws;
  s.part_key = (uint2*)(s.part_sum + items);
  s.part_ref = (float*)(s.part_key + items * s.n);
  const dim3 grid((uint32_t)((items + 3) / 4));
  if (dt == LR_BF16) hipLaunchKernelGGL(beam_runs_kernel<uint16_t>, grid, dim3(256), 0, st, s);
  else hipLaunchKernelGGL(beam_runs_kernel<float>, grid, dim3(256), 0, st, s);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(beam_merge_kernel, dim3((uint32_t)(s.rows / s.beams)), dim3(256), 0, st, s);
  return hipGetLastError();
}

}  // namespace lrb
