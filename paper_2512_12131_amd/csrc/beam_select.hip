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

// 2^t in 64 bits for t <= 1000, within 6e-11 of it (from -1000 down 2^-1000, also for -infinity; a NaN is lost): 2^k 2^g with whole k, |g| <= 1/2, and the
// polynomial through 2^g at the Chebyshev points of degree 7.  Adding 1.5 * 2^52 leaves k in the low bits.
__device__ __forceinline__ double pow2_64(double t) {
  constexpr double C = 6755399441055744.0;
  const double m = __builtin_fmax(t, -1000.0) + C;
  const double g = __builtin_fmax(t, -1000.0) - (m - C);
  double p = 1.5303699001378845e-05;
  p = fma(p, g, 0.00015469729140704658);
  p = fma(p, g, 0.0013333478480888061);
  p = fma(p, g, 0.009618025613598036);
  p = fma(p, g, 0.055504109063177154);
  p = fma(p, g, 0.24022651213495422);
  p = fma(p, g, 0.6931471805568341);
  p = fma(p, g, 0.9999999999595622);
  return __hiloint2double(__double2hiint(p) + (__double2loint(m) << 20), __double2loint(p));
}
constexpr double LOG2E = 1.4426950408889634;


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

// 16 bytes of logits
template <class T> struct Vec;
template <> struct Vec<uint16_t> {
  static constexpr int N = 8;
  uint4 q;
  __device__ __forceinline__ void load(const uint16_t* p) { q = *reinterpret_cast<const uint4*>(p); }
  __device__ __forceinline__ void load(const uint16_t* p, int from, int end) {      // those of the indices from .. end, -infinity elsewhere
    uint32_t w[4];
#pragma unroll
    for (int j = 0; j < 8; j++) {
      const uint32_t b = j >= from && j < end ? p[j] : 0xff80u;
      w[j / 2] = j % 2 ? w[j / 2] | b << 16 : b;
    }
    q = make_uint4(w[0], w[1], w[2], w[3]);
  }
  __device__ __forceinline__ void floats(float* f) const { unpack8(q, f); }
};
template <> struct Vec<float> {
  static constexpr int N = 4;
  float4 q;
  __device__ __forceinline__ void load(const float* p) { q = *reinterpret_cast<const float4*>(p); }
  __device__ __forceinline__ void load(const float* p, int from, int end) {
    float v[4];
#pragma unroll
    for (int j = 0; j < 4; j++) v[j] = j >= from && j < end ? p[j] : -INFINITY;
    q = make_float4(v[0], v[1], v[2], v[3]);
  }
  __device__ __forceinline__ void floats(float* f) const { f[0] = q.x; f[1] = q.y; f[2] = q.z; f[3] = q.w; }
};

// E: logits per lane and piece
template <class T, int E>
__global__ __launch_bounds__(256) void beam_runs_kernel(BeamSelect s) {
  constexpr int N = Vec<T>::N, NV = E / N, PIECE = 64 * E;
  const int lane = threadIdx.x & 63;
  const int item = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = item / s.parts, part = item - row * s.parts;
  if (row >= s.rows || (s.done && s.done[row] != 0)) return;
  const T* x = (const T*)s.logits + (int64_t)row * s.ld;
  // vectors start on 16 bytes; the first may reach before the row
  const int shift = (int)(((uintptr_t)x & 15) / sizeof(T));
  const int begin = part * s.run - shift, end = min(begin + s.run, s.V);
  auto load = [&](int p0, Vec<T> (&v)[NV]) {
#pragma unroll
    for (int j = 0; j < NV; j++) {
      const int i0 = p0 + (j * 64 + lane) * N;
      if (p0 >= 0 && p0 + PIECE <= end) v[j].load(x + i0);
      else v[j].load(x + i0, max(-i0, 0), end - i0);
    }
  };
  Best best;
  float ref = -INFINITY;
  double sum = 0, ref2 = 0;                            // ref2: ref * log2(e)
  bool bad = false;
  Vec<T> cur[NV], nxt[NV];
  load(begin, cur);
  for (int p0 = begin; p0 < end; p0 += PIECE) {
    if (p0 + PIECE < end) load(p0 + PIECE, nxt);
    float most = -INFINITY;
#pragma unroll
    for (int j = 0; j < NV; j++) {
      float f[N];
      cur[j].floats(f);
#pragma unroll
      for (int e = 0; e < N; e += 2) {
        bad |= __builtin_isunordered(f[e], f[e + 1]);
        most = fmaxf(fmaxf(most, f[e]), f[e + 1]);
      }
    }
    // the exponentials refer to the largest logit of the first piece that has any, or of one that is far above it
    if (__ballot(most > ref + 500.f || (ref == -INFINITY && most > ref)) != 0) {
      float top = most;
#pragma unroll
      for (int d = 32; d > 0; d >>= 1) top = fmaxf(top, __shfl_xor(top, d));
      if (ref > -INFINITY) sum *= pow2_64(((double)ref - top) * LOG2E);
      ref = top;
      ref2 = (double)ref * LOG2E;
    }
    if (ref > -INFINITY) {
#pragma unroll
      for (int j = 0; j < NV; j++) {
        float f[N];
        cur[j].floats(f);
#pragma unroll
        for (int e = 0; e < N; e++) sum += pow2_64(fma((double)f[e], LOG2E, -ref2));
      }
    }
    // Candidates: at least n lanes have one that reaches `floor`, or the list is full and ends with it.
    uint32_t last_hi = lane_value(best.hi, s.n - 1), last_lo = lane_value(best.lo, s.n - 1);
    const uint32_t least = last_hi != 0 ? last_hi : nth_of_lanes(most > -INFINITY ? ordered(most + 0.f) : 0, s.n);
    const float floor = least != 0 ? unordered(least) : -INFINITY;
    if (__ballot(most >= floor && most > -INFINITY) != 0) {
#pragma unroll 1
      for (int j = 0; j < NV; j++) {
        Vec<T> v = cur[0];
#pragma unroll
        for (int i = 1; i < NV; i++)
          if (i == j) v = cur[i];
        float f[N], top = -INFINITY;
        v.floats(f);
#pragma unroll
        for (int e = 0; e < N; e += 2) top = fmaxf(fmaxf(top, f[e]), f[e + 1]);
        if (__ballot(top >= floor) == 0) continue;
#pragma unroll
        for (int e = 0; e < N; e++) {
          uint64_t m = __ballot(f[e] >= floor && f[e] > -INFINITY);
          if (m == 0) continue;
          const uint32_t hi = ordered(f[e] + 0.f);                              // (-0 is 0)
          const uint32_t lo = ~(uint32_t)(p0 + (j * 64 + lane) * N + e);
          m &= __ballot(hi > last_hi || (hi == last_hi && lo > last_lo));
          while (m != 0) {
            const int from = __builtin_ctzll(m);
            best.insert(lane_value(hi, from), lane_value(lo, from), lane);
            last_hi = lane_value(best.hi, s.n - 1);
            last_lo = lane_value(best.lo, s.n - 1);
            m &= ~(1ull << from) & __ballot(hi > last_hi || (hi == last_hi && lo > last_lo));
          }
        }
      }
    }
#pragma unroll
    for (int j = 0; j < NV; j++) cur[j] = nxt[j];
  }
#pragma unroll
  for (int d = 32; d > 0; d >>= 1) sum += __shfl_xor(sum, d);
  if (__ballot(bad) != 0 || !(ref < INFINITY)) sum = __builtin_nan("");
  if (lane == 0) {
    s.part_ref[item] = ref;
    s.part_sum[item] = sum;
  }
  if (lane < s.n) s.part_key[(int64_t)item * s.n + lane] = make_uint2(best.hi, best.lo);
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

// A wavefront's candidates (one per lane) into its list: was one added?
__device__ __forceinline__ bool merge(Scored& best, uint64_t score, uint32_t at, int n, int lane) {
  uint64_t last = lane_value64(best.score, n - 1);
  uint32_t last_at = lane_value(best.at, n - 1);
  const uint32_t floor = last == 0 ? nth_of_lanes((uint32_t)(score >> 32), n) : 0;      // (no full list yet)
  uint64_t m = __ballot(score != 0 && (uint32_t)(score >> 32) >= floor && (score > last || (score == last && at > last_at)));
  const bool added = m != 0;
  while (m != 0) {
    const int from = __builtin_ctzll(m);
    best.insert(lane_value64(score, from), lane_value(at, from), lane);
    last = lane_value64(best.score, n - 1);
    last_at = lane_value(best.at, n - 1);
    m &= ~(1ull << from) & __ballot(score > last || (score == last && at > last_at));
  }
  return added;
}

__global__ __launch_bounds__(256) void beam_merge_kernel(BeamSelect s) {
  // a candidate's score is (logit - largest logit) - logarithm of the sum + score, in this order: the logits may be far from zero
  __shared__ double log_sum[BEAM_MOST];                // NaN: the beam offers nothing
  __shared__ float largest[BEAM_MOST], score_in[BEAM_MOST];
  __shared__ uint64_t list_score[4 * 64];
  __shared__ uint32_t list_at[4 * 64];
  constexpr int AHEAD = 4;                             // candidates of a list that are asked for at once
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int prompt = blockIdx.x, row0 = prompt * s.beams;
  // The runs' lists fall from candidate to candidate: all first ones, then the second ones, until none is added
  const int lists = s.beams * s.parts;
  const uint2* keys = s.part_key + (int64_t)row0 * s.parts * s.n;
  uint2 key[AHEAD];
  auto ask = [&](int l) {
#pragma unroll
    for (int r = 0; r < AHEAD; r++) key[r] = l < lists && r < s.n ? keys[(int64_t)l * s.n + r] : make_uint2(0, 0);
  };
  ask(lane * 4 + wave);
  // sixteen lanes per beam
  for (int w0 = 0; w0 < s.beams; w0 += 16) {
    const int w = w0 + (int)threadIdx.x / 16, sub = threadIdx.x & 15;
    const bool in = w < s.beams && !(s.done && s.done[row0 + w] != 0);      // (an ended beam's logits were not looked at)
    const int64_t item = (int64_t)(row0 + w) * s.parts;
    float top = -INFINITY;
    double sum = 0;
    bool bad = false;
    for (int p = sub; in && p < s.parts; p += 16) {
      const float ref = s.part_ref[item + p];
      const double t = s.part_sum[item + p];
      bad |= !(t == t);
      if (ref > top) {                                 // (the sum so far refers to the larger one)
        sum = top > -INFINITY ? sum * pow2_64(((double)top - ref) * LOG2E) : 0;
        top = ref;
      }
      if (ref > -INFINITY) sum += t * pow2_64(((double)ref - top) * LOG2E);
    }
    float most = top;
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) most = fmaxf(most, __shfl_xor(most, d));
    sum = top > -INFINITY ? sum * pow2_64(((double)top - most) * LOG2E) : 0;
    int wrong = bad;
#pragma unroll
    for (int d = 8; d > 0; d >>= 1) {
      sum += __shfl_xor(sum, d);
      wrong |= __shfl_xor(wrong, d);
    }
    if (sub == 0 && w < s.beams) {
      const float score = s.score[row0 + w];
      const bool none = !in || wrong || !(most > -INFINITY) || !(__builtin_fabsf(score) < INFINITY);
      log_sum[w] = none ? __builtin_nan("") : log(sum);
      largest[w] = most;
      score_in[w] = score;
    }
  }
  __syncthreads();
  Scored best;
  for (int l0 = 0; l0 < lists; l0 += 256) {
    const int l = l0 + lane * 4 + wave, w = min(l / s.parts, s.beams - 1);
    const double less = log_sum[w];
    const bool some = l < lists && less == less;
    if (l0 > 0) ask(l);
    auto step = [&](uint2 k) {
      uint64_t score = 0;
      if (some && k.x != 0) score = ordered(((double)unordered(k.x) - largest[w] - less) + score_in[w] + 0.0);
      return merge(best, score, ~((uint32_t)w << 20 | ~k.y), s.n, lane);
    };
    bool more = true;
#pragma unroll
    for (int r = 0; r < AHEAD; r++)
      if (more && r < s.n) more = step(key[r]);
    for (int r = AHEAD; more && r < s.n; r++) more = step(l < lists ? keys[(int64_t)l * s.n + r] : make_uint2(0, 0));
  }
  if (s.done && wave == 0) {                           // an ended beam goes on with one token, at its score
    const int w = lane;
    uint64_t score = 0;
    if (w < s.beams && s.done[row0 + w] != 0 && __builtin_fabsf(s.score[row0 + w]) < INFINITY) score = ordered((double)s.score[row0 + w] + 0.0);
    merge(best, score, ~((uint32_t)w << 20 | (uint32_t)s.done_token), s.n, lane);
  }
  list_score[wave * 64 + lane] = lane < s.n ? best.score : 0;
  list_at[wave * 64 + lane] = best.at;
  __syncthreads();
  // A candidate's place is the number of those above it, in the four lists
  const uint64_t mine = list_score[threadIdx.x];
  const uint32_t at = list_at[threadIdx.x];
  int place = 0, all = 0;
  for (int l = 0; l < 4; l++)
    for (int i = 0; i < s.n; i++) {
      const uint64_t other = list_score[l * 64 + i];
      place += other > mine || (other == mine && list_at[l * 64 + i] > at);
      all += other != 0;
    }
  const int64_t o = (int64_t)prompt * s.n;
  if (mine != 0 && place < s.n) {
    s.parent[o + place] = row0 + (int)(~at >> 20);
    s.token[o + place] = (int)(~at & 0xfffffu);
    s.score_out[o + place] = (float)unordered(mine);
  }
  if ((int)threadIdx.x < s.n && (int)threadIdx.x >= all) {
    s.parent[o + threadIdx.x] = s.token[o + threadIdx.x] = -1;
    s.score_out[o + threadIdx.x] = -INFINITY;
  }
}

// A run for a wavefront: pieces of 512 logits where those of 2048 are too few for the chip, else as many as give every SIMD four wavefronts.
struct Runs { int elems; int64_t run, parts; };
Runs runs_of(int64_t rows, int64_t V) {
  const int64_t span = V + 7;                          // (a row may start up to 7 logits behind 16 bytes)
  const int elems = rows * ((span + 2047) / 2048) < 1024 ? 8 : 32;
  const int64_t piece = 64 * elems, pieces = (span + piece - 1) / piece;
  int64_t parts = rows > 0 ? (4096 + rows - 1) / rows : 1;
  if (parts > pieces) parts = pieces;
  const int64_t per = (pieces + parts - 1) / parts;
  return {elems, per * piece, (pieces + per - 1) / per};
}

template <class T>
hipError_t launch_runs(const BeamSelect& s, int elems, int64_t items, hipStream_t st) {
  const dim3 grid((uint32_t)((items + 3) / 4));
  if (elems == 8) hipLaunchKernelGGL((beam_runs_kernel<T, 8>), grid, dim3(256), 0, st, s);
  else hipLaunchKernelGGL((beam_runs_kernel<T, 32>), grid, dim3(256), 0, st, s);
  return hipGetLastError();
}

}  // namespace

size_t beam_select_ws_bytes(int64_t rows, int64_t V, int64_t n) {
  return (size_t)(rows * runs_of(rows, V).parts) * (sizeof(double) + (size_t)n * sizeof(uint2) + sizeof(float));
}
hipError_t k_beam_select(BeamSelect s, int dt, void* ws, hipStream_t st) {
  const Runs r = runs_of(s.rows, s.V);
  s.parts = (int)r.parts;
  s.run = (int)r.run;
  const int64_t items = (int64_t)s.rows * s.parts;
  s.part_sum = (double*)ws;
  s.part_key = (uint2*)(s.part_sum + items);
  s.part_ref = (float*)(s.part_key + items * s.n);
  const hipError_t e = dt == LR_BF16 ? launch_runs<uint16_t>(s, r.elems, items, st) : launch_runs<float>(s, r.elems, items, st);
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL(beam_merge_kernel, dim3((uint32_t)(s.rows / s.beams)), dim3(256), 0, st, s);
  return hipGetLastError();
}

}  // namespace lrb
