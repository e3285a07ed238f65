// The candidates of highest score over the beams of a prompt and the vocabulary: score[w] + logit[w, v] - log sum_u exp(logit[w, u]), the n
// largest for each prompt, ties to the lower beam; within a beam the order is that of the logits, ties to the lower token.
//
// Scores are formed in 64 bits: candidates of different beams are compared through two such sums, and 32 bits would change the
// order of those that lie next to each other.  Logits that differ by less than a last place of their scores have one score, and still an order: score, beam,
// logit and token together order all candidates, in the runs (one beam: logit and token) and in the merge alike, so that the first ones are the same however many
// are asked for.
//
// First launch: a wavefront takes a run of one beam's logits.  Within a beam the order of the scores is that of the logits, so it keeps the
// n largest logits of the run, one per lane, and the sum of exponentials relative to the largest logit of its first piece.  Second launch:
// a workgroup per prompt adds up the beams' sums and merges their lists by score.
#include "lanes.h"

namespace lrb {
namespace {

__device__ __forceinline__ int lanes_in(uint64_t m) { return __popcll(m); }
// the value of the lane before (lane 0: its own)
__device__ __forceinline__ uint32_t from_lane_before(uint32_t v) { return from_lane<0x138, 0xf>(v, v); }      // wave_shr:1

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

// 2^t in 64 bits for t <= 1000, within 4e-16 of it, two last places (from -1000 down 2^-1000, also for -infinity; a NaN is lost): 2^k 2^g with whole k, |g| <= 1/2,
// and the polynomial through 2^g at the Chebyshev points of degree 10 (3.1e-16; degree 9 has 1.8e-14, degree 7 5.5e-11).  Adding 1.5 * 2^52 leaves k in the low bits.
__device__ __forceinline__ double pow2_64(double t) {
  constexpr double C = 6755399441055744.0;
  const double m = __builtin_fmax(t, -1000.0) + C;
  const double g = __builtin_fmax(t, -1000.0) - (m - C);
  double p = 7.072585949269223e-09;
  p = fma(p, g, 1.0208690299958306e-07);
  p = fma(p, g, 1.321544258792169e-06);
  p = fma(p, g, 1.5252657260200837e-05);
  p = fma(p, g, 0.0001540353044173605);
  p = fma(p, g, 0.0013333558230164974);
  p = fma(p, g, 0.009618129107606888);
  p = fma(p, g, 0.05550410866444772);
  p = fma(p, g, 0.24022650695910097);
  p = fma(p, g, 0.69314718055995);
  p = fma(p, g, 1.0);
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

// The largest value that at least n lanes reach (0: fewer have any), without its lowest 12 bits.
__device__ __forceinline__ uint32_t nth_of_lanes(uint32_t v, int n) {
  uint32_t t = 0;
#pragma unroll
  for (int b = 31; b >= 12; b--) {
    const uint32_t u = t | (1u << b);
    if (lanes_in(__ballot(v >= u)) >= n) t = u;
  }
  return t;
}

// 16 bytes of logits; a row may start on any element
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x4_anywhere __attribute__((ext_vector_type(4), aligned(2)));
template <class T> struct Vec;
template <> struct Vec<uint16_t> {
  static constexpr int N = 8;
  static constexpr uint32_t NONE = 0xff80ff80u;        // two of -infinity
  __device__ static __forceinline__ void floats(u32x4 q, float* f) { unpack8(make_uint4(q[0], q[1], q[2], q[3]), f); }
  __device__ static __forceinline__ float one(const uint16_t* p) { return bf16_bits_to_f32(*p); }
  __device__ static __forceinline__ float element(u32x4 q, int i) {      // (i < 8)
    const uint32_t w = i & 4 ? (i & 2 ? q[3] : q[2]) : (i & 2 ? q[1] : q[0]);
    return __uint_as_float(i & 1 ? w & 0xffff0000u : w << 16);
  }
  __device__ static __forceinline__ u32x4 less(u32x4 q, float by) {
    float f[8];
    floats(q, f);
#pragma unroll
    for (int j = 0; j < 4; j++) q[j] = pack_bf16x2(f[2 * j] - by, f[2 * j + 1] - by);
    return q;
  }
};
template <> struct Vec<float> {
  static constexpr int N = 4;
  static constexpr uint32_t NONE = 0xff800000u;
  __device__ static __forceinline__ void floats(u32x4 q, float* f) {
#pragma unroll
    for (int j = 0; j < 4; j++) f[j] = __uint_as_float(q[j]);
  }
  __device__ static __forceinline__ float one(const float* p) { return *p; }
  __device__ static __forceinline__ float element(u32x4 q, int i) { return __uint_as_float(i & 2 ? (i & 1 ? q[3] : q[2]) : (i & 1 ? q[1] : q[0])); }
  __device__ static __forceinline__ u32x4 less(u32x4 q, float by) {
#pragma unroll
    for (int j = 0; j < 4; j++) q[j] = __float_as_uint(__uint_as_float(q[j]) - by);
    return q;
  }
};

// A wavefront's n largest logits and its sum of exponentials.
struct RunState {
  Best best;
  uint32_t last_hi = 0, last_lo = 0;                   // the n-th of them, 0: there are fewer
  float ref = -INFINITY;                               // what the exponentials refer to
  // Exponents are logit * log2(e) - ref2 with ref2 = ref * log2(e), whose rounding is 2^-53 |ref2|, as that of a logarithm of this size in 64 bits; `far` for
  // |ref| >= 2^20, where logits are made differences to ref first (neighbours' differences are exact, and the others' exponentials 0) and ref2 is 0.
  double sum = 0, ref2 = 0;
  bool far = false;
  bool bad = false;                                    // a NaN was there
  // `most`: the lane's largest of what comes next.  The exponentials refer to the largest logit of the first piece that has any, or of one that is far above it.
  __device__ __forceinline__ void refer(float most) {
    if (__ballot(most > ref + 500.f || (ref == -INFINITY && most > ref)) == 0) return;
    const float top = wave_max(most);
    if (ref > -INFINITY) sum *= pow2_64(((double)ref - top) * LOG2E);
    ref = top;
    far = __builtin_fabsf(ref) >= 1048576.f;
    ref2 = far ? 0.0 : (double)ref * LOG2E;
  }
  // below it no lane's logit is among the row's n largest: at least n lanes have one that reaches it, or the list is full and ends with it, or
  // another run of the row says so (`known`, 0: none did)
  __device__ __forceinline__ uint32_t floor(float most, uint32_t known, int n) const {
    known = max(known, last_hi);
    return known != 0 ? known : nth_of_lanes(most > -INFINITY ? ordered(most + 0.f) : 0, n);
  }
  // a logit per lane; at: its token
  __device__ __forceinline__ void offer(float f, int at, float floor, int n, int lane) {
    uint64_t m = __ballot(f >= floor && f > -INFINITY);
    if (m == 0) return;
    const uint32_t hi = ordered(f + 0.f), lo = ~(uint32_t)at;      // (-0 is 0)
    m &= __ballot(hi > last_hi || (hi == last_hi && lo > last_lo));
    while (m != 0) {
      const int from = __builtin_ctzll(m);
      best.insert(value_of_lane(hi, from), value_of_lane(lo, from), lane);
      last_hi = value_of_lane(best.hi, n - 1);
      last_lo = value_of_lane(best.lo, n - 1);
      m &= ~(1ull << from) & __ballot(hi > last_hi || (hi == last_hi && lo > last_lo));
    }
  }
};

// E: logits per lane and piece.  Bound: vector instructions (71 % of all cycles), 19 for an exponential, most of them in 64 bits, which are as fast as those of 32
// here.  64 prompts of 8 beams, 131072 tokens in bf16: 72 us (134 MB, 1.9 TB/s; without exponentials and candidates 22); one prompt of 4 beams, 32000 tokens: 5.6.
// Every piece asks for the same number of vectors, the next one's before this one is worked on, so that the compiler can count which have arrived:
// behind the last vector it is that one once more.
template <class T, int E>
__global__ __launch_bounds__(256) void beam_runs_kernel(BeamSelect s) {
  constexpr int N = Vec<T>::N, NV = E / N;
  const int lane = threadIdx.x & 63;
  const int item = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int row = item / s.parts, part = item - row * s.parts;
  // the floors of the workgroup's rows: what falls below any run's cannot be among the row's n largest
  __shared__ uint32_t floors[4];
  if (threadIdx.x < 4) floors[threadIdx.x] = 0;
  __syncthreads();
  uint32_t* known = floors + (row - (int)blockIdx.x * 4 / s.parts);
  const bool live = row < s.rows && !(s.done && s.done[row] != 0);
  const T* x = (const T*)s.logits + (int64_t)(live ? row : 0) * s.ld;
  // Runs, pieces and vectors are the same in every row, wherever it starts: rows of the same logits have the same sum, and equal candidates stay equal.
  const int vecs = s.V / N, tail = s.V - vecs * N;
  const int begin = part * s.run, end = min(begin + s.run, vecs);
  const u32x4_anywhere* px = reinterpret_cast<const u32x4_anywhere*>(x);
  u32x4 cur[NV], nxt[NV];
  auto ask = [&](int v0, u32x4 (&v)[NV]) {
#pragma unroll
    for (int j = 0; j < NV; j++) v[j] = px[min(v0 + j * 64 + lane, vecs - 1)];
  };
  auto cut = [&](int v0) {                             // what of `cur` lies behind the run
    if (v0 + 64 * NV > end) {
#pragma unroll
      for (int j = 0; j < NV; j++)
        if (v0 + j * 64 + lane >= end) cur[j] = u32x4{Vec<T>::NONE, Vec<T>::NONE, Vec<T>::NONE, Vec<T>::NONE};
    }
  };
  // the largest logit of every vector, and of them all (a NaN comes through, and comparisons with it are false)
  auto largest = [&](float (&top)[NV]) {
    float most = -INFINITY;
#pragma unroll
    for (int j = 0; j < NV; j++) {
      float f[N];
      Vec<T>::floats(cur[j], f);
      top[j] = f[0];
#pragma unroll
      for (int e = 1; e < N; e++) top[j] = __builtin_elementwise_maximum(top[j], f[e]);
      most = __builtin_elementwise_maximum(most, top[j]);
    }
    return most;
  };
  // all first pieces' floors before any of them is searched
  if (live && begin < end) {
    ask(begin, cur);
    cut(begin);
    float top[NV];
    const float most = largest(top);
    const uint32_t least = nth_of_lanes(most > -INFINITY ? ordered(most + 0.f) : 0, s.n);
    if (lane == 0) __hip_atomic_fetch_max(known, least, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
  }
  __syncthreads();
  if (!live) return;
  RunState st;
  if (part == 0 && tail > 0) {
    const int at = vecs * N + lane;
    const float f = lane < tail ? Vec<T>::one(x + at) : -INFINITY;
    st.bad |= f != f;
    st.refer(f);
    if (st.ref > -INFINITY) st.sum += lane < tail ? pow2_64(((double)f - st.ref) * LOG2E) : 0.0;
    st.offer(f, at, -INFINITY, s.n, lane);
  }
  for (int v0 = begin; v0 < end; v0 += 64 * NV) {
    ask(v0 + 64 * NV, nxt);
    cut(v0);
    float top[NV];
    const float most = largest(top);
    st.bad |= most != most;
    st.refer(most);
    const uint32_t least = st.floor(most, __hip_atomic_load(known, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP), s.n);
    const float floor = least != 0 ? unordered(least) : -INFINITY;
    uint32_t which = 0;                                // vectors that hold candidates
#pragma unroll
    for (int j = 0; j < NV; j++) which |= __ballot(top[j] >= floor && top[j] > -INFINITY) != 0 ? 1u << j : 0u;
    while (which != 0) {
      const int j = __builtin_ctz(which);
      which &= which - 1;
      u32x4 v = cur[0];
      float mine = top[0];
#pragma unroll
      for (int i = 1; i < NV; i++)
        if (i == j) {
          v = cur[i];
          mine = top[i];
        }
      // one lane's vector at a time: a logit of it per lane
      uint64_t m = __ballot(mine >= floor && mine > -INFINITY);
      while (m != 0) {
        const int from = __builtin_ctzll(m);
        m &= m - 1;
        u32x4 w;
#pragma unroll
        for (int i = 0; i < 4; i++) w[i] = value_of_lane(v[i], from);
        const float f = Vec<T>::element(w, lane);
        st.offer(lane < N ? f : -INFINITY, (v0 + j * 64 + from) * N + lane, floor, s.n, lane);
      }
    }
    if (lane == 0) __hip_atomic_fetch_max(known, max(least, st.last_hi), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_WORKGROUP);
    if (st.far) {
#pragma unroll
      for (int j = 0; j < NV; j++) cur[j] = Vec<T>::less(cur[j], st.ref);
    }
    if (st.ref > -INFINITY) {
#pragma unroll
      for (int j = 0; j < NV; j++) {
        float f[N];
        Vec<T>::floats(cur[j], f);
#pragma unroll
        for (int e = 0; e < N; e++) st.sum += pow2_64(fma((double)f[e], LOG2E, -st.ref2));
      }
    }
#pragma unroll
    for (int j = 0; j < NV; j++) cur[j] = nxt[j];
  }
  double sum = wave_sum(st.sum);
  if (__ballot(st.bad) != 0 || !(st.ref < INFINITY)) sum = __builtin_nan("");
  if (lane == 0) {
    s.part_ref[item] = st.ref;
    s.part_sum[item] = sum;
  }
  if (lane < s.n) s.part_key[(int64_t)item * s.n + lane] = make_uint2(st.best.hi, st.best.lo);
}

// One workgroup per prompt.  The n best candidates so far lie in LDS; with up to 256 more of them, a candidate's new place is the number of those
// above it.  Bound: latency, of the first launch's results and of the steps that wait for each other:
// one prompt of 4 beams 4.6 us, 64 of 8 beams 9.0.
__global__ __launch_bounds__(256) void beam_merge_kernel(BeamSelect s) {
  // a candidate's score is (logit - largest logit) - logarithm of the sum + score, in this order: the logits may be far from zero
  __shared__ double log_sum[BEAM_MOST];                // NaN: the beam offers nothing
  __shared__ float largest[BEAM_MOST], score_in[BEAM_MOST];
  __shared__ uint64_t best_score[2][BEAM_MOST + 256];  // (double's order; 0: none)
  __shared__ uint64_t best_at[2][BEAM_MOST + 256];     // order_of: of equal scores the larger is the earlier
  __shared__ uint32_t floors[4];
  __shared__ int added;
  constexpr int AHEAD = 4;                             // candidates of a list that are asked for at once
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int prompt = blockIdx.x, row0 = prompt * s.beams;
  // The runs' lists fall from candidate to candidate, in the order that the merge has: all first ones, then the second ones, until none is added
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
    const float score = w < s.beams ? s.score[row0 + w] : 0.f;
    float top = -INFINITY;
    double sum = 0;
    bool bad = false;
    for (int p0 = 0; in && p0 < s.parts; p0 += 64) {   // four runs of a lane are on their way at once
      float ref[4], high = top;
      double t[4];
#pragma unroll
      for (int j = 0; j < 4; j++) {
        const int p = p0 + 16 * j + sub, q = min(p, s.parts - 1);
        ref[j] = s.part_ref[item + q];
        t[j] = s.part_sum[item + q];
        if (p >= s.parts) ref[j] = -INFINITY, t[j] = 0;
      }
#pragma unroll
      for (int j = 0; j < 4; j++) {
        bad |= !(t[j] == t[j]);
        high = fmaxf(high, ref[j]);
      }
      if (high > -INFINITY) {                          // (the sum so far refers to the largest one; a run without any has 0)
        sum *= pow2_64(((double)top - high) * LOG2E);
#pragma unroll
        for (int j = 0; j < 4; j++) sum += t[j] * pow2_64(((double)ref[j] - high) * LOG2E);
        top = high;
      }
    }
    const float most = row_all(top, [](float a, float b) { return fmaxf(a, b); });
    sum = top > -INFINITY ? sum * pow2_64(((double)top - most) * LOG2E) : 0;
    sum = row_all(sum, [](double a, double b) { return a + b; });
    const int wrong = row_all((int)bad, [](int a, int b) { return a | b; });
    if (sub == 0 && w < s.beams) {
      const bool none = !in || wrong || !(most > -INFINITY) || !(__builtin_fabsf(score) < INFINITY);
      log_sum[w] = none ? __builtin_nan("") : log(sum);
      largest[w] = most;
      score_in[w] = score;
    }
  }
  __syncthreads();
  // the lower beam of the prompt, the larger logit (as `ordered` numbers it), the lower token
  auto order_of = [](int w, uint32_t logit, uint32_t token) { return (uint64_t)(BEAM_MOST - 1 - w) << 52 | (uint64_t)logit << 20 | (0xfffffu - token); };
  int have = 0, side = 0;                              // candidates in best_*[side], the best first
  // a candidate per thread: was one added?
  auto offer = [&](uint64_t score, uint64_t at) {
    bool in;
    if (threadIdx.x == 0) added = 0;
    if (have == s.n) {
      const uint64_t last = best_score[side][s.n - 1];
      in = score > last || (score == last && score != 0 && at > best_at[side][s.n - 1]);
      __syncthreads();
    } else {
      // n of a wavefront's candidates reach its floor: those below the highest of the four are not among the best
      const uint32_t floor = nth_of_lanes((uint32_t)(score >> 32), s.n);
      if (lane == 0) floors[wave] = floor;
      __syncthreads();
      in = score != 0 && (uint32_t)(score >> 32) >= max(max(floors[0], floors[1]), max(floors[2], floors[3]));
    }
    const uint64_t m = __ballot(in);
    int to = 0;
    if (lane == 0 && m != 0) to = atomicAdd(&added, lanes_in(m));
    to = have + __builtin_amdgcn_readfirstlane(to) + __builtin_amdgcn_mbcnt_hi((uint32_t)(m >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)m, 0u));
    if (in) {
      best_score[side][to] = score;
      best_at[side][to] = at;
    }
    __syncthreads();
    const int more = added, all = have + more;
    if (more == 0) return false;
    // sixteen lanes per candidate
    for (int i0 = 0; i0 < all; i0 += 16) {
      const int i = min(i0 + (int)threadIdx.x / 16, all - 1);
      const uint64_t mine = best_score[side][i];
      const uint64_t mine_at = best_at[side][i];
      int place = 0;
      for (int j = threadIdx.x & 15; j < all; j += 16) {
        const uint64_t other = best_score[side][j];
        const uint64_t other_at = best_at[side][j];
        place += other > mine || (other == mine && other_at > mine_at);
      }
      place = row_all(place, [](int a, int b) { return a + b; });
      if ((threadIdx.x & 15) == 0 && i0 + (int)threadIdx.x / 16 < all && place < s.n) {
        best_score[side ^ 1][place] = mine;
        best_at[side ^ 1][place] = mine_at;
      }
    }
    __syncthreads();
    side ^= 1;
    have = min(all, s.n);
    return true;
  };
  for (int l0 = 0; l0 < lists; l0 += 256) {
    const int l = l0 + lane * 4 + wave, w = min(l / s.parts, s.beams - 1);
    const double less = log_sum[w];
    const bool some = l < lists && less == less;
    if (l0 > 0) ask(l);
    auto step = [&](uint2 k) {
      uint64_t score = 0;
      if (some && k.x != 0) score = ordered(((double)unordered(k.x) - largest[w] - less) + score_in[w] + 0.0);
      return offer(score, order_of(w, k.x, ~k.y & 0xfffffu));
    };
    bool more = true;
#pragma unroll 1
    for (int r = 0; more && r < s.n; r++)
      more = step(r == 0 ? key[0] : r == 1 ? key[1] : r == 2 ? key[2] : r == 3 ? key[3] : l < lists ? keys[(int64_t)l * s.n + r] : make_uint2(0, 0));
  }
  if (s.done) {                                        // an ended beam goes on with one token, at its score
    const int w = threadIdx.x;
    uint64_t score = 0;
    if (w < s.beams && s.done[row0 + w] != 0 && __builtin_fabsf(score_in[w]) < INFINITY) score = ordered((double)score_in[w] + 0.0);
    offer(score, order_of(w & (BEAM_MOST - 1), 0, (uint32_t)s.done_token));
  }
  if ((int)threadIdx.x < s.n) {
    const int64_t o = (int64_t)prompt * s.n + threadIdx.x;
    const bool some = (int)threadIdx.x < have;
    const uint64_t at = some ? best_at[side][threadIdx.x] : 0;
    s.parent[o] = some ? row0 + BEAM_MOST - 1 - (int)(at >> 52) : -1;
    s.token[o] = some ? (int)(0xfffffu - (uint32_t)(at & 0xfffffu)) : -1;
    s.score_out[o] = some ? (float)unordered(best_score[side][threadIdx.x]) : -INFINITY;
  }
}

// A run for a wavefront: pieces of 512 logits where those of 2048 are too few for the chip, else as many as give every SIMD four wavefronts.
struct Runs { int elems; int64_t run, parts; };        // run: in vectors of 16 bytes
Runs runs_of(int64_t rows, int64_t V, int dt) {
  const int64_t per_vec = dt == LR_BF16 ? 8 : 4;
  const int elems = rows * ((V + 2047) / 2048) < 1024 ? 8 : 32;
  const int64_t piece = 64 * elems, pieces = V >= piece ? (V + piece - 1) / piece : 1;
  int64_t parts = rows > 0 ? (4096 + rows - 1) / rows : 1;
  if (parts > pieces) parts = pieces;
  const int64_t per = (pieces + parts - 1) / parts;
  return {elems, per * piece / per_vec, (pieces + per - 1) / per};
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
  return (size_t)(rows * runs_of(rows, V, LR_BF16).parts)      // (the same for either type)
         * (sizeof(double) + (size_t)n * sizeof(uint2) + sizeof(float));
}
hipError_t k_beam_select(BeamSelect s, int dt, void* ws, hipStream_t st) {
  const Runs r = runs_of(s.rows, s.V, dt);
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
