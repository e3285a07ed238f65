// Rotary positions: the tables of the angles, the rotation of rows at given positions, and the keys and values of new tokens
// written into the pages of a cache with the rotation applied on the way.
//
// The pair (a, b) of a head turns by the angle of the token's position: (a c - b s, b c + a s), in 32 bits, rounded once to the
// storage type.  Pairs are (i, i + rot / 2) or, interleaved, (2i, 2i + 1); columns from rot on are left as they are.
#include "common.h"

namespace lrb {
namespace {

// ---- tables ------------------------------------------------------------------------------------------
// cos / sin [n, rot / 2] of (first + p) w_i.  The frequencies w_i = base^(-2i / rot), scaled for long contexts frequency by
// frequency: one that turns at least `high` times over the `context` trained on is kept, one that turns at most `low` times is divided
// by `factor`, linearly in between.
// Angles of far positions (2^31 at most, the caller refuses others) need all of 64 bits; there the reduction to [-pi/4, pi/4] is exact to 1e-16 with pi / 2 in two parts,
// and Taylor's polynomials of degree 13 and 14 are to 2e-14: vector units multiply and add 64 bits as fast as 32.
__device__ __forceinline__ void sincos_f64(double a, double* sn, double* cs) {
  const double k = rint(a * 0.63661977236758134308);
  double r = fma(-k, 1.57079632679489655800, a);
  r = fma(-k, 6.12323399573676603587e-17, r);
  const double z = r * r;
  double s = 1.0 / 6227020800.0, c = -1.0 / 87178291200.0;
  s = fma(s, z, -1.0 / 39916800.0);
  s = fma(s, z, 1.0 / 362880.0);
  s = fma(s, z, -1.0 / 5040.0);
  s = fma(s, z, 1.0 / 120.0);
  s = fma(s, z, -1.0 / 6.0);
  s = fma(s * z, r, r);
  c = fma(c, z, 1.0 / 479001600.0);
  c = fma(c, z, -1.0 / 3628800.0);
  c = fma(c, z, 1.0 / 40320.0);
  c = fma(c, z, -1.0 / 720.0);
  c = fma(c, z, 1.0 / 24.0);
  c = fma(c, z, -0.5);
  c = fma(c, z, 1.0);
  const int q = (int)((int64_t)k & 3);
  const double u = (q & 1) ? c : s, v = (q & 1) ? s : c;
  *sn = (q & 2) ? -u : u;
  *cs = ((q + 1) & 2) ? -v : v;
}

// A lane stays in one column and walks down a workgroup's rows, `step` at a time: the first angle is formed as above, the next ones by turning it by
// step * w (four products of 64 bits; 16 of them are off by some 2^-49).  Bound: the writes.  131072 rows of 64 (67 MB), a call: 20 us with an
// angle of its own for every entry, now 12.
__global__ __launch_bounds__(256) void rope_table_kernel(float* __restrict__ cs, float* __restrict__ sn, int64_t n, int half, int rows,
                                                         int64_t first, double log2_base, double inv_factor, double turns, double low,
                                                         double inv_span, double mscale) {
  const int wide = half < 256 ? half : 256, step = 256 / wide, row = (int)threadIdx.x / wide;
  if (row >= step) return;
  const int64_t row0 = (int64_t)blockIdx.x * rows, end = row0 + rows < n ? row0 + rows : n;
  for (int i = (int)threadIdx.x % wide; i < half; i += 256) {
    double w = exp2(-log2_base * (double)i / (double)half);
    const double keep = turns > 0.0 ? fmin(1.0, fmax(0.0, (turns * w - low) * inv_span)) : 0.0;
    w *= keep + (1.0 - keep) * inv_factor;
    double s, c, ds = 0.0, dc = 1.0;
    sincos_f64((double)(first + row0 + row) * w, &s, &c);
    if (rows > step) sincos_f64((double)step * w, &ds, &dc);
    s *= mscale;
    c *= mscale;
    for (int64_t p = row0 + row; p < end; p += step) {
      cs[p * half + i] = (float)c;
      sn[p * half + i] = (float)s;
      const double t = c * dc - s * ds;
      s = s * dc + c * ds;
      c = t;
    }
  }
}

// ---- rotation ----------------------------------------------------------------------------------------
// One lane's share of a head, a unit: as many pairs as 16 bytes hold elements (two vectors, i and i + rot / 2 or neighbours), or one
// vector of the columns that are copied.  fp32 rows that may start anywhere: one pair or one column.
template <typename E, int VEC> struct Vec;
template <> struct Vec<uint16_t, 8> {
  typedef uint4 T;
  static __device__ __forceinline__ void get(const T& q, float* v) { unpack8(q, v); }
  static __device__ __forceinline__ T put(const float* v) { return pack8(v); }
};
template <> struct Vec<float, 4> {
  typedef float4 T;
  static __device__ __forceinline__ void get(const T& q, float* v) { v[0] = q.x; v[1] = q.y; v[2] = q.z; v[3] = q.w; }
  static __device__ __forceinline__ T put(const float* v) { return make_float4(v[0], v[1], v[2], v[3]); }
};
template <> struct Vec<float, 1> {
  typedef float T;
  static __device__ __forceinline__ void get(const T& q, float* v) { v[0] = q; }
  static __device__ __forceinline__ T put(const float* v) { return v[0]; }
};
// a and b: the first and second elements of VEC pairs, or, interleaved, the first and second half of them
template <int VEC, bool INTER>
__device__ __forceinline__ void turn(const float* a, const float* b, const float* c, const float* s, float* oa, float* ob) {
  if constexpr (INTER && VEC > 1) {
#pragma unroll
    for (int i = 0; i < VEC / 2; i++) {
      oa[2 * i] = a[2 * i] * c[i] - a[2 * i + 1] * s[i];
      oa[2 * i + 1] = a[2 * i + 1] * c[i] + a[2 * i] * s[i];
      ob[2 * i] = b[2 * i] * c[VEC / 2 + i] - b[2 * i + 1] * s[VEC / 2 + i];
      ob[2 * i + 1] = b[2 * i + 1] * c[VEC / 2 + i] + b[2 * i] * s[VEC / 2 + i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < VEC; i++) {
      oa[i] = a[i] * c[i] - b[i] * s[i];
      ob[i] = b[i] * c[i] + a[i] * s[i];
    }
  }
}
template <int VEC>
__device__ __forceinline__ void table_entries(const float* p, float* v) {
  if constexpr (VEC == 1) {
    v[0] = *p;
  } else {
#pragma unroll
    for (int i = 0; i < VEC; i += 4) {
      const float4 q = *reinterpret_cast<const float4*>(p + i);
      v[i] = q.x; v[i + 1] = q.y; v[i + 2] = q.z; v[i + 3] = q.w;
    }
  }
}
// Unit u of a head, x to out.  A lane does one: two heads or four per lane, sharing the table's entries, were slower (16384 tokens of 32 heads 42 us ->
// 51 and 53: the entries are in the nearest cache, and the lanes are fewer).
template <typename E, int VEC, bool INTER>
__device__ __forceinline__ void turn_unit(int u, int rot, const float* cs, const float* sn, float sgn, const E* x, E* out) {
  using V = Vec<E, VEC>;
  const int at = INTER ? u * 2 * VEC : u * VEC, other = INTER ? VEC : rot / 2;
  const typename V::T qa = *reinterpret_cast<const typename V::T*>(x + at), qb = *reinterpret_cast<const typename V::T*>(x + at + other);
  float c[VEC], s[VEC], va[VEC], vb[VEC], oa[VEC], ob[VEC];
  table_entries<VEC>(cs + u * VEC, c);
  table_entries<VEC>(sn + u * VEC, s);
#pragma unroll
  for (int i = 0; i < VEC; i++) s[i] *= sgn;
  V::get(qa, va);
  V::get(qb, vb);
  turn<VEC, INTER>(va, vb, c, s, oa, ob);
  *reinterpret_cast<typename V::T*>(out + at) = V::put(oa);
  *reinterpret_cast<typename V::T*>(out + at + other) = V::put(ob);
}

struct RopeArgs {
  const void* x;
  void* out;
  int64_t ldx, ldo, T, table_rows;
  const int32_t* pos;
  const float *cs, *sn;
  int H, hd, rot;
  int nrot, units;        // units of a head that turn, and all of them
  int rows, parts;        // rows of a workgroup, or workgroups of a row
  FastDiv by_units, by_row, by_parts;
  float sgn;
};

// A pair (a, b) by the angle of its row's position: (a c - b s, b c + a s) in fp32; the transpose, which is the gradient, turns by -s.  Rows of small
// heads share a workgroup.  Bound: memory, 16384 tokens of 32 heads of 128 in bf16 (0.27 GB in and out) 43 us, 6.5 TB/s (some of it stays in the
// 256 MB cache between calls; a copy of 1 GB 5.1).
template <typename E, int VEC, bool INTER>
__global__ __launch_bounds__(256) void rope_at_kernel(RopeArgs a) {
  const uint32_t group = a.by_parts.div(blockIdx.x), idx = (blockIdx.x - group * a.parts) * 256 + threadIdx.x;
  const uint32_t r = a.by_row.div(idx), rem = idx - r * (uint32_t)(a.H * a.units);
  const int64_t row = (int64_t)group * a.rows + r;
  if (r >= (uint32_t)a.rows || row >= a.T) return;
  const int64_t p = a.pos ? (int64_t)a.pos[row] : row;
  if (p < 0 || p >= a.table_rows) return;
  const int h = (int)a.by_units.div(rem), u = (int)rem - h * a.units;
  const E* x = (const E*)a.x + row * a.ldx + h * a.hd;
  E* out = (E*)a.out + row * a.ldo + h * a.hd;
  if (u < a.nrot) {
    turn_unit<E, VEC, INTER>(u, a.rot, a.cs + p * (a.rot / 2), a.sn + p * (a.rot / 2), a.sgn, x, out);
  } else {
    const int at = a.rot + (u - a.nrot) * VEC;
    *reinterpret_cast<typename Vec<E, VEC>::T*>(out + at) = *reinterpret_cast<const typename Vec<E, VEC>::T*>(x + at);
  }
}

// ---- new keys and values into the pages of a cache -----------------------------------------------------
struct AppendArgs {
  KvCache c;
  const uint16_t *k, *v, *q;
  uint16_t* q_out;
  int64_t ldk, ldv, ldq, ldqo, T, table_rows;
  const float *cs, *sn;
  int H, rot;
  int nrot, units, vunits;  // units of a key or query head, as above; vectors of a value head
  int parts;                // workgroups that share a token's units out
  FastDiv by_units, by_vunits, by_tok, by_parts;
};

// Where a workgroup's tokens go is found once, a token per wavefront: its sequence is the number of boundaries at or before it, 64 of them compared
// at a time.  Then the lanes share out the units of all of them.  Bound: memory, 16384 tokens of 32 heads, each with keys and values of its own,
// 162 us (0.81 GB in and out, 5.0 TB/s; a copy of 1 GB 5.1).
template <bool INTER, int TOKENS>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs a) {
  __shared__ int s_pos[TOKENS];
  __shared__ int64_t s_row[TOKENS];            // element offset of the token's row in the cache
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const uint32_t group = a.by_parts.div(blockIdx.x), part = blockIdx.x - group * a.parts;
  const int64_t tok0 = (int64_t)group * TOKENS;
  const int Hkv = a.c.n_kv_heads, hd = a.c.head_dim;
  if (wave < TOKENS) {
    const int64_t t = tok0 + wave;
    int pos = -1;
    int64_t at = 0;
    if (t < a.T) {
      int before = 0;                          // sequences that end at or before t
      for (int i = 0; i < a.c.batch; i += 64) {
        const bool in = i + lane < a.c.batch;
        before += __popcll(__ballot(in && a.c.cu_q[in ? i + lane + 1 : 0] <= t));
      }
      if (before < a.c.batch && a.c.cu_q[before] <= t) {
        // (counted from the sequence's last token, whether or not the call has that)
        const int64_t p = (int64_t)a.c.kv_len[before] - ((int64_t)a.c.cu_q[before + 1] - t);
        if (p >= 0 && p < a.c.capacity && (a.rot == 0 || p < a.table_rows)) {
          const int col = (int)a.c.by_page.div((uint32_t)p);
          const int page = a.c.page_table[before * a.c.table_ld + col];
          if ((uint32_t)page < (uint32_t)a.c.n_pages) {
            pos = (int)p;
            at = page * a.c.page_stride + (p - (int64_t)col * a.c.page_size) * a.c.token_stride;
          }
        }
      }
    }
    if (lane == 0) { s_pos[wave] = pos; s_row[wave] = at; }
  }
  __syncthreads();
  const int nqk = (Hkv + a.H) * a.units, per_tok = nqk + Hkv * a.vunits;
  for (int idx = (int)part * 256 + tid; idx < TOKENS * per_tok; idx += a.parts * 256) {
    const int tl = TOKENS == 1 ? 0 : (int)a.by_tok.div((uint32_t)idx);
    const int rem = idx - tl * per_tok, pos = s_pos[tl];
    if (pos < 0) continue;                     // (also where the call has no such token)
    const int64_t t = tok0 + tl, row = s_row[tl];
    if (rem < nqk) {
      const int h = (int)a.by_units.div((uint32_t)rem), u = rem - h * a.units;
      const uint16_t* x = h < Hkv ? a.k + t * a.ldk + h * hd : a.q + t * a.ldq + (h - Hkv) * hd;
      uint16_t* out = h < Hkv ? a.c.k + row + h * a.c.head_stride : a.q_out + t * a.ldqo + (h - Hkv) * hd;
      if (u < a.nrot) {
        const int64_t at = (int64_t)pos * (a.rot / 2);
        turn_unit<uint16_t, 8, INTER>(u, a.rot, a.cs + at, a.sn + at, 1.f, x, out);
      } else {
        const int at = a.rot + (u - a.nrot) * 8;
        *reinterpret_cast<uint4*>(out + at) = *reinterpret_cast<const uint4*>(x + at);
      }
    } else {                                   // values
      const int h = (int)a.by_vunits.div((uint32_t)(rem - nqk)), at = (rem - nqk - h * a.vunits) * 8;
      *reinterpret_cast<uint4*>(a.c.v + row + h * a.c.head_stride + at) = *reinterpret_cast<const uint4*>(a.v + t * a.ldv + h * hd + at);
    }
  }
}

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

}  // namespace

hipError_t k_rope_table(float* cs, float* sn, int64_t n, int half, int64_t first, double base, double factor, double context, double low,
                        double high, double mscale, hipStream_t st) {
  const int wide = half < 256 ? half : 256, step = 256 / wide;
  // 2048 workgroups, of 16 steps at most while that is a grid
  int64_t rows = (n + 2047) / 2048;
  rows = (rows + step - 1) / step * step;
  if (rows > 16 * step && (n + 16 * step - 1) / (16 * step) < (1 << 22)) rows = 16 * step;
  hipLaunchKernelGGL(rope_table_kernel, dim3((unsigned)((n + rows - 1) / rows)), dim3(256), 0, st, cs, sn, n, half, (int)rows, first, log2(base),
                     1.0 / factor, context / 6.283185307179586477, low, 1.0 / (high - low), mscale);
  return hipGetLastError();
}

hipError_t k_rope_at(const void* x, int64_t ldx, void* out, int64_t ldo, const int32_t* pos, const float* cs, const float* sn,
                     int64_t table_rows, int64_t T, int H, int hd, int rot, int interleaved, int inverse, int dt, hipStream_t st) {
  RopeArgs a;
  a.x = x; a.out = out; a.ldx = ldx; a.ldo = ldo; a.T = T; a.table_rows = table_rows; a.pos = pos; a.cs = cs; a.sn = sn;
  a.H = H; a.hd = hd; a.rot = rot; a.sgn = inverse ? -1.f : 1.f;
  // fp32 in vectors of four where rows, heads and the two halves of the pairs start on 16 bytes
  const bool whole = (((uintptr_t)x | (uintptr_t)out | (uintptr_t)cs | (uintptr_t)sn) & 15) == 0 && (ldx | ldo | hd) % 4 == 0 && rot % 8 == 0;
  const int vec = dt == LR_BF16 ? 8 : whole ? 4 : 1;
  a.nrot = rot / 2 / vec;
  a.units = a.nrot + (x == out ? 0 : (hd - rot) / vec);
  const int per_row = H * a.units;
  a.rows = per_row >= 256 ? 1 : 256 / per_row;
  a.parts = ceil_div(per_row, 256);
  a.by_units = FastDiv::of(a.units);
  a.by_row = FastDiv::of(per_row);
  a.by_parts = FastDiv::of(a.parts);
  const int64_t groups = (T + a.rows - 1) / a.rows * a.parts;
  if (groups >= (int64_t)1 << 24) return hipErrorNotSupported;      // 2^32 lanes
  const dim3 grid((unsigned)groups), block(256);
  if (dt == LR_BF16 && interleaved) hipLaunchKernelGGL((rope_at_kernel<uint16_t, 8, true>), grid, block, 0, st, a);
  else if (dt == LR_BF16) hipLaunchKernelGGL((rope_at_kernel<uint16_t, 8, false>), grid, block, 0, st, a);
  else if (whole && interleaved) hipLaunchKernelGGL((rope_at_kernel<float, 4, true>), grid, block, 0, st, a);
  else if (whole) hipLaunchKernelGGL((rope_at_kernel<float, 4, false>), grid, block, 0, st, a);
  else if (interleaved) hipLaunchKernelGGL((rope_at_kernel<float, 1, true>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((rope_at_kernel<float, 1, false>), grid, block, 0, st, a);
  return hipGetLastError();
}

hipError_t k_kv_append(const KvCache& c, const void* k, int64_t ldk, const void* v, int64_t ldv, const void* q, int64_t ldq, void* q_out,
                       int64_t ldqo, int64_t T, int H, const float* cs, const float* sn, int64_t table_rows, int rot, int interleaved,
                       hipStream_t st) {
  AppendArgs a;
  a.c = c; a.k = (const uint16_t*)k; a.v = (const uint16_t*)v; a.q = (const uint16_t*)q; a.q_out = (uint16_t*)q_out;
  a.ldk = ldk; a.ldv = ldv; a.ldq = ldq; a.ldqo = ldqo; a.T = T; a.table_rows = table_rows; a.cs = cs; a.sn = sn; a.H = H; a.rot = rot;
  a.nrot = rot / 16;
  a.units = a.nrot + (c.head_dim - rot) / 8;
  a.vunits = c.head_dim / 8;
  const int per_tok = (c.n_kv_heads + H) * a.units + c.n_kv_heads * a.vunits;
  // Few tokens: as many workgroups to each as its units fill, so that a lane has one; else four tokens to a workgroup, found side by side.
  const bool few = T * per_tok <= 256 * 1024;
  a.parts = few ? ceil_div(per_tok, 256) : 1;
  a.by_units = FastDiv::of(a.units);
  a.by_vunits = FastDiv::of(a.vunits);
  a.by_tok = FastDiv::of(per_tok);
  a.by_parts = FastDiv::of(a.parts);
  const dim3 grid((unsigned)(few ? T * a.parts : (T + 3) / 4)), block(256);
  if (few && interleaved) hipLaunchKernelGGL((kv_append_kernel<true, 1>), grid, block, 0, st, a);
  else if (few) hipLaunchKernelGGL((kv_append_kernel<false, 1>), grid, block, 0, st, a);
  else if (interleaved) hipLaunchKernelGGL((kv_append_kernel<true, 4>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((kv_append_kernel<false, 4>), grid, block, 0, st, a);
  return hipGetLastError();
}

}  // namespace lrb
