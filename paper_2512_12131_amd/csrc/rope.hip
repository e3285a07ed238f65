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
// Angles of far positions (2^31 at most) need all of 64 bits; there the reduction to [-pi/4, pi/4] is exact to 1e-16 with pi / 2 in two parts,
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

// A workgroup writes `rows` rows; its columns' frequencies are formed once, in LDS.
__global__ __launch_bounds__(256) void rope_table_kernel(float* __restrict__ cs, float* __restrict__ sn, int64_t n, int half, int rows,
                                                         FastDiv by_half, int64_t first, double log2_base, double inv_factor,
                                                         double turns, double low, double inv_span, double mscale) {
  extern __shared__ double freq[];
  for (int i = threadIdx.x; i < half; i += 256) {
    const double w = exp2(-log2_base * (double)i / (double)half);
    const double keep = turns > 0.0 ? fmin(1.0, fmax(0.0, (turns * w - low) * inv_span)) : 0.0;
    freq[i] = w * (keep + (1.0 - keep) * inv_factor);
  }
  __syncthreads();
  const int64_t row0 = (int64_t)blockIdx.x * rows;
  const int count = (int)(n - row0 < rows ? n - row0 : rows) * half;
  for (int e = threadIdx.x; e < count; e += 256) {
    const int p = (int)by_half.div((uint32_t)e), i = e - p * half;
    double s, c;
    sincos_f64((double)(first + row0 + p) * freq[i], &s, &c);
    cs[row0 * half + e] = (float)(c * mscale);
    sn[row0 * half + e] = (float)(s * mscale);
  }
}

// ---- rotation ----------------------------------------------------------------------------------------
// One lane's share of a head, a unit: 8 pairs of bf16 (two 16-byte vectors: i and i + rot / 2, or neighbours), or one vector of the
// columns that are copied.  fp32: one pair or one column, since rows may start anywhere.
template <bool INTER>
__device__ __forceinline__ void turn8(const float* a, const float* b, const float* c, const float* s, float* oa, float* ob) {
  if constexpr (INTER) {      // a: pairs 0..3, b: pairs 4..7
#pragma unroll
    for (int i = 0; i < 4; i++) {
      oa[2 * i] = a[2 * i] * c[i] - a[2 * i + 1] * s[i];
      oa[2 * i + 1] = a[2 * i + 1] * c[i] + a[2 * i] * s[i];
      ob[2 * i] = b[2 * i] * c[4 + i] - b[2 * i + 1] * s[4 + i];
      ob[2 * i + 1] = b[2 * i + 1] * c[4 + i] + b[2 * i] * s[4 + i];
    }
  } else {
#pragma unroll
    for (int i = 0; i < 8; i++) {
      oa[i] = a[i] * c[i] - b[i] * s[i];
      ob[i] = b[i] * c[i] + a[i] * s[i];
    }
  }
}
__device__ __forceinline__ void load8f(const float* p, float* v) {
  const float4 a = reinterpret_cast<const float4*>(p)[0], b = reinterpret_cast<const float4*>(p)[1];
  v[0] = a.x; v[1] = a.y; v[2] = a.z; v[3] = a.w; v[4] = b.x; v[5] = b.y; v[6] = b.z; v[7] = b.w;
}

struct RopeArgs {
  const void* x;
  void* out;
  int64_t ldx, ldo, T, table_rows;
  const int32_t* pos;
  const float *cs, *sn;
  int H, hd, rot;
  int nrot, units;        // units of a head that turn, and all of them
  int groups, rows;       // head groups of a row (a lane works on heads g, g + groups, ...); rows of a workgroup
  FastDiv by_units, by_row;
  float sgn;
};

template <typename E, bool INTER, int HPT>
__global__ __launch_bounds__(256) void rope_at_kernel(RopeArgs a) {
  constexpr bool BF = sizeof(E) == 2;
  const int per_row = a.groups * a.units, half = a.rot / 2;
  const int64_t row0 = (int64_t)blockIdx.x * a.rows;
  const int count = (int)(a.T - row0 < a.rows ? a.T - row0 : a.rows) * per_row;
  for (int idx = threadIdx.x; idx < count; idx += 256) {
    const int r = (int)a.by_row.div((uint32_t)idx), rem = idx - r * per_row;
    const int g = (int)a.by_units.div((uint32_t)rem), u = rem - g * a.units;
    const int64_t row = row0 + r;
    const int64_t p = a.pos ? (int64_t)a.pos[row] : row;
    if (p < 0 || p >= a.table_rows) continue;
    const E* x = (const E*)a.x + row * a.ldx;
    E* out = (E*)a.out + row * a.ldo;
    if constexpr (BF) {
      if (u < a.nrot) {
        const int at = INTER ? u * 16 : u * 8, other = INTER ? 8 : half;
        float c[8], s[8];
        load8f(a.cs + p * half + u * 8, c);
        load8f(a.sn + p * half + u * 8, s);
#pragma unroll
        for (int i = 0; i < 8; i++) s[i] *= a.sgn;
        uint4 qa[HPT], qb[HPT];
#pragma unroll
        for (int j = 0; j < HPT; j++) {
          const int h = g + j * a.groups;
          if (h < a.H) {
            qa[j] = *reinterpret_cast<const uint4*>(x + h * a.hd + at);
            qb[j] = *reinterpret_cast<const uint4*>(x + h * a.hd + at + other);
          }
        }
#pragma unroll
        for (int j = 0; j < HPT; j++) {
          const int h = g + j * a.groups;
          if (h < a.H) {
            float va[8], vb[8], oa[8], ob[8];
            unpack8(qa[j], va);
            unpack8(qb[j], vb);
            turn8<INTER>(va, vb, c, s, oa, ob);
            *reinterpret_cast<uint4*>(out + h * a.hd + at) = pack8(oa);
            *reinterpret_cast<uint4*>(out + h * a.hd + at + other) = pack8(ob);
          }
        }
      } else {
        const int at = a.rot + (u - a.nrot) * 8;
        for (int h = g; h < a.H; h += a.groups)
          *reinterpret_cast<uint4*>(out + h * a.hd + at) = *reinterpret_cast<const uint4*>(x + h * a.hd + at);
      }
    } else {
      if (u < a.nrot) {
        const int i0 = INTER ? 2 * u : u, i1 = INTER ? i0 + 1 : u + half;
        const float c = a.cs[p * half + u], s = a.sn[p * half + u] * a.sgn;
        float va[HPT], vb[HPT];
#pragma unroll
        for (int j = 0; j < HPT; j++) {
          const int h = g + j * a.groups;
          if (h < a.H) { va[j] = x[h * a.hd + i0]; vb[j] = x[h * a.hd + i1]; }
        }
#pragma unroll
        for (int j = 0; j < HPT; j++) {
          const int h = g + j * a.groups;
          if (h < a.H) {
            out[h * a.hd + i0] = va[j] * c - vb[j] * s;
            out[h * a.hd + i1] = vb[j] * c + va[j] * s;
          }
        }
      } else {
        const int at = a.rot + u - a.nrot;
        for (int h = g; h < a.H; h += a.groups) out[h * a.hd + at] = x[h * a.hd + at];
      }
    }
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
  int nrot, units;          // of a key or query head, as above
  int groups, vunits, vgroups;    // head groups (keys' and queries' heads in one row of them); vectors of a value head, its groups
  FastDiv by_units, by_vunits, by_tok;
};

constexpr int APPEND_TOKENS = 4;       // a workgroup's: one for each wavefront to look up

// Where the workgroup's tokens go is found once, a token per wavefront: its sequence is the number of boundaries at or before it, 64 of them
// compared at a time.  Then the lanes share out the units of all of them.
template <bool INTER, int HPT>
__global__ __launch_bounds__(256) void kv_append_kernel(AppendArgs a) {
  __shared__ int s_pos[APPEND_TOKENS];
  __shared__ int64_t s_row[APPEND_TOKENS];     // element offset of the token's row in the cache
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int64_t tok0 = (int64_t)blockIdx.x * APPEND_TOKENS;
  const int Hkv = a.c.n_kv_heads, hd = a.c.head_dim;
  {
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
        const int64_t end = a.c.cu_q[before + 1] < a.T ? a.c.cu_q[before + 1] : a.T;
        const int64_t p = (int64_t)a.c.kv_len[before] - (end - t);
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
  const int heads = Hkv + a.H, half = a.rot / 2;
  const int nqk = a.groups * a.units, per_tok = nqk + a.vgroups * a.vunits;
  for (int idx = tid; idx < APPEND_TOKENS * per_tok; idx += 256) {
    const int tl = (int)a.by_tok.div((uint32_t)idx);
    int rem = idx - tl * per_tok;
    const int pos = s_pos[tl];
    if (pos < 0) continue;                     // (also where the call has no such token)
    const int64_t t = tok0 + tl, row = s_row[tl];
    if (rem >= nqk) {                          // values
      rem -= nqk;
      const int g = (int)a.by_vunits.div((uint32_t)rem), at = (rem - g * a.vunits) * 8;
      uint4 w[HPT];
#pragma unroll
      for (int j = 0; j < HPT; j++) {
        const int h = g + j * a.vgroups;
        if (h < Hkv) w[j] = *reinterpret_cast<const uint4*>(a.v + t * a.ldv + h * hd + at);
      }
#pragma unroll
      for (int j = 0; j < HPT; j++) {
        const int h = g + j * a.vgroups;
        if (h < Hkv) *reinterpret_cast<uint4*>(a.c.v + row + h * a.c.head_stride + at) = w[j];
      }
      continue;
    }
    const int g = (int)a.by_units.div((uint32_t)rem), u = rem - g * a.units;
    auto src = [&](int h) { return h < Hkv ? a.k + t * a.ldk + h * hd : a.q + t * a.ldq + (h - Hkv) * hd; };
    auto dst = [&](int h) { return h < Hkv ? a.c.k + row + h * a.c.head_stride : a.q_out + t * a.ldqo + (h - Hkv) * hd; };
    if (u < a.nrot) {
      const int at = INTER ? u * 16 : u * 8, other = INTER ? 8 : half;
      float c[8], s[8];
      load8f(a.cs + (int64_t)pos * half + u * 8, c);
      load8f(a.sn + (int64_t)pos * half + u * 8, s);
      uint4 qa[HPT], qb[HPT];
#pragma unroll
      for (int j = 0; j < HPT; j++) {
        const int h = g + j * a.groups;
        if (h < heads) {
          const uint16_t* p = src(h) + at;
          qa[j] = *reinterpret_cast<const uint4*>(p);
          qb[j] = *reinterpret_cast<const uint4*>(p + other);
        }
      }
#pragma unroll
      for (int j = 0; j < HPT; j++) {
        const int h = g + j * a.groups;
        if (h < heads) {
          float va[8], vb[8], oa[8], ob[8];
          unpack8(qa[j], va);
          unpack8(qb[j], vb);
          turn8<INTER>(va, vb, c, s, oa, ob);
          uint16_t* p = dst(h) + at;
          *reinterpret_cast<uint4*>(p) = pack8(oa);
          *reinterpret_cast<uint4*>(p + other) = pack8(ob);
        }
      }
    } else {
      const int at = a.rot + (u - a.nrot) * 8;
      for (int h = g; h < heads; h += a.groups) *reinterpret_cast<uint4*>(dst(h) + at) = *reinterpret_cast<const uint4*>(src(h) + at);
    }
  }
}

int ceil_div(int64_t a, int64_t b) { return (int)((a + b - 1) / b); }

}  // namespace

hipError_t k_rope_table(float* cs, float* sn, int64_t n, int half, int64_t first, double base, double factor, double context, double low,
                        double high, double mscale, hipStream_t st) {
  int64_t rows = 4096 / half < 1 ? 1 : 4096 / half;
  if ((n + rows - 1) / rows < 1024) rows = n / 1024 < 1 ? 1 : n / 1024;
  hipLaunchKernelGGL(rope_table_kernel, dim3((unsigned)((n + rows - 1) / rows)), dim3(256), half * sizeof(double), st, cs, sn, n, half,
                     (int)rows, FastDiv::of(half), first, log2(base), 1.0 / factor, context / 6.283185307179586477, low, 1.0 / (high - low),
                     mscale);
  return hipGetLastError();
}

hipError_t k_rope_at(const void* x, int64_t ldx, void* out, int64_t ldo, const int32_t* pos, const float* cs, const float* sn,
                     int64_t table_rows, int64_t T, int H, int hd, int rot, int interleaved, int inverse, int dt, hipStream_t st) {
  RopeArgs a;
  a.x = x; a.out = out; a.ldx = ldx; a.ldo = ldo; a.T = T; a.table_rows = table_rows; a.pos = pos; a.cs = cs; a.sn = sn;
  a.H = H; a.hd = hd; a.rot = rot; a.sgn = inverse ? -1.f : 1.f;
  const int vec = dt == LR_BF16 ? 8 : 1;
  a.nrot = rot / 2 / vec;
  a.units = a.nrot + (x == out ? 0 : (hd - rot) / vec);
  auto launch = [&](auto HPTc) {
    constexpr int HPT = decltype(HPTc)::value;
    a.groups = ceil_div(H, HPT);
    const int per_row = a.groups * a.units;
    a.rows = per_row >= 256 ? 1 : 256 / per_row;
    a.by_units = FastDiv::of(a.units);
    a.by_row = FastDiv::of(per_row);
    const dim3 grid((unsigned)((T + a.rows - 1) / a.rows)), block(256);
    if (dt == LR_BF16 && interleaved) hipLaunchKernelGGL((rope_at_kernel<uint16_t, true, HPT>), grid, block, 0, st, a);
    else if (dt == LR_BF16) hipLaunchKernelGGL((rope_at_kernel<uint16_t, false, HPT>), grid, block, 0, st, a);
    else if (interleaved) hipLaunchKernelGGL((rope_at_kernel<float, true, HPT>), grid, block, 0, st, a);
    else hipLaunchKernelGGL((rope_at_kernel<float, false, HPT>), grid, block, 0, st, a);
    return hipGetLastError();
  };
  return launch(std::integral_constant<int, 1>{});
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
  constexpr int HPT = 1;
  a.groups = ceil_div(c.n_kv_heads + H, HPT);
  a.vgroups = ceil_div(c.n_kv_heads, HPT);
  a.by_units = FastDiv::of(a.units);
  a.by_vunits = FastDiv::of(a.vunits);
  a.by_tok = FastDiv::of(a.groups * a.units + a.vgroups * a.vunits);
  const dim3 grid((unsigned)((T + APPEND_TOKENS - 1) / APPEND_TOKENS)), block(256);
  if (interleaved) hipLaunchKernelGGL((kv_append_kernel<true, HPT>), grid, block, 0, st, a);
  else hipLaunchKernelGGL((kv_append_kernel<false, HPT>), grid, block, 0, st, a);
  return hipGetLastError();
}

}  // namespace lrb
