// Causal attention of each sequence's new tokens over its pages of a key / value cache, heads of 128, bf16 in / fp32 softmax, for gfx950.
//
// Rows.  A sequence's n new tokens and the grp query heads that share a key / value head are n * grp rows against the same keys; row r is
// token r / grp, head r % grp.  Up to 32 rows (decoding: single tokens, a few of them) are one narrow item of work, more are wide
// items of 128 rows:
//   narrow   a workgroup's four wavefronts take a quarter of the keys each, with all 32 rows, through LDS rings of their own and no barrier
//            before the end, where they join their sums.  Bound by memory: every key and value is read once (64 single tokens over 4600 keys on
//            average, 32 / 8 heads, 1.2 GB: 193 us, 6.2 TB/s).
//   wide     the four wavefronts take 32 rows each, keys and values pass through LDS in tiles of 64 for all of them.  Bound by the matrix
//            and vector units (4 x 2048 tokens over 8192 keys: 0.93 - 0.98 ms, 0.98 - 1.03 PFLOP/s, matrix units busy for 55 % of the cycles at
//            the 1.7 GHz that the power limit leaves).
// Both compute S^T = K Q^T and O^T += V^T P^T on 32 x 32 x 16 MFMAs with the running maximum and sum of a softmax (one lane column per row),
// as attention.hip does.
//
// Keys.  Nothing but the lists knows how long sequences are, and they stay on the device.  So every workgroup adds the work of all
// sequences up by itself (64 of them at a time, one per lane), and sequences are cut into splits of equal length such that all of them
// together are some rounds of the chip; a second kernel joins what was split, in the order of the splits (4 - 8 us).  No atomics: the same
// lists give the same bits.  A workgroup's way in (lists, search, page numbers, first keys: loads that wait for each other) is 4 - 5 us.
//
// Pages.  Eight keys that start at a multiple of eight lie in one page.  A lane looks one such group up and keeps its place in the cache in
// units of 16 bytes; 64 groups (512 keys) are a window, the next one's page numbers are asked for while this one is worked on.  The place
// becomes the base of a buffer descriptor that ends with the last key: rows past it, and pages that are none, arrive as zeros.
#include <algorithm>
#include <cmath>

#include "attn_tile.h"

namespace lrb {
namespace {

constexpr int R_NARROW = 32, R_WIDE = 128;
constexpr int MIN_SPLIT = 2;                      // 64-key tiles of a split: 32 keys for each wavefront of a narrow item
constexpr uint32_t PLACES = 512;                  // workgroups that the chip holds at once
constexpr int ROUNDS = 2048;                      // splits that all the work is cut into at most, four for each place on the chip
constexpr uint32_t RUN = 16;                      // blocks of rows that read the same keys on one XCD at a time
constexpr int LDS_JOIN_LD = 132;                  // floats of a row of sums in LDS
constexpr int LDS_BYTES = 4 * R_NARROW * LDS_JOIN_LD * 4 + 1024;
static_assert(LDS_BYTES >= 4 * TILE_BYTES && LDS_BYTES <= 80 * 1024, "two workgroups share a CU");

constexpr int AHEAD = 4;                          // MFMAs that their LDS operands are read ahead of

struct PagedArgs {
  KvCache c;
  const uint16_t* q;
  uint16_t* o;
  float* lse;
  float* part_o;          // [part_rows][128] unnormalised sums of splits
  float2* part_ml;        // their maximum and sum
  uint32_t part_rows;
  int64_t ldq, ldo;
  int T, H, grp, runs;          // runs: consecutive items on one XCD
  FastDiv by_grp;
  float scale;
};

// The arguments once more, from where they are: what only the way in or out needs does not hold scalar registers in between (a hundred are too
// few for everything, and those that do not fit would be read back lane by lane inside the loops).
typedef const __attribute__((address_space(4))) PagedArgs* ArgPtr;
__device__ __forceinline__ ArgPtr args_again() {
  ArgPtr p = (ArgPtr)__builtin_amdgcn_kernarg_segment_ptr();
  asm volatile("" : "+s"(p));
  return p;
}
__device__ __forceinline__ uint32_t div_by(uint32_t n, uint32_t mul, uint32_t shift) { return (uint32_t)(((uint64_t)n * mul) >> shift); }

// The running maximum of a row that has seen no key: finite, so that no difference of two of them is undefined, and below the score of any
// logit that the library takes (2^26 in magnitude, at factors c from 2^-100 on).
__device__ __forceinline__ float no_score(float c) { return -3.0e38f / fmaxf(c, 1.f); }

// ---- the split of the work ------------------------------------------------------------------------------
__device__ __forceinline__ int uni(int x) { return __builtin_amdgcn_readfirstlane(x); }
// The lane moves of an inclusive scan in the vector unit (a shuffle goes through LDS: eighteen of them were 1.5 us on the way in).
template <class F>
__device__ __forceinline__ void down_the_lanes(F&& step) {
  using std::integral_constant;
  using All = integral_constant<int, 0xf>;
  step(integral_constant<int, 0x111>{}, All{});      // from 1, 2, 4, 8 lanes down within a row of 16
  step(integral_constant<int, 0x112>{}, All{});
  step(integral_constant<int, 0x114>{}, All{});
  step(integral_constant<int, 0x118>{}, All{});
  step(integral_constant<int, 0x142>{}, integral_constant<int, 0xa>{});   // a row's last lane to the next row: rows 1 and 3
  step(integral_constant<int, 0x143>{}, integral_constant<int, 0xc>{});   // lane 31 to rows 2 and 3
}
// Inclusive sum over the lanes.
__device__ __forceinline__ uint32_t wave_scan(uint32_t x) {
  down_the_lanes([&](auto Ctrl, auto Rows) {
    x += (uint32_t)__builtin_amdgcn_update_dpp(0, (int)x, decltype(Ctrl)::value, decltype(Rows)::value, 0xf, false);
  });
  return x;
}
__device__ __forceinline__ uint32_t last_lane(uint32_t x) { return __builtin_amdgcn_readlane(x, 63); }

struct Seq {              // of one sequence
  int tok0, n, kv;        // first token, new tokens and keys with them: of the tokens that the call has
  int keys, tiles;        // keys that its last token sees, in 64-key tiles (at least one)
  int rows, blocks;       // rows per key / value head and items of them
};
__device__ __forceinline__ Seq load_seq(const PagedArgs& a, int b) {
  Seq s;
  const int c0 = a.c.cu_q[b], c1 = a.c.cu_q[b + 1];
  s.kv = max(a.c.kv_len[b], 0) - max(max(c1, 0) - a.T, 0);      // (without those that are not there)
  s.tok0 = min(max(c0, 0), a.T);
  s.n = max(min(max(c1, 0), a.T) - s.tok0, 0);
  s.keys = (int)min((int64_t)max(s.kv, 0), a.c.capacity);
  s.tiles = max((s.keys + KT - 1) / KT, 1);
  s.rows = s.n * a.grp;                          // (below 2^31: T * H is)
  s.blocks = s.rows <= R_NARROW ? (s.rows > 0) : (s.rows + R_WIDE - 1) / R_WIDE;
  return s;
}
// 64-key tiles of a split, from w, the number of them in all items.
//   narrow  w / ROUNDS, but more than sqrt(w / 64): a split's way in and out costs as much as some tiles, so splits should grow with the work: s
//           splits save w (1 - 1 / s) and cost s.  While w is few times PLACES, w / PLACES, so that every item finds a place on the chip at
//           once (one sequence of 4096 keys 12.4 -> 10.6 us, 8 of 2000 20.4 -> 16.8, one of 16384 20.1 -> 18.0).
//   wide    w / PLACES (of little work half of the places, a CU each): more splits than places save nothing.  And no less than
//           sqrt(x / 6150), x the tiles times their rows: len tiles take len * 1.6
//           us, and x / len rows of sums 0.26 ns each on their way through memory.  A sequence of two of the latter, or of three tiles, is not
//           split, since the join takes some us by itself.  (us, against the narrow rule for both: a prompt of 777 tokens 31.0 -> 26.9, of
//           2048 74 -> 58, 512 tokens over 8192 keys 97 -> 87, over 32768 314 -> 284, 6 chunks of up to 256
//           tokens beside 18 single ones over up to 4096 keys, the mixed batch below, 101 -> 93.  Four tiles split in two: 10
//           tokens over 250 keys 12.7 -> 11.3; three: the same within 1.5 %, 6 batches of up to 180 keys.)
struct SplitLen { uint32_t narrow, wide, whole; };      // whole: wide sequences of up to so many tiles are not split
// Sum over the lanes, in an order of its own: both kernels get the same bits.  (Products and sums are rounded one by one wherever this is inlined.)
__device__ __forceinline__ float lanes_sum(float x) {
  auto step = [&](auto Ctrl, auto Rows) {
    constexpr int ctrl = decltype(Ctrl)::value, rows = decltype(Rows)::value;
    x = __fadd_rn(x, __uint_as_float(__builtin_amdgcn_update_dpp(0, (int)__float_as_uint(x), ctrl, rows, 0xf, false)));
  };
  down_the_lanes(step);
  return __uint_as_float(last_lane(__float_as_uint(x)));
}
// first: of the lane's sequence among the first 64, loaded already.
__device__ __forceinline__ SplitLen split_len(const PagedArgs& a, const Seq& first) {
  const int lane = threadIdx.x & 63;
  float w = 0.f, x = 0.f;
  for (int b0 = 0; b0 < a.c.batch; b0 += 64) {
    float tiles = 0.f, rows = 0.f;
    if (b0 + lane < a.c.batch) {
      const Seq s = b0 == 0 ? first : load_seq(a, b0 + lane);
      tiles = __fmul_rn((float)s.blocks, (float)s.tiles);
      rows = s.rows > R_NARROW ? __fmul_rn((float)s.rows, (float)s.tiles) : 0.f;
    }
    w = __fadd_rn(w, lanes_sum(tiles));
    if (__builtin_amdgcn_ballot_w64(rows > 0.f)) x = __fadd_rn(x, lanes_sum(rows));
  }
  w = __fmul_rn(w, (float)a.c.n_kv_heads);
  x = __fmul_rn(x, (float)a.c.n_kv_heads);
  auto part = [&](float n) { return (uint32_t)uni((int)ceilf(fminf(__fmul_rn(w, 1.f / n), 1e9f))); };      // (n: a power of two)
  auto root = [&](float y, float f) { return (uint32_t)uni((int)__builtin_amdgcn_sqrtf(__fmul_rn(y, f))) + 1; };
  const float places = PLACES;
  const uint32_t narrow = w <= 4.f * places ? part(places) : max(part(ROUNDS), root(w, 1.f / 64.f));
  const uint32_t traffic = max(root(x, 1.f / 6150.f), (uint32_t)MIN_SPLIT), fill = max(part(places), min(part(places / 2), 8u));
  return SplitLen{max(narrow, (uint32_t)MIN_SPLIT), max(fill, traffic), max(2 * root(x, 1.f / 6150.f), 3u)};
}
// (rounded to the nearer number, wide ones' up from a quarter, since the longest item decides: the mixed batch 97 -> 92 us, 16 chunks of up to 256
// tokens beside 16 single ones 204 either way; as even as they can be)
__device__ __forceinline__ uint32_t splits_of(const Seq& s, const SplitLen& l) {
  const bool wide = s.rows > R_NARROW;
  const uint32_t len = wide ? l.wide : l.narrow, n = ((uint32_t)s.tiles + (wide ? len * 3 / 4 : len / 2)) / len;
  return wide && (uint32_t)s.tiles <= l.whole ? 1u : max(n, 1u);
}
// rows of sums that a sequence keeps: [key / value head][split][row]
__device__ __forceinline__ uint32_t part_rows_of(const PagedArgs& a, const Seq& s, uint32_t splits) {
  return splits > 1 ? (uint32_t)a.c.n_kv_heads * splits * (uint32_t)s.rows : 0;
}

// ---- pages ----------------------------------------------------------------------------------------------
// Of the 64 groups of one window: place, and bytes from there on that are read (0: none).
struct Pages {
  uint32_t place, bytes;
};
struct PageSource {
  const int32_t* row;     // of the page table
  int end;                // keys that are read end here
  uint32_t head;          // of the key / value head, in units of 16 bytes
  int* spot;              // in LDS, the wavefront's own: the next window's page numbers
};
constexpr int SPOTS = 4 * TILE_BYTES;      // behind the tiles, 256 bytes for a wavefront
static_assert(SPOTS + 4 * 256 <= LDS_BYTES, "page numbers behind the tiles");
__device__ __forceinline__ int ask_pages(ArgPtr a, const PageSource& p, int w, int lane) {
  const uint32_t key = (uint32_t)w * 512u + (uint32_t)lane * 8u;
  return key < (uint32_t)p.end ? p.row[div_by(key, a->c.by_page.mul, a->c.by_page.shift)] : -1;
}
// ... into the spot, on the way while others are worked on.  A load into registers would not do: the compiler waits for it where the loop comes round,
// and so for all tiles' loads before it (a prompt of 2048 tokens 57.5 -> 53.8 us without, 64 single tokens over 1000 keys 47.1 -> 45.5, at the time of
// a maximum in steps).
__device__ __forceinline__ void ask_ahead(ArgPtr a, const PageSource& p, int w, int lane) {
  const uint32_t col = div_by((uint32_t)w * 512u + (uint32_t)lane * 8u, a->c.by_page.mul, a->c.by_page.shift);
  const uint32_t cols = div_by((uint32_t)p.end - 1u, a->c.by_page.mul, a->c.by_page.shift) + 1u;
  const uint64_t row = (uint64_t)(uintptr_t)p.row;
  lds_dma4_at(rsrc_t{(uint32_t)row, (uint32_t)(row >> 32), cols * 4u, 0x00020000u}, (uint32_t)(uintptr_t)LRB_LDS_PTR(p.spot), col * 4u);
}
__device__ __forceinline__ void places(ArgPtr a, Pages& pg, int raw, const PageSource& p, int w, int lane) {
  const uint32_t key = (uint32_t)w * 512u + (uint32_t)lane * 8u, row = (uint32_t)(a->c.token_stride >> 3);
  const uint32_t in = key - div_by(key, a->c.by_page.mul, a->c.by_page.shift) * (uint32_t)a->c.page_size;
  pg.place = (uint32_t)((uint64_t)(uint32_t)raw * (uint64_t)(a->c.page_stride >> 3) + (uint64_t)in * row) + p.head;
  const int rows = min(p.end - (int)key, 8);
  pg.bytes = (uint32_t)raw < (uint32_t)a->c.n_pages && rows > 0 ? (uint32_t)(rows - 1) * row * 16u + 256u : 0u;
}
// Before the loads of tile t, TILES of them to a window: the next window where t is its first one; its page numbers are asked for half a window ahead, and
// have landed by now, since the loop waits for younger loads.
template <int TILES>
__device__ __forceinline__ void next_window(Pages& pg, const PageSource& p, int t, int lane) {
  Pages n = pg;
  if ((t & (TILES - 1)) == 0) places(args_again(), n, p.spot[lane], p, t / TILES, lane);
  else if ((t & (TILES - 1)) == TILES / 2) ask_ahead(args_again(), p, t / TILES + 1, lane);
  pg = n;
}
template <int TILES>
__device__ __forceinline__ void first_window(ArgPtr a, Pages& pg, const PageSource& p, int t, int lane) {
  const int raw = ask_pages(a, p, t / TILES, lane);
  p.spot[lane] = ask_pages(a, p, t / TILES + 1, lane);
  places(a, pg, raw, p, t / TILES, lane);
}
// Descriptors of a group's keys and values: the same place in both.
struct Group { uint64_t at; uint32_t bytes; };
// A vector write of a scalar needs five wait states before a load's descriptor has it, and the compiler does not see the loads: asked for right before
// them, a group waits (the machine code is checked for it).
__device__ __forceinline__ Group group(const Pages& pg, int g) {
  const uint32_t place = __builtin_amdgcn_readlane(pg.place, g & 63);
  uint32_t bytes = __builtin_amdgcn_readlane(pg.bytes, g & 63);
  asm volatile("s_nop 4" : "+s"(bytes));
  return Group{(uint64_t)place << 4, bytes};
}
__device__ __forceinline__ rsrc_t group_rsrc(const Group& g, const uint16_t* base) {
  const uint64_t addr = (uint64_t)(uintptr_t)base + g.at;
  return rsrc_t{(uint32_t)addr, (uint32_t)(addr >> 32), g.bytes, 0x00020000u};
}

// For long runs of tiles: the groups' addresses in one of the caches, so that a descriptor is three lanes' values and nothing else (24 scalar
// instructions less per tile and wavefront than from places: a wavefront that is alone on its SIMD is bound by how many instructions it issues).
// Asked for a slot of other work before the load, a descriptor does not have to wait (no SETTLE; the machine code is checked for either).
struct Spots { uint32_t lo, hi, bytes; };
__device__ __forceinline__ Spots spots(const Pages& pg, const uint16_t* base) {
  const uint64_t at = (uint64_t)(uintptr_t)base + ((uint64_t)pg.place << 4);
  return Spots{(uint32_t)at, (uint32_t)(at >> 32), pg.bytes};
}
template <bool SETTLE>
__device__ __forceinline__ rsrc_t spot_rsrc(const Spots& s, int g) {
  uint32_t lo = __builtin_amdgcn_readlane(s.lo, g & 63), hi = __builtin_amdgcn_readlane(s.hi, g & 63);
  uint32_t bytes = __builtin_amdgcn_readlane(s.bytes, g & 63);
  if constexpr (SETTLE) asm volatile("s_nop 4" : "+s"(lo), "+s"(hi), "+s"(bytes));
  return rsrc_t{lo, hi, bytes, 0x00020000u};
}
// lds_dma_at a fixed distance from an address
template <uint32_t OFF>
__device__ __forceinline__ void lds_dma_from(rsrc_t rs, uint32_t lds, uint32_t voff) {
  asm volatile("s_add_u32 m0, %0, %1\n\ts_nop 0\n\tbuffer_load_dwordx4 %2, %3, 0 offen lds" ::"s"(lds), "i"(OFF), "v"(voff), "s"(rs) : "m0", "scc", "memory");
}

// ---- one wavefront's share of a tile: 32 rows, NB blocks of 32 keys ------------------------------------------
struct Rows {
  f32x16 o[4];            // O^T: column = row of the wavefront
  float m, l;             // running maximum; sum of this lane's keys
};
__device__ __forceinline__ void rows_init(Rows& s, float c) {
#pragma unroll
  for (int hb = 0; hb < 4; hb++)
#pragma unroll
    for (int e = 0; e < 16; e++) s.o[hb][e] = 0.f;
  s.m = no_score(c);
  s.l = 0.f;
}
// queries: lane's row r in the B operand layout
__device__ __forceinline__ void load_queries(ArgPtr a, bf16x8 (&qf)[8], const Seq& s, int kvh, int r, int lane) {
  const bool ok = r < s.rows;
  const int tok = ok ? (int)div_by((uint32_t)r, a->by_grp.mul, a->by_grp.shift) : 0, h = ok ? r - tok * a->grp : 0;
  const uint16_t* p = a->q + (int64_t)(s.tok0 + tok) * a->ldq + (kvh * a->grp + h) * HD + (lane >> 5) * 8;
#pragma unroll
  for (int ks = 0; ks < 8; ks++)
    qf[ks] = __builtin_bit_cast(bf16x8, ok ? *reinterpret_cast<const uint4*>(p + ks * 16) : make_uint4(0, 0, 0, 0));
}
// keys that row r sees
__device__ __forceinline__ int row_limit(ArgPtr a, const Seq& s, int r) {
  const int64_t lim = (int64_t)s.kv - s.n + (int)div_by((uint32_t)min(r, s.rows - 1), a->by_grp.mul, a->by_grp.shift) + 1;
  return (int)min(max(lim, (int64_t)0), (int64_t)s.keys);
}

template <int NB>
__device__ __forceinline__ void scores(f32x16 (&st)[NB], const bf16x8 (&qf)[8], const unsigned char* sK, int lane) {
  constexpr f32x16 zero = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  bf16x8 fr[AHEAD];       // operands read ahead, slot i in fr[i % AHEAD]
  auto read = [&](int i) { return swz_row_frag(sK, i % NB * 32, i / NB, lane); };
#pragma unroll
  for (int i = 0; i < AHEAD; i++) fr[i] = read(i);
#pragma unroll
  for (int i = 0; i < 8 * NB; i++) {
    st[i % NB] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[i % AHEAD], qf[i / NB], i < NB ? zero : st[i % NB], 0, 0, 0);
    if (i + AHEAD < 8 * NB) fr[i % AHEAD] = read(i + AHEAD);
    __builtin_amdgcn_sched_barrier(0);
  }
}
// Keys from the row's limit on: minus infinity.
template <int NB>
__device__ __forceinline__ void mask(f32x16 (&st)[NB], int lim, int lane) {
  lim -= 4 * (lane >> 5);
#pragma unroll
  for (int nb = 0; nb < NB; nb++)
#pragma unroll
    for (int e = 0; e < 16; e++) st[nb][e] = nb * 32 + acc_row(e, 0) >= lim ? -INFINITY : st[nb][e];
}
// Probabilities from scores, as bf16 operands (half a step, 2^-9 relative on average, is what their product with V on the matrix cores costs; the
// sum adds them unrounded).  Exponents refer to the maximum of all scores so far, so that a row's largest probability is 1, which bf16 holds: a
// maximum that only follows in steps of 2^8 saves wide items rescalings (4 x 2048 tokens over 8192 keys 928 -> 890 us, a prompt of 2048 57 -> 53), but
// rounds the probability that counts most (error of o 0.0019 -> 0.0023 of its RMS, of which 0.0017 is its own rounding).
template <int NB>
__device__ __forceinline__ void softmax(Rows& s, f32x16 (&st)[NB], bf16x8 (&pf)[NB * 2], float c) {
  float mx = st[0][0];
#pragma unroll
  for (int nb = 0; nb < NB; nb++)
#pragma unroll
    for (int e = 0; e < 16; e++) mx = fmaxf(mx, st[nb][e]);
  const float mn = fmaxf(s.m, half_max(mx)), alpha = fast_exp2((s.m - mn) * c), mc = mn * c;
  s.m = mn;
  float sum = 0.f;
#pragma unroll
  for (int nb = 0; nb < NB; nb++)
#pragma unroll
    for (int e = 0; e < 16; e++) {
      st[nb][e] = fast_exp2(fmaf(st[nb][e], c, -mc));
      sum += st[nb][e];
    }
  s.l = s.l * alpha + sum;
#pragma unroll
  for (int t = 0; t < NB * 2; t++) pf[t] = pack_acc_half(st[t >> 1], t & 1);
  if (__builtin_amdgcn_ballot_w64(alpha != 1.f) != 0) {
#pragma unroll
    for (int hb = 0; hb < 4; hb++)
#pragma unroll
      for (int e = 0; e < 16; e++) s.o[hb][e] *= alpha;
  }
}
template <int NB>
__device__ __forceinline__ void output(Rows& s, const bf16x8 (&pf)[NB * 2], const unsigned char* sV, int lane) {
  bf16x8 fr[AHEAD];
  auto read = [&](int i) { return swz_tr_frag(sV, (i >> 2) * 16, (i & 3) * 32, lane); };
#pragma unroll
  for (int i = 0; i < AHEAD; i++) fr[i] = read(i);
#pragma unroll
  for (int i = 0; i < 8 * NB; i++) {
    s.o[i & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[i % AHEAD], pf[i >> 2], s.o[i & 3], 0, 0, 0);
    if (i + AHEAD < 8 * NB) fr[i % AHEAD] = read(i + AHEAD);
    __builtin_amdgcn_sched_barrier(0);
  }
}
// A tile with keys that some rows must not see: there 0 * infinity and 0 * NaN would carry a later token's value into earlier rows.  Values
// that are no numbers are taken out of the tile in LDS (16 bytes per lane and step, `bytes` of it from `at` on), and in the end added to the rows
// that see them.
__device__ __forceinline__ bool take_out(unsigned char* at, int bytes, int lane) {
  uint32_t top = 0;
  typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));
  auto high = [&](uint32_t w) {
    const u16x2 x = __builtin_elementwise_max(__builtin_bit_cast(u16x2, top), __builtin_bit_cast(u16x2, w & 0x7fff7fffu));
    top = __builtin_bit_cast(uint32_t, x);
  };
  for (int i = lane * 16; i < bytes; i += 1024) {
    const uint4 q = *reinterpret_cast<const uint4*>(at + i);
    high(q.x); high(q.y); high(q.z); high(q.w);
  }
  const bool bad = (top & 0xffffu) >= 0x7f80u || (top >> 16) >= 0x7f80u;
  if (bad) {
#pragma unroll 1
    for (int i = lane * 16; i < bytes; i += 1024)
#pragma unroll 1
      for (int k = 0; k < 16; k += 2) {
        uint16_t* x = reinterpret_cast<uint16_t*>(at + i + k);
        if ((*x & 0x7f80u) == 0x7f80u) *x = 0;
      }
  }
  return __builtin_amdgcn_ballot_w64(bad) != 0;
}
__device__ __forceinline__ void put_back(Rows& s, const int32_t* table, int kvh, int k0, int k1, int lim, int lane) {
  const ArgPtr a = args_again();
#pragma unroll 1
  for (int k = k0; k < k1; k++) {
    const int col = (int)div_by((uint32_t)k, a->c.by_page.mul, a->c.by_page.shift), page = table[col];
    if ((uint32_t)page >= (uint32_t)a->c.n_pages) continue;
    const uint16_t* p = a->c.v + page * a->c.page_stride + (int64_t)(k - col * a->c.page_size) * a->c.token_stride + kvh * a->c.head_stride + 4 * (lane >> 5);
    auto seen = [&](uint32_t x) { return (x & 0x7f80u) == 0x7f80u && k < lim ? bf16_bits_to_f32(x) : 0.f; };
#pragma unroll
    for (int hb = 0; hb < 4; hb++)
#pragma unroll
      for (int g4 = 0; g4 < 4; g4++) {
        const uint2 w = *reinterpret_cast<const uint2*>(p + hb * 32 + 8 * g4);
        s.o[hb][g4 * 4] += seen(w.x & 0xffffu);
        s.o[hb][g4 * 4 + 1] += seen(w.x >> 16);
        s.o[hb][g4 * 4 + 2] += seen(w.y & 0xffffu);
        s.o[hb][g4 * 4 + 3] += seen(w.y >> 16);
        __builtin_amdgcn_sched_barrier(0);
      }
  }
}

// 4 consecutive columns of a row that is complete
__device__ __forceinline__ void store4(uint16_t* p, float a, float b, float c, float d) {
  uint2 w;
  w.x = pack_bf16x2(a, b);
  w.y = pack_bf16x2(c, d);
  *reinterpret_cast<uint2*>(p) = w;
}

// All but the last N loads into LDS have landed; what was read from LDS is in registers.
template <int N>
__device__ __forceinline__ void landed() {
  asm volatile("" ::: "memory");
  wait_vm<N>();
  asm volatile("" ::: "memory");
}
__device__ __forceinline__ void read_done() {
  asm volatile("" ::: "memory");
  wait_lgkm0();
  asm volatile("" ::: "memory");
}

// lds_dma_at past the caches' retention: what is read once leaves room for nothing that is read again (decoding 64 sequences, 1.2 GB: 5.5 -> 6.1 TB/s;
// a plain read of 4 GB reaches 6.3).
__device__ __forceinline__ void lds_dma_once(rsrc_t rs, uint32_t lds, uint32_t voff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds" ::"s"(lds), "v"(voff), "s"(rs) : "m0", "memory");
}

// ---- narrow items -----------------------------------------------------------------------------------------
__device__ __forceinline__ void narrow_item(const Seq& s, const int32_t* table, int kvh, int key_lo, int key_hi, bool whole,
                                            uint32_t part0, unsigned char* smem) {
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6), r = lane & 31;
  const ArgPtr in = args_again();
  const uint16_t *cK = in->c.k, *cV = in->c.v;
  const float c = in->scale * LOG2E;
  const int blocks = (max(key_hi - key_lo, 0) + 31) / 32, share = (blocks + 3) / 4;
  const int j0 = min(wave * share, blocks) + key_lo / 32, j1 = min((wave + 1) * share, blocks) + key_lo / 32;
  const PageSource src = {table, min(key_hi, j1 * 32), (uint32_t)((int64_t)kvh * in->c.head_stride >> 3), (int*)(smem + SPOTS + wave * 256)};
  unsigned char* sK = smem + wave * 16384;
  unsigned char* sV = sK + 8192;
  const uint32_t ldsK = (uint32_t)(uintptr_t)LRB_LDS_PTR(sK), ldsV = ldsK + 8192;
  const int ts = (int)in->c.token_stride * 2, r4 = lane >> 4, pc = lane & 15;
  uint32_t offK[4], offV[2];              // of load i: offK[i % 4], offV[i % 2]
#pragma unroll
  for (int i = 0; i < 4; i++) offK[i] = (uint32_t)(((i & 1) * 4 + r4) * ts + ((pc ^ (i * 4 + r4)) << 4));
#pragma unroll
  for (int i = 0; i < 2; i++) offV[i] = (uint32_t)((i * 4 + r4) * ts + ((pc ^ (r4 << 2)) << 4));

  Rows st;
  rows_init(st, c);
  if (j0 < j1) {
    bf16x8 qf[8];
    load_queries(in, qf, s, kvh, r, lane);
    const int lim = row_limit(in, s, r), lim0 = uni(row_limit(in, s, 0)), all = uni(row_limit(in, s, s.rows - 1));
    Pages pg;
    first_window<16>(in, pg, src, j0, lane);
    auto dma = [&](bool isV, int j) {     // 8 loads of 4 keys each
#pragma unroll
      for (int g = 0; g < 4; g++) {
        const rsrc_t rs = group_rsrc(group(pg, j * 4 + g), isV ? cV : cK);
#pragma unroll
        for (int i = g * 2; i < g * 2 + 2; i++) lds_dma_once(rs, (isV ? ldsV : ldsK) + i * 1024, isV ? offV[i & 1] : offK[i & 3]);
        __builtin_amdgcn_sched_barrier(0);
      }
    };
    bool bad = false;
    dma(false, j0);
    dma(true, j0);
    for (int j = j0; j < j1; j++) {
      const int key0 = j * 32;
      f32x16 x[1];
      bf16x8 pf[2];
      landed<8>();                        // K; behind it V
      scores<1>(x, qf, sK, lane);
      read_done();
      const bool more = j + 1 < j1;       // (a load that asks for nothing still takes 95 cycles to issue)
      if (more) {
        next_window<16>(pg, src, j + 1, lane);
        dma(false, j + 1);
      }
      const bool masked = key0 + 32 > lim0;
      if (masked) mask<1>(x, lim - key0, lane);
      softmax<1>(st, x, pf, c);
      if (more) landed<8>();              // V; behind it the next K
      else landed<0>();
      if (masked && lim0 < all) bad |= take_out(sV, 8192, lane);
      output<1>(st, pf, sV, lane);
      if (more) {
        read_done();
        dma(true, j + 1);
      }
    }
    if (bad) put_back(st, table, kvh, max(j0 * 32, lim0 & ~31), min(min(j1 * 32, key_hi), all), lim, lane);
  }
  landed<0>();                            // no load is on its way into LDS
  __syncthreads();
  // the four wavefronts' sums, [wave][row][column]
  float* sum = (float*)smem;
  float2* ml = (float2*)(smem + 4 * R_NARROW * LDS_JOIN_LD * 4);
  st.l = half_sum(st.l);
  if (r < s.rows) {
    float* p = sum + (wave * R_NARROW + r) * LDS_JOIN_LD;
#pragma unroll
    for (int hb = 0; hb < 4; hb++)
#pragma unroll
      for (int g4 = 0; g4 < 4; g4++)
        *reinterpret_cast<float4*>(p + hb * 32 + 8 * g4 + 4 * (lane >> 5)) =
            make_float4(st.o[hb][g4 * 4], st.o[hb][g4 * 4 + 1], st.o[hb][g4 * 4 + 2], st.o[hb][g4 * 4 + 3]);
    if (lane < 32) ml[wave * R_NARROW + r] = make_float2(st.m, st.l);
  }
  __syncthreads();
  const ArgPtr a = args_again();
  const int col = (tid & 31) * 4;
  for (int row = tid >> 5; row < s.rows; row += 8) {
    float2 w[4];
    float m = no_score(c), l = 0.f;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      w[i] = ml[i * R_NARROW + row];
      m = fmaxf(m, w[i].x);
    }
    float v[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const float f = fast_exp2((w[i].x - m) * c);
      const float4 x = *reinterpret_cast<const float4*>(sum + (i * R_NARROW + row) * LDS_JOIN_LD + col);
      l += w[i].y * f;
      v[0] += x.x * f; v[1] += x.y * f; v[2] += x.z * f; v[3] += x.w * f;
    }
    if (whole) {
      const int tok = (int)div_by((uint32_t)row, a->by_grp.mul, a->by_grp.shift), head = kvh * a->grp + row - tok * a->grp;
      const int64_t t = s.tok0 + tok;
      const float inv = l == 0.f ? 0.f : 1.f / l;
      store4(a->o + t * a->ldo + head * HD + col, v[0] * inv, v[1] * inv, v[2] * inv, v[3] * inv);
      if (a->lse && col == 0) a->lse[t * a->H + head] = l == 0.f ? -INFINITY : m * a->scale + logf(l);
    } else {
      *reinterpret_cast<float4*>(a->part_o + (int64_t)(part0 + row) * HD + col) = make_float4(v[0], v[1], v[2], v[3]);
      if (col == 0) a->part_ml[part0 + row] = make_float2(m, l);
    }
  }
}

// ---- wide items -------------------------------------------------------------------------------------------
struct WideTiles {
  unsigned char* smem;
  const uint16_t *cK, *cV;
  uint32_t lds0, offK, offV;      // LDS address of the wavefront's first load; lane offsets in K and V, the same for every load
  int t0, t1, tw;                 // 64-key tiles of the item, and the end of the wavefront's
  int lim0, first, end;           // keys that the wavefront's and the item's first rows see, and that any row sees
  int r, wave, lane;
};
// Takes what is no number out of V of tile t, if that has keys that some rows must not see.
__device__ __forceinline__ bool careful(const WideTiles& w, int t) {
  if (!(t * KT + KT > w.first && w.first < w.end)) return false;
  return __syncthreads_or(take_out(w.smem + (2 + ((t - w.t0) & 1)) * TILE_BYTES + w.wave * 4096, 4096, w.lane)) != 0;
}

// A few tiles: one after the other.
__device__ __forceinline__ bool wide_short(ArgPtr in, Rows& st, const WideTiles& w, const Seq& s, const PageSource& src, const bf16x8 (&qf)[8], float c) {
  Pages pg;
  first_window<8>(in, pg, src, w.t0, w.lane);
  auto dma = [&](int t) {                 // K and V of tile t into the slots of its parity
    const uint32_t slot = w.lds0 + (uint32_t)((t - w.t0) & 1) * TILE_BYTES;
#pragma unroll
    for (int i = 0; i < 4; i++) {
      const Group g = group(pg, t * 8 + i * 2 + (w.wave >> 1));
      lds_dma_at(group_rsrc(g, w.cK), slot + i * 4096, w.offK);
      lds_dma_at(group_rsrc(g, w.cV), slot + 2 * TILE_BYTES + i * 4096, w.offV);
      __builtin_amdgcn_sched_barrier(0);
    }
  };
  bool bad = false;
  if (w.t0 < w.t1) dma(w.t0);
  for (int t = w.t0; t < w.t1; t++) {
    landed<0>();
    __syncthreads();                      // the tile has landed for everyone, and everyone has left the one before
    if (t + 1 < w.t1) {
      next_window<8>(pg, src, t + 1, w.lane);
      dma(t + 1);
    }
    bad |= careful(w, t);
    if (t >= w.tw) continue;
    const unsigned char* sK = w.smem + ((t - w.t0) & 1) * TILE_BYTES;
    f32x16 x[2];
    bf16x8 pf[4];
    scores<2>(x, qf, sK, w.lane);
    if (t * KT + KT > w.lim0) mask<2>(x, row_limit(args_again(), s, w.r) - t * KT, w.lane);
    softmax<2>(st, x, pf, c);
    output<2>(st, pf, sK + 2 * TILE_BYTES, w.lane);
  }
  return bad;
}

template <int N>
__device__ __forceinline__ void lds_reads_left() { __builtin_amdgcn_s_waitcnt(0xc07f | N << 8); }
// An iteration works on two key tiles, as the dense forward's does: the scores of tile t + 1 and the output of tile t, with the softmax of tile t and
// the maximum of the new scores threaded between their MFMAs, one barrier in the middle.
// (A barrier of its own for V's slot, which gives the loads half an iteration more, was 1 - 2 % slower.)
constexpr int BARRIER = 12;
constexpr int softmax_elems(int n) { return n < 0 ? 0 : n < 16 ? 5 * (n + 1) / 4 : n < 28 ? 5 + n : 32; }   // done by the end of slot n

__device__ __forceinline__ bool wide_long(ArgPtr in, Rows& st, const WideTiles& w, const Seq& s, const PageSource& src, const bf16x8 (&qf)[8], float c) {
  unsigned char* const smem = w.smem;
  const int t0 = w.t0, t1 = w.t1, tw = w.tw, lim0 = w.lim0, wave = w.wave, lane = w.lane;
  Pages pg;
  first_window<8>(in, pg, src, t0, lane);
  Spots pk = spots(pg, w.cK), pv = spots(pg, w.cV);      // windows of K's loads and of V's, which follow two tiles behind
  auto next = [&](int t) {
    next_window<8>(pg, src, t, lane);
    Spots n = pk;
    if ((t & 7) == 0) {
      asm volatile("");                         // (a branch, not three selections per tile)
      n = spots(pg, w.cK);
    }
    pk = n;
  };
  auto dma = [&](bool isV, int t, int i) {     // load i of tile t into the slot of its parity; past the keys: zeros
    lds_dma_at(spot_rsrc<true>(isV ? pv : pk, t * 8 + i * 2 + (wave >> 1)), w.lds0 + (uint32_t)((isV ? 2 : 0) + ((t - t0) & 1)) * TILE_BYTES + i * 4096,
               isV ? w.offV : w.offK);
  };
  if (t0 < t1) {
#pragma unroll
    for (int i = 0; i < 4; i++) dma(false, t0, i);
#pragma unroll
    for (int i = 0; i < 4; i++) dma(true, t0, i);
    next(t0 + 1);
#pragma unroll
    for (int i = 0; i < 4; i++) dma(false, t0 + 1, i);
    next(t0 + 2);
  }
  f32x16 sa[2], sb[2];                          // scores of the tile whose softmax comes next, and of the one after it
  bf16x8 fr[AHEAD];                             // operands read ahead, slot n in fr[n % AHEAD]
  float alpha = 1.f, mc = 0.f, sum = 0.f, plow = 0.f;
  uint32_t pw[16];                              // probabilities as bf16 pairs
  bool bad = false;
  // operand of slot n: 0..15 scores (k16 step n / 2, key block n % 2), 16..31 output (16 keys each four slots)
  auto read = [&](auto Nc, const unsigned char* sK, const unsigned char* sV) {
    constexpr int n = decltype(Nc)::value;
    if constexpr (n < 16) fr[n % AHEAD] = swz_row_frag(sK, (n & 1) * 32, n >> 1, lane);
    else fr[n % AHEAD] = swz_tr_frag(sV, ((n - 16) >> 2) * 16, (n & 3) * 32, lane);
  };
  // maximum of a tile's scores from key0 on; mx where no key of it is hidden, else masked first
  auto masked_max = [&](f32x16 (&x)[2], int key0, float mx) -> float {
    if (key0 + KT > lim0) {
      mask<2>(x, row_limit(args_again(), s, w.r) - key0, lane);
      mx = x[0][0];
#pragma unroll
      for (int nb = 0; nb < 2; nb++)
#pragma unroll
        for (int e = 0; e < 16; e++) mx = fmaxf(mx, x[nb][e]);
    }
    return mx;
  };
  auto new_max = [&](float mx) {
    const float mn = fmaxf(st.m, half_max(mx));
    alpha = fast_exp2((st.m - mn) * c);
    st.m = mn;
    mc = mn * c;
  };
  auto rescale = [&] {
    if (__builtin_amdgcn_ballot_w64(alpha != 1.f) != 0) {
#pragma unroll
      for (int hb = 0; hb < 4; hb++)
#pragma unroll
        for (int e = 0; e < 16; e++) st.o[hb][e] *= alpha;
    }
  };
  // everyone has read K of tile t + 1 and V of tile t - 1, and K of t + 2 and V of t have landed
  auto turn = [&] {
    read_done();
    landed<0>();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
  };
  // loads 0 .. 7 of tile t's iteration, into the slots just left: V of t + 1, K of t + 3
  auto next_load = [&](int t, int i) { dma(i < 4, t + (i < 4 ? 1 : 3), i & 3); };
  auto next_rsrc = [&](int t, int i) { return spot_rsrc<false>(i < 4 ? pv : pk, (t + (i < 4 ? 1 : 3)) * 8 + (i & 3) * 2 + (wave >> 1)); };
  auto windows = [&](int t) {                   // of the loads of tile t's iteration
    next(t + 3);
    Spots n = pv;
    if (((t + 1) & 7) == 0) {
      asm volatile("");
      n = spots(pg, w.cV);
    }
    pv = n;
  };
  // elements F .. T - 1 of a tile's softmax
  auto softmax_to = [&](const f32x16 (&x)[2], auto Fc, auto Tc) {
    constexpr int f = decltype(Fc)::value, t = decltype(Tc)::value;
    unroll_for<t - f>([&](auto I) {
      constexpr int e = f + decltype(I)::value;
      const float p = fast_exp2(fmaf(x[e >> 4][e & 15], c, -mc));
      sum += p;
      if constexpr (e & 1) pw[e >> 1] = pack_bf16x2(plow, p);
      else plow = p;
    });
  };
  auto out = [&](auto Nc) {
    constexpr int n = decltype(Nc)::value, kk = (n - 16) >> 2;
    const bf16x8 pf = __builtin_bit_cast(bf16x8, make_uint4(pw[kk * 4], pw[kk * 4 + 1], pw[kk * 4 + 2], pw[kk * 4 + 3]));
    st.o[n & 3] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[n % AHEAD], pf, st.o[n & 3], 0, 0, 0);
  };
  // softmax and output of tile t (scores sc), scores of tile t + 1 (into sn).  LAST: near the end, where keys may be hidden
  auto iteration = [&](int t, auto par, auto LAST, f32x16 (&sc)[2], f32x16 (&sn)[2]) {
    const unsigned char* sK1 = smem + (par ^ 1) * TILE_BYTES;             // K of tile t + 1
    const unsigned char* sK2 = smem + par * TILE_BYTES;                   // K of tile t + 2
    const unsigned char* sV = smem + (2 + par) * TILE_BYTES;              // V of tile t
    windows(t);
    rescale();
    sum = 0.f;
#pragma unroll
    for (int nb = 0; nb < 2; nb++)
#pragma unroll
      for (int e = 0; e < 16; e++) sn[nb][e] = 0.f;
    float mx0 = -INFINITY, mx1 = -INFINITY;
    rsrc_t ahead = {};
    unroll_for<32>([&](auto Nc) {
      constexpr int n = decltype(Nc)::value;
      if constexpr (n % 2 == 0 && n != BARRIER) {      // the last two operands may be on their way
        lds_reads_left<(n < 14 || n >= 30 ? 2 : 4)>();
        __builtin_amdgcn_sched_barrier(0);
      }
      if constexpr (n < 16) sn[n & 1] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fr[n % AHEAD], qf[n >> 1], sn[n & 1], 0, 0, 0);
      else out(Nc);
      if constexpr (n == BARRIER) {
        turn();
        if constexpr (decltype(LAST)::value) bad |= careful(w, t);
      }
      // operands, two at a time (half of the waits for them): V only from behind the barrier, then K of the tile after next
      unroll_for<32>([&](auto I) {
        constexpr int x = decltype(I)::value + AHEAD;               // slot that reads
        constexpr int early = (x - AHEAD) | 1, at = early < BARRIER && x >= 16 ? BARRIER : early;
        if constexpr (at == n) {
          if constexpr (x < 32) read(std::integral_constant<int, x>{}, sK1, sV);
          else read(std::integral_constant<int, x - 32>{}, sK2, sV);
        }
      });
      if constexpr (n > BARRIER && n <= BARRIER + 8) {
        constexpr uint32_t V = n - BARRIER <= 4, slot = V * 2 * TILE_BYTES + ((n - BARRIER - 1) & 3) * 4096;
        if constexpr (decltype(LAST)::value) lds_dma_at(ahead, w.lds0 + (par ^ 1) * TILE_BYTES + slot, V ? w.offV : w.offK);
        else lds_dma_from<(decltype(par)::value ^ 1) * TILE_BYTES + slot>(ahead, w.lds0, V ? w.offV : w.offK);
      }
      softmax_to(sc, std::integral_constant<int, softmax_elems(n - 1)>{}, std::integral_constant<int, softmax_elems(n)>{});
      if constexpr (n >= 18 && n < 26) {                            // maximum of the new scores
        constexpr int e = (n - 18) * 2;
        mx0 = fmaxf(fmaxf(mx0, sn[0][e]), sn[0][e + 1]);
        mx1 = fmaxf(fmaxf(mx1, sn[1][e]), sn[1][e + 1]);
      }
      if constexpr (softmax_elems(n - 1) != softmax_elems(n)) asm volatile("" : "+v"(sum));
      if constexpr (n >= BARRIER && n < BARRIER + 8) ahead = next_rsrc(t, n - BARRIER);
      if constexpr (n == 25) asm volatile("" : "+v"(mx0), "+v"(mx1));
      __builtin_amdgcn_sched_barrier(0);
    });
    st.l = st.l * alpha + sum;
    float mx = fmaxf(mx0, mx1);
    if constexpr (decltype(LAST)::value) mx = masked_max(sn, (t + 1) * KT, mx);
    new_max(mx);
  };

  landed<0>();
  __syncthreads();
  if (t0 < tw) {                                // scores of the first tile
    scores<2>(sa, qf, smem, lane);
    float mx = sa[0][0];
#pragma unroll
    for (int nb = 0; nb < 2; nb++)
#pragma unroll
      for (int e = 0; e < 16; e++) mx = fmaxf(mx, sa[nb][e]);
    new_max(masked_max(sa, t0 * KT, mx));
    if (t0 + 1 < tw) unroll_for<AHEAD>([&](auto I) { read(I, smem + TILE_BYTES, smem); });
  }
  read_done();
  __builtin_amdgcn_s_barrier();                 // nobody reads K of the first tile any more
  asm volatile("" ::: "memory");
  if (t0 < t1) {
#pragma unroll
    for (int i = 0; i < 4; i++) dma(false, t0 + 2, i);
  }
  const int plain = min(w.first / KT, tw);        // tiles without a hidden key
  int t = t0;
  for (; t + 2 < plain; t += 2) {
    iteration(t, std::integral_constant<int, 0>{}, std::false_type{}, sa, sb);
    iteration(t + 1, std::integral_constant<int, 1>{}, std::false_type{}, sb, sa);
  }
  for (; t + 1 < tw; t++) {
    iteration(t, (t - t0) & 1, std::true_type{}, sa, sb);
#pragma unroll
    for (int nb = 0; nb < 2; nb++) sa[nb] = sb[nb];
  }
  if (t < tw) {                                 // this wavefront's last tile
    const unsigned char* sV = smem + (2 + ((t - t0) & 1)) * TILE_BYTES;
    windows(t);
    rescale();
    sum = 0.f;
    turn();
    bad |= careful(w, t);
    unroll_for<AHEAD>([&](auto I) { read(std::integral_constant<int, 16 + decltype(I)::value>{}, smem, sV); });
    if (t + 1 < t1) {
#pragma unroll
      for (int i = 0; i < 8; i++) next_load(t, i);
    }
    softmax_to(sa, std::integral_constant<int, 0>{}, std::integral_constant<int, 16>{});
    unroll_for<16>([&](auto I) {
      constexpr int n = 16 + decltype(I)::value;
      out(std::integral_constant<int, n>{});
      if constexpr (n + AHEAD < 32) read(std::integral_constant<int, n + AHEAD>{}, smem, sV);
      if constexpr (n < 24) softmax_to(sa, std::integral_constant<int, 16 + (n - 16) * 2>{}, std::integral_constant<int, 18 + (n - 16) * 2>{});
    });
    st.l = st.l * alpha + sum;
    t++;
  }
  for (; t < t1; t++) {                         // nothing left for this wavefront but its share of the loads
    windows(t);
    turn();
    bad |= careful(w, t);
    if (t + 1 < t1) {
#pragma unroll
      for (int i = 0; i < 8; i++) next_load(t, i);
    }
  }
  return bad;
}

// Tiles from which on the long form is faster, whose code and way in are longer (16 prompts of 256 tokens 38.0 -> 40.3 us with it from 4 tiles on, a prompt
// of 640 23.4 -> 24.7 without it up to 12).
constexpr int LONG = 8;

__device__ __forceinline__ void wide_item(const Seq& s, const int32_t* table, int kvh, int row0, int key_lo, int key_hi, bool whole,
                                          uint32_t part0, unsigned char* smem) {
  const int tid = threadIdx.x, lane = tid & 63, wave = uni(tid >> 6);
  const ArgPtr in = args_again();
  const uint16_t *cK = in->c.k, *cV = in->c.v;
  const float c = in->scale * LOG2E;
  const int wrow0 = row0 + wave * 32, r = wrow0 + (lane & 31);
  const bool busy = wrow0 < s.rows;
  const int lim0 = uni(row_limit(in, s, wrow0)), all = uni(row_limit(in, s, wrow0 + 31));
  const int end = min(key_hi, uni(row_limit(in, s, row0 + R_WIDE - 1)));      // keys that any row of the item sees
  const int first = uni(row_limit(in, s, row0));
  const int t0 = key_lo / KT, t1 = max((end + KT - 1) / KT, t0);
  const int tw = busy ? min(t1, max((min(all, end) + KT - 1) / KT, t0)) : t0;   // ... and of the wavefront
  const PageSource src = {table, end, (uint32_t)((int64_t)kvh * in->c.head_stride >> 3), (int*)(smem + SPOTS + wave * 256)};
  const uint32_t lds0 = (uint32_t)(uintptr_t)LRB_LDS_PTR(smem) + (uint32_t)wave * 1024u;
  const int ts = (int)in->c.token_stride * 2, r4 = lane >> 4, pc = lane & 15, rg = (wave & 1) * 4 + r4;
  // load i of a tile: keys (i * 4 + wave) * 4 .., the same lane offset for every i
  const uint32_t offK = (uint32_t)(rg * ts + ((pc ^ (wave * 4 + r4)) << 4)), offV = (uint32_t)(rg * ts + ((pc ^ (r4 << 2)) << 4));

  Rows st;
  rows_init(st, c);
  bf16x8 qf[8];
  load_queries(in, qf, s, kvh, r, lane);
  const WideTiles w = {smem, cK, cV, lds0, offK, offV, t0, t1, tw, lim0, first, end, r, wave, lane};
  const bool bad = t1 - t0 >= LONG ? wide_long(in, st, w, s, src, qf, c) : wide_short(in, st, w, s, src, qf, c);
  landed<0>();
  if (bad && busy) put_back(st, table, kvh, max(t0 * KT, first & ~(KT - 1)), min(all, end), row_limit(args_again(), s, r), lane);
  const float l = half_sum(st.l);
  if (r >= s.rows) return;
  const ArgPtr a = args_again();
  if (whole) {
    const int tok = (int)div_by((uint32_t)r, a->by_grp.mul, a->by_grp.shift), head = kvh * a->grp + r - tok * a->grp;
    const int64_t t = s.tok0 + tok;
    store_acc_T(a->o + t * a->ldo + head * HD, st.o, l == 0.f ? 0.f : 1.f / l, lane);
    if (a->lse && lane < 32) a->lse[t * a->H + head] = l == 0.f ? -INFINITY : st.m * a->scale + logf(l);
  } else {
    if (lane < 32) a->part_ml[part0 + r] = make_float2(st.m, l);
    if (t0 >= t1) return;               // (a split behind all of the block's keys: its sums are not read)
    float* p = a->part_o + (int64_t)(part0 + r) * HD;
#pragma unroll
    for (int hb = 0; hb < 4; hb++)
#pragma unroll
      for (int g4 = 0; g4 < 4; g4++)
        *reinterpret_cast<float4*>(p + hb * 32 + 8 * g4 + 4 * (lane >> 5)) =
            make_float4(st.o[hb][g4 * 4], st.o[hb][g4 * 4 + 1], st.o[hb][g4 * 4 + 2], st.o[hb][g4 * 4 + 3]);
  }
}

// One workgroup per item: sequence, run of blocks, key / value head, split, block of rows in the run.
__global__ __launch_bounds__(256, 2) void paged_kernel(PagedArgs a) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int lane = threadIdx.x & 63;
  Seq s = {};
  if (lane < a.c.batch) s = load_seq(a, lane);
  const SplitLen len = split_len(a, s);
  // The hardware deals workgroups to the 8 XCDs in rotation; a run, which reads the same keys, stays on one.
  uint32_t v = blockIdx.x;
  if (a.runs) {
    const uint32_t x = v % 8, j = v / 8;
    v = (j / RUN * 8 + x) * RUN + j % RUN;
  }
  uint32_t item0 = 0, part0 = 0, item_end, part_end, splits, items, parts;
  uint64_t hit = 0;
  int b0 = 0;
  for (; b0 < a.c.batch; b0 += 64) {
    splits = items = parts = 0;
    if (b0 + lane < a.c.batch) {
      if (b0 > 0) s = load_seq(a, b0 + lane);
      splits = splits_of(s, len);
      items = (uint32_t)a.c.n_kv_heads * splits * (uint32_t)s.blocks;
      parts = part_rows_of(a, s, splits);
    }
    // wide sequences' items before the others' of the same 64
    const uint32_t wide = s.rows > R_NARROW ? items : 0, wide_end = wave_scan(wide), other_end = wave_scan(items - wide);
    item_end = item0 + (wide > 0 ? wide_end : last_lane(wide_end) + other_end);
    part_end = part0 + wave_scan(parts);
    hit = __builtin_amdgcn_ballot_w64(v - (item_end - items) < items);
    if (hit) break;
    item0 += last_lane(wide_end) + last_lane(other_end);
    part0 = last_lane(part_end);
  }
  if (hit == 0) return;
  const int at = __builtin_ctzll(hit);
  Seq q;
  q.tok0 = __builtin_amdgcn_readlane(s.tok0, at); q.n = __builtin_amdgcn_readlane(s.n, at); q.kv = __builtin_amdgcn_readlane(s.kv, at);
  q.keys = __builtin_amdgcn_readlane(s.keys, at); q.tiles = __builtin_amdgcn_readlane(s.tiles, at);
  q.rows = __builtin_amdgcn_readlane(s.rows, at); q.blocks = __builtin_amdgcn_readlane(s.blocks, at);
  splits = __builtin_amdgcn_readlane(splits, at);
  items = __builtin_amdgcn_readlane(items, at);
  parts = __builtin_amdgcn_readlane(parts, at);
  const uint32_t local = v - (__builtin_amdgcn_readlane(item_end, at) - items), part = __builtin_amdgcn_readlane(part_end, at) - parts;
  // (lists that are no batch's: nothing that has no room)
  if (local >= items || part > a.part_rows || parts > a.part_rows - part) return;
  // blocks in runs, the last (longest) ones of all heads first
  int kvh, split, block = 0;
  if (q.blocks == 1) {
    kvh = uni((int)(local / splits));
    split = (int)(local - (uint32_t)kvh * splits);
  } else {
    const uint32_t runs = ((uint32_t)q.blocks + RUN - 1) / RUN, of_run = RUN * (uint32_t)a.c.n_kv_heads * splits,
                   run = (uint32_t)uni((int)min(local / of_run, runs - 1));
    const uint32_t size = min((uint32_t)q.blocks - run * RUN, RUN), of_head = size * splits;
    uint32_t rem = local - run * of_run;
    kvh = uni((int)(rem / of_head));
    rem -= (uint32_t)kvh * of_head;
    split = uni((int)(rem / size));
    block = q.blocks - 1 - (int)(run * RUN + rem - (uint32_t)split * size);
  }
  const int64_t l64 = (int64_t)(((uint32_t)q.tiles + splits - 1) / splits) * KT;
  const int lo = (int)min(split * l64, (int64_t)q.keys), hi = (int)min((split + 1) * l64, (int64_t)q.keys);
  const uint32_t p0 = part + ((uint32_t)kvh * splits + (uint32_t)split) * (uint32_t)q.rows;
  const int32_t* table = a.c.page_table + (int64_t)(b0 + at) * a.c.table_ld;
  if (q.rows <= R_NARROW) narrow_item(q, table, kvh, lo, hi, splits == 1, p0, smem);
  else wide_item(q, table, kvh, block * R_WIDE, lo, hi, splits == 1, p0, smem);
}

// ---- joining the splits -------------------------------------------------------------------------------------
// Rows (token and head) of the sequences that were split, numbered through.  A row is half a wavefront's, four columns per lane, the halves on
// neighbouring heads; WAVES wavefronts share a row's splits out.  Splits that a row's limit leaves without keys have a sum of zero.
constexpr int JOIN_BATCH = 4;      // splits whose sums are on their way at once

template <int WAVES>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedArgs a) {
  __shared__ float4 s_sum[4][64];
  __shared__ float2 s_ml[4][2];
  const int lane = threadIdx.x & 63, wave = uni(threadIdx.x >> 6), half = lane >> 5, col = (lane & 31) * 4;
  Seq s = {};
  if (lane < a.c.batch) s = load_seq(a, lane);
  const SplitLen len = split_len(a, s);
  const float c = a.scale * LOG2E;
  const int pairs = (a.H + 1) / 2;
  uint32_t part0 = 0, item0 = 0;
  uint32_t i = WAVES == 1 ? blockIdx.x * 4 + (uint32_t)wave : blockIdx.x;      // (token, pair of heads)
  const uint32_t stride = WAVES == 1 ? gridDim.x * 4 : gridDim.x;
  for (int b0 = 0; b0 < a.c.batch; b0 += 64) {
    uint32_t splits = 0, parts = 0;
    if (b0 + lane < a.c.batch) {
      if (b0 > 0) s = load_seq(a, b0 + lane);
      splits = splits_of(s, len);
      parts = part_rows_of(a, s, splits);
    }
    const uint32_t items = parts > 0 ? (uint32_t)s.n * (uint32_t)pairs : 0;
    const uint32_t part_end = part0 + wave_scan(parts), item_end = item0 + wave_scan(items);
    part0 = last_lane(part_end);
    item0 = last_lane(item_end);
    for (; i < item0; i += stride) {
      const int at = __builtin_ctzll(__builtin_amdgcn_ballot_w64(i < item_end));
      const int tok0 = __builtin_amdgcn_readlane(s.tok0, at);
      const uint32_t rows = __builtin_amdgcn_readlane(s.rows, at), sp = __builtin_amdgcn_readlane(splits, at),
                     np = __builtin_amdgcn_readlane(parts, at), part = __builtin_amdgcn_readlane(part_end, at) - np;
      const uint32_t local = i - (__builtin_amdgcn_readlane(item_end, at) - __builtin_amdgcn_readlane(items, at));
      if (part > a.part_rows || np > a.part_rows - part) continue;
      const int tok = uni((int)(local / (uint32_t)pairs)), head = uni((int)(local % (uint32_t)pairs)) * 2 + half;
      const bool there = head < a.H;
      const int kvh = (int)a.by_grp.div((uint32_t)(there ? head : a.H - 1)), in_grp = (there ? head : a.H - 1) - kvh * a.grp;
      const int64_t row = part + (int64_t)((uint32_t)kvh * sp * rows) + (tok * a.grp + in_grp);
      const uint32_t share = WAVES == 1 ? sp : (sp + WAVES - 1) / WAVES;
      const uint32_t k0 = WAVES == 1 ? 0 : min((uint32_t)wave * share, sp), k1 = WAVES == 1 ? sp : min(k0 + share, sp);
      const float2* ml = a.part_ml + row;
      const float* o = a.part_o + row * HD + col;
      float m = no_score(c), l = 0.f;
      float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
      for (uint32_t k = k0; k < k1; k += JOIN_BATCH) {
        float2 w[JOIN_BATCH];
        float4 v[JOIN_BATCH];
#pragma unroll
        for (int j = 0; j < JOIN_BATCH; j++) {
          w[j] = make_float2(m, 0.f);
          if (k + j < k1) {
            w[j] = ml[(k + j) * rows];
            v[j] = *reinterpret_cast<const float4*>(o + (int64_t)((k + j) * rows) * HD);
          }
        }
        float mn = m;
#pragma unroll
        for (int j = 0; j < JOIN_BATCH; j++) mn = fmaxf(mn, w[j].x);
        const float al = fast_exp2((m - mn) * c);
        l *= al; x.x *= al; x.y *= al; x.z *= al; x.w *= al;
        m = mn;
#pragma unroll
        for (int j = 0; j < JOIN_BATCH; j++) {
          if (w[j].y == 0.f) continue;           // (nothing there, or no key: its sums were not formed)
          const float f = fast_exp2((w[j].x - m) * c);
          l += w[j].y * f;
          x.x += v[j].x * f; x.y += v[j].y * f; x.z += v[j].z * f; x.w += v[j].w * f;
        }
      }
      if constexpr (WAVES > 1) {
        __syncthreads();                 // (the row before has been read)
        s_sum[wave][lane] = x;
        if ((lane & 31) == 0) s_ml[wave][half] = make_float2(m, l);
        __syncthreads();
        if (wave > 0) continue;
        float mn = m;
#pragma unroll
        for (int j = 1; j < WAVES; j++) mn = fmaxf(mn, s_ml[j][half].x);
        float f = fast_exp2((m - mn) * c);
        l *= f; x.x *= f; x.y *= f; x.z *= f; x.w *= f;
#pragma unroll
        for (int j = 1; j < WAVES; j++) {
          const float2 w = s_ml[j][half];
          const float4 v = s_sum[j][lane];
          f = fast_exp2((w.x - mn) * c);
          l += w.y * f;
          x.x += v.x * f; x.y += v.y * f; x.z += v.z * f; x.w += v.w * f;
        }
        m = mn;
      }
      if (!there) continue;
      const float inv = l == 0.f ? 0.f : 1.f / l;
      const int64_t t = tok0 + tok;
      store4(a.o + t * a.ldo + head * HD + col, x.x * inv, x.y * inv, x.z * inv, x.w * inv);
      if (a.lse && col == 0) a.lse[t * a.H + head] = l == 0.f ? -INFINITY : m * a.scale + logf(l);
    }
  }
}

// What can be said of a call without its lists.
struct Bounds {
  int64_t items, part_rows;
  bool split;
};
bool runs_of(int64_t T, int grp, int batch) { return T * grp >= 2 * (int64_t)R_WIDE * batch; }
Bounds bounds(int64_t T, int H, int Hkv, int batch, int64_t capacity) {
  const int64_t tiles = (capacity + KT - 1) / KT, rows = T * (H / Hkv);
  const int64_t blocks = (batch < T ? batch : T) + rows / R_WIDE;      // of rows: a sequence's last one may be short
  const int64_t most = (tiles + MIN_SPLIT - 1) / MIN_SPLIT;           // splits of a sequence
  // ... and of all beside one for each item: w / len, which grows with w; wide ones at most PLACES
  const double w = (double)Hkv * (double)blocks * (double)tiles;
  const int64_t cuts = std::min<int64_t>(ROUNDS, std::max<int64_t>((int64_t)(8.0 * std::sqrt(w)) + 2, PLACES)), wide = rows > R_NARROW ? PLACES : 0;
  Bounds b;
  b.split = most > 1;
  b.items = std::min(Hkv * blocks * most, Hkv * blocks + cuts + wide);
  // rows of sums: all rows in every split, or those of the splits there are (rounded as they are, two or more are at most 4 / 3 of a sequence's share,
  // wide ones 8 / 5)
  b.part_rows = b.split ? std::min(T * H * most, cuts * std::min<int64_t>(rows, R_NARROW) * 4 / 3 + wide * R_WIDE * 8 / 5 + 1) : 0;
  return b;
}

int64_t grid_of(int64_t T, int H, int Hkv, int batch, int64_t capacity) {
  const int64_t items = bounds(T, H, Hkv, batch, capacity).items;
  return runs_of(T, H / Hkv, batch) ? (items + 8 * RUN - 1) / (8 * RUN) * (8 * RUN) : items;
}

}  // namespace

bool attention_paged_fits(int64_t T, int H, int Hkv, int batch, int64_t capacity) {
  return grid_of(T, H, Hkv, batch, capacity) < (int64_t)1 << 24;      // 2^32 lanes
}

size_t attention_paged_ws_bytes(int64_t T, int H, int Hkv, int batch, int64_t capacity) {
  return T == 0 || batch == 0 ? 0 : (size_t)bounds(T, H, Hkv, batch, capacity).part_rows * (HD * sizeof(float) + sizeof(float2));
}

hipError_t attention_paged_bf16(const KvCache& c, const void* q, int64_t ldq, void* o, int64_t ldo, float* lse, int64_t T, int H, float scale,
                                void* ws, hipStream_t st) {
  static const hipError_t attr_err = hipFuncSetAttribute((const void*)paged_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, LDS_BYTES);
  if (attr_err != hipSuccess) return attr_err;
  const Bounds b = bounds(T, H, c.n_kv_heads, c.batch, c.capacity);
  PagedArgs a;
  a.c = c; a.q = (const uint16_t*)q; a.o = (uint16_t*)o; a.lse = lse;
  a.part_rows = (uint32_t)b.part_rows;
  a.part_o = (float*)ws;
  a.part_ml = (float2*)((float*)ws + b.part_rows * HD);
  a.ldq = ldq; a.ldo = ldo; a.T = (int)T; a.H = H; a.grp = H / c.n_kv_heads; a.scale = scale;
  a.by_grp = FastDiv::of(a.grp);
  a.runs = runs_of(T, a.grp, c.batch);
  const int64_t grid = grid_of(T, H, c.n_kv_heads, c.batch, c.capacity);
  hipLaunchKernelGGL(paged_kernel, dim3((unsigned)grid), dim3(256), LDS_BYTES, st, a);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || !b.split) return e;
  // four wavefronts per pair of rows where the chip has places for all of them
  const int64_t pairs = T * ((H + 1) / 2);
  if (pairs <= 1024) hipLaunchKernelGGL(paged_join_kernel<4>, dim3((unsigned)pairs), dim3(256), 0, st, a);
  else hipLaunchKernelGGL(paged_join_kernel<1>, dim3((unsigned)std::min<int64_t>((pairs + 3) / 4, 2048)), dim3(256), 0, st, a);
  return hipGetLastError();
}

}  // namespace lrb
