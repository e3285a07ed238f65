// What the attention kernels share: 256-byte rows (heads of 128, bf16) moved straight from memory into LDS, the operand reads of
// such tiles, accumulator layouts.  For attention.hip and attention_paged.hip.
#pragma once
#include "common.h"

namespace lrb {
namespace {

constexpr int HD = 128;
constexpr int KT = 64;            // keys (or queries, in the dkv kernel) per streamed tile
constexpr float LOG2E = 1.4426950408889634f;

typedef short s16x4 __attribute__((ext_vector_type(4)));

// raw v_exp_f32 (2^x): the arguments here are differences to a running maximum, never denormal-critical
__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

__device__ __forceinline__ bf16x8 lds_b128(const unsigned char* p) { return *reinterpret_cast<const bf16x8*>(p); }

// 8 consecutive accumulator values (v = t*8 .. t*8+7) packed as the bf16 B operand of one k16 step.
__device__ __forceinline__ bf16x8 pack_acc_half(const f32x16& a, int t) {
  uint4 q;
  q.x = pack_bf16x2(a[t * 8 + 0], a[t * 8 + 1]);
  q.y = pack_bf16x2(a[t * 8 + 2], a[t * 8 + 3]);
  q.z = pack_bf16x2(a[t * 8 + 4], a[t * 8 + 5]);
  q.w = pack_bf16x2(a[t * 8 + 6], a[t * 8 + 7]);
  return __builtin_bit_cast(bf16x8, q);
}

// Row index of accumulator element v inside a 32-row block.
__device__ __forceinline__ int acc_row(int v, int lane) { return 8 * (v >> 2) + 4 * (lane >> 5) + (v & 3); }

// Query-row fragments kept in registers: B operand (rows = queries) for all 8 k16 steps over h.
template <int MB>
__device__ __forceinline__ void load_row_frags(bf16x8 (&f)[MB][8], const uint16_t* base, int64_t ld, int row0,
                                               int nrows, int lane) {
#pragma unroll
  for (int mb = 0; mb < MB; mb++) {
    const int row = row0 + mb * 32 + (lane & 31);
    const bool ok = row < nrows;
#pragma unroll
    for (int ks = 0; ks < 8; ks++) {
      uint4 q = ok ? *reinterpret_cast<const uint4*>(base + (int64_t)row * ld + ks * 16 + (lane >> 5) * 8)
                   : make_uint4(0, 0, 0, 0);
      f[mb][ks] = __builtin_bit_cast(bf16x8, q);
    }
  }
}

// Writes a transposed accumulator block set acc[hb][.] (rows = h, column = the lane's token) as
// out[token][h], 4 consecutive h (8 bytes) at a time, scaled by `mul`.
__device__ __forceinline__ void store_acc_T(uint16_t* out_row, const f32x16 (&acc)[4], float mul, int lane) {
#pragma unroll
  for (int hb = 0; hb < 4; hb++)
#pragma unroll
    for (int g4 = 0; g4 < 4; g4++) {
      const int h = hb * 32 + 8 * g4 + 4 * (lane >> 5);
      uint2 w;
      w.x = pack_bf16x2(acc[hb][g4 * 4 + 0] * mul, acc[hb][g4 * 4 + 1] * mul);
      w.y = pack_bf16x2(acc[hb][g4 * 4 + 2] * mul, acc[hb][g4 * 4 + 3] * mul);
      *reinterpret_cast<uint2*>(out_row + h) = w;
    }
}

// ----------------------------------------------------------------------------------------------
// 64-row x 128-column bf16 tiles moved global -> LDS without passing through registers.
// One buffer_load_dwordx4 ... lds per wavefront writes 1 KB = 4 tile rows of 256 bytes; lane L's 16
// bytes land at base + 16 L, i.e. row L/16, physical chunk L%16.  Rows are not padded; instead the
// 16-byte chunks of a row are XOR-swizzled and each lane fetches the logical chunk that belongs in its
// slot.  Two swizzles, one per read pattern:
//   SWZ_ROW16  chunk ^ (row % 16)        16 consecutive rows x one logical chunk (ds_read_b128 of
//                                        MFMA operand rows) cover all 64 banks
//   SWZ_ROW4   chunk ^ ((row % 4) * 4)   4 consecutive rows x 64 bytes (the LDS transpose read)
//                                        cover all 64 banks
// Rows at or past `nrows` are fetched with an out-of-range offset: the load returns zeros.
// ----------------------------------------------------------------------------------------------
constexpr int TILE_BYTES = KT * HD * 2;
constexpr uint32_t DMA_OOB = 0x80000000u;
enum { SWZ_ROW16 = 0, SWZ_ROW4 = 1, SWZ_BOTH = 2 };
//   SWZ_BOTH   chunk ^ ((row % 4) * 4 + (row / 4) % 4)   serves both read patterns of a tile that is
//                                        needed row-wise and transposed: 16 consecutive rows see 16
//                                        different terms, 4 consecutive rows 4 different 64-byte groups
#define LRB_LDS_PTR(p) ((__attribute__((address_space(3))) void*)(p))

// Buffer resource as four scalar words: base address, stride 0, size in bytes, data format word.
typedef uint32_t rsrc_t __attribute__((ext_vector_type(4)));
__device__ __forceinline__ rsrc_t make_rsrc(const void* base, uint32_t bytes) {
  const uint64_t a = (uint64_t)(uintptr_t)base;
  rsrc_t r = {(uint32_t)a, (uint32_t)(a >> 32) & 0xffffu, bytes, 0x00020000u};
  // Five wait states have to pass between a vector write of a scalar (v_readfirstlane) and a buffer instruction that reads
  // it; the compiler does not look for buffer instructions inside lds_dma's assembly.
  asm volatile("s_nop 4" : "+s"(r));
  return r;
}
__device__ __forceinline__ rsrc_t tile_rsrc(const uint16_t* base) { return make_rsrc(base, 0x7fffffffu); }

// One global -> LDS load of BYTES (4 or 16) per lane: lane L's data lands at lds + BYTES * L.  Issued
// as inline assembly on purpose: through the builtin the compiler treats every later LDS read as a
// possible read of this load's destination and makes it wait for ALL global loads in flight, i.e. the
// tile being worked on would wait for the next tile's loads.  Completion is tracked by hand instead
// (wait_vm0 before the barrier that publishes a tile).  `lds` must be wavefront-uniform.
template <int BYTES>
__device__ __forceinline__ void lds_dma(rsrc_t rs, const unsigned char* lds, uint32_t voff) {
  const uint32_t m0v = __builtin_amdgcn_readfirstlane((uint32_t)(uintptr_t)LRB_LDS_PTR(lds));
  if constexpr (BYTES == 16)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(m0v), "v"(voff), "s"(rs) : "m0", "memory");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(m0v), "v"(voff), "s"(rs) : "m0", "memory");
}

// Per-lane byte offsets (row * ld + logical chunk) of the 16 / NW wavefront loads that a wavefront of
// an NW-wavefront workgroup contributes to one tile.
template <int SWZ, int NL>
__device__ __forceinline__ void dma_lane_offsets(uint32_t (&off)[NL], int (&row)[NL], int64_t ld, int wave, int lane) {
  constexpr int NW = 16 / NL;
#pragma unroll
  for (int i = 0; i < NL; i++) {
    const int r = (i * NW + wave) * 4 + (lane >> 4);
    const int pc = lane & 15;
    const int lc = SWZ == SWZ_ROW16 ? (pc ^ (r & 15))
                 : SWZ == SWZ_ROW4 ? (pc ^ ((r & 3) << 2))
                                   : (pc ^ (((r & 3) << 2) | ((r >> 2) & 3)));
    row[i] = r;
    off[i] = (uint32_t)(r * (int)ld + lc * 8) * 2u;
  }
}
template <int NL>
__device__ __forceinline__ void dma_tile(rsrc_t rs, unsigned char* tile, const uint32_t (&off)[NL],
                                         const int (&row)[NL], int row0, int nrows, int64_t ld, int wave) {
  constexpr int NW = 16 / NL;
  const uint32_t base = (uint32_t)row0 * (uint32_t)ld * 2u;
#pragma unroll
  for (int i = 0; i < NL; i++) {
    const uint32_t o = (row0 + row[i]) < nrows ? base + off[i] : DMA_OOB;
    lds_dma<16>(rs, tile + (i * NW + wave) * 1024, o);
  }
}
// s_waitcnt vmcnt(0) alone (gfx9 encoding), and lgkmcnt(0) alone
__device__ __forceinline__ void wait_vm0() { __builtin_amdgcn_s_waitcnt(0x0f70); }
__device__ __forceinline__ void wait_lgkm0() { __builtin_amdgcn_s_waitcnt(0xc07f); }
// s_waitcnt vmcnt(N) alone, N < 64: bits 3:0 and 15:14 hold vmcnt, the other counters stay at "no wait"
template <int N>
__device__ __forceinline__ void wait_vm() {
  static_assert(N >= 0 && N < 64, "vmcnt is a 6-bit counter");
  __builtin_amdgcn_s_waitcnt(0x0f70 | (N & 15) | ((N >> 4) << 14));
}

// A operand (32 rows = tile rows r0 + lane%32, k slots = logical chunk ks*2 + lane/32) from a
// SWZ_ROW16 tile.  r0 is a multiple of 16, so the swizzle term depends on the lane only.
__device__ __forceinline__ bf16x8 swz_row_frag(const unsigned char* tile, int r0, int ks, int lane) {
  const int row = r0 + (lane & 31);
  return lds_b128(tile + row * 256 + (((ks * 2 + (lane >> 5)) ^ (lane & 15)) << 4));
}
// Transposed A operand from a SWZ_ROW4 tile stored [k][col]: rows = columns c0..c0+31 (c0 a multiple
// of 32), k slots (half = lane / 32, e = 0..7) = tile rows k0 + (e/4)*8 + half*4 + e%4 (k0 a multiple
// of 16), which is the row order of a 32x32 accumulator.  Inside each group of 16 lanes the transpose
// read hands lane i the i-th 16-bit column of the 4 x 16 block that the 16 lanes fetched as 4 rows x
// 4 lanes x 8 bytes.
__device__ __forceinline__ bf16x8 swz_tr_frag(const unsigned char* tile, int k0, int c0, int lane) {
  const int g = lane >> 4, s = lane & 15;
  const int rl = (g >> 1) * 4 + (s >> 2);                       // row inside the 16-row group; rl % 4 = s / 4
  const int chunk = (c0 >> 3) + (g & 1) * 2 + ((s & 3) >> 1);   // logical 16-byte chunk
  const unsigned char* p0 = tile + (k0 + rl) * 256 + ((chunk ^ ((s >> 2) << 2)) << 4) + (s & 1) * 8;
  const unsigned char* p1 = p0 + 8 * 256;
  s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(p0));
  s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(p1));
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  s16x8 r = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  return __builtin_bit_cast(bf16x8, r);
}

// The same two operand reads for a SWZ_BOTH tile (r0 and k0 multiples of 16, c0 a multiple of 32).
__device__ __forceinline__ bf16x8 both_row_frag(const unsigned char* tile, int r0, int ks, int lane) {
  const int l31 = lane & 31;
  const int f = ((l31 & 3) << 2) | ((l31 >> 2) & 3);
  return lds_b128(tile + (r0 + l31) * 256 + (((ks * 2 + (lane >> 5)) ^ f) << 4));
}
__device__ __forceinline__ bf16x8 both_tr_frag(const unsigned char* tile, int k0, int c0, int lane) {
  const int g = lane >> 4, s = lane & 15;
  const int rl = (g >> 1) * 4 + (s >> 2);
  const int f0 = ((s >> 2) << 2) | (g >> 1);                    // rows k0 + rl; rows + 8 flip bit 1 of the term
  const int chunk = (c0 >> 3) + (g & 1) * 2 + ((s & 3) >> 1);
  const unsigned char* rowp = tile + (k0 + rl) * 256 + (s & 1) * 8;
  s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((s16x4 __attribute__((address_space(3)))*)(rowp + ((chunk ^ f0) << 4)));
  s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16(
      (s16x4 __attribute__((address_space(3)))*)(rowp + 8 * 256 + ((chunk ^ f0 ^ 2) << 4)));
  typedef short s16x8 __attribute__((ext_vector_type(8)));
  s16x8 r = {lo[0], lo[1], lo[2], lo[3], hi[0], hi[1], hi[2], hi[3]};
  return __builtin_bit_cast(bf16x8, r);
}

// Compile-time loop over std::integral_constant indices: register arrays indexed by them stay in registers.
template <int N, class F, int I = 0>
__device__ __forceinline__ void unroll_for(F&& f) {
  if constexpr (I < N) {
    f(std::integral_constant<int, I>{});
    unroll_for<N, F, I + 1>(static_cast<F&&>(f));
  }
}
// Buffer resource of S rows of 256 bytes, ld elements apart: rows at or past S are out of range by themselves.
__device__ __forceinline__ rsrc_t rows_rsrc(const uint16_t* base, int S, int64_t ld) {
  return make_rsrc(base, (uint32_t)(S - 1) * (uint32_t)ld * 2u + 256u);
}
// The same resource from byte `off` on (scalar arithmetic only); empty, so that loads deliver zeros, where !valid.
__device__ __forceinline__ rsrc_t rsrc_from(rsrc_t r, uint32_t off, bool valid) {
  const uint64_t a = (((uint64_t)r.y << 32) | r.x) + (valid ? off : 0u);
  return rsrc_t{(uint32_t)a, (uint32_t)(a >> 32), valid ? r.z - off : 0u, r.w};
}
// lds_dma<16> with the LDS address as a number
__device__ __forceinline__ void lds_dma_at(rsrc_t rs, uint32_t lds, uint32_t voff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(voff), "s"(rs) : "m0", "memory");
}
__device__ __forceinline__ void lds_dma4_at(rsrc_t rs, uint32_t lds, uint32_t voff) {
  asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(lds), "v"(voff), "s"(rs) : "m0", "memory");
}
// max / sum of the two lanes l and l + 32
__device__ __forceinline__ float half_max(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float half_sum(float x) {
  const auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

}  // namespace
}  // namespace lrb
