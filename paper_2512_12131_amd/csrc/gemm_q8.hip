// Products of 8-bit integers: C[m, n] = sa[m] sb[n] sum_k A[m, k] B[n, k], both operands k-contiguous in rows that start on 16 bytes, the sum
// exact in 32-bit integers, scaled in 32 bits (the row's scale first) and rounded once.
//
// v_mfma_i32_32x32x32_i8 takes twice the k of the bf16 instruction in the same registers (a lane holds 16 bytes of one row), places and
// cycles, so tiles, LDS layout and loads are those of the bf16 kernels, with a slice of 128 k where they have 64: rows of 128 bytes, loaded
// straight into LDS, 16-byte chunks XORed by (row / 2) % 8.
//
// What lies in a row behind K may be anything (the weight of K = 5461 in rows of 5472, a view of a wider matrix): TAIL masks it out of
// A's operand of the last chunk, so that it is multiplied with zeros.  Chunks past the last one are not loaded.
#include "gemm_ring.h"
#include "quant_row.h"

namespace lrb {
namespace {

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x16 __attribute__((ext_vector_type(16)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint16_t u16x2 __attribute__((ext_vector_type(2)));

// A's operand of chunk c with what lies behind K cleared
struct Tail {
  int chunk;                 // the last chunk, of which `mask` is kept
  i32x4 mask;
  __device__ __forceinline__ explicit Tail(int K) : chunk((K - 1) / 16) {
    const int n = K - chunk * 16;
#pragma unroll
    for (int j = 0; j < 4; j++) mask[j] = n >= 4 * j + 4 ? -1 : n <= 4 * j ? 0 : (1 << (8 * (n - 4 * j))) - 1;
  }
  __device__ __forceinline__ i32x4 of(i32x4 v, int c) const {
#pragma unroll
    for (int j = 0; j < 4; j++) v[j] &= c == chunk ? mask[j] : -1;
    return v;
  }
};

// ---- epilogue ---------------------------------------------------------------------------------
// The accumulators hold the transposed 32 x 32 blocks: lane -> row lane % 32, registers 4g .. 4g + 3 -> columns 8g + 4 (lane / 32) + 0..3.  They go
// through LDS (the wavefront's own space; see gemm_tile.h for the two staging forms) and leave as rows of eight columns per lane.
template <class T, class Stage>
struct Q8Scales {
  static constexpr int NJ = T::TN / Stage::SC, NH = 32 / Stage::SR;
  float row[T::FM][NH];      // of the rows this lane stages
  f32x4 col[NJ][2];          // of the columns this lane stores
  __device__ __forceinline__ void load(const Q8Op& op, int m0, int n0, int wave, int lane) {
    const int wm = wave / T::WN, wn = wave % T::WN, cg = lane % (Stage::SC / 8);
    // (whole scales behind the last row and column are read as zeros)
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)(op.sa + m0), 0, (uint32_t)min(op.M - m0, T::BM) * 4u, 0x00020000);
    const __amdgpu_buffer_rsrc_t cs = __builtin_amdgcn_make_buffer_rsrc((void*)(op.sb + n0), 0, (uint32_t)min(op.N - n0, T::BN) * 4u, 0x00020000);
#pragma unroll
    for (int i = 0; i < T::FM; i++)
#pragma unroll
      for (int h = 0; h < NH; h++)
        row[i][h] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(rs, (wm * T::TM + i * 32 + h * Stage::SR + lane % Stage::SR) * 4, 0, 0));
#pragma unroll
    for (int jj = 0; jj < NJ; jj++)
#pragma unroll
      for (int x = 0; x < 2; x++) {
#pragma unroll
        for (int r = 0; r < 4; r++)
          col[jj][x][r] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(cs, (wn * T::TN + jj * Stage::SC + cg * 8 + x * 4 + r) * 4, 0, 0));
      }
  }
};

// OUT: LR_BF16 or LR_F32.  EDGE: N is no multiple of 8; the vector with the last columns is stored element by element.
template <class T, int OUT, bool EDGE, class Stage>
__device__ __forceinline__ void q8_epilogue(const Q8Op& op, i32x16 (&acc)[T::FM][T::FN], const Q8Scales<T, Stage>& s, const Stage& stage, int wave, int lane,
                                            int m0, int n0) {
  constexpr int ES = OUT == LR_BF16 ? 2 : 4;
  constexpr int LPR = Stage::SC / 8, RPP = 64 / LPR, PPS = Stage::SR / RPP, NJ = T::TN / Stage::SC, NH = 32 / Stage::SR;
  constexpr uint32_t OOB = 0x80000000u;
  const int wm = wave / T::WN, wn = wave % T::WN, cg = lane % LPR, rsub = lane / LPR;
  const int rows = min(T::BM, op.M - m0);
  const __amdgpu_buffer_rsrc_t rsC = __builtin_amdgcn_make_buffer_rsrc((void*)((char*)op.C + (int64_t)m0 * op.ldc * ES), 0,
                                                                       (uint32_t)rows * (uint32_t)op.ldc * ES, 0x00020000);
  const uint32_t ld = (uint32_t)op.ldc * ES;
  static_for<T::FM * NH * NJ>([&](auto Q) {
    constexpr int q = decltype(Q)::value, i = q / (NH * NJ), h = q / NJ % NH, jj = q % NJ;
    if constexpr (Stage::SR == 16 && h == 0 && jj == 0) {
      // rows 0..15 of two neighbouring blocks come together, then their rows 16..31
      static_for<T::FN / 2>([&](auto J) {
        constexpr int j = decltype(J)::value;
#pragma unroll
        for (int v = 0; v < 16; v++) {
          const auto sw = __builtin_amdgcn_permlane16_swap((uint32_t)acc[i][2 * j][v], (uint32_t)acc[i][2 * j + 1][v], false, false);
          acc[i][2 * j][v] = (int)sw[0];
          acc[i][2 * j + 1][v] = (int)sw[1];
        }
      });
    }
    auto put = [&](int row, int chunk, const i32x16& a) {
#pragma unroll
      for (int g = 0; g < 4; g++) {
        f32x4 v;
#pragma unroll
        for (int r = 0; r < 4; r++) v[r] = (float)a[4 * g + r] * s.row[i][h];
        *reinterpret_cast<f32x4*>(stage.at(row, chunk + 2 * g)) = v;
      }
    };
    if constexpr (Stage::SR == 32)
      static_for<T::FN>([&](auto J) { put(lane & 31, decltype(J)::value * 8 + (lane >> 5), acc[i][decltype(J)::value]); });
    else
      put(lane & 15, (lane >> 4 & 1) * 8 + (lane >> 5), acc[i][2 * jj + h]);
    const int n = n0 + wn * T::TN + jj * Stage::SC + cg * 8;
    const bool whole = !EDGE || n + 8 <= op.N;
    const uint32_t off_n = n < op.N && whole ? (uint32_t)n * ES : OOB;
#pragma unroll
    for (int p = 0; p < PPS; p++) {
      const int rl = p * RPP + rsub, lm = wm * T::TM + i * 32 + h * Stage::SR + rl;
      const f32x4 lo = *reinterpret_cast<const f32x4*>(stage.at(rl, 2 * cg)) * s.col[jj][0];
      const f32x4 hi = *reinterpret_cast<const f32x4*>(stage.at(rl, 2 * cg + 1)) * s.col[jj][1];
      const uint32_t off = (uint32_t)lm * ld + off_n;
      if constexpr (OUT == LR_BF16) {
        const u32x4 v = {pack_bf16x2(lo[0], lo[1]), pack_bf16x2(lo[2], lo[3]), pack_bf16x2(hi[0], hi[1]), pack_bf16x2(hi[2], hi[3])};
        __builtin_amdgcn_raw_buffer_store_b128(v, rsC, (int)off, 0, 0);
        if (EDGE && !whole) {
#pragma unroll
          for (int e = 0; e < 8; e++)
            __builtin_amdgcn_raw_buffer_store_b16((uint16_t)(v[e / 2] >> (16 * (e % 2))), rsC, (int)(n + e < op.N ? (uint32_t)lm * ld + (uint32_t)(n + e) * 2u : OOB), 0, 0);
        }
      } else {
        const u32x4 a = __builtin_bit_cast(u32x4, lo), b = __builtin_bit_cast(u32x4, hi);
        __builtin_amdgcn_raw_buffer_store_b128(a, rsC, (int)off, 0, 0);
        __builtin_amdgcn_raw_buffer_store_b128(b, rsC, (int)(off + 16u), 0, 0);
        if (EDGE && !whole) {
#pragma unroll
          for (int e = 0; e < 8; e++)
            __builtin_amdgcn_raw_buffer_store_b32(e < 4 ? a[e % 4] : b[e % 4], rsC, (int)(n + e < op.N ? (uint32_t)lm * ld + (uint32_t)(n + e) * 4u : OOB), 0, 0);
        }
      }
    }
  });
}

// ---- ring tiles: a workgroup per output tile ----------------------------------------------------
// dma16 past the caches' retention, for what is read once
template <bool FIRST>
__device__ __forceinline__ void dma16_once(rsrc_words rs, uint32_t lds, uint32_t voff) {
  if constexpr (FIRST)
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 4\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds" ::"s"(lds), "v"(voff), "s"(rs) : "m0", "memory");
  else
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds" ::"s"(lds), "v"(voff), "s"(rs) : "m0", "memory");
}

// (rows of 128 bytes are 64 elements of the bf16 kernels' offsets)
// ONCE: one row of tiles and a weight that comes from memory.  Its rows are 4 KB or so apart, and workgroups that all walk k from its start ask for the
// same few channels at a time: each column of tiles starts 5 slices further instead, and the weight passes by the caches.  us, weights from
// memory, plain / starts apart / both: 64 x 32000 x 4096 32.7 / 27.7 / 24.4 (5.4 TB/s), 128 x 32000 x 4096 on 128 x 128 tiles 34.1 / 29.8 / 28.3, 64 x 11008 x
// 4096 on 64 x 64 14.9 / 14.1 / 13.5; of a weight that the caches keep, 64 x 1000 x 4000, 11.5 / 11.6 / 17.3, so it has to be 16 MB.
template <class T, int OUT, bool EDGE, bool TAIL, bool ONCE>
__global__ __launch_bounds__(T::NT) void q8_ring_kernel(Q8Op op, int tiles_m, int tiles_n) {
  static_assert(T::NL == 0, "every wavefront loads and multiplies");
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / T::WN, wn = wave % T::WN;
  int tm, tn, bz;
  tile_of_block(blockIdx.x, gridDim.x, tiles_m, tiles_n, tm, tn, bz);
  const int m0 = tm * T::BM, n0 = tn * T::BN;
  const int klen = (op.K + 15) / 16 * 8;                 // pairs of bytes that are loaded of a row
  constexpr int KST = T::SUB * BK, KSTEPS = T::SUB * 4;
  const int nit = (klen + KST - 1) / KST;
  const rsrc_words rsA = operand_rsrc(op.A + (int64_t)m0 * op.lda), rsB = operand_rsrc(op.B + (int64_t)n0 * op.ldb);
  const uint32_t sbase = (uint32_t)(uintptr_t)LRB_LDS_PTR(smem);
  uint32_t offA[T::LA], offB[T::LB];
  int kl = 0;
  lane_offsets<T, false, T::BM>(offA, kl, op.lda / 2, m0, op.M, wave, lane);
  lane_offsets<T, false, T::BN>(offB, kl, op.ldb / 2, n0, op.N, wave, lane);
  const int start = ONCE ? tn * 5 % nit : 0;
  auto stage_of = [&](int it) { return !ONCE || it >= nit ? it : it + start >= nit ? it + start - nit : it + start; };
  auto issue_one = [&](int it, int slot, auto I, auto FIRST) {
    constexpr int s = decltype(I)::value / (T::LA + T::LB), j = decltype(I)::value % (T::LA + T::LB);
    constexpr bool is_a = j < T::LA;
    constexpr int i = is_a ? j : j - T::LA;
    const int k0 = stage_of(it) * KST + s * BK;
    const uint32_t dst = sbase + (uint32_t)(slot * T::STAGE + s * T::SLICE + (is_a ? 0 : T::A_BYTES)) + (uint32_t)(wave + T::NWL * i) * 1024u;
    const uint32_t off = k0 + kl < klen ? (is_a ? offA[is_a ? i : 0] : offB[is_a ? 0 : i]) + (uint32_t)k0 * 2u : RING_OOB;
    if constexpr (ONCE && !is_a) dma16_once<decltype(FIRST)::value>(rsB, dst, off);
    else dma16<decltype(FIRST)::value>(is_a ? rsA : rsB, dst, off);
  };
  i32x16 acc[T::FM][T::FN] = {};
  const Tail tail(op.K);
#pragma unroll
  for (int s = 0; s < T::NS - 1; s++) static_for<T::LPS>([&](auto I) { issue_one(s, s, I, std::true_type{}); });
  const int frow = lane & 31, fhalf = lane >> 5, fsw = (frow >> 1) & 7;
  int rd = 0, wr = T::NS - 1;
  for (int it = 0; it < nit; it++) {
    asm volatile("" ::: "memory");
    wait_vmcnt<(T::NS - 2) * T::LPS>();
    wait_lgkmcnt0();
    __builtin_amdgcn_s_barrier();
    asm volatile("" ::: "memory");
    if (TAIL && stage_of(it) == nit - 1) {
      // what lies behind K is cleared in LDS, once (a mask on the way into every product, us: 777 x 2047 x 5461 with rows of 5504 23.3, so 20.9; 300 x 3001 x 4001 15.2, so 12.0)
      static_assert(T::BM <= T::NT, "a thread per row");
      if (tid < T::BM) {
        i32x4* last = reinterpret_cast<i32x4*>(smem + rd * T::STAGE + tail.chunk / 8 % T::SUB * T::SLICE + tid * 128 + ((tail.chunk % 8 ^ (tid >> 1 & 7)) << 4));
        *last = tail.of(*last, tail.chunk);
      }
      wait_lgkmcnt0();
      __builtin_amdgcn_s_barrier();
      asm volatile("" ::: "memory");
    }
    i32x4 af[KSTEPS][T::FM], bf[KSTEPS][T::FN];
#pragma unroll
    for (int kk = 0; kk < KSTEPS; kk++) {
      const unsigned char* sa = smem + rd * T::STAGE + (kk / 4) * T::SLICE;
      const int co = ((kk % 4 * 2 + fhalf) ^ fsw) << 4;
#pragma unroll
      for (int i = 0; i < T::FM; i++) af[kk][i] = *reinterpret_cast<const i32x4*>(sa + (wm * T::TM + i * 32 + frow) * 128 + co);
#pragma unroll
      for (int j = 0; j < T::FN; j++) bf[kk][j] = *reinterpret_cast<const i32x4*>(sa + T::A_BYTES + (wn * T::TN + j * 32 + frow) * 128 + co);
    }
    asm volatile("" ::: "memory");
    static_for<KSTEPS>([&](auto KK) {
      constexpr int kk = decltype(KK)::value;
      constexpr int l0 = kk * T::LPS / KSTEPS, l1 = (kk + 1) * T::LPS / KSTEPS;
      static_for<l1 - l0>([&](auto L) { issue_one(it + T::NS - 1, wr, std::integral_constant<int, l0 + decltype(L)::value>{}, std::false_type{}); });
#pragma unroll
      for (int i = 0; i < T::FM; i++) {
#pragma unroll
        for (int j = 0; j < T::FN; j++) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(bf[kk][j], af[kk][i], acc[i][j], 0, 0, 0);
      }
      __builtin_amdgcn_sched_barrier(0);
    });
    rd = rd + 1 == T::NS ? 0 : rd + 1;
    wr = wr + 1 == T::NS ? 0 : wr + 1;
  }
  Q8Scales<T, typename T::EpiStage> scales;
  scales.load(op, m0, n0, wave, lane);
  wait_vmcnt<0>();
  __syncthreads();           // the ring is dead from here on
  q8_epilogue<T, OUT, EDGE>(op, acc, scales, typename T::EpiStage{smem + wave * T::STAGE_BYTES}, wave, lane, m0, n0);
}

template <class T, int OUT, bool EDGE, bool TAIL, bool ONCE>
hipError_t launch_q8_ring_as(const Q8Op& op, hipStream_t st) {
  auto kern = q8_ring_kernel<T, OUT, EDGE, TAIL, ONCE>;
  // one-time opt-in to more than 64 KB of dynamic LDS (thread-safe function-local static)
  static const hipError_t attr_err = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, T::LDS_BYTES);
  if (attr_err != hipSuccess) return attr_err;
  const int tiles_m = (op.M + T::BM - 1) / T::BM, tiles_n = (op.N + T::BN - 1) / T::BN;
  hipLaunchKernelGGL(kern, dim3((uint32_t)tiles_m * tiles_n), dim3(T::NT), T::LDS_BYTES, st, op, tiles_m, tiles_n);
  return hipGetLastError();
}
template <class T, int OUT, bool EDGE, bool TAIL>
hipError_t launch_q8_ring(const Q8Op& op, hipStream_t st) {
  const bool once = op.M <= T::BM && (int64_t)op.N * op.K >= 16 << 20;
  return once ? launch_q8_ring_as<T, OUT, EDGE, TAIL, true>(op, st) : launch_q8_ring_as<T, OUT, EDGE, TAIL, false>(op, st);
}

// ---- 256 x 256 tiles: at most one workgroup per CU, which walks its tiles in one stream of slices --------
// The schedule of the bf16 kernel of these tiles (gemm_bf16.hip, where it is explained): three A and two B slots of LDS, loads up to two
// slices ahead and into the next tile, a slice in four steps whose operands are read one step ahead.
struct Big {
  static constexpr int BM = 256, BN = 256, WM = 4, WN = 2, NW = 8, NT = 512;
  static constexpr int TM = 64, TN = 128, FM = 2, FN = 4;
  static constexpr int A_BYTES = BM * 128, B_BYTES = BN * 128;
  static constexpr int WLA = BM / 8 / NW, WLB = BN / 8 / NW, NSA = 3, NSB = 2;
  static constexpr int LDS_BYTES = NSA * A_BYTES + NSB * B_BYTES;
  struct EpiStage {          // 16 rows x 64 columns per wavefront in four 1 KB pieces of the free A slot that its own loads fill
    static constexpr int SR = 16, SC = 64;
    unsigned char* p;
    __device__ __forceinline__ unsigned char* at(int row, int chunk) const {
      return p + (row >> 2) * (NW * 1024) + (row & 3) * 256 + ((chunk ^ row) << 4);
    }
  };
};
constexpr int Q8_CUS = 256;

template <int OUT, bool EDGE, bool TAIL>
__global__ __launch_bounds__(Big::NT) void q8_big_kernel(Q8Op op, int tiles_m, int tiles_n, int total) {
  using T = Big;
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int wm = wave / T::WN, wn = wave % T::WN;
  const int bid = blockIdx.x, nwg = gridDim.x, xcd = bid % NXCD;
  const int step = nwg / NXCD + (xcd < nwg % NXCD ? 1 : 0);
  const int tiles_first = xcd * (total / NXCD) + min(xcd, total % NXCD);
  const int tiles_end = tiles_first + total / NXCD + (xcd < total % NXCD ? 1 : 0);
  const int kbytes = (op.K + 15) / 16 * 16;
  const int nk = max((kbytes + 127) / 128, total > nwg ? 2 : 1);      // (two slices of the next tile are under way before an epilogue)
  struct Source {
    const int8_t *a, *b;
    uint32_t rec_a, rec_b;   // bytes behind them that may be read; what lies beyond arrives as zeros
    int m0, n0;
  };
  auto source = [&](int nid) -> Source {
    Source s;
    int tm, tn, bz;
    tile_of_index(nid, tiles_m, tiles_n, tm, tn, bz);
    s.m0 = tm * T::BM;
    s.n0 = tn * T::BN;
    s.a = op.A + (int64_t)s.m0 * op.lda;
    s.b = op.B + (int64_t)s.n0 * op.ldb;
    s.rec_a = (uint32_t)((min(T::BM, op.M - s.m0) - 1) * (int)op.lda + kbytes);
    s.rec_b = (uint32_t)((min(T::BN, op.N - s.n0) - 1) * (int)op.ldb + kbytes);
    return s;
  };
  int nid = tiles_first + bid / NXCD;
  Source cur = source(nid), nxt = cur;
  constexpr uint32_t OOB = 0x80000000u;
  const int lrow = lane >> 3, lchunk = (lane & 7) ^ (((wave & 1) << 2) | (lrow >> 1));
  uint32_t goff[T::WLA + T::WLB];
#pragma unroll
  for (int i = 0; i < T::WLA + T::WLB; i++) {
    const bool is_a = i < T::WLA;
    const int g = wave + T::NW * (is_a ? i : i - T::WLA);
    goff[i] = (uint32_t)((g * 8 + lrow) * (int)(is_a ? op.lda : op.ldb) + lchunk * 16);
  }
  uint32_t a0 = 0, a1 = T::A_BYTES, a2 = 2 * T::A_BYTES, b0 = T::NSA * T::A_BYTES, b1 = b0 + T::B_BYTES;
  auto issue = [&](int kt, uint32_t slot, auto IS_A, auto HALF) {      // HALF: 0, 1 or both (2)
    constexpr bool is_a = decltype(IS_A)::value;
    constexpr int half = decltype(HALF)::value;
    const bool here = kt < nk;
    const int ks = here ? kt : kt - nk;
    const uint32_t skip = (uint32_t)ks * 128u;
    const __amdgpu_buffer_rsrc_t rs = __builtin_amdgcn_make_buffer_rsrc((void*)(here ? (is_a ? cur.a : cur.b) : (is_a ? nxt.a : nxt.b)), 0,
                                                                        here ? (is_a ? cur.rec_a : cur.rec_b) : (is_a ? nxt.rec_a : nxt.rec_b), 0x00020000);
    const uint32_t mask = (int)skip + lchunk * 16 < kbytes ? 0u : OOB;
    unsigned char* dst = smem + slot + wave * 1024;
    constexpr int F0 = is_a ? 0 : T::WLA, F1 = is_a ? T::WLA : T::WLA + T::WLB;
    constexpr int I0 = half == 1 ? (F0 + F1) / 2 : F0, I1 = half == 0 ? (F0 + F1) / 2 : F1;
#pragma unroll
    for (int i = I0; i < I1; i++)
      __builtin_amdgcn_raw_ptr_buffer_load_lds(rs, LRB_LDS_PTR(dst + (i - F0) * (T::NW * 1024)), 16, (int)((goff[i] + skip) | mask), 0, 0, 0);
  };
  using Half0 = std::integral_constant<int, 0>;
  using Half1 = std::integral_constant<int, 1>;
  using Whole = std::integral_constant<int, 2>;
  constexpr std::true_type OPA{};
  constexpr std::false_type OPB{};
  const Tail tail(op.K);
  i32x16 acc[T::FM][T::FN];
  const int frow = lane & 31, fk = lane >> 5, fsw = (frow >> 1) & 7;
  i32x4 af[2][T::FM], bf[2][T::FN];
  auto load_frags = [&](int buf, uint32_t slot_a, uint32_t slot_b, int kk) {
    const unsigned char* sa = smem + slot_a + (wm * T::TM + frow) * 128;
    const unsigned char* sb = smem + slot_b + (wn * T::TN + frow) * 128;
    const int co = ((kk * 2 + fk) ^ fsw) << 4;
#pragma unroll
    for (int i = 0; i < T::FM; i++) af[buf][i] = *reinterpret_cast<const i32x4*>(sa + i * 32 * 128 + co);
#pragma unroll
    for (int j = 0; j < T::FN; j++) bf[buf][j] = *reinterpret_cast<const i32x4*>(sb + j * 32 * 128 + co);
  };
  auto multiply = [&](int buf, int chunk, auto ZERO) {
    constexpr i32x16 zero = {0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0};
#pragma unroll
    for (int i = 0; i < T::FM; i++) {
      const i32x4 a = TAIL ? tail.of(af[buf][i], chunk) : af[buf][i];
#pragma unroll
      for (int j = 0; j < T::FN; j++) acc[i][j] = __builtin_amdgcn_mfma_i32_32x32x32_i8(bf[buf][j], a, decltype(ZERO)::value ? zero : acc[i][j], 0, 0, 0);
    }
  };
  constexpr int MPR = (T::FM * T::FN) / (T::FM + T::FN);
  auto interleave = [&](auto N) {      // the operand reads and N loads among the MFMAs
    constexpr int n = decltype(N)::value;
#pragma unroll
    for (int i = 0; i < T::FM + T::FN; i++) {
      __builtin_amdgcn_sched_group_barrier(0x008, MPR, 0);
      __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      if (i * n / (T::FM + T::FN) != (i + 1) * n / (T::FM + T::FN)) __builtin_amdgcn_sched_group_barrier(0x020, 1, 0);
    }
    __builtin_amdgcn_sched_barrier(0);
  };
  constexpr int STORES = T::TM * T::TN / (64 * 8) * (OUT == LR_F32 ? 2 : 1);      // that an epilogue certainly issues
  static_assert(T::WLA + STORES < 64, "vmcnt is a 6-bit counter");
  bool stores_fly = false;
  auto slice = [&](int kt, auto FIRST) {
    constexpr bool first = decltype(FIRST)::value;
    static_for<3>([&](auto KK) {
      constexpr int kk = decltype(KK)::value;
      load_frags((kk + 1) & 1, a0, b0, kk + 1);
      if constexpr (kk == 0 && !first) issue(kt + 1, b1, OPB, Half1{});
      if constexpr (kk == 1) issue(kt + 2, a2, OPA, Half0{});
      if constexpr (kk == 2) issue(kt + 2, a2, OPA, Half1{});
      multiply(kk & 1, kt * 8 + kk * 2 + fk, std::integral_constant<bool, first && kk == 0>{});
      interleave(std::integral_constant<int, (kk > 0 ? T::WLA / 2 : first ? 0 : T::WLB / 2)>{});
    });
    // (behind an epilogue the scales' loads lie between its stores and this slice's loads, so most of its stores are waited for too)
    if (first && stores_fly) wait_vmcnt<(T::WLA + STORES)>();
    else wait_vmcnt<T::WLA>();
    wait_lgkmcnt0();
    __builtin_amdgcn_s_barrier();
    __builtin_amdgcn_sched_barrier(0);
    issue(kt + 2, b0, OPB, Half0{});
    load_frags(0, a1, b1, 0);
    multiply(1, kt * 8 + 6 + fk, std::false_type{});
    interleave(std::integral_constant<int, T::WLB / 2>{});
    const uint32_t a = a0, b = b0;
    a0 = a1; a1 = a2; a2 = a;
    b0 = b1; b1 = b;
  };
  issue(0, a0, OPA, Whole{});
  issue(0, b0, OPB, Whole{});
  issue(1, a1, OPA, Whole{});
  issue(1, b1, OPB, Whole{});
  wait_vmcnt<T::WLA + T::WLB>();
  __builtin_amdgcn_s_barrier();
  while (true) {
    const int nid_next = nid + step;
    const bool more = nid_next < tiles_end;
    if (more) nxt = source(nid_next);
    else nxt.rec_a = nxt.rec_b = 0;
    Q8Scales<T, Big::EpiStage> scales;      // (asked for here, they don't wait behind the next tile's slices)
    scales.load(op, cur.m0, cur.n0, wave, lane);
    load_frags(0, a0, b0, 0);
    slice(0, std::true_type{});
    for (int kt = 1; kt < nk; kt++) slice(kt, std::false_type{});
    int elane = lane, ewave = wave;
    asm volatile("" : "+v"(elane), "+s"(ewave));      // (the epilogue's addresses stay out of the loop over tiles)
    issue(nk + 1, b1, OPB, Half1{});
    __builtin_amdgcn_sched_barrier(0);
    q8_epilogue<T, OUT, EDGE>(op, acc, scales, Big::EpiStage{smem + a2 + wave * 1024}, ewave, elane, cur.m0, cur.n0);
    if (!more) break;
    stores_fly = true;
    nid = nid_next;
    cur = nxt;
  }
  wait_vmcnt<STORES>();      // no load into LDS outlives its workgroup
}

template <int OUT, bool EDGE, bool TAIL>
hipError_t launch_q8_big(const Q8Op& op, hipStream_t st) {
  auto kern = q8_big_kernel<OUT, EDGE, TAIL>;
  static const hipError_t attr_err = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, Big::LDS_BYTES);
  if (attr_err != hipSuccess) return attr_err;
  const int tiles_m = (op.M + 255) / 256, tiles_n = (op.N + 255) / 256, total = tiles_m * tiles_n;
  hipLaunchKernelGGL(kern, dim3((uint32_t)(total < Q8_CUS ? total : Q8_CUS)), dim3(Big::NT), Big::LDS_BYTES, st, op, tiles_m, tiles_n, total);
  return hipGetLastError();
}

// ---- 16 x 16 pieces: few rows --------------------------------------------------------------------
// A workgroup takes 16 rows and NT * 16 columns over all of k: A and B lie in LDS as they are (up to `chunk` k at a time), its 16 wavefronts take every
// 16th step of 64 k each (v_mfma_i32_16x16x64_i8) and the 16 sums are added up through LDS.
//
// QUADS: A comes as rows of type KIND, which every workgroup quantises for itself, a wavefront a row: it holds the row (of up to 64 * 4 * QUADS columns) in
// registers, whose largest element needs no other wavefront.  Bound: the way in and out of a launch, and what a CU takes in.
// The layer 4096 -> 1024 -> 4096 of 16 tokens, us: 11.3 so in its second product, 12.7 with a launch for the quantisation between the products.  In the first
// product, where every workgroup does the rows' whole work, up to 2^15 elements: of 1 / 8 / 16 tokens, with a launch before it, 10.1 / 10.6 / 11.3, without
// 8.2 / 9.1 / 11.2; 1024 -> 256 -> 1024 9.2 / 9.2 / 9.4 and 6.0 / 6.0 / 6.5; 4096 -> 4096 -> 4096 in fp32 13.9 / 15.8 / 17.2 and 12.1 / 14.8 / 17.2.
constexpr int R16_W = 16, R16_SLICE = 2048, R16_LDS = 160 * 1024;
constexpr int rows16_lds(int chunk, int nt) { return chunk / 128 * R16_SLICE * (1 + nt) + R16_W * nt * 1024; }

// four elements of a row, as they are stored (fp32 rows may start anywhere) and as floats
typedef float f32x4_anywhere __attribute__((ext_vector_type(4), aligned(4)));
typedef uint32_t u32x2_t __attribute__((ext_vector_type(2)));
template <Rows KIND> struct Four { typedef f32x4_anywhere In; typedef f32x4 V; typedef float X; };
template <> struct Four<Rows::BF16> { typedef u32x2_t In, V; typedef uint16_t X; };
__device__ __forceinline__ void floats_of(const f32x4& v, float* f) {
#pragma unroll
  for (int e = 0; e < 4; e++) f[e] = v[e];
}
__device__ __forceinline__ void floats_of(const u32x2_t& v, float* f) {
#pragma unroll
  for (int e = 0; e < 4; e++) f[e] = __uint_as_float(e & 1 ? v[e / 2] & 0xffff0000u : v[e / 2] << 16);
}

template <int QUADS, Rows KIND, int NT, int OUT, bool TAIL>
__global__ __launch_bounds__(R16_W * 64) void q8_rows16_kernel(Q8Op op, const void* xs, int64_t ldx, int chunk) {
  extern __shared__ __attribute__((aligned(16))) unsigned char smem[];
  __shared__ float row_scale[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int m0 = blockIdx.y * 16, n0 = blockIdx.x * (NT * 16);
  const int kbytes = (op.K + 15) / 16 * 16, slices = chunk / 128;
  unsigned char* sB = smem + slices * R16_SLICE;                 // then NT of these
  int* part = reinterpret_cast<int*>(sB + NT * slices * R16_SLICE);
  const uint32_t lds = (uint32_t)(uintptr_t)LRB_LDS_PTR(smem);
  const rsrc_words rsB = operand_rsrc(op.B + (int64_t)n0 * op.ldb), rsA = operand_rsrc(QUADS ? op.B : op.A + (int64_t)m0 * op.lda);
  // Loads of 8 rows x 128 bytes: the rows of A (as int8), then those of B, slice by slice
  constexpr int FIRST_OP = QUADS ? 1 : 0, PER = 2 * (1 + NT - FIRST_OP);
  auto load = [&](int k0) {
    for (int id = wave; id < slices * PER; id += R16_W) {
      const int slice = id / PER, w = id % PER + 2 * FIRST_OP, o = w >> 1;      // o: 0 A, then the 16 columns of B
      const int row = (w & 1) * 8 + (lane >> 3), lc = (lane & 7) ^ ((row >> 1) & 7);
      const int k = k0 + slice * 128 + lc * 16;
      const bool in = k < kbytes && (o == 0 ? m0 + row < op.M : n0 + (o - 1) * 16 + row < op.N);
      const uint32_t off = in ? (o == 0 ? (uint32_t)row * (uint32_t)op.lda : (uint32_t)((o - 1) * 16 + row) * (uint32_t)op.ldb) + (uint32_t)k : RING_OOB;
      dma16<true>(o == 0 ? rsA : rsB, lds + (uint32_t)((o * slices + slice) * R16_SLICE + (w & 1) * 1024), off);
    }
  };
  i32x4 acc[NT] = {};
  const Tail tail(op.K);
  auto multiply = [&](int k0) {
    const int row = lane & 15, sw = (row >> 1) & 7;
    for (int step = wave; step < 2 * slices; step += R16_W) {
      const int at = (step >> 1) * R16_SLICE + row * 128 + ((((step & 1) * 4 + (lane >> 4)) ^ sw) << 4);
      i32x4 fa = *reinterpret_cast<const i32x4*>(smem + at);
      if constexpr (!QUADS && TAIL) fa = tail.of(fa, (k0 + step * 64) / 16 + (lane >> 4));
#pragma unroll
      for (int j = 0; j < NT; j++)
        acc[j] = __builtin_amdgcn_mfma_i32_16x16x64_i8(*reinterpret_cast<const i32x4*>(sB + j * slices * R16_SLICE + at), fa, acc[j], 0, 0, 0);
    }
  };
  if constexpr (!QUADS) {
    for (int k0 = 0; k0 < kbytes; k0 += chunk) {
      load(k0);
      wait_vmcnt<0>();
      __syncthreads();
      multiply(k0);
      __syncthreads();
    }
    if (tid < 16) row_scale[tid] = m0 + tid < op.M ? op.sa[m0 + tid] : 0.f;
  } else {
    typename Four<KIND>::V v[QUADS];
    const bool has = m0 + wave < op.M;
    using F = Four<KIND>;
    const typename F::X* px = (const typename F::X*)xs + (int64_t)(m0 + wave) * ldx;
#pragma unroll
    for (int i = 0; i < QUADS; i++) {
      const int k = (i * 64 + lane) * 4;
      v[i] = typename F::V{};
      if (has && k < op.K) v[i] = *reinterpret_cast<const typename F::In*>(px + k);
    }
    load(0);
    if (has) {                                         // (behind the last row anything: its products are not stored)
      uint32_t most = 0;
#pragma unroll
      for (int i = 0; i < QUADS; i++) {
        float f[4];
        floats_of(v[i], f);
#pragma unroll
        for (int e = 0; e < 4; e++) most = max(most, __float_as_uint(f[e]) & 0x7fffffffu);
      }
      most = wave_max(most);
      const Scale<KIND> sc(most);
      if (lane == 0) row_scale[wave] = sc.scale;
      const int sw = (wave >> 1) & 7;
#pragma unroll
      for (int i = 0; i < QUADS; i++) {
        const int k = (i * 64 + lane) * 4;
        float f[4];
        floats_of(v[i], f);
        // (of a row without a scale anything: it is multiplied with NaN)
        if (k < chunk) *reinterpret_cast<uint32_t*>(smem + (k >> 7) * R16_SLICE + wave * 128 + ((((k >> 4) & 7) ^ sw) << 4) + (k & 15)) = sc.bytes(f);
      }
    }
    wait_vmcnt<0>();
    __syncthreads();
    multiply(0);
  }
  // operands exchanged: lane -> row lane % 16, columns 4 (lane / 16) + 0..3
#pragma unroll
  for (int j = 0; j < NT; j++) *reinterpret_cast<i32x4*>(part + wave * (NT * 256) + j * 256 + lane * 4) = acc[j];
  __syncthreads();
  for (int t = tid; t < NT * 256; t += R16_W * 64) {
    int sum = 0;
#pragma unroll
    for (int w = 0; w < R16_W; w++) sum += part[w * (NT * 256) + t];
    const int l = (t >> 2) & 63, m = l & 15, n = n0 + (t >> 8) * 16 + (l >> 4) * 4 + (t & 3);
    if (m0 + m < op.M && n < op.N) {
      const float c = act_f((float)sum * row_scale[m] * op.sb[n], op.act);
      if constexpr (OUT == LR_BF16) ((uint16_t*)op.C)[(int64_t)(m0 + m) * op.ldc + n] = (uint16_t)f32_to_bf16_bits(c);
      else ((float*)op.C)[(int64_t)(m0 + m) * op.ldc + n] = c;
    }
  }
}

// 16-column pieces of a workgroup that quantises its rows: as many as leave about a workgroup per CU
int rows16_nt(int64_t N) { return N <= 256 * 16 ? 1 : N <= 512 * 16 ? 2 : 4; }

template <int QUADS, Rows KIND, int NT, int OUT, bool TAIL>
hipError_t launch_rows16_nt(const Q8Op& op, const void* x, int64_t ldx, hipStream_t st) {
  auto kern = q8_rows16_kernel<QUADS, KIND, NT, OUT, TAIL>;
  // one-time opt-in to more than 64 KB of dynamic LDS (thread-safe function-local static)
  static const hipError_t attr_err = hipFuncSetAttribute((const void*)kern, hipFuncAttributeMaxDynamicSharedMemorySize, R16_LDS - 256);
  if (attr_err != hipSuccess) return attr_err;
  const int whole = (op.K + 127) / 128 * 128;
  int chunk = whole;
  while (rows16_lds(chunk, NT) > R16_LDS - 256) chunk = (chunk / 2 + 127) / 128 * 128;      // (int8 alone: several turns of even length)
  if (QUADS && (chunk != whole || op.K > QUADS * 256)) return hipErrorInvalidValue;
  const dim3 grid((uint32_t)((op.N + NT * 16 - 1) / (NT * 16)), (uint32_t)((op.M + 15) / 16));
  hipLaunchKernelGGL(kern, grid, dim3(R16_W * 64), rows16_lds(chunk, NT), st, op, x, ldx, chunk);
  return hipGetLastError();
}
template <int QUADS, Rows KIND, int OUT>
hipError_t launch_rows16_of(const Q8Op& op, const void* x, int64_t ldx, hipStream_t st) {
  switch (rows16_nt(op.N)) {
    case 1: return launch_rows16_nt<QUADS, KIND, 1, OUT, false>(op, x, ldx, st);
    case 2: return launch_rows16_nt<QUADS, KIND, 2, OUT, false>(op, x, ldx, st);
    default: return launch_rows16_nt<QUADS, KIND, 4, OUT, false>(op, x, ldx, st);
  }
}
template <Rows KIND, int OUT>
hipError_t launch_rows16_from(const Q8Op& op, const void* x, int64_t ldx, hipStream_t st) {
  return op.K <= 1024 ? launch_rows16_of<4, KIND, OUT>(op, x, ldx, st) : launch_rows16_of<16, KIND, OUT>(op, x, ldx, st);
}

using R64x128 = RingTile<64, 128, 2, 2, 1, 3>;      // two workgroups per CU
using R128 = RingTile<128, 128, 2, 4, 1, 5>;
using R64 = RingTile<64, 64, 2, 2, 2, 5>;

enum Q8Tile : int { Q8_BIG, Q8_R128, Q8_R64X128, Q8_R64, Q8_ROWS16 };

template <int OUT, bool EDGE, bool TAIL>
hipError_t launch_q8(const Q8Op& op, int tile, hipStream_t st) {
  switch (tile) {
    case Q8_BIG: return launch_q8_big<OUT, EDGE, TAIL>(op, st);
    case Q8_R128: return launch_q8_ring<R128, OUT, EDGE, TAIL>(op, st);
    case Q8_R64X128: return launch_q8_ring<R64x128, OUT, EDGE, TAIL>(op, st);
    case Q8_R64: return launch_q8_ring<R64, OUT, EDGE, TAIL>(op, st);
    default: return launch_rows16_nt<0, Rows::F32, 1, OUT, TAIL>(op, nullptr, 0, st);
  }
}

// The tile with the shortest estimate: a launch's fixed time, and for every round of `slots` workgroups one of its own and s0 + s1 for each slice of
// 128 k; of the last round, as much of e1 and s1 as its share of the slots.  Fitted to 375 shapes (16 to 16384 rows, 256 to 32000 columns, k 64 to 11008;
// estimates are off by 2 % in the median, 8 to 16 % at the 95th percentile); taking the shortest estimate loses 0.3 % on average and 28 % at most to the
// fastest tile.  us, 256 x 256 / 128 x 128 / 64 x 128 / 64 x 64: 16384 x 4096 x 4096 225 / 328 / 361 / 555, 4096 x 2048 x 1024 18.5 / 16.6 / 16.8 / 32.7,
// 1031 x 4096 x 256 9.5 / 10.0 / 8.4 / 15.1, 512 x 1024 x 4096 37.7 / 16.4 / 12.8 / 9.9.
// Up to 512 pieces of 16 x 16, two for each CU, run as those: 16 x 1024 x 4096 3.8 (9.4 on 64 x 64), 64 x 1024 x 1024 4.1 (5.5), 16 x 8192 x 4096 10.8 (13.1),
// 128 x 1024 x 4096 7.9 (9.9); with 1024 of them, 128 x 2048 x 1024, 6.7 (5.5).
int q8_tile(const Q8Op& op) {
  auto up = [](int64_t a, int64_t b) { return (a + b - 1) / b; };
  if (up(op.M, 16) * up(op.N, 16) <= 512) return Q8_ROWS16;
  struct Cost { int rows, cols, slots, threads; double f, e, e1, s0, s1; };      // threads: of a workgroup per tile
  static constexpr Cost cost[] = {{256, 256, 256, 0, 4.06, 2.35, 3.45, 0.935, 0.568}, {128, 128, 256, R128::NT, 2.53, 2.07, 0.95, 0.345, 0.186},
                                  {64, 128, 512, R64x128::NT, 3.00, 0.95, 1.40, 0.252, 0.353}, {64, 64, 256, R64::NT, 2.27, 2.00, 0.22, 0.159, 0.050}};
  const double slices = (double)up(op.K, 128);
  int best = 0;
  double least = 0;
  for (int t = 0; t < 4; t++) {
    const Cost& c = cost[t];
    const int64_t tiles = up(op.M, c.rows) * up(op.N, c.cols);
    if (tiles * c.threads >= (int64_t)1 << 32) continue;      // more than a launch may have (2^30 rows and a few columns); the stream of 256 x 256 tiles has 256 workgroups
    const double fill = (double)(tiles % c.slots) / c.slots;
    double us = c.f + (double)(tiles / c.slots) * (c.e + c.e1 + slices * (c.s0 + c.s1));
    if (fill > 0) us += c.e + c.e1 * fill + slices * (c.s0 + c.s1 * fill);
    if (t == 0 || us < least) {
      best = t;
      least = us;
    }
  }
  return best;
}

}  // namespace

void gemm_q8_tile_size(const Q8Op& op, int* rows, int* cols) {
  static constexpr int size[][2] = {{256, 256}, {128, 128}, {64, 128}, {64, 64}, {16, 16}};
  const int tile = q8_tile(op);
  *rows = size[tile][0];
  *cols = size[tile][1];
}
bool gemm_q8_acts(const Q8Op& op) { return q8_tile(op) == Q8_ROWS16; }
bool gemm_q8_quantises(int64_t M, int64_t N, int64_t K) {
  return M <= 16 && K <= 4096 && K % 4 == 0 && rows16_lds((int)(K + 127) / 128 * 128, rows16_nt(N)) <= R16_LDS - 256;
}
hipError_t gemm_q8_from(const Q8Op& op, const void* x, int64_t ldx, int dt, hipStream_t st) {
  if (dt == LR_BF16) return op.dt == LR_F32 ? launch_rows16_from<Rows::BF16, LR_F32>(op, x, ldx, st) : hipErrorInvalidValue;
  return op.dt == LR_BF16 ? launch_rows16_from<Rows::F32, LR_BF16>(op, x, ldx, st) : launch_rows16_from<Rows::F32, LR_F32>(op, x, ldx, st);
}

hipError_t gemm_q8(const Q8Op& op, hipStream_t st) {
  const int tile = q8_tile(op);
  const bool edge = op.N % 8 != 0, tail = op.K % 16 != 0;
  const int form = (op.dt == LR_F32) * 4 + edge * 2 + tail;
  switch (form) {
    case 0: return launch_q8<LR_BF16, false, false>(op, tile, st);
    case 1: return launch_q8<LR_BF16, false, true>(op, tile, st);
    case 2: return launch_q8<LR_BF16, true, false>(op, tile, st);
    case 3: return launch_q8<LR_BF16, true, true>(op, tile, st);
    case 4: return launch_q8<LR_F32, false, false>(op, tile, st);
    case 5: return launch_q8<LR_F32, false, true>(op, tile, st);
    case 6: return launch_q8<LR_F32, true, false>(op, tile, st);
    default: return launch_q8<LR_F32, true, true>(op, tile, st);
  }
}

}  // namespace lrb
