// Pages of a key / value cache: who holds them (fork), where they lie (compact), and their copies.
//
// A page's count says how many entries of page tables hold it (and whoever else does); pages of count 0 are free.  Fork and compact
// read the old lists and write new ones, so that a step that finds too few pages can be taken back.  Fresh pages are the lowest free
// ones, given to the sequences in order: sums of whole numbers and prefix counts, so the same lists give the same result.
#include "lanes.h"

namespace lrb {
namespace {

__device__ __forceinline__ int lane_id() { return __builtin_amdgcn_mbcnt_hi(~0u, __builtin_amdgcn_mbcnt_lo(~0u, 0u)); }
__device__ __forceinline__ int lanes_below(uint64_t mask) {
  return __builtin_amdgcn_mbcnt_hi((uint32_t)(mask >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)mask, 0u));
}

// Sum of v over the workgroup's threads before this one, and over all of them.  scratch: one entry for each of its NW wavefronts, free again after the call.
template <class V, int NW>
__device__ __forceinline__ V block_prefix(V v, V (&scratch)[NW], V* total) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const V incl = wave_prefix(v);
  if (lane == 63) scratch[wave] = incl;
  __syncthreads();
  V before = 0, all = 0;
#pragma unroll
  for (int w = 0; w < NW; w++) {
    const V s = scratch[w];
    before += w < wave ? s : 0;
    all += s;
  }
  __syncthreads();
  *total = all;
  return before + incl - v;
}

constexpr int PLAN_T = 1024;      // threads of the planning workgroup
constexpr int PLAN_PER = 8;       // counts per thread and step of its search for free pages

// What the new sequence i is made of.
struct Child {
  int parent;                // -1: none
  int64_t old, now;          // keys so far, with the new ones
  int full, part;            // whole pages of the keys so far, keys behind them
};
__device__ __forceinline__ Child child_of(const KvFork& f, int i) {
  Child c;
  const int p = f.parent[i];
  c.parent = p >= 0 && p < f.n_in ? p : -1;
  c.old = c.parent >= 0 ? max(f.len_in[c.parent], 0) : 0;
  c.now = c.old + max(f.grow[i], 0);
  c.full = (int)f.by_page.div((uint32_t)c.old);
  c.part = (int)c.old - c.full * f.page_size;
  return c;
}
__device__ __forceinline__ bool is_page(const KvFork& f, int e) { return (uint32_t)e < (uint32_t)f.n_pages; }

// Workgroup 0 plans: the first child of every parent, how many fresh pages each child takes, and the first so many free ones.  The
// others copy the counts, which the second launch moves on.
//
// Bound: latency, of the lists that lead to each other and of the search through the counts: PLAN_T * PLAN_PER of them per step of
// about a microsecond, no further than needed.  48 sequences 4.7 us, 512 beams 6.1.
__global__ __launch_bounds__(PLAN_T) void fork_plan_kernel(KvFork f) {
  const int tid = threadIdx.x;
  if (blockIdx.x > 0) {
    for (int64_t i = (int64_t)(blockIdx.x - 1) * PLAN_T + tid; i < f.n_pages; i += (int64_t)(gridDim.x - 1) * PLAN_T) f.refs_out[i] = f.refs_in[i];
    return;
  }
  extern __shared__ int first[];          // [n_in] the first child of a parent, then [n_in] its children
  __shared__ int64_t scratch[PLAN_T / 64];
  __shared__ int steps[PLAN_T / 64];
  __shared__ unsigned long long beyond;   // pages that no column of the table is left for
  if (tid == 0) beyond = 0;
  int* count = first + f.n_in;
  for (int p = tid; p < f.n_in; p += PLAN_T) {
    first[p] = 0x7fffffff;
    count[p] = 0;
  }
  __syncthreads();
  for (int i = tid; i < f.n_out; i += PLAN_T) {
    const int p = f.parent[i];
    if (p >= 0 && p < f.n_in) {
      atomicMin(&first[p], i);
      atomicAdd(&count[p], 1);
    }
  }
  __syncthreads();
  int64_t want = 0;                       // fresh pages so far
  for (int i0 = 0; i0 < f.n_out; i0 += PLAN_T) {
    const int i = i0 + tid;
    int64_t need = 0, over = 0;
    if (i < f.n_out) {
      const Child c = child_of(f, i);
      const int last = (int)min((c.now + f.page_size - 1) / f.page_size, (int64_t)f.max_pages);      // columns with keys
      over = (c.now + f.page_size - 1) / f.page_size - last;
      const bool heir = c.parent >= 0 && first[c.parent] == i;
      int flags = heir ? 1 : 0;
      need = max(last - c.full, 0);
      if (heir) {
        const int32_t* row = f.table_in + (int64_t)c.parent * f.ld_in;
        // the half filled page stays where nobody else holds it
        if (c.part > 0 && c.full < f.max_pages) {
          const int e = row[c.full];
          if (is_page(f, e) && f.refs_in[e] == 1) {
            flags |= 2;
            need--;
          }
        }
#pragma unroll 8
        for (int col = c.full + (c.part > 0 ? 1 : 0); col < last; col++) need -= is_page(f, row[col]) ? 1 : 0;
      }
      f.flags[i] = flags;
    }
    int64_t all;
    const int64_t at = want + block_prefix(need, scratch, &all);
    if (i < f.n_out) f.offset[i] = (int)min(at, (int64_t)f.n_pages);
    want += all;
    if (over > 0) atomicAdd(&beyond, (unsigned long long)over);
  }
  __syncthreads();
  for (int p = tid; p < f.n_in; p += PLAN_T) {
    f.first[p] = first[p];
    f.count[p] = count[p];
  }
  int64_t found = 0;
  const bool vec = ((uintptr_t)f.refs_in & 15) == 0;
  for (int64_t p0 = 0; p0 < f.n_pages && found < want; p0 += PLAN_T * PLAN_PER) {
    const int64_t p = p0 + tid * PLAN_PER;
    int r[PLAN_PER];
    if (vec && p + PLAN_PER <= f.n_pages) {
#pragma unroll
      for (int j = 0; j < PLAN_PER; j += 4) *reinterpret_cast<int4*>(r + j) = *reinterpret_cast<const int4*>(f.refs_in + p + j);
    } else {
#pragma unroll
      for (int j = 0; j < PLAN_PER; j++) r[j] = p + j < f.n_pages ? f.refs_in[p + j] : 1;
    }
    int mine = 0, all;
#pragma unroll
    for (int j = 0; j < PLAN_PER; j++) mine += r[j] == 0;
    int64_t at = found + block_prefix(mine, steps, &all);
#pragma unroll
    for (int j = 0; j < PLAN_PER; j++)
      if (r[j] == 0 && at < f.n_pages) f.fresh[at++] = (int)(p + j);
    found += all;
  }
  if (tid == 0) {
    const int64_t lack = max(want - found, (int64_t)0) + (int64_t)beyond;
    *f.found = (int)min(found, (int64_t)f.n_pages);
    *f.missing = (int)min(lack, (int64_t)0x7fffffff);
  }
}

// One wavefront per row: the new tables, lengths and copies, and how the old tables' pages change hands.  Bound: latency; 512 beams 3.8 us.
__global__ __launch_bounds__(256) void fork_rows_kernel(KvFork f) {
  const int lane = threadIdx.x & 63;
  const int row = (int)blockIdx.x * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  if (row < f.n_out) {
    const int i = row;
    const Child c = child_of(f, i);
    const int flags = f.flags[i], found = *f.found;
    const bool heir = flags & 1, alone = flags & 2;
    const int32_t* in = f.table_in + (int64_t)max(c.parent, 0) * f.ld_in;
    int32_t* out = f.table_out + (int64_t)i * f.ld_out;
    int at = f.offset[i];
    bool copied = false;
    for (int c0 = 0; c0 < f.max_pages; c0 += 64) {
      const int col = c0 + lane;
      const int e = c.parent >= 0 && col < f.max_pages ? in[col] : -1;
      const bool page = is_page(f, e), half = col == c.full && c.part > 0 && page;
      const bool keep = page && (col < c.full || (heir && (!half || alone)));
      const bool take = col < f.max_pages && col >= c.full && !keep && (int64_t)col * f.page_size < c.now;
      const uint64_t takers = __ballot(take);
      const int slot = at + lanes_below(takers);
      at = min(at + __popcll(takers), f.n_pages);      // (no more than there are: a table may have 2^31 columns, and slots are counted in 32 bits)
      const int got = take && slot < found ? f.fresh[slot] : -1;
      if (col < f.max_pages) out[col] = keep ? e : got;
      if (got >= 0) f.refs_out[got] = 1;
      const bool copy = half && got >= 0;
      if (copy) {
        f.copy_src[i] = e;
        f.copy_dst[i] = got;
        f.copy_rows[i] = c.part;
      }
      copied |= __ballot(copy) != 0;
    }
    if (lane == 0) {
      if (!copied) {
        f.copy_src[i] = f.copy_dst[i] = -1;
        f.copy_rows[i] = 0;
      }
      f.len_out[i] = (int)min(c.now, (int64_t)0x7fffffff);
    }
    return;
  }
  const int p = row - f.n_out;
  if (p >= f.n_in) return;
  const int children = f.count[p];
  const bool alone = children > 0 && (f.flags[f.first[p]] & 2);
  const uint32_t old = (uint32_t)max(f.len_in[p], 0);
  const int full = (int)f.by_page.div(old), part = (int)old - full * f.page_size;
  const int32_t* in = f.table_in + (int64_t)p * f.ld_in;
  for (int col = lane; col < f.max_pages; col += 64) {
    const int e = in[col];
    if (!is_page(f, e)) continue;
    // whole pages go to every child, the half filled one to an heir that nobody else shares it with, those behind to the heir
    const int by = col < full ? children - 1 : children == 0 || (col == full && part > 0 && !alone) ? -1 : 0;
    if (by != 0) atomicAdd(&f.refs_out[e], by);
  }
}

constexpr int SPAN_T = 256, SPAN_PER = 8, SPAN = SPAN_T * SPAN_PER;   // pages of a workgroup
constexpr int SPANS_FEW = 64 / SPAN_PER;       // spans whose pages every workgroup can count by itself

typedef int i32x4_anywhere __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ int held_mask(const KvCompact& c, int64_t p) {      // of SPAN_PER pages from p
  int m = 0;
  if (p + SPAN_PER <= c.n_pages) {
#pragma unroll
    for (int j = 0; j < SPAN_PER; j += 4) {
      const i32x4_anywhere r = *reinterpret_cast<const i32x4_anywhere*>(c.refs_in + p + j);
#pragma unroll
      for (int i = 0; i < 4; i++) m |= (r[i] > 0) << (j + i);
    }
  } else {
#pragma unroll
    for (int j = 0; j < SPAN_PER; j++) m |= (p + j < c.n_pages && c.refs_in[p + j] > 0) << j;
  }
  return m;
}

// Pages held of every span.
__global__ __launch_bounds__(SPAN_T) void compact_count_kernel(KvCompact c) {
  __shared__ int scratch[SPAN_T / 64];
  int all;
  block_prefix((int)__popc(held_mask(c, (int64_t)blockIdx.x * SPAN + threadIdx.x * SPAN_PER)), scratch, &all);
  if (threadIdx.x == 0) c.span_held[blockIdx.x] = all;
}

// With H the number of held pages: the j-th held page from H on moves into the j-th free one below H.  A page p below H has p - (held
// pages before it) free ones before it, one from H on (held pages before it) - (held pages below H) movers.
template <bool FEW>
__global__ __launch_bounds__(SPAN_T) void compact_lists_kernel(KvCompact c) {
  __shared__ int scratch[SPAN_T / 64];
  const int64_t p = (int64_t)blockIdx.x * SPAN + threadIdx.x * SPAN_PER;
  int held, low, rank, m;                        // held pages: of all, below page H, before this thread's; the latter's
  if constexpr (FEW) {                           // no count before: every workgroup looks at all pages, SPAN_PER bits of `all` per span
    __shared__ int64_t sums[SPAN_T / 64];
    uint64_t all = 0;
#pragma unroll
    for (int s = 0; s < SPANS_FEW; s++) all |= (uint64_t)held_mask(c, (int64_t)s * SPAN + threadIdx.x * SPAN_PER) << (s * SPAN_PER);
    const int shift = (int)blockIdx.x * SPAN_PER;
    m = (int)(all >> shift) & ((1 << SPAN_PER) - 1);
    // three sums at once, of 20 bits each: of all, of the spans before this one, of this one
    int64_t total;
    const int64_t below = block_prefix((int64_t)__popcll(all) | (int64_t)__popcll(all & ((1ull << shift) - 1)) << 20 | (int64_t)__popc(m) << 40, sums, &total);
    held = (int)(total & 0xfffff);
    rank = (int)(total >> 20 & 0xfffff) + (int)(below >> 40);
    int mine = 0;
#pragma unroll
    for (int s = 0; s < SPANS_FEW; s++) {
      const int n = held - (s * SPAN + (int)threadIdx.x * SPAN_PER), b = (int)(all >> (s * SPAN_PER)) & ((1 << SPAN_PER) - 1);
      mine += n <= 0 ? 0 : __popc(n >= SPAN_PER ? b : b & ((1 << n) - 1));
    }
    block_prefix(mine, scratch, &low);
  } else {
    int before = 0, all;
    held = low = 0;
    for (int s = threadIdx.x; s < c.spans; s += SPAN_T) {
      const int n = c.span_held[s];
      held += n;
      if (s < (int)blockIdx.x) before += n;
    }
    block_prefix(held, scratch, &all);
    held = all;
    block_prefix(before, scratch, &all);
    before = all;
    const int cut = held / SPAN;                 // the span of page H (held == n_pages: one behind the last)
    for (int s = threadIdx.x; s < min(cut, c.spans); s += SPAN_T) low += c.span_held[s];
    const int64_t pc = (int64_t)cut * SPAN + threadIdx.x * SPAN_PER, n = held - pc;
    const int b = held_mask(c, pc);
    low += n <= 0 ? 0 : __popc(n >= SPAN_PER ? b : b & ((1 << n) - 1));
    block_prefix(low, scratch, &all);
    low = all;
    m = held_mask(c, p);
    rank = before + block_prefix((int)__popc(m), scratch, &all);
  }
  const int moves = held - low, room = (int)(c.n_pages / 2);
#pragma unroll
  for (int j = 0; j < SPAN_PER; j++) {
    const int64_t page = p + j;
    if (page >= c.n_pages) break;
    const bool is = (m >> j) & 1;
    int to = -1;
    if (page < held) {
      if (is) to = (int)page;
      else if ((int)page - rank < room) c.copy_dst[(int)page - rank] = (int)page;
    } else if (is && rank - low < room) {
      c.copy_src[rank - low] = (int)page;
      to = -2 - (rank - low);                    // the third launch puts the page there
    }
    c.turn[page] = to;
    rank += is;
  }
  for (int64_t j = (int64_t)blockIdx.x * SPAN_T + threadIdx.x; j < room; j += (int64_t)gridDim.x * SPAN_T)
    if (j >= moves) c.copy_src[j] = c.copy_dst[j] = -1;
  if (blockIdx.x == 0 && threadIdx.x == 0) *c.n_live = held;
}

// The pages' new numbers, in the map, the counts and the table.  Bound: latency; 8192 pages 4.7 us.
__global__ __launch_bounds__(256) void compact_apply_kernel(KvCompact c) {
  const int64_t cells = (int64_t)c.batch * c.max_pages, total = c.n_pages + cells;
  const int held = *c.n_live;
  for (int64_t k = (int64_t)blockIdx.x * 256 + threadIdx.x; k < total; k += (int64_t)gridDim.x * 256) {
    if (k < c.n_pages) {
      const int t = c.turn[k], to = t <= -2 ? c.copy_dst[-2 - t] : t;
      c.page_map[k] = to;
      if (to >= 0) c.refs_out[to] = c.refs_in[k];
      if (k >= held) c.refs_out[k] = 0;          // (below it every page is somebody's new place)
    } else {
      const int64_t row = (k - c.n_pages) / c.max_pages, col = (k - c.n_pages) % c.max_pages;
      const int e = c.table_in[row * c.ld_in + col];
      int to = -1;
      if ((uint32_t)e < (uint32_t)c.n_pages) {
        const int t = c.turn[e];
        to = t <= -2 ? c.copy_dst[-2 - t] : t;
      }
      c.table_out[row * c.ld_out + col] = to;
    }
  }
}

// The first rows[i] tokens (NULL: all) of page src[i] onto page dst[i], keys and values.
//
// Bound: HBM.  A workgroup takes up to 256 * PER vectors of 16 bytes of a pair's keys or values at a time, PER per lane, in the order token, head, column.
// 2048 pages of 64 KB 37 - 43 us (268 MB read and written, 6.3 TB/s and more), the half filled pages of 512 beams, 47 MB, 11.9.
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
template <int PER>
__global__ __launch_bounds__(256) void kv_copy_kernel(KvCopy c) {
  const int part = blockIdx.x, run = part >> 1;
  uint16_t* const base = (part & 1) ? c.v : c.k;
  int token[PER];
  int64_t off[PER];                              // of this lane's vectors inside a page, in elements
#pragma unroll
  for (int j = 0; j < PER; j++) {
    const int v = (run * PER + j) * 256 + threadIdx.x;
    token[j] = (int)c.by_row.div((uint32_t)v);
    const int w = v - token[j] * c.row_vecs, h = (int)c.by_head.div((uint32_t)w);
    off[j] = token[j] * c.token_stride + h * c.head_stride + (w - h * c.head_vecs) * 8;
  }
  for (int64_t pair = blockIdx.y; pair < c.n; pair += gridDim.y) {
    const int src = c.src[pair], dst = c.dst[pair];
    const int rows = c.rows ? min(max(c.rows[pair], 0), c.page_size) : c.page_size;
    if ((uint32_t)src >= (uint32_t)c.n_pages || (uint32_t)dst >= (uint32_t)c.n_pages || src == dst) continue;
    const uint16_t* from = base + (int64_t)src * c.page_stride;
    uint16_t* to = base + (int64_t)dst * c.page_stride;
    u32x4 q[PER];
#pragma unroll
    for (int j = 0; j < PER; j++) {
      q[j] = u32x4{0, 0, 0, 0};
      if (token[j] < rows) q[j] = *reinterpret_cast<const u32x4*>(from + off[j]);
    }
#pragma unroll
    for (int j = 0; j < PER; j++)
      if (token[j] < rows) *reinterpret_cast<u32x4*>(to + off[j]) = q[j];
  }
}

}  // namespace

size_t kv_fork_ws_bytes(int64_t n_in, int64_t n_out, int64_t n_pages) {
  return (size_t)(2 * n_in + 2 * n_out + n_pages + 1) * sizeof(int32_t);
}
hipError_t k_kv_fork(KvFork f, void* ws, hipStream_t st) {
  int32_t* w = (int32_t*)ws;
  f.found = w;
  f.first = w + 1;
  f.count = f.first + f.n_in;
  f.flags = f.count + f.n_in;
  f.offset = f.flags + f.n_out;
  f.fresh = f.offset + f.n_out;
  // one-time opt-in to more than 64 KB of dynamic LDS (thread-safe function-local static)
  static const hipError_t attr_err =
      hipFuncSetAttribute((const void*)fork_plan_kernel, hipFuncAttributeMaxDynamicSharedMemorySize, 2 * KV_FORK_MOST * (int)sizeof(int));
  if (attr_err != hipSuccess) return attr_err;
  const int64_t copies = (f.n_pages + 4 * PLAN_T - 1) / (4 * PLAN_T);
  hipLaunchKernelGGL(fork_plan_kernel, dim3((uint32_t)(1 + (copies < 255 ? copies : 255))), dim3(PLAN_T), (size_t)2 * f.n_in * sizeof(int), st, f);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int rows = f.n_in + f.n_out;
  if (rows > 0) hipLaunchKernelGGL(fork_rows_kernel, dim3((uint32_t)((rows + 3) / 4)), dim3(256), 0, st, f);
  return hipGetLastError();
}

size_t kv_compact_ws_bytes(int64_t n_pages) { return (size_t)(n_pages + (n_pages + SPAN - 1) / SPAN) * sizeof(int32_t); }
hipError_t k_kv_compact(KvCompact c, void* ws, hipStream_t st) {
  c.spans = (int)((c.n_pages + SPAN - 1) / SPAN);
  c.turn = (int32_t*)ws;
  c.span_held = c.turn + c.n_pages;
  hipError_t e;
  if (c.spans <= SPANS_FEW) {      // us of the lists, 1000 pages 6.0 / 9.0 with a launch that counts, 8192 pages 7.0 / 12.5
    hipLaunchKernelGGL(compact_lists_kernel<true>, dim3((uint32_t)c.spans), dim3(SPAN_T), 0, st, c);
  } else {
    hipLaunchKernelGGL(compact_count_kernel, dim3((uint32_t)c.spans), dim3(SPAN_T), 0, st, c);
    e = hipGetLastError();
    if (e != hipSuccess) return e;
    hipLaunchKernelGGL(compact_lists_kernel<false>, dim3((uint32_t)c.spans), dim3(SPAN_T), 0, st, c);
  }
  e = hipGetLastError();
  if (e != hipSuccess) return e;
  const int64_t blocks = (c.n_pages + (int64_t)c.batch * c.max_pages + 255) / 256;
  hipLaunchKernelGGL(compact_apply_kernel, dim3((uint32_t)(blocks < 8192 ? blocks : 8192)), dim3(256), 0, st, c);
  return hipGetLastError();
}

hipError_t k_kv_copy(KvCopy c, hipStream_t st) {
  const int64_t vecs = (int64_t)c.page_size * c.row_vecs;
  auto run = [&](auto kern, int per) {
    const int64_t runs = (vecs + 256 * per - 1) / (256 * per), most = ((int64_t)1 << 22) / runs + 1;
    hipLaunchKernelGGL(kern, dim3((uint32_t)(2 * runs), (uint32_t)(c.n < most ? (c.n < 65535 ? c.n : 65535) : (most < 65535 ? most : 65535))), dim3(256), 0, st, c);
    return hipGetLastError();
  };
  // us, two vectors a lane / four: 2000 pages of 4 KB 5.3 / 6.4, 2048 pages of 64 KB that no cache holds, with their lists, 67.4 / 66.6, 512 beams and their lists 22.0 / 21.0
  return vecs <= 512 ? run(kv_copy_kernel<2>, 2) : run(kv_copy_kernel<4>, 4);
}

}  // namespace lrb
