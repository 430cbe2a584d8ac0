// pages.cu — a store's pages kept on the GPU: the free list, pages handed out and taken
// back from lengths, the slot map and positions of a step.
//
// Nothing but integers moves.  A call's order of pages is that of its definition, the
// exclusive sums over segments of what each gives back and takes, so the same call
// gives the same table; the only atomics set bits.
#include <algorithm>

#include "../../include/certkv.h"
#include "common.cuh"
#include "internal.cuh"
#include "store.cuh"

namespace certkv {
namespace {

struct Pages {
  int32_t *held, *free, *free_count;
};

int pages_of(const certkv_pages* p, Pages* out) {
  if (!p || !p->held || !p->free || !p->free_count) return CERTKV_EINVAL;
  if (((uintptr_t)p->held | (uintptr_t)p->free | (uintptr_t)p->free_count) % 4 != 0) return CERTKV_EINVAL;
  *out = {p->held, p->free, p->free_count};
  return CERTKV_OK;
}

struct ReserveArgs {
  Store st;
  Pages pg;
  const int32_t *room, *want;
  int per_seq;     // segments of a sequence
  int per_block;   // segments of a block
  longlong2* sums;  // [blocks] pages given back and asked for
  int* n0;          // the free pages before the call
};

constexpr int kThreads = 256;
constexpr int kMovePages = 128;  // pages of a segment that a block moves

// What segment u gives back and asks for.
struct Change {
  int held, need;
  int64_t slots;
  bool cut;
  __device__ __forceinline__ int back() const { return max(held - need, 0); }
  __device__ __forceinline__ int more() const { return max(need - held, 0); }
};
__device__ __forceinline__ Change change_of(const ReserveArgs& p, int u) {
  Change c = {0, 0, 0, false};
  if (u >= p.st.units) return c;
  c.held = min(max(p.pg.held[u], 0), p.st.max_pages);
  const int64_t s = (int64_t)(p.want ? p.want[u] : p.st.counts[u]) + (p.room ? p.room[u / p.per_seq] : 0);
  const int64_t most = (int64_t)p.st.max_pages * kPage;
  c.cut = s > most;
  c.slots = min(max(s, (int64_t)0), most);
  c.need = (int)((c.slots + kPage - 1) / kPage);
  return c;
}

// Exclusive sums of two counts over the block's threads (kThreads of them); the block's
// totals in `all`.  64 bits: what is asked for may be any multiple of the pool.
__device__ __forceinline__ longlong2 block_scan(longlong2 v, longlong2* all) {
  __shared__ longlong2 part[kThreads / 32];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  longlong2 x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long a = __shfl_up_sync(kFull, x.x, o), b = __shfl_up_sync(kFull, x.y, o);
    if (lane >= o) x.x += a, x.y += b;
  }
  if (lane == 31) part[warp] = x;
  __syncthreads();
  longlong2 before = make_longlong2(0, 0), sum = make_longlong2(0, 0);
#pragma unroll
  for (int w = 0; w < kThreads / 32; ++w) {
    if (w < warp) before.x += part[w].x, before.y += part[w].y;
    sum.x += part[w].x, sum.y += part[w].y;
  }
  __syncthreads();
  *all = sum;
  return make_longlong2(before.x + x.x - v.x, before.y + x.y - v.y);
}

__global__ void __launch_bounds__(kThreads) pages_sum_kernel(const ReserveArgs p) {
  longlong2 sum = make_longlong2(0, 0), all;
  release_next();
  for (int i = threadIdx.x; i < p.per_block; i += kThreads) {
    const int64_t u = (int64_t)blockIdx.x * p.per_block + i;
    const Change c = change_of(p, u < p.st.units ? (int)u : p.st.units);
    sum.x += c.back();
    sum.y += c.more();
  }
  block_scan(sum, &all);
  if (threadIdx.x == 0) p.sums[blockIdx.x] = all;
  if (threadIdx.x == 0 && blockIdx.x == 0) *p.n0 = min(max(*p.pg.free_count, 0), p.st.pool_pages);
}

// Sums of the blocks before this one, and of all.
__device__ __forceinline__ void block_base(const ReserveArgs& p, longlong2* base, longlong2* total) {
  longlong2 b = make_longlong2(0, 0), t = make_longlong2(0, 0);
  for (int i = threadIdx.x; i < gridDim.x; i += kThreads) {
    const longlong2 s = p.sums[i];
    t.x += s.x, t.y += s.y;
    if (i < blockIdx.x) b.x += s.x, b.y += s.y;
  }
  block_scan(b, base);
  block_scan(t, total);
}

// A segment's pages [first, first + n) of its table row, number num, num + 1, .. of the call.
struct Run {
  int u, first, n;
  long long num;
};
// Page k of a run goes to the list (TAKE false) or comes from it; false: not as it should.
template <bool TAKE>
__device__ __forceinline__ bool move_page(const ReserveArgs& p, const Run& r, int k, int n0, int top) {
  int32_t* e = p.st.table + (int64_t)r.u * p.st.max_pages + r.first + k;
  const long long place = top - 1 - (r.num + k);
  if (TAKE) {
    const int page = p.pg.free[place];  // 0 <= place: n is what is left
    *e = page;
    return page >= 0 && page < p.st.pool_pages;
  }
  if (place >= n0) p.pg.free[place] = *e;
  *e = -1;
  return place >= n0;
}
template <bool TAKE>
__device__ __forceinline__ Run run_of(int u, const Change& c, const longlong2& before, int top) {
  const long long num = TAKE ? before.y : before.x;
  return {u, TAKE ? c.held : c.need, TAKE ? (int)min((long long)c.more(), max(top - num, 0ll)) : c.back(), num};
}
// The account of segment u, n pages handed out; false: cut or short.
__device__ __forceinline__ bool settle(const ReserveArgs& p, int u, const Change& c, int n) {
  p.pg.held[u] = min(c.held, c.need) + n;
  if (p.st.counts[u] > c.slots) p.st.counts[u] = (int)c.slots;
  return !c.cut && n == c.more();
}

// TAKE false: the pages given back go to the list.  TAKE true: pages are handed out, and
// the account is brought up to date.  A segment's pages are moved by its thread where
// they are few, by a warp where there are many, the block's warps taking turns, kMovePages of them
// by each of the blocks of a column of the grid (a 131072-token sequence's 524288 pages taken back
// and handed out: 275 us with one block a segment, 48 with one warp a block, 35 so).
template <bool TAKE>
__global__ void __launch_bounds__(kThreads) pages_move_kernel(const ReserveArgs p) {
  await_previous();
  release_next();
  longlong2 at, total;
  block_base(p, &at, &total);
  const int n0 = *p.n0, top = (int)min(n0 + total.x, (long long)p.st.pool_pages);
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, k0 = blockIdx.y * kMovePages;
  __shared__ Run runs[kThreads];
  bool bad = false;
  for (int i0 = 0; i0 < p.per_block; i0 += kThreads) {
    const int i = i0 + threadIdx.x;
    const int64_t unit = (int64_t)blockIdx.x * p.per_block + i;
    const int u = i < p.per_block && unit < p.st.units ? (int)unit : p.st.units;
    const Change c = change_of(p, u);
    longlong2 all;
    longlong2 in = block_scan(make_longlong2(c.back(), c.more()), &all);
    in.x += at.x, in.y += at.y;
    at.x += all.x, at.y += all.y;
    const Run r = run_of<TAKE>(u, c, in, top);
    constexpr int kFew = 4;
    if (r.n <= kFew && k0 == 0)
      for (int k = 0; k < r.n; ++k) bad |= !move_page<TAKE>(p, r, k, n0, top);
    if (__syncthreads_or(r.n > kFew && r.n > k0)) {
      runs[threadIdx.x] = r;
      __syncthreads();
      for (int j = warp; j < kThreads && j < p.per_block - i0; j += kThreads / 32) {
        const Run x = runs[j];
        if (x.n <= kFew) continue;
        const int k1 = min(x.n, k0 + kMovePages);
#pragma unroll 4
        for (int k = k0 + lane; k < k1; k += 32) bad |= !move_page<TAKE>(p, x, k, n0, top);
      }
      __syncthreads();
    }
    // behind every read of the account: those of the column's other blocks too, which have to
    // see the same; the first block's threads settle it in a launch of their own where there
    // are others
    if (TAKE && gridDim.y == 1 && u < p.st.units) bad |= !settle(p, u, c, r.n);
  }
  if (TAKE && gridDim.y == 1 && blockIdx.x == 0 && threadIdx.x == 0)
    *p.pg.free_count = top - (int)min(total.y, (long long)top);
  if (bad) p.st.raise();
}

// The accounts, behind a grid of several blocks a segment.
__global__ void __launch_bounds__(kThreads) pages_settle_kernel(const ReserveArgs p) {
  await_previous();
  longlong2 at, total;
  block_base(p, &at, &total);
  const int top = (int)min(*p.n0 + total.x, (long long)p.st.pool_pages);
  bool bad = false;
  for (int i0 = 0; i0 < p.per_block; i0 += kThreads) {
    const int i = i0 + threadIdx.x;
    const int64_t unit = (int64_t)blockIdx.x * p.per_block + i;
    const int u = i < p.per_block && unit < p.st.units ? (int)unit : p.st.units;
    const Change c = change_of(p, u);
    longlong2 all;
    longlong2 in = block_scan(make_longlong2(c.back(), c.more()), &all);
    in.x += at.x, in.y += at.y;
    at.x += all.x, at.y += all.y;
    if (u < p.st.units) bad |= !settle(p, u, c, run_of<true>(u, c, in, top).n);
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *p.pg.free_count = top - (int)min(total.y, (long long)top);
  if (bad) p.st.raise();
}

// Few segments of few pages: everything by one block, which saves the launches.  The host knows sizes
// but not how much moves, and a step, which is what most calls are, moves a page or so of some segments
// (us a call, and by the launches below: 64 segments x 16 entries, one page each 3.9 and 6.6; 1024 x 128,
// one 4.7 and 6.7, four 8.8 and 7.7, eight 16.1 and 16.2).  Sequences that begin or end whole pay for
// it, since a thread moves its segments' pages one after the other: 64 x 16 pages 12 and 10, 64 x 128
// 56 and 13, 256 x 128 67 and 30, 1024 x 64 112 and 22, 1024 x 128 222 and 30.
constexpr int kSmallUnits = 4 * kThreads, kSmallPages = 128;
__global__ void __launch_bounds__(kThreads) pages_small_kernel(const ReserveArgs p) {
  constexpr int kEach = kSmallUnits / kThreads;
  Change c[kEach];
  longlong2 sum = make_longlong2(0, 0), total;
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int u = kEach * (int)threadIdx.x + i;
    c[i] = change_of(p, min(u, p.st.units));
    sum.x += c[i].back(), sum.y += c[i].more();
  }
  const int n0 = min(max(*p.pg.free_count, 0), p.st.pool_pages);
  longlong2 in = block_scan(sum, &total);
  const int top = (int)min(n0 + total.x, (long long)p.st.pool_pages);
  bool bad = false;
  Run take[kEach];
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    const int u = min(kEach * (int)threadIdx.x + i, p.st.units);
    take[i] = run_of<true>(u, c[i], in, top);
    const Run r = run_of<false>(u, c[i], in, top);
    for (int k = 0; k < r.n; ++k) bad |= !move_page<false>(p, r, k, n0, top);
    in.x += c[i].back(), in.y += c[i].more();
  }
  __syncthreads();  // the list holds what was given back
#pragma unroll
  for (int i = 0; i < kEach; ++i) {
    for (int k = 0; k < take[i].n; ++k) bad |= !move_page<true>(p, take[i], k, n0, top);
    if (take[i].u < p.st.units) bad |= !settle(p, take[i].u, c[i], take[i].n);
  }
  if (threadIdx.x == 0) *p.pg.free_count = top - (int)min(total.y, (long long)top);
  if (bad) p.st.raise();
}

// ------------------------------------------------------------ free list --
// One warp per table row: how far it reaches, and a bit for each of its pages.
__global__ void __launch_bounds__(kThreads) pages_mark_kernel(const Store st, int32_t* held, uint32_t* used) {
  const int64_t u = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> 5;
  const int lane = threadIdx.x & 31;
  release_next();
  if (u >= st.units) return;
  int reach = 0;
#pragma unroll 4
  for (int i = lane; i < st.max_pages; i += 32) {
    const int page = st.table[u * st.max_pages + i];
    if (page < 0 || page >= st.pool_pages) continue;
    reach = i + 1;
    atomicOr(used + (page >> 5), 1u << (page & 31));
  }
  reach = __reduce_max_sync(kFull, reach);
  if (lane == 0) held[u] = reach;
}

constexpr int kWords = kThreads;  // words of 32 pages a block

__device__ __forceinline__ uint32_t free_bits(const uint32_t* used, int64_t w, int pool) {
  if (w * 32 >= pool) return 0u;
  const int n = (int)min((int64_t)32, pool - w * 32);
  return ~used[w] & (0xffffffffu >> (32 - n));
}

__global__ void __launch_bounds__(kThreads) pages_free_sum_kernel(const uint32_t* used, int pool, longlong2* sums) {
  await_previous();
  release_next();
  longlong2 all;
  block_scan(make_longlong2(__popc(free_bits(used, (int64_t)blockIdx.x * kWords + threadIdx.x, pool)), 0), &all);
  if (threadIdx.x == 0) sums[blockIdx.x] = all;
}

__global__ void __launch_bounds__(kThreads) pages_free_kernel(const uint32_t* used, int pool, const longlong2* sums,
                                                              int32_t* list, int32_t* count) {
  await_previous();
  longlong2 b = make_longlong2(0, 0), base;
  for (int i = threadIdx.x; i < gridDim.x; i += kThreads) {
    b.x += sums[i].x;
    if (i < blockIdx.x) b.y += sums[i].x;
  }
  block_scan(b, &base);
  const int total = (int)base.x;
  const int lane = threadIdx.x & 31;
  const int64_t w = (int64_t)blockIdx.x * kWords + threadIdx.x;
  const uint32_t mine = free_bits(used, w, pool);
  longlong2 all;
  const int rank = (int)base.y + (int)block_scan(make_longlong2(__popc(mine), 0), &all).x;
  // a word's pages side by side (each by its thread alone, and four words a thread: 8 us more for a list
  // of 280000 pages)
#pragma unroll 4
  for (int i = 0; i < 32; ++i) {
    const uint32_t x = __shfl_sync(kFull, mine, i);
    const int at = total - 1 - __shfl_sync(kFull, rank, i) - __popc(x & ((1u << lane) - 1u));
    if (x >> lane & 1u) list[at] = (int32_t)((w - lane + i) * 32 + lane);
  }
  if (blockIdx.x == 0 && threadIdx.x == 0) *count = total;
}

// ------------------------------------------------------------- slot map --
struct MapArgs {
  Store st;
  int batch, tokens, per_seq;
  const int32_t *rows, *start, *base;
  const uint64_t* mask;
  int32_t *slots, *positions;
  int per;         // warps (step) or blocks of a segment
  int64_t chunks;  // of all segments
};
// Position e of the output, if there is one.
__device__ __forceinline__ void position(const MapArgs& p, int64_t e) {
  if (!p.positions || e >= (int64_t)p.batch * p.tokens) return;
  const int b = (int)(e / p.tokens), t = (int)(e - (int64_t)b * p.tokens);
  int depth = t;
  if (p.mask) depth = __popcll(p.mask[e] & (~0ull >> (64 - p.tokens)) & ~(1ull << t));
  p.positions[e] = (int32_t)((uint32_t)(p.base ? p.base[b] : 0) + (uint32_t)depth);
}

// A step's rows, a warp 32 of a segment; one launch's latency.
constexpr int kStepRows = 512;  // up to this many rows a segment
__global__ void __launch_bounds__(kThreads) slot_map_step_kernel(const MapArgs p) {
  const int64_t w = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> 5;
  const int lane = threadIdx.x & 31;
  if (w < p.chunks) {
    const int u = (int)(w / p.per), i = (int)(w - (int64_t)u * p.per) * 32 + lane;
    const int n = p.rows ? min(max(p.rows[u / p.per_seq], 0), p.tokens) : p.tokens;
    if (i >= p.tokens) return;
    int64_t at = -1;
    if (i < n) {
      const int64_t s = (int64_t)(p.start ? p.start[u] : p.st.counts[u]) + i;
      if (s >= 0 && s < (int64_t)p.st.max_pages * kPage) at = p.st.slot(u, (int)s);
      if (at < 0) p.st.raise();
    }
    p.slots[(int64_t)u * p.tokens + i] = (int32_t)at;
    return;
  }
  position(p, (w - p.chunks) * 32 + lane);
}

constexpr int kRows = 16384;  // rows of a segment that a block takes
constexpr int kMapEach = kRows / 4 / kThreads;

// Many rows: bound by the bytes it writes (a 131071-token prompt of 256 segments, 137 MB).  A
// thread writes 16 bytes at a time wherever a row of the output begins; its four rows lie in one
// page or two, whose entries are the only thing that it reads (with the rows that cross from one
// to the next on a path of their own, which every warp took, 44 us for 27).
__global__ void __launch_bounds__(kThreads) slot_map_kernel(const MapArgs p) {
  if (blockIdx.x >= p.chunks) {
    position(p, (blockIdx.x - p.chunks) * kThreads + threadIdx.x);
    return;
  }
  const int u = (int)(blockIdx.x / p.per), part = (int)(blockIdx.x - (int64_t)u * p.per);
  const int n = p.rows ? min(max(p.rows[u / p.per_seq], 0), p.tokens) : p.tokens;
  const int64_t start = p.start ? p.start[u] : p.st.counts[u], most = (int64_t)p.st.max_pages * kPage;
  // rows [lo, hi) have a place in the table
  const int lo = (int)min(max(-start, (int64_t)0), (int64_t)p.tokens), hi = (int)max(min((int64_t)n, most - start), (int64_t)lo);
  int32_t* out = p.slots + (int64_t)u * p.tokens;
  const int early = (int)(reinterpret_cast<uintptr_t>(out) / 4 & 3);  // rows from the boundary before to the first
  const int32_t* row = p.st.table + (int64_t)u * p.st.max_pages;
  const int i0 = part * kRows - early, s0 = (int)start;
  bool bad = (lo > 0 || hi < n) && n > 0 && part == 0;
  int page[kMapEach], next[kMapEach];  // of a thread's first row and of its last
#pragma unroll
  for (int j = 0; j < kMapEach; ++j) {
    const int i = i0 + 4 * (j * kThreads + (int)threadIdx.x);
    const bool all = i >= lo && i + 4 <= hi;
    page[j] = all ? __ldg(row + ((s0 + i) >> 6)) : -1;
    next[j] = all ? __ldg(row + ((s0 + i + 3) >> 6)) : -1;
  }
#pragma unroll
  for (int j = 0; j < kMapEach; ++j) {
    const int i = i0 + 4 * (j * kThreads + (int)threadIdx.x), s = (int)((uint32_t)s0 + (uint32_t)i);
    if (page[j] >= 0 && page[j] < p.st.pool_pages && next[j] >= 0 && next[j] < p.st.pool_pages) {
      const int v = page[j] * kPage + (s & 63), w = (next[j] - 1) * kPage + (s & 63), left = kPage - (s & 63);
      *reinterpret_cast<int4*>(out + i) = make_int4(v, (left > 1 ? v : w) + 1, (left > 2 ? v : w) + 2, (left > 3 ? v : w) + 3);
      continue;
    }
    int v[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      v[k] = -1;
      if (i + k < lo || i + k >= hi) continue;
      const int pg = __ldg(row + ((s + k) >> 6));
      if (pg >= 0 && pg < p.st.pool_pages) v[k] = pg * kPage + ((s + k) & 63);
      else bad = true;
    }
    if (i >= 0 && i + 4 <= p.tokens) {
      *reinterpret_cast<int4*>(out + i) = make_int4(v[0], v[1], v[2], v[3]);
    } else {
#pragma unroll
      for (int k = 0; k < 4; ++k)
        if (i + k >= 0 && i + k < p.tokens) out[i + k] = v[k];
    }
  }
  if (bad) p.st.raise();
}

size_t align256(size_t x) { return (x + 255) / 256 * 256; }
// launch_kernel of a grid of two dimensions, early.
bool launch_grid(void (*kernel)(ReserveArgs), dim3 grid, cudaStream_t st, const ReserveArgs& p) {
  cudaLaunchAttribute at;
  at.id = cudaLaunchAttributeProgrammaticStreamSerialization;
  at.val.programmaticStreamSerializationAllowed = 1;
  cudaLaunchConfig_t c = {};
  c.gridDim = grid;
  c.blockDim = dim3(kThreads);
  c.stream = st;
  c.attrs = &at;
  c.numAttrs = 1;
  return cudaLaunchKernelEx(&c, kernel, p) == cudaSuccess;
}
int64_t free_blocks(int pool) { return ((int64_t)(pool + 31) / 32 + kWords - 1) / kWords; }

}  // namespace
}  // namespace certkv

extern "C" size_t certkv_pages_workspace_bytes(int32_t units, int32_t pool_pages) {
  using namespace certkv;
  if (units < 1 || units > (1 << 24) || pool_pages < 1 || pool_pages >= (1 << 25)) return 0;
  const size_t bits = align256(((size_t)pool_pages + 31) / 32 * 4);
  const size_t blocks = std::max((size_t)(units + 7) / 8, (size_t)free_blocks(pool_pages));
  return bits + align256((blocks + 1) * sizeof(longlong2));
}

extern "C" int certkv_pages_list(const certkv_store* store, const certkv_pages* pages, void* workspace,
                                 size_t workspace_bytes, void* stream) {
  using namespace certkv;
  Store st;
  Pages pg;
  int rc;
  if ((rc = store_of(store, &st)) || (rc = pages_of(pages, &pg))) return rc;
  if (!workspace || (uintptr_t)workspace % 256 != 0 ||
      workspace_bytes < certkv_pages_workspace_bytes(st.units, st.pool_pages))
    return CERTKV_EWORKSPACE;
  const size_t bits = align256(((size_t)st.pool_pages + 31) / 32 * 4);
  uint32_t* used = reinterpret_cast<uint32_t*>(workspace);
  longlong2* sums = reinterpret_cast<longlong2*>(reinterpret_cast<char*>(workspace) + bits);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const unsigned blocks = (unsigned)free_blocks(st.pool_pages);
  if (cudaMemsetAsync(used, 0, bits, s) != cudaSuccess) return cuda_failed();
  {
    TraceScope ts_("pages_mark", s);
    if (!launch_kernel(false, pages_mark_kernel, (unsigned)(((int64_t)st.units * 32 + kThreads - 1) / kThreads),
                       kThreads, 0, s, st, pg.held, used))
      return cuda_failed();
  }
  {
    TraceScope ts_("pages_free_sum", s);
    if (!launch_kernel(true, pages_free_sum_kernel, blocks, kThreads, 0, s, used, st.pool_pages, sums))
      return cuda_failed();
  }
  {
    TraceScope ts_("pages_free", s);
    launch_kernel(true, pages_free_kernel, blocks, kThreads, 0, s, used, st.pool_pages, sums, pg.free,
                  pg.free_count);
  }
  return cudaGetLastError() == cudaSuccess ? CERTKV_OK : CERTKV_ECUDA;
}

extern "C" int certkv_pages_reserve(int32_t batch, const int32_t* room, const int32_t* want,
                                    const certkv_store* store, const certkv_pages* pages, void* workspace,
                                    size_t workspace_bytes, void* stream) {
  using namespace certkv;
  ReserveArgs p;
  int rc;
  if ((rc = store_of(store, &p.st)) || (rc = pages_of(pages, &p.pg))) return rc;
  if (batch < 1 || p.st.units % batch != 0) return CERTKV_EINVAL;
  if (((uintptr_t)room | (uintptr_t)want) % 4 != 0) return CERTKV_EINVAL;
  if (!workspace || (uintptr_t)workspace % 256 != 0 ||
      workspace_bytes < certkv_pages_workspace_bytes(p.st.units, p.st.pool_pages))
    return CERTKV_EWORKSPACE;
  p.room = room;
  p.want = want;
  p.per_seq = p.st.units / batch;
  p.per_block = p.st.max_pages >= 256 ? 8 : kThreads;
  p.n0 = reinterpret_cast<int*>(workspace);
  p.sums = reinterpret_cast<longlong2*>(workspace) + 1;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (p.st.units <= kSmallUnits && p.st.max_pages <= kSmallPages) {
    TraceScope ts_("pages_small", s);
    return launch_kernel(false, pages_small_kernel, 1, kThreads, 0, s, p) ? CERTKV_OK : cuda_failed();
  }
  const unsigned blocks = (unsigned)((p.st.units + p.per_block - 1) / p.per_block);
  const dim3 grid(blocks, (unsigned)((p.st.max_pages + kMovePages - 1) / kMovePages));
  {
    TraceScope ts_("pages_sum", s);
    if (!launch_kernel(false, pages_sum_kernel, blocks, kThreads, 0, s, p)) return cuda_failed();
  }
  {
    TraceScope ts_("pages_back", s);
    if (!launch_grid(pages_move_kernel<false>, grid, s, p)) return cuda_failed();
  }
  {
    TraceScope ts_("pages_out", s);
    if (!launch_grid(pages_move_kernel<true>, grid, s, p)) return cuda_failed();
  }
  if (grid.y > 1) {
    TraceScope ts_("pages_settle", s);
    launch_kernel(true, pages_settle_kernel, blocks, kThreads, 0, s, p);
  }
  return cudaGetLastError() == cudaSuccess ? CERTKV_OK : CERTKV_ECUDA;
}

extern "C" int certkv_slot_map(int32_t batch, int32_t tokens, const int32_t* rows, const int32_t* start,
                               const int32_t* base, const uint64_t* mask, const certkv_store* store,
                               int32_t* slots, int32_t* positions, void* stream) {
  using namespace certkv;
  MapArgs p;
  int rc;
  if ((rc = store_of(store, &p.st))) return rc;
  if (batch < 1 || p.st.units % batch != 0 || tokens < 1 || tokens > 1 << 30 || (mask && tokens > 64))
    return CERTKV_EINVAL;
  if (((uintptr_t)rows | (uintptr_t)start | (uintptr_t)base | (uintptr_t)slots | (uintptr_t)positions) % 4 != 0 ||
      (uintptr_t)mask % 8 != 0 || (!slots && !positions))
    return CERTKV_EINVAL;
  if ((int64_t)p.st.units * tokens >= (int64_t)1 << 40) return CERTKV_EINVAL;
  p.batch = batch;
  p.tokens = tokens;
  p.per_seq = p.st.units / batch;
  p.rows = rows;
  p.start = start;
  p.base = base;
  p.mask = mask;
  p.slots = slots;
  p.positions = positions;
  const bool step = tokens <= kStepRows;
  // one block more where a segment's entries do not begin on a 16-byte boundary: its parts then
  // begin up to 3 rows early
  const bool early = tokens % 4 != 0 || (uintptr_t)slots % 16 != 0;
  p.per = step ? (tokens + 31) / 32 : (tokens + kRows - 1) / kRows + early;
  p.chunks = slots ? (int64_t)p.st.units * p.per : 0;
  const int64_t rest = positions ? (int64_t)batch * tokens : 0, per_warp = kThreads / 32;
  const int64_t blocks = step ? (p.chunks + (rest + 31) / 32 + per_warp - 1) / per_warp
                              : p.chunks + (rest + kThreads - 1) / kThreads;
  if (blocks > INT32_MAX) return CERTKV_EINVAL;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  TraceScope ts_("slot_map", s);
  return launch_kernel(false, step ? slot_map_step_kernel : slot_map_kernel, (unsigned)blocks, kThreads, 0, s, p)
             ? CERTKV_OK
             : cuda_failed();
}
