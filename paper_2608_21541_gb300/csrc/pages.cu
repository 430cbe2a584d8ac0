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
  longlong2* sums; // [blocks] pages given back and asked for
};

constexpr int kThreads = 256;

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

// TAKE false: the pages given back go to the list.  TAKE true: pages are handed out, and
// the account is brought up to date.  A segment's pages are moved by its thread where
// they are few, by its whole warp where there are many.
template <bool TAKE>
__global__ void __launch_bounds__(kThreads) pages_move_kernel(const ReserveArgs p) {
  await_previous();
  release_next();
  longlong2 at, total;
  block_base(p, &at, &total);
  const int pool = p.st.pool_pages, n0 = min(max(*p.pg.free_count, 0), pool);
  const int top = (int)min(n0 + total.x, (long long)pool);
  const int lane = threadIdx.x & 31;
  bool bad = false;
  for (int i0 = 0; i0 < p.per_block; i0 += kThreads) {
    const int i = i0 + threadIdx.x;
    const int64_t unit = (int64_t)blockIdx.x * p.per_block + i;
    const int u = i < p.per_block && unit < p.st.units ? (int)unit : p.st.units;
    const Change c = change_of(p, u);
    longlong2 all;
    const longlong2 in = block_scan(make_longlong2(c.back(), c.more()), &all);
    // pages [first, first + n) of the row; page k of them is number num + k of the call
    const long long num = TAKE ? at.y + in.y : at.x + in.x;
    at.x += all.x, at.y += all.y;
    const int first = TAKE ? c.held : c.need;
    const int n = TAKE ? (int)min((long long)c.more(), max(top - num, 0ll)) : c.back();
    auto move = [&](int seg, int k, int s_first, long long s_num) {
      int32_t* e = p.st.table + (int64_t)seg * p.st.max_pages + s_first + k;
      const long long place = top - 1 - (s_num + k);
      if (TAKE) {
        const int page = p.pg.free[place];  // 0 <= place: n is what is left
        if (page < 0 || page >= pool) bad = true;
        *e = page;
      } else {
        if (place >= n0) p.pg.free[place] = *e;
        else bad = true;
        *e = -1;
      }
    };
    constexpr int kFew = 4;
    if (n <= kFew)
      for (int k = 0; k < n; ++k) move(u, k, first, num);
    for (uint32_t many = __ballot_sync(kFull, n > kFew); many; many &= many - 1) {
      const int src = __ffs(many) - 1;
      const int s_u = __shfl_sync(kFull, u, src), s_n = __shfl_sync(kFull, n, src);
      const int s_first = __shfl_sync(kFull, first, src);
      const long long s_num = __shfl_sync(kFull, num, src);
#pragma unroll 4
      for (int k = lane; k < s_n; k += 32) move(s_u, k, s_first, s_num);
    }
    if (TAKE && u < p.st.units) {
      p.pg.held[u] = min(c.held, c.need) + n;
      if (p.st.counts[u] > c.slots) p.st.counts[u] = (int)c.slots;
      if (c.cut || n < c.more()) bad = true;
    }
  }
  if (bad) p.st.raise();
}

// Behind every block that reads the count it replaces.
__global__ void __launch_bounds__(kThreads) pages_count_kernel(const ReserveArgs p, int blocks) {
  await_previous();
  longlong2 t = make_longlong2(0, 0), all;
  for (int i = threadIdx.x; i < blocks; i += kThreads) t.x += p.sums[i].x, t.y += p.sums[i].y;
  block_scan(t, &all);
  if (threadIdx.x == 0) {
    const int pool = p.st.pool_pages, n0 = min(max(*p.pg.free_count, 0), pool);
    const int top = (int)min(n0 + all.x, (long long)pool);
    *p.pg.free_count = top - (int)min(all.y, (long long)top);
  }
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

constexpr int kWords = 4 * kThreads;  // words of 32 pages a block

__device__ __forceinline__ uint32_t free_bits(const uint32_t* used, int64_t w, int pool) {
  if (w * 32 >= pool) return 0u;
  const int n = (int)min((int64_t)32, pool - w * 32);
  return ~used[w] & (0xffffffffu >> (32 - n));
}

__global__ void __launch_bounds__(kThreads) pages_free_sum_kernel(const uint32_t* used, int pool, longlong2* sums) {
  await_previous();
  release_next();
  longlong2 n = make_longlong2(0, 0), all;
  for (int i = 0; i < kWords; i += kThreads)
    n.x += __popc(free_bits(used, (int64_t)blockIdx.x * kWords + i + threadIdx.x, pool));
  block_scan(n, &all);
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
  int before = (int)base.y;
  for (int i = 0; i < kWords; i += kThreads) {
    const int64_t w = (int64_t)blockIdx.x * kWords + i + threadIdx.x;
    uint32_t x = free_bits(used, w, pool);
    longlong2 all;
    int rank = before + (int)block_scan(make_longlong2(__popc(x), 0), &all).x;
    before += (int)all.x;
    for (; x; x &= x - 1) list[total - 1 - rank++] = (int32_t)(w * 32 + __ffs(x) - 1);
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
  int64_t chunks;  // of kRows rows, of all segments
};
constexpr int kRows = 128;  // rows of a warp

__global__ void __launch_bounds__(kThreads) slot_map_kernel(const MapArgs p) {
  const int64_t w = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> 5;
  const int lane = threadIdx.x & 31;
  if (w < p.chunks) {
    const int per = (p.tokens + kRows - 1) / kRows;
    const int u = (int)(w / per), i0 = (int)(w - (int64_t)u * per) * kRows;
    const int n = p.rows ? min(max(p.rows[u / p.per_seq], 0), p.tokens) : p.tokens;
    const int64_t start = p.start ? p.start[u] : p.st.counts[u];
    bool bad = false;
#pragma unroll
    for (int j = 0; j < kRows; j += 32) {
      const int i = i0 + j + lane;
      if (i >= p.tokens) break;
      int64_t at = -1;
      if (i < n) {
        const int64_t s = start + i;
        if (s >= 0 && s < (int64_t)p.st.max_pages * kPage) at = p.st.slot(u, (int)s);
        if (at < 0) bad = true;
      }
      p.slots[(int64_t)u * p.tokens + i] = (int32_t)at;
    }
    if (bad) p.st.raise();
    return;
  }
  const int64_t e = (w - p.chunks) * 32 + lane;
  if (!p.positions || e >= (int64_t)p.batch * p.tokens) return;
  const int b = (int)(e / p.tokens), t = (int)(e - (int64_t)b * p.tokens);
  int depth = t;
  if (p.mask) depth = __popcll(p.mask[e] & (~0ull >> (64 - p.tokens)) & ~(1ull << t));
  p.positions[e] = (int32_t)((uint32_t)(p.base ? p.base[b] : 0) + (uint32_t)depth);
}

size_t align256(size_t x) { return (x + 255) / 256 * 256; }
int64_t free_blocks(int pool) { return ((int64_t)(pool + 31) / 32 + kWords - 1) / kWords; }

}  // namespace
}  // namespace certkv

extern "C" size_t certkv_pages_workspace_bytes(int32_t units, int32_t pool_pages) {
  using namespace certkv;
  if (units < 1 || units > (1 << 24) || pool_pages < 1 || pool_pages >= (1 << 25)) return 0;
  const size_t bits = align256(((size_t)pool_pages + 31) / 32 * 4);
  const size_t blocks = std::max((size_t)(units + 7) / 8, (size_t)free_blocks(pool_pages));
  return bits + align256(blocks * sizeof(longlong2));
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
  p.sums = reinterpret_cast<longlong2*>(workspace);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const unsigned blocks = (unsigned)((p.st.units + p.per_block - 1) / p.per_block);
  {
    TraceScope ts_("pages_sum", s);
    if (!launch_kernel(false, pages_sum_kernel, blocks, kThreads, 0, s, p)) return cuda_failed();
  }
  {
    TraceScope ts_("pages_back", s);
    if (!launch_kernel(true, pages_move_kernel<false>, blocks, kThreads, 0, s, p)) return cuda_failed();
  }
  {
    TraceScope ts_("pages_out", s);
    if (!launch_kernel(true, pages_move_kernel<true>, blocks, kThreads, 0, s, p)) return cuda_failed();
  }
  {
    TraceScope ts_("pages_count", s);
    launch_kernel(true, pages_count_kernel, 1, kThreads, 0, s, p, (int)blocks);
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
  if (batch < 1 || p.st.units % batch != 0 || tokens < 1 || (mask && tokens > 64)) return CERTKV_EINVAL;
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
  p.chunks = slots ? (int64_t)p.st.units * ((tokens + kRows - 1) / kRows) : 0;
  const int64_t warps = p.chunks + (positions ? ((int64_t)batch * tokens + 31) / 32 : 0);
  const int64_t blocks = (warps * 32 + kThreads - 1) / kThreads;
  if (blocks > INT32_MAX) return CERTKV_EINVAL;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  TraceScope ts_("slot_map", s);
  return launch_kernel(false, slot_map_kernel, (unsigned)blocks, kThreads, 0, s, p) ? CERTKV_OK : cuda_failed();
}
