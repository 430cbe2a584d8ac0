// store.cu — the paged store: quantising rows as they are written, from the
// packed cache or from token rows, and reading them back.
//
// Eight lanes hold a row: lane i elements 8 i .. 8 i + 7 and 64 + 8 i .., so that
// every load and store of the eight lanes is one run of whole sectors (with
// sixteen consecutive elements a lane each access would touch half of every
// sector: reading back 131072 8-bit rows took 22.7 us instead of 20.4).  A scale
// group of the 4-bit format is a pair of lanes.  Every row is read once and
// written once; the kernels are bound by those bytes.
#include "../../include/certkv.h"
#include "common.cuh"
#include "internal.cuh"
#include "rows.cuh"
#include "store.cuh"

namespace certkv {
namespace {

constexpr int kStoreThreads = 256;
constexpr int kLoadBlocks = 4;  // resident blocks per SM of the load kernel
constexpr float kTiny = 7.8886091e-31f;  // 2^-100: rows below are held as zeros

struct Words16 {
  uint32_t w[8];  // sixteen bf16: elements 8 sub .., then 64 + 8 sub ..
};

// This lane's elements of the bf16 row at `row`.
__device__ __forceinline__ Words16 load_row(const uint16_t* row, int sub) {
  Words16 x;
  const uint4 a = __ldg(reinterpret_cast<const uint4*>(row + 8 * sub));
  const uint4 b = __ldg(reinterpret_cast<const uint4*>(row + 64 + 8 * sub));
  x.w[0] = a.x; x.w[1] = a.y; x.w[2] = a.z; x.w[3] = a.w;
  x.w[4] = b.x; x.w[5] = b.y; x.w[6] = b.z; x.w[7] = b.w;
  return x;
}
__device__ __forceinline__ void store_row(uint16_t* row, int sub, const Words16& x) {
  *reinterpret_cast<uint4*>(row + 8 * sub) = make_uint4(x.w[0], x.w[1], x.w[2], x.w[3]);
  *reinterpret_cast<uint4*>(row + 64 + 8 * sub) = make_uint4(x.w[4], x.w[5], x.w[6], x.w[7]);
}
// Largest magnitude of eight bf16 as fp32 bits; a NaN or infinity stays one.
__device__ __forceinline__ uint32_t top8(const uint32_t* w) {
  uint32_t two = w[0] & 0x7fff7fffu;
#pragma unroll
  for (int i = 1; i < 4; ++i) asm("max.NaN.bf16x2 %0, %0, %1;" : "+r"(two) : "r"(w[i] & 0x7fff7fffu));
  return max(two << 16, two & 0xffff0000u);
}

// Encode the row held by this lane's group of eight lanes (sub = lane & 7) and
// write it to pool slot `to` (to < 0: nowhere).  Every lane of the warp takes
// part in the shuffles.
template <int FMT>
__device__ __forceinline__ void put_row(const Words16& x, int sub, int64_t to, uint8_t* codes,
                                        uint8_t* group, float* scale) {
  if (FMT == CERTKV_STORE_BF16) {
    if (to >= 0) store_row(reinterpret_cast<uint16_t*>(codes) + to * kD, sub, x);
    return;
  }
  // maxima of the lane pair's elements in either half of the row (4-bit scale
  // groups sub / 2 and 4 + sub / 2), then of the row
  uint32_t half[2] = {top8(x.w), top8(x.w + 4)};
  if (FMT == CERTKV_STORE_FP4) {
    half[0] = max(half[0], __shfl_xor_sync(kFull, half[0], 1));
    half[1] = max(half[1], __shfl_xor_sync(kFull, half[1], 1));
  }
  uint32_t top = max(half[0], half[1]);
  if (FMT != CERTKV_STORE_FP4) top = max(top, __shfl_xor_sync(kFull, top, 1));
  top = max(top, __shfl_xor_sync(kFull, top, 2));
  top = max(top, __shfl_xor_sync(kFull, top, 4));
  const float amax = __uint_as_float(top);
  const float kTop = FMT == CERTKV_STORE_FP8 ? 448.f : 2688.f;
  const bool bad = top >= 0x7f800000u;
  const bool zero = amax < kTiny || bad;
  const float s = bad ? __int_as_float(0x7fc00000) : zero ? 1.f : __fmul_rn(amax, 1.f / kTop);
  const float r = zero ? 0.f : __fmul_rn(__frcp_rn(amax), kTop);
  if (to < 0) return;
  if (sub == 0) scale[to] = s;
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    float m = r;
    if (FMT == CERTKV_STORE_FP4) {
      const uint32_t g8 = bad ? 0u : e4m3x2(__fmul_rn(__fmul_rn(__uint_as_float(half[h]), r), 1.f / 6.f), 0.f) & 0xffu;
      const float gs = f16x2_to_f32(e4m3x2_to_f16x2(g8)).x;
      m = gs > 0.f ? __fmul_rn(r, __frcp_rn(gs)) : 0.f;
      if ((sub & 1) == h) group[to * kGroups + 4 * h + (sub >> 1)] = (uint8_t)g8;
    }
    const float2 m2 = make_float2(m, m);
    float2 v[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] = fmul2(make_float2(bf16lo(x.w[4 * h + i]), bf16hi(x.w[4 * h + i])), m2);
    if (FMT == CERTKV_STORE_FP8) {
      const uint32_t a = bad ? 0u : e4m3x2(v[0].x, v[0].y) | (e4m3x2(v[1].x, v[1].y) << 16);
      const uint32_t b = bad ? 0u : e4m3x2(v[2].x, v[2].y) | (e4m3x2(v[3].x, v[3].y) << 16);
      *reinterpret_cast<uint2*>(codes + to * 128 + 64 * h + sub * 8) = make_uint2(a, b);
    } else {
      *reinterpret_cast<uint32_t*>(codes + to * 64 + 32 * h + sub * 4) = bad ? 0u : e2m1x8(v[0], v[1], v[2], v[3]);
    }
  }
}

// This lane's elements of pool slot `at` as bf16 words.
template <int FMT>
__device__ __forceinline__ Words16 get_row(int sub, int64_t at, const uint8_t* codes,
                                           const uint8_t* group, const float* scale) {
  if (FMT == CERTKV_STORE_BF16) return load_row(reinterpret_cast<const uint16_t*>(codes) + at * kD, sub);
  Words16 x;
  const float s = scale[at];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    uint32_t f16[4];
    float gs = 1.f;
    if (FMT == CERTKV_STORE_FP8) {
      const uint2 c = __ldg(reinterpret_cast<const uint2*>(codes + at * 128 + 64 * h + sub * 8));
      f16[0] = e4m3x2_to_f16x2(c.x & 0xffffu);
      f16[1] = e4m3x2_to_f16x2(c.x >> 16);
      f16[2] = e4m3x2_to_f16x2(c.y & 0xffffu);
      f16[3] = e4m3x2_to_f16x2(c.y >> 16);
    } else {
      const uint32_t c = __ldg(reinterpret_cast<const uint32_t*>(codes + at * 64 + 32 * h + sub * 4));
      gs = f16x2_to_f32(e4m3x2_to_f16x2(group[at * kGroups + 4 * h + (sub >> 1)])).x;
      f16[0] = e2m1x2_to_f16x2<0>(c);
      f16[1] = e2m1x2_to_f16x2<1>(c);
      f16[2] = e2m1x2_to_f16x2<2>(c);
      f16[3] = e2m1x2_to_f16x2<3>(c);
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float2 f = f16x2_to_f32(f16[i]);
      if (FMT == CERTKV_STORE_FP4) f = make_float2(f.x * gs, f.y * gs);
      const __nv_bfloat162 b = __floats2bfloat162_rn(f.x * s, f.y * s);
      x.w[4 * h + i] = *reinterpret_cast<const uint32_t*>(&b);
    }
  }
  return x;
}

// ------------------------------------------------------------------ load --
// One block: first[u] = pages of the segments before u (as wanted, not cut),
// first[units] = their sum, saturating at INT32_MAX.
__global__ void __launch_bounds__(1024) load_plan_kernel(int units, const int32_t* __restrict__ real,
                                                         int tail_slot, int reserve,
                                                         int32_t* __restrict__ first) {
  __shared__ long long wsum[32];
  __shared__ long long carry;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) carry = 0;
  __syncthreads();
  for (int base = 0; base < units; base += 1024) {
    const int u = base + threadIdx.x;
    const long long v =
        u < units ? ((long long)max(real[u], 0) + tail_slot + reserve + kPage - 1) / kPage : 0;
    long long x = v;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(kFull, x, o);
      if (lane >= o) x += y;
    }
    if (lane == 31) wsum[warp] = x;
    __syncthreads();
    if (warp == 0) {
      long long w = wsum[lane];
#pragma unroll
      for (int o = 1; o < 32; o <<= 1) {
        const long long y = __shfl_up_sync(kFull, w, o);
        if (lane >= o) w += y;
      }
      wsum[lane] = w;
    }
    __syncthreads();
    const long long excl = carry + (warp > 0 ? wsum[warp - 1] : 0) + x - v;
    if (u < units) first[u] = (int32_t)min(excl, (long long)INT32_MAX);
    __syncthreads();
    if (threadIdx.x == 0) carry += wsum[31];
    __syncthreads();
  }
  if (threadIdx.x == 0) first[units] = (int32_t)min(carry, (long long)INT32_MAX);
}

// Persistent: tables and counts, then the pages, one page of K and V rows per
// block and step.  Four blocks an SM, whose registers hold two rows of K and V a
// thread in flight, are the fastest (1.7 GB of bf16 rows into 8 bits: 400 us, 96 %
// of the copy bandwidth; five blocks 424, eight with one row at a time 495).
template <int FMT>
__global__ void __launch_bounds__(kStoreThreads, kLoadBlocks) load_kernel(
    Store st, const uint16_t* __restrict__ pk, const uint16_t* __restrict__ pv,
    const int64_t* __restrict__ offsets, const int32_t* __restrict__ real, int tail_slot,
    int64_t capacity, const int32_t* __restrict__ first) {
  const int64_t entries = (int64_t)st.units * st.max_pages;
  const int64_t tid = (int64_t)blockIdx.x * kStoreThreads + threadIdx.x;
  const int64_t step = (int64_t)gridDim.x * kStoreThreads;
  for (int64_t e = tid; e < entries; e += step) {
    const int u = (int)(e / st.max_pages), i = (int)(e - (int64_t)u * st.max_pages);
    const int64_t page = (int64_t)first[u] + i;
    st.table[e] = page < first[u + 1] && page < st.pool_pages ? (int)page : -1;
  }
  for (int64_t u = tid; u < st.units; u += step) {
    const int64_t n = (int64_t)max(real[u], 0) + tail_slot;
    const int64_t have = min((int64_t)min(first[u + 1], st.pool_pages) - min(first[u], st.pool_pages),
                             (int64_t)st.max_pages) * kPage;
    const bool outside = !lies_in(offsets[u], n, capacity);
    st.counts[u] = outside ? 0 : (int)min(n, have);
    if (outside || n > have) st.raise();
  }
  const int total = min(first[st.units], st.pool_pages);
  const int grp = threadIdx.x >> 3, sub = threadIdx.x & 7;  // 32 rows at a time
  for (int page = blockIdx.x; page < total; page += gridDim.x) {
    int lo = 0, hi = st.units;  // the segment of this page: the last u with first[u] <= page
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (first[mid] <= page) lo = mid;
      else hi = mid;
    }
    const int u = lo, s0 = (page - first[u]) * kPage;
    const int64_t n = (int64_t)max(real[u], 0) + tail_slot;
    if (!lies_in(offsets[u], n, capacity) || page - first[u] >= st.max_pages) continue;  // uniform over the block
#pragma unroll 2
    for (int half = 0; half < 2; ++half) {
      const int s = s0 + half * 32 + grp;
      const bool live = s < n;
      const int64_t from = (offsets[u] + s) * kD;
      Words16 a = {}, b = {};
      if (live) {
        a = load_row(pk + from, sub);
        b = load_row(pv + from, sub);
      }
      const int64_t to = live ? (int64_t)page * kPage + half * 32 + grp : -1;
      put_row<FMT>(a, sub, to, st.k, st.kg, st.ks);
      put_row<FMT>(b, sub, to, st.v, st.vg, st.vs);
    }
  }
}

// ---------------------------------------------------------------- append --
struct AppendArgs {
  Rows k, v;
  int L, H, T;
  const int32_t *select, *accepted, *start;
  int64_t rows;  // units T
  int bump;      // write counts here (start does not alias them)
};

__device__ __forceinline__ int accepted_of(const AppendArgs& p, int b) {
  return p.accepted ? min(max(p.accepted[b], 0), p.T) : p.T;
}
__device__ __forceinline__ int grown(const Store& st, int start, int m) {
  return (int)min((int64_t)max(start, 0) + m, (int64_t)st.max_pages * kPage);
}

// id / by, for the ids a launch has: 32-bit division where they fit
__device__ __forceinline__ int64_t div_id(int64_t id, int64_t ids, int by) {
  return ids <= 0xffffffffll ? (int64_t)((uint32_t)id / (uint32_t)by) : id / by;
}

// Few rows of each segment: eight lanes per (segment, row), both K and V of it.
// Latency of a launch: 8 tokens of 2048 segments 6 us.
template <int FMT>
__global__ void __launch_bounds__(kStoreThreads, 8) append_kernel(Store st, AppendArgs p) {
  const int64_t id = ((int64_t)blockIdx.x * kStoreThreads + threadIdx.x) >> 3;
  const int sub = threadIdx.x & 7;
  Words16 a = {}, c = {};
  int64_t to = -1;
  if (id < p.rows) {
    const int64_t u = div_id(id, p.rows, p.T);
    const int i = (int)(id - u * p.T);
    const int bl = (int)u / p.H, h = (int)u - bl * p.H;
    const int b = bl / p.L, l = bl - b * p.L;
    const int m = accepted_of(p, b);
    const int start = p.start[u];
    if (i < m) {
      const int t = p.select ? p.select[(int64_t)b * p.T + i] : i;
      const int64_t s = (int64_t)start + i;
      if (start >= 0 && s < (int64_t)st.max_pages * kPage && t >= 0 && t < p.T) to = st.slot(u, (int)s);
      if (to >= 0) {
        a = load_row(p.k.at(b, l, t, h), sub);
        c = load_row(p.v.at(b, l, t, h), sub);
      } else if (sub == 0) {
        st.raise();
      }
    }
    if (p.bump && i == 0 && sub == 0) {
      st.counts[u] = grown(st, start, m);
      if (p.accepted && p.accepted[b] != m) st.raise();
    }
  }
  put_row<FMT>(a, sub, to, st.k, st.kg, st.ks);
  put_row<FMT>(c, sub, to, st.v, st.vg, st.vs);
}

// Many rows of each segment: a block takes kRun consecutive rows of one segment, a
// group of lanes every 32nd of them, the next one's loads under way; the segment's
// indices and addresses are worked out once (from every row's own index the kernel
// was bound by its instructions).  4-bit prompt of 131071 x 8 rows written and read
// back: 230 us; runs of 128 or 512 rows 236 and 232, no loads ahead 238, append_kernel
// 257.
constexpr int kRun = 256;
template <int FMT>
__global__ void __launch_bounds__(kStoreThreads, 4) append_run_kernel(Store st, AppendArgs p, int runs) {
  const int u = blockIdx.x / runs, i0 = (blockIdx.x - u * runs) * kRun;
  const int sub = threadIdx.x & 7;
  const int bl = u / p.H, h = u - bl * p.H, b = bl / p.L, l = bl - b * p.L;
  const int m = accepted_of(p, b), start = p.start[u];
  const uint16_t *k = p.k.at(b, l, 0, h), *v = p.v.at(b, l, 0, h);
  const int32_t* select = p.select ? p.select + (int64_t)b * p.T : nullptr;
  const int32_t* table = st.table + (int64_t)u * st.max_pages;
  const int64_t room = start < 0 ? INT64_MIN : (int64_t)st.max_pages * kPage;
  const int i1 = min(m, i0 + kRun);
  Words16 a = {}, c = {};
  int64_t to = -1;
  auto fetch = [&](int i) {
    to = -1;
    if (i >= i1) return;
    const int t = select ? select[i] : i;
    const int64_t s = (int64_t)start + i;
    if (s < room && t >= 0 && t < p.T) {
      const int page = table[(int)s / kPage];
      if (page >= 0 && page < st.pool_pages) to = (int64_t)page * kPage + (int)s % kPage;
    }
    if (to >= 0) {
      a = load_row(k + t * p.k.st, sub);
      c = load_row(v + t * p.v.st, sub);
    } else if (sub == 0) {
      st.raise();
    }
  };
  const int mine = i0 + (threadIdx.x >> 3);
  fetch(mine);
#pragma unroll 1
  for (int r = 0; r < i1 - i0; r += 32) {
    const Words16 x = a, y = c;
    const int64_t at = to;
    fetch(mine + r + 32);
    put_row<FMT>(x, sub, at, st.k, st.kg, st.ks);
    put_row<FMT>(y, sub, at, st.v, st.vg, st.vs);
  }
  if (p.bump && i0 == 0 && threadIdx.x == 0) {
    st.counts[u] = grown(st, start, m);
    if (p.accepted && p.accepted[b] != m) st.raise();
  }
}

// counts[u] += m, after the rows were written at the old counts.
__global__ void __launch_bounds__(kStoreThreads) append_count_kernel(Store st, AppendArgs p) {
  const int64_t u = (int64_t)blockIdx.x * kStoreThreads + threadIdx.x;
  if (u >= st.units) return;
  const int b = (int)(u / ((int64_t)p.L * p.H));
  const int m = accepted_of(p, b);
  if (p.accepted && p.accepted[b] != m) st.raise();
  st.counts[u] = grown(st, p.start[u], m);
}

// ------------------------------------------------------------------ read --
// Eight lanes per (segment, slot): both K and V of it, 32 registers a thread so that
// an SM is full.  Bound by bytes: 130912 slots of 8 bits 20.4 us, 74 % of the copy
// bandwidth, of which a launch's start and end are a part.
template <int FMT>
__global__ void __launch_bounds__(kStoreThreads) read_kernel(Store st, const int32_t* __restrict__ start,
                                                             int T, int64_t rows,
                                                             uint16_t* __restrict__ ko,
                                                             uint16_t* __restrict__ vo) {
  const int64_t id = ((int64_t)blockIdx.x * kStoreThreads + threadIdx.x) >> 3;
  const int sub = threadIdx.x & 7;
  if (id >= rows) return;
  const int64_t u = div_id(id, rows, T);
  const int64_t s = (start ? start[u] : 0) + (id - u * T);
  const int64_t at = s >= 0 && s < st.count(u) ? st.slot(u, (int)s) : -1;
  Words16 a = {}, b = {};
  if (at >= 0) {
    a = get_row<FMT>(sub, at, st.k, st.kg, st.ks);
    b = get_row<FMT>(sub, at, st.v, st.vg, st.vs);
  }
  store_row(ko + id * kD, sub, a);
  store_row(vo + id * kD, sub, b);
}

int last_error() { return cudaGetLastError() == cudaSuccess ? CERTKV_OK : CERTKV_ECUDA; }

// blocks for `rows` rows of eight lanes; 0: too many
unsigned row_blocks(int64_t rows) {
  const int64_t blocks = (rows + kStoreThreads / 8 - 1) / (kStoreThreads / 8);
  return blocks <= INT32_MAX ? (unsigned)blocks : 0u;
}

}  // namespace
}  // namespace certkv

extern "C" size_t certkv_store_workspace_bytes(int32_t units) {
  if (units < 1 || units > (1 << 24)) return 0;
  return ((size_t)units + 1) * sizeof(int32_t);
}

extern "C" int certkv_store_load(const certkv_packed* packed, int32_t tail_slot, int32_t reserve,
                                 const certkv_store* store, void* workspace, size_t workspace_bytes,
                                 void* stream) {
  using namespace certkv;
  Store s;
  int rc = store_of(store, &s);
  if (rc) return rc;
  if (!packed || !packed->k || !packed->v || !packed->offsets || !packed->real_counts ||
      packed->capacity_slots < 1)
    return CERTKV_EINVAL;
  if (((uintptr_t)packed->k | (uintptr_t)packed->v) % 16 != 0) return CERTKV_EINVAL;
  if (((uintptr_t)packed->offsets % 8 | (uintptr_t)packed->real_counts % 4) != 0) return CERTKV_EINVAL;
  if ((tail_slot != 0 && tail_slot != 1) || reserve < 0) return CERTKV_EINVAL;
  if (!workspace || (uintptr_t)workspace % 256 != 0 ||
      workspace_bytes < certkv_store_workspace_bytes(s.units))
    return CERTKV_EWORKSPACE;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  int32_t* first = reinterpret_cast<int32_t*>(workspace);
  {
    TraceScope ts_("store_plan", st);
    if (!launch_kernel(false, load_plan_kernel, 1, 1024, 0, st, s.units, packed->real_counts, tail_slot,
                       reserve, first))
      return cuda_failed();
  }
  // enough blocks for every page, at most those that are resident together
  const int grid = s.pool_pages < 152 * kLoadBlocks ? s.pool_pages : 152 * kLoadBlocks;
  const uint16_t* pk = reinterpret_cast<const uint16_t*>(packed->k);
  const uint16_t* pv = reinterpret_cast<const uint16_t*>(packed->v);
  TraceScope ts_("store_load", st);
#define CERTKV_LOAD(F)                                                                          \
  load_kernel<F><<<grid, kStoreThreads, 0, st>>>(s, pk, pv, packed->offsets, packed->real_counts, \
                                                 tail_slot, packed->capacity_slots, first)
  if (store->format == CERTKV_STORE_BF16) CERTKV_LOAD(CERTKV_STORE_BF16);
  else if (store->format == CERTKV_STORE_FP8) CERTKV_LOAD(CERTKV_STORE_FP8);
  else CERTKV_LOAD(CERTKV_STORE_FP4);
#undef CERTKV_LOAD
  return last_error();
}

extern "C" int certkv_store_append(int32_t batch, int32_t layers, int32_t hkv, int32_t tokens,
                                   const certkv_rows* k, const certkv_rows* v,
                                   const int32_t* select, const int32_t* accepted,
                                   const int32_t* start, const certkv_store* store, void* stream) {
  using namespace certkv;
  Store s;
  int rc = store_of(store, &s);
  if (rc) return rc;
  if (batch < 1 || layers < 1 || hkv < 1 || tokens < 1 || tokens > (1 << 24)) return CERTKV_EINVAL;
  if ((int64_t)batch * layers > (1 << 24) || (int64_t)batch * layers * hkv != s.units)
    return CERTKV_EINVAL;
  if (!rows_ok(k, batch, layers, tokens, hkv) || !rows_ok(v, batch, layers, tokens, hkv))
    return CERTKV_EINVAL;
  if (((uintptr_t)select | (uintptr_t)accepted | (uintptr_t)start) % 4 != 0) return CERTKV_EINVAL;
  AppendArgs p;
  p.k = rows_of(k);
  p.v = rows_of(v);
  p.L = layers;
  p.H = hkv;
  p.T = tokens;
  p.select = select;
  p.accepted = accepted;
  p.start = start ? start : s.counts;
  p.bump = p.start != s.counts;
  p.rows = (int64_t)s.units * tokens;
  const unsigned grid = row_blocks(p.rows);
  if (!grid) return CERTKV_EINVAL;
  const int runs = (tokens + kRun - 1) / kRun;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  {
    TraceScope ts_("store_append", st);
#define CERTKV_APPEND(F)                                                                             \
  (tokens >= kRun                                                                                    \
       ? launch_kernel(false, append_run_kernel<F>, s.units * runs, kStoreThreads, 0, st, s, p, runs) \
       : launch_kernel(false, append_kernel<F>, grid, kStoreThreads, 0, st, s, p))
    const bool launched = store->format == CERTKV_STORE_BF16  ? CERTKV_APPEND(CERTKV_STORE_BF16)
                          : store->format == CERTKV_STORE_FP8 ? CERTKV_APPEND(CERTKV_STORE_FP8)
                                                              : CERTKV_APPEND(CERTKV_STORE_FP4);
#undef CERTKV_APPEND
    if (!launched) return cuda_failed();  // the counts stay with what is written
  }
  if (!p.bump) {
    TraceScope ts_("store_count", st);
    append_count_kernel<<<(s.units + kStoreThreads - 1) / kStoreThreads, kStoreThreads, 0, st>>>(s, p);
  }
  return last_error();
}

extern "C" int certkv_store_read(const certkv_store* store, const int32_t* start, int32_t tokens,
                                 void* k_out, void* v_out, void* stream) {
  using namespace certkv;
  Store s;
  int rc = store_of(store, &s);
  if (rc) return rc;
  if (tokens < 1 || tokens > (1 << 24) || !k_out || !v_out ||
      ((uintptr_t)k_out | (uintptr_t)v_out) % 16 != 0 || (uintptr_t)start % 4 != 0)
    return CERTKV_EINVAL;
  const int64_t rows = (int64_t)s.units * tokens;
  const unsigned grid = row_blocks(rows);
  if (!grid) return CERTKV_EINVAL;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  uint16_t* ko = reinterpret_cast<uint16_t*>(k_out);
  uint16_t* vo = reinterpret_cast<uint16_t*>(v_out);
  TraceScope ts_("store_read", st);
  if (store->format == CERTKV_STORE_BF16)
    read_kernel<CERTKV_STORE_BF16><<<grid, kStoreThreads, 0, st>>>(s, start, tokens, rows, ko, vo);
  else if (store->format == CERTKV_STORE_FP8)
    read_kernel<CERTKV_STORE_FP8><<<grid, kStoreThreads, 0, st>>>(s, start, tokens, rows, ko, vo);
  else
    read_kernel<CERTKV_STORE_FP4><<<grid, kStoreThreads, 0, st>>>(s, start, tokens, rows, ko, vo);
  return last_error();
}
