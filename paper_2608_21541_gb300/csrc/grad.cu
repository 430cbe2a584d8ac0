// grad.cu — gradients of tree attention over the paged store.
//
// For query row r and what it sees, slot or draft s:
//   p = exp(scale <q_r, k_s> - lse_r),  e = scale p (<dout_r, v_s> - delta_r),
//   delta_r = <dout_r, out_r> - dlse_r,
//   dq_r = sum_s e k_s,  dk_s = sum_r e q_r,  dv_s = sum_r p dout_r.
//
// Launches: what is known of each row, and the segments' tiles (grad_rows); the stored slots
// (grad_q.cu for dq, grad_kv.cu for dk and dv; with few rows grad_kv.cu for all three); the
// drafts' own keys and values, with what the shares left of dq (grad_drafts); and the sums over
// what is left in parts (grad_merge), in one order.
//
// What a row does not see cannot reach it, nor the row that, though matrix products sum over all
// rows and drafts of a tile: rows that take no part enter them as zeros with probability 0, and
// rows or keys with a NaN or infinity as zeros too, with the probabilities of what sees them NaN.
#include <float.h>
#include <math.h>

#include <algorithm>
#include <atomic>

#include "../../include/certkv.h"
#include "common.cuh"
#include "grad.cuh"
#include "internal.cuh"

namespace certkv {
namespace {

constexpr int kThreads = 256;
constexpr int kChunkRows = 128;  // query rows of a block of the drafts' kernel

__device__ __forceinline__ void store4(uint16_t* row, int lane, float4 a) {
  const __nv_bfloat162 lo = __floats2bfloat162_rn(a.x, a.y), hi = __floats2bfloat162_rn(a.z, a.w);
  *reinterpret_cast<uint2*>(row + 4 * lane) =
      make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
}
// Block 0: the tiles of the segments before each.  Latency of one launch.
__device__ __forceinline__ void scan_tiles(const GradArgs& p) {
  __shared__ long long part[kThreads / 32];
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  long long carry = 0;
  constexpr int kEach = 16;
  for (int base = 0; base < p.units; base += kEach * kThreads) {
    int n[kEach];
    long long sum = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int u = base + kEach * (int)threadIdx.x + i;
      n[i] = u < p.units ? (p.st.count(u) + kGradTile - 1) / kGradTile : 0;
      sum += n[i];
    }
    long long x = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(kFull, x, o);
      if (lane >= o) x += y;
    }
    if (lane == 31) part[warp] = x;
    __syncthreads();
    long long before = carry;
#pragma unroll
    for (int w = 0; w < kThreads / 32; ++w) {
      if (w < warp) before += part[w];
      carry += part[w];
    }
    before += x - sum;
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int u = base + kEach * (int)threadIdx.x + i;
      if (u < p.units) p.first[u] = before;
      before += n[i];
    }
    __syncthreads();
  }
  if (threadIdx.x == 0) p.first[p.units] = carry;
}

// Sixteen lanes per row: its log-sum-exp in the log2 domain and delta; +inf and 0 where it takes
// no part; NaN where its query or its output's gradient holds a NaN or infinity, or the log-sum-exp
// is +inf.  Both rows are laid out for the matrix units (grad_pack): a unit's rows are read again for
// each of its tiles, and as they lie, 16 bytes a copy, that took longer than the products (1024 rows
// over 32768 slots: the slots' gradients 247 us, 225 as bulk copies, both with p and e in one part; 279
// with the two that they have).
__global__ void __launch_bounds__(kThreads) grad_rows_kernel(const __grid_constant__ GradArgs p) {
  release_next();
  if (blockIdx.x == 0) {
    scan_tiles(p);
    return;
  }
  const int lane = threadIdx.x & 31, c = lane & 15;
  const int64_t all = (int64_t)p.units * p.padded;
  const int64_t w0 = ((int64_t)(blockIdx.x - 1) * kThreads + threadIdx.x) >> 4, w = min(w0, all - 1);
  const int u = (int)(w / p.padded), to = (int)(w - (int64_t)u * p.padded), r = min(to, p.rows - 1);
  const int t = r / p.G, g = r - t * p.G;
  const GradUnit x(p, u);
  const int qh = x.h * p.G + g;
  const int64_t at = (((int64_t)x.b * p.L + x.l) * p.T + t) * p.H * p.G + qh;
  const uint4 q = *(reinterpret_cast<const uint4*>(p.q.at(x.b, x.l, t, qh)) + c);
  const uint4 d = *(reinterpret_cast<const uint4*>(p.go.at(x.b, x.l, t, qh)) + c);
  const uint4 o = *(reinterpret_cast<const uint4*>(p.o.at(x.b, x.l, t, qh)) + c);
  const float lse = p.lse[at], dlse = p.dlse ? p.dlse[at] : 0.f;
  const uint32_t qw[4] = {q.x, q.y, q.z, q.w}, dw[4] = {d.x, d.y, d.z, d.w}, ow[4] = {o.x, o.y, o.z, o.w};
  float delta = 0.f;
  bool odd = false;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    delta = fmaf(bf16lo(dw[i]), bf16lo(ow[i]), delta);
    delta = fmaf(bf16hi(dw[i]), bf16hi(ow[i]), delta);
    odd |= (qw[i] & 0x7f80u) == 0x7f80u || (qw[i] & 0x7f800000u) == 0x7f800000u || (dw[i] & 0x7f80u) == 0x7f80u ||
           (dw[i] & 0x7f800000u) == 0x7f800000u;
  }
#pragma unroll
  for (int s = 8; s >= 1; s >>= 1) delta += __shfl_xor_sync(kFull, delta, s);
  odd = (__ballot_sync(kFull, odd) & (0xffffu << (lane & 16))) != 0u;
  if (w0 >= all) return;
  const float2 f = to >= p.rows || lse == -INFINITY ? make_float2(INFINITY, 0.f)
                   : odd || lse == INFINITY         ? make_float2(nanf(""), nanf(""))
                                                    : make_float2(lse * 1.4426950408889634f, delta - dlse);
  if (c == 0) {
    if (to < p.rows) p.row[(int64_t)u * p.rows + to] = f;
    p.neg[(int64_t)(2 * u) * p.padded + to] = -f.x;
    p.neg[(int64_t)(2 * u + 1) * p.padded + to] = -f.y;
  }
  const bool on = fabsf(f.x) < INFINITY;
  const uint4 none = make_uint4(0u, 0u, 0u, 0u);
  const int chunk = ((c & 7) ^ (to & 7)) << 4;
  *reinterpret_cast<uint4*>(grad_pack(p, u, c >> 3, to) + chunk) = on ? q : none;
  *reinterpret_cast<uint4*>(grad_pack(p, u, 2 + (c >> 3), to) + chunk) = on ? d : none;
}

// The records of unit u: shares c0 .. c1 (c1 < c0: none), of which folding leaves the first.
struct Records {
  int c0, c1;
  __device__ __forceinline__ Records(const GradArgs& p, int u, bool folded) {
    const int64_t f0 = p.first[u], f1 = p.first[u + 1], per = tiles_per_share(p);
    c0 = f1 > f0 ? (int)(f0 / per) : 1;
    c1 = f1 > f0 ? (folded ? c0 : (int)((f1 - 1) / per)) : 0;
  }
};
__device__ __forceinline__ void add4(float4& a, const float* from) {
  const float4 x = *reinterpret_cast<const float4*>(from);
  a.x += x.x;
  a.y += x.y;
  a.z += x.z;
  a.w += x.w;
}

// Few segments, of which each met many shares: one block per row adds their records up into the
// first, each warp every eighth of them, so that no warp goes through all.
__global__ void __launch_bounds__(kThreads) grad_fold_kernel(const __grid_constant__ GradArgs p) {
  __shared__ float4 part[kThreads / 32][32];
  const int u = blockIdx.x / p.rows, r = blockIdx.x - u * p.rows, warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  await_previous();
  release_next();
  const Records c(p, u, false);
  if (c.c1 <= c.c0) return;
  const int blk = r / p.rb, at = grad_at(p, r - blk * p.rb, 4 * lane);
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
  for (int i = c.c0 + warp; i <= c.c1; i += kThreads / 32) add4(a, grad_record(p, i, u, blk) + at);
  part[warp][lane] = a;
  __syncthreads();
  if (warp > 0) return;
#pragma unroll
  for (int w = 1; w < kThreads / 32; ++w) add4(a, &part[w][lane].x);
  *reinterpret_cast<float4*>(grad_record(p, c.c0, u, blk) + at) = a;
}

// Without drafts one warp per query row: the records of the shares that met its segment.  With
// them one per draft and gradient: its chunks, where there are several.
__global__ void __launch_bounds__(kThreads) grad_merge_kernel(const __grid_constant__ GradArgs p) {
  int64_t w = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> 5;
  const int lane = threadIdx.x & 31;
  await_previous();
  const int64_t rows = p.dq.p && !p.kn.p ? (int64_t)p.units * p.rows : 0;
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  if (w < rows) {
    const int u = (int)(w / p.rows), r = (int)(w - (int64_t)u * p.rows), t = r / p.G, g = r - t * p.G;
    const GradUnit x(p, u);
    const int blk = r / p.rb, at = grad_at(p, r - blk * p.rb, 4 * lane);
    const Records c(p, u, p.folded);
#pragma unroll 4
    for (int i = c.c0; i <= c.c1; ++i) add4(a, grad_record(p, i, u, blk) + at);
    // a row that takes no part: its zeros times a slot's NaN or infinity are NaN
    if (p.row[(int64_t)u * p.rows + r].x == INFINITY) a = make_float4(0.f, 0.f, 0.f, 0.f);
    store4(p.dq.at(x.b, x.l, t, x.h * p.G + g), lane,
           make_float4(a.x * p.scale, a.y * p.scale, a.z * p.scale, a.w * p.scale));
    return;
  }
  w -= rows;
  if (!p.dkn.p || p.chunks == 1 || w >= (int64_t)p.units * p.T * 2) return;
  const int u = (int)(w / (2 * p.T)), i = (int)(w - (int64_t)u * 2 * p.T), key = i < p.T, j = key ? i : i - p.T;
  const GradUnit x(p, u);
#pragma unroll 4
  for (int c = 0; c < p.chunks; ++c) add4(a, p.part + (((int64_t)u * p.chunks + c) * 2 * p.T + i) * kD + 4 * lane);
  const float f = key ? p.scale : 1.f;
  store4((key ? p.dkn : p.dvn).at(x.b, x.l, j, x.h), lane, make_float4(a.x * f, a.y * f, a.z * f, a.w * f));
}

// ----------------------------------------------------------------- drafts --
__device__ __forceinline__ uint32_t smem(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void ldm4(uint32_t a, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(a)
               : "memory");
}
__device__ __forceinline__ void ldm4t(uint32_t a, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(a)
               : "memory");
}
__device__ __forceinline__ void mma(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, "
      "{%0, %1, %2, %3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}

constexpr int kPitch = 2 * kD + 16;  // bytes of a row of 128 elements in shared memory: odd in 16 bytes
template <int TD>
struct Drafts {  // TD: the drafts, filled up with zeros
  static constexpr int kWide = 2 * TD + 16;
  static constexpr int kKeyOff = 0, kValueOff = TD * kPitch;
  static constexpr int kRowOff = 2 * TD * kPitch, kGradOff = kRowOff + kChunkRows * kPitch;
  static constexpr int kPOff = kGradOff + kChunkRows * kPitch, kEOff = kPOff + kChunkRows * kWide;
  static constexpr int kRest = 2 * kChunkRows * kWide;  // p and e's roundings' remainders lie so far behind them
  static constexpr int kInfoOff = kEOff + kChunkRows * kWide + kRest, kSeenOff = kInfoOff + kChunkRows * 8;
  static constexpr int kBadOff = kSeenOff + kChunkRows * 8, kBytes = kBadOff + 16;
};

__device__ __forceinline__ void copy16(uint32_t to, const void* from, bool on) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(on ? 16 : 0) : "memory");
}

// N elements from d0 on of dq of a warp's 16 rows, from s0 on: what the shares left of them, all
// loads of a share under way, and the drafts' part.  A row that takes no part gets 0, whatever its
// zeros made of a slot's NaN or infinity.
template <int TD, int N>
__device__ __forceinline__ void drafts_dq(const GradArgs& p, const GradUnit& x, int u, int r0, int rows, int s0, int d0,
                                          uint32_t base, const float2* info) {
  using D = Drafts<TD>;
  const int lane = threadIdx.x & 31, g8 = lane >> 2, t4 = lane & 3;
  const int lr = lane & 7, l8 = lane >> 3 & 1, l16 = lane >> 4;
  float acc[N / 8][4];
  const Records part(p, u, p.folded);
  const float* from[2];
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int br = min(r0 + s0 + g8 + 8 * h, p.rows - 1), blk = br / p.rb;
    from[h] = grad_record(p, part.c0, u, blk) + grad_at(p, br - blk * p.rb, d0 + 2 * t4);
  }
#pragma unroll
  for (int h = 0; h < 2; ++h)
#pragma unroll
    for (int n = 0; n < N / 8; ++n) {
      const float2 y = part.c0 <= part.c1 ? __ldcg(reinterpret_cast<const float2*>(from[h] + n * p.rb * 8)) : make_float2(0.f, 0.f);
      acc[n][2 * h] = y.x, acc[n][2 * h + 1] = y.y;
    }
  const int64_t share = (int64_t)p.nblk * p.rb * kD;
#pragma unroll 1
  for (int i = part.c0 + 1; i <= part.c1; ++i) {
    float2 y[2][N / 8];
#pragma unroll
    for (int h = 0; h < 2; ++h) {
      from[h] += share;
#pragma unroll
      for (int n = 0; n < N / 8; ++n) y[h][n] = __ldcg(reinterpret_cast<const float2*>(from[h] + n * p.rb * 8));
    }
#pragma unroll
    for (int h = 0; h < 2; ++h)
#pragma unroll
      for (int n = 0; n < N / 8; ++n) acc[n][2 * h] += y[h][n].x, acc[n][2 * h + 1] += y[h][n].y;
  }
#pragma unroll
  for (int k = 0; k < TD / 16; ++k) {
    uint32_t a[4], ar[4];
    const uint32_t at = base + (uint32_t)(D::kEOff + (s0 + lr + 8 * l8) * D::kWide + 32 * k + 16 * l16);
    ldm4(at, a);
    ldm4(at + D::kRest, ar);
#pragma unroll
    for (int d = 0; d < N / 16; ++d) {
      uint32_t b[4];
      ldm4t(base + (uint32_t)(D::kKeyOff + (16 * k + lr + 8 * l8) * kPitch + 2 * d0 + 32 * d + 16 * l16), b);
      mma(acc[2 * d], a, b[0], b[1]);
      mma(acc[2 * d + 1], a, b[2], b[3]);
      mma(acc[2 * d], ar, b[0], b[1]);
      mma(acc[2 * d + 1], ar, b[2], b[3]);
    }
  }
#pragma unroll
  for (int h = 0; h < 2; ++h) {
    const int br = r0 + s0 + g8 + 8 * h, tok = br / p.G;
    if (s0 + g8 + 8 * h >= rows) continue;
    uint16_t* out = p.dq.at(x.b, x.l, tok, x.h * p.G + br - tok * p.G) + d0 + 2 * t4;
    const bool on = info[s0 + g8 + 8 * h].x != INFINITY;
#pragma unroll
    for (int n = 0; n < N / 8; ++n)
      *reinterpret_cast<uint32_t*>(out + 8 * n) = on ? pack2(acc[n][2 * h] * p.scale, acc[n][2 * h + 1] * p.scale) : 0u;
  }
}

// One block per (unit, 128 query rows), on mma.sync: products of at most 128 x 64 x 128, whose
// time is that of bringing the rows in.  A warp makes p and e of 16 rows; then each warp 16 elements
// of dk and dv over all rows; then each its rows' dq.  All but the last runs while the last CTAs of
// the kernel before, which leave the records, still do (8-bit trees 173 us, 180 behind them): that
// kernel lets this one start behind its own wait for grad_rows_kernel, whose rows are thus there.
// Where there is no kernel between the two this one is not started early.
template <int TD>
__global__ void __launch_bounds__(kThreads) grad_drafts_kernel(const __grid_constant__ GradArgs p) {
  using D = Drafts<TD>;
  extern __shared__ __align__(128) char sm[];
  const int u = blockIdx.x / p.chunks, chunk = blockIdx.x - u * p.chunks;
  const int r0 = chunk * kChunkRows, rows = min(p.rows - r0, kChunkRows), strips = (rows + 15) / 16;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const GradUnit x(p, u);
  float2* info = reinterpret_cast<float2*>(sm + D::kInfoOff);
  uint64_t* sees = reinterpret_cast<uint64_t*>(sm + D::kSeenOff);
  unsigned long long* bad = reinterpret_cast<unsigned long long*>(sm + D::kBadOff);
  if (tid == 0) *bad = 0ull;
  if (tid < kChunkRows) {
    info[tid] = tid < rows ? __ldcg(p.row + (int64_t)u * p.rows + r0 + tid) : make_float2(INFINITY, 0.f);
    sees[tid] = tid < rows && info[tid].x != INFINITY ? grad_seen(p, x.b, (r0 + tid) / p.G) : 0ull;
  }
  __syncthreads();
  const int c = tid & 15;  // 16 lanes a row, 16 bytes each
  const uint32_t base = smem(sm);
  {
    const uint16_t *q0 = p.q.at(x.b, x.l, 0, x.h * p.G) + 8 * c, *g0 = p.go.at(x.b, x.l, 0, x.h * p.G) + 8 * c;
#pragma unroll
    for (int i = 0; i < kChunkRows / (kThreads / 16); ++i) {
      const int r = (tid >> 4) + i * (kThreads / 16);
      if (r >= 16 * strips) break;
      const bool on = fabsf(info[r].x) < INFINITY;
      const int br = r0 + r, tok = br / p.G, g = br - tok * p.G;
      copy16(base + D::kRowOff + r * kPitch + 16 * c, on ? q0 + tok * p.q.st + g * p.q.sh : q0, on);
      copy16(base + D::kGradOff + r * kPitch + 16 * c, on ? g0 + tok * p.go.st + g * p.go.sh : g0, on);
    }
  }
  {
    constexpr int kEach = TD / (kThreads / 16) > 0 ? TD / (kThreads / 16) : 1;
    uint4 k[kEach], v[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int j = (tid >> 4) + i * (kThreads / 16);
      k[i] = v[i] = make_uint4(0u, 0u, 0u, 0u);
      if (j < p.T) {
        k[i] = *(reinterpret_cast<const uint4*>(p.kn.at(x.b, x.l, j, x.h)) + c);
        v[i] = *(reinterpret_cast<const uint4*>(p.vn.at(x.b, x.l, j, x.h)) + c);
      }
    }
#pragma unroll
    for (int i = 0; i < kEach; ++i) {  // keys with a NaN or infinity as zeros, and noted
      const int j = (tid >> 4) + i * (kThreads / 16);
      const uint32_t w[4] = {k[i].x, k[i].y, k[i].z, k[i].w};
      bool odd = false;
#pragma unroll
      for (int n = 0; n < 4; ++n) odd |= (w[n] & 0x7f80u) == 0x7f80u || (w[n] & 0x7f800000u) == 0x7f800000u;
      const uint32_t any = __ballot_sync(kFull, odd) & (0xffffu << (lane & 16));
      if (any) {
        k[i] = make_uint4(0u, 0u, 0u, 0u);
        if (c == 0) atomicOr(bad, 1ull << j);
      }
      *reinterpret_cast<uint4*>(sm + D::kKeyOff + j * kPitch + 16 * c) = k[i];
      *reinterpret_cast<uint4*>(sm + D::kValueOff + j * kPitch + 16 * c) = v[i];
    }
  }
  const int g8 = lane >> 2, t4 = lane & 3;
  asm volatile("cp.async.commit_group;\ncp.async.wait_group 0;" ::: "memory");
  __syncthreads();
  // lane's address offsets of 16 x 16 blocks: rows as they lie (A), rows as columns of B, and
  // transposed (B from [k][n], A from [k][m])
  const int lr = lane & 7, l8 = lane >> 3 & 1, l16 = lane >> 4;
  const int s0 = 16 * warp;
  if (warp < strips) {
    float s[TD / 8][4], r[TD / 8][4];
#pragma unroll
    for (int n = 0; n < TD / 8; ++n)
#pragma unroll
      for (int i = 0; i < 4; ++i) s[n][i] = r[n][i] = 0.f;
#pragma unroll
    for (int k = 0; k < kD / 16; ++k) {
      uint32_t aq[4], ag[4];
      const uint32_t at = base + (uint32_t)((s0 + lr + 8 * l8) * kPitch + 32 * k + 16 * l16);
      ldm4(at + D::kRowOff, aq);
      ldm4(at + D::kGradOff, ag);
#pragma unroll
      for (int n = 0; n < TD / 16; ++n) {
        uint32_t bk[4], bv[4];
        const uint32_t to = base + (uint32_t)((16 * n + lr + 8 * l16) * kPitch + 32 * k + 16 * l8);
        ldm4(to + D::kKeyOff, bk);
        ldm4(to + D::kValueOff, bv);
        mma(s[2 * n], aq, bk[0], bk[1]);
        mma(s[2 * n + 1], aq, bk[2], bk[3]);
        mma(r[2 * n], ag, bv[0], bv[1]);
        mma(r[2 * n + 1], ag, bv[2], bv[3]);
      }
    }
    const unsigned long long odd = *bad;
    const float2 i0 = info[s0 + g8], i1 = info[s0 + g8 + 8];
    const uint64_t see0 = sees[s0 + g8], see1 = sees[s0 + g8 + 8];
#pragma unroll
    for (int n = 0; n < TD / 8; ++n) {
      float pr[4], er[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int j = 8 * n + 2 * t4 + (i & 1);
        const float2 inf = i < 2 ? i0 : i1;
        const bool on = (i < 2 ? see0 : see1) >> j & 1u;
        pr[i] = on ? (odd >> j & 1u ? nanf("") : exp2f(fmaf(s[n][i], p.scale_log2, -inf.x))) : 0.f;
        er[i] = on ? pr[i] * (r[n][i] - inf.y) : 0.f;
      }
      const int at = (s0 + g8) * D::kWide + 16 * n + 4 * t4;
      const uint32_t p0 = pack2(pr[0], pr[1]), p1 = pack2(pr[2], pr[3]);
      const uint32_t e0 = pack2(er[0], er[1]), e1 = pack2(er[2], er[3]);
      auto put = [&](int off, uint32_t lo, uint32_t hi) {
        *reinterpret_cast<uint32_t*>(sm + off + at) = lo;
        *reinterpret_cast<uint32_t*>(sm + off + at + 8 * D::kWide) = hi;
      };
      put(D::kPOff, p0, p1);
      put(D::kPOff + D::kRest, pack2(pr[0] - bf16lo(p0), pr[1] - bf16hi(p0)), pack2(pr[2] - bf16lo(p1), pr[3] - bf16hi(p1)));
      put(D::kEOff, e0, e1);
      put(D::kEOff + D::kRest, pack2(er[0] - bf16lo(e0), er[1] - bf16hi(e0)), pack2(er[2] - bf16lo(e1), er[3] - bf16hi(e1)));
    }
  }
  __syncthreads();
  if (p.dkn.p) {
    float dk[TD / 16][2][4], dv[TD / 16][2][4];
#pragma unroll
    for (int i = 0; i < TD / 16; ++i)
#pragma unroll
      for (int n = 0; n < 2; ++n)
#pragma unroll
        for (int k = 0; k < 4; ++k) dk[i][n][k] = dv[i][n][k] = 0.f;
    for (int k = 0; k < strips; ++k) {
      uint32_t bq[4], bg[4];
      const uint32_t at = base + (uint32_t)((16 * k + lr + 8 * l8) * kPitch + 32 * warp + 16 * l16);
      ldm4t(at + D::kRowOff, bq);
      ldm4t(at + D::kGradOff, bg);
#pragma unroll
      for (int i = 0; i < TD / 16; ++i) {
#pragma unroll
        for (int part = 0; part < 2; ++part) {
          uint32_t ap[4], ae[4];
          const uint32_t to = base + (uint32_t)(part * D::kRest + (16 * k + lr + 8 * l16) * D::kWide + 32 * i + 16 * l8);
          ldm4t(to + D::kPOff, ap);
          ldm4t(to + D::kEOff, ae);
          mma(dv[i][0], ap, bg[0], bg[1]);
          mma(dv[i][1], ap, bg[2], bg[3]);
          mma(dk[i][0], ae, bq[0], bq[1]);
          mma(dk[i][1], ae, bq[2], bq[3]);
        }
      }
    }
#pragma unroll
    for (int i = 0; i < TD / 16; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int j = 16 * i + g8 + 8 * h;
        if (j >= p.T) continue;
#pragma unroll
        for (int n = 0; n < 2; ++n) {
          const int d = 16 * warp + 8 * n + 2 * t4;
          if (p.chunks == 1) {
            *reinterpret_cast<uint32_t*>(p.dkn.at(x.b, x.l, j, x.h) + d) =
                pack2(dk[i][n][2 * h] * p.scale, dk[i][n][2 * h + 1] * p.scale);
            *reinterpret_cast<uint32_t*>(p.dvn.at(x.b, x.l, j, x.h) + d) = pack2(dv[i][n][2 * h], dv[i][n][2 * h + 1]);
          } else {
            float* o = p.part + (((int64_t)u * p.chunks + chunk) * 2 * p.T + j) * kD + d;
            *reinterpret_cast<float2*>(o) = make_float2(dk[i][n][2 * h], dk[i][n][2 * h + 1]);
            *reinterpret_cast<float2*>(o + (int64_t)p.T * kD) = make_float2(dv[i][n][2 * h], dv[i][n][2 * h + 1]);
          }
        }
      }
  }
  await_previous();  // the records
  release_next();
  if (!p.dq.p) return;
  // a strip's elements shared out over the warps that have none of their own (1 token x 4 heads in a
  // graph: 21 -> 15 us)
  if (strips > 4) {
    if (warp < strips) drafts_dq<TD, 128>(p, x, u, r0, rows, 16 * warp, 0, base, info);
  } else if (strips > 2) {
    if (warp / 2 < strips) drafts_dq<TD, 64>(p, x, u, r0, rows, 16 * (warp / 2), 64 * (warp & 1), base, info);
  } else if (strips > 1) {
    drafts_dq<TD, 32>(p, x, u, r0, rows, 16 * (warp / 4), 32 * (warp & 3), base, info);
  } else {
    drafts_dq<TD, 16>(p, x, u, r0, rows, 0, 16 * warp, base, info);
  }
}

template <int TD>
bool launch_drafts(const GradArgs& p, bool early, cudaStream_t st) {
  constexpr int bytes = Drafts<TD>::kBytes;
  static_assert(bytes <= 232448, "over the 227 KB of shared memory a CTA can have");
  static std::atomic<uint64_t> ready{0};  // devices on which the shared memory is opted in to
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  if (dev > 63 || !(ready.load() >> dev & 1u)) {
    if (cudaFuncSetAttribute(grad_drafts_kernel<TD>, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes) != cudaSuccess)
      return false;
    if (dev < 64) ready.fetch_or(1ull << dev);
  }
  return launch_kernel(early, grad_drafts_kernel<TD>, (unsigned)((int64_t)p.units * p.chunks), kThreads, bytes, st, p);
}

int grad_shape(const certkv_shape* s, int32_t tokens) {
  if (!s || s->batch < 1 || s->layers < 1 || s->hq < 1 || s->hkv < 1) return CERTKV_EINVAL;
  if (s->d != kD || s->hq % s->hkv != 0 || s->hq / s->hkv > CERTKV_TREE_MAX_GROUP) return CERTKV_EINVAL;
  if (tokens < 1 || tokens > CERTKV_TREE_MAX_TOKENS) return CERTKV_EINVAL;
  if ((int64_t)s->batch * s->layers > (1 << 24) || (int64_t)s->batch * s->layers * s->hkv > (1 << 24))
    return CERTKV_EINVAL;
  return CERTKV_OK;
}

constexpr int kMaxCtas = 1024;  // records are sized for at most this many

struct GradLayout {
  int padded, nblk, rb, chunks;
  size_t row, first, pack, neg, rec, part, total;
  GradLayout(int64_t units, int tokens, int rows) {
    auto a = [](size_t x) { return (x + 255) / 256 * 256; };
    nblk = (rows + kGradRows - 1) / kGradRows;
    rb = ((rows + nblk - 1) / nblk + 7) / 8 * 8;
    padded = (rows + 15) / 16 * 16;
    chunks = (rows + kChunkRows - 1) / kChunkRows;
    const size_t n = (size_t)units * rows;
    row = 0;
    first = row + a(n * sizeof(float2));
    pack = first + a(((size_t)units + 1) * sizeof(int64_t));
    neg = pack + (size_t)units * 4 * padded * 128;
    rec = neg + a((size_t)units * 2 * padded * sizeof(float));
    part = rec + ((size_t)units * nblk + kMaxCtas) * rb * kD * sizeof(float);
    total = part + (chunks > 1 ? (size_t)units * chunks * 2 * tokens * kD * sizeof(float) : 0);
  }
};

unsigned warps(int64_t n) { return (unsigned)((n * 32 + kThreads - 1) / kThreads); }

}  // namespace
}  // namespace certkv

extern "C" size_t certkv_tree_grad_workspace_bytes(const certkv_shape* shape, int32_t tokens) {
  using namespace certkv;
  if (grad_shape(shape, tokens)) return 0;
  return GradLayout((int64_t)shape->batch * shape->layers * shape->hkv, tokens, tokens * (shape->hq / shape->hkv)).total;
}

extern "C" int certkv_tree_attn_grad(const certkv_shape* shape, int32_t tokens, const certkv_rows* q,
                                     const certkv_rows* k_new, const certkv_rows* v_new, const uint64_t* mask,
                                     const certkv_store* store, float scale, const certkv_rows* out,
                                     const float* lse, const certkv_rows* dout, const float* dlse,
                                     const certkv_rows* dq, const certkv_rows* dk_new, const certkv_rows* dv_new,
                                     void* dk_store, void* dv_store, void* workspace, size_t workspace_bytes,
                                     void* stream) {
  using namespace certkv;
  int rc = grad_shape(shape, tokens);
  if (rc) return rc;
  const int B = shape->batch, L = shape->layers, Hq = shape->hq, H = shape->hkv;
  GradArgs p;
  if ((rc = store_of(store, &p.st))) return rc;
  if ((int64_t)B * L * H != p.st.units) return CERTKV_EINVAL;
  if (!rows_ok(q, B, L, tokens, Hq) || !rows_ok(out, B, L, tokens, Hq) || !rows_ok(dout, B, L, tokens, Hq))
    return CERTKV_EINVAL;
  if (!lse || ((uintptr_t)lse | (uintptr_t)dlse) % 4 != 0 || (uintptr_t)mask % 8 != 0) return CERTKV_EINVAL;
  if ((k_new == nullptr) != (v_new == nullptr) || (dk_new == nullptr) != (dv_new == nullptr) ||
      (dk_store == nullptr) != (dv_store == nullptr))
    return CERTKV_EINVAL;
  if (k_new && (!rows_ok(k_new, B, L, tokens, H) || !rows_ok(v_new, B, L, tokens, H))) return CERTKV_EINVAL;
  if (dq && !rows_out_ok(dq, B, L, tokens, Hq)) return CERTKV_EINVAL;
  if (dk_new && (!k_new || !rows_out_ok(dk_new, B, L, tokens, H) || !rows_out_ok(dv_new, B, L, tokens, H)))
    return CERTKV_EINVAL;
  if (((uintptr_t)dk_store | (uintptr_t)dv_store) % 128 != 0 || (!dq && !dk_new && !dk_store)) return CERTKV_EINVAL;
  if (!(scale >= 0.0f) || !isfinite(scale)) return CERTKV_EINVAL;
  if (!workspace || (uintptr_t)workspace % 256 != 0 ||
      workspace_bytes < certkv_tree_grad_workspace_bytes(shape, tokens))
    return CERTKV_EWORKSPACE;
  p.L = L;
  p.H = H;
  p.G = Hq / H;
  p.T = tokens;
  p.units = p.st.units;
  p.rows = tokens * p.G;
  p.q = rows_of(q);
  p.kn = rows_of(k_new);
  p.vn = rows_of(v_new);
  p.o = rows_of(out);
  p.go = rows_of(dout);
  p.dq = rows_of(dq);
  p.dkn = rows_of(dk_new);
  p.dvn = rows_of(dv_new);
  p.mask = mask;
  p.lse = lse;
  p.dlse = dlse;
  p.scale = (float)(scale > 0.0f ? scale : 1.0 / sqrt((double)kD));
  // a number whose reciprocal there is: the queries' kernel divides by it
  p.scale_log2 = std::max((float)((scale > 0.0f ? scale : 1.0 / sqrt((double)kD)) * 1.4426950408889634), FLT_MIN);
  p.dks = reinterpret_cast<uint16_t*>(dk_store);
  p.dvs = reinterpret_cast<uint16_t*>(dv_store);
  const GradLayout ly(p.units, tokens, p.rows);
  p.padded = ly.padded;
  p.nblk = ly.nblk;
  p.rb = ly.rb;
  p.chunks = ly.chunks;
  char* ws = reinterpret_cast<char*>(workspace);
  p.row = reinterpret_cast<float2*>(ws + ly.row);
  p.first = reinterpret_cast<int64_t*>(ws + ly.first);
  p.pack = reinterpret_cast<uint8_t*>(ws + ly.pack);
  p.neg = reinterpret_cast<float*>(ws + ly.neg);
  p.rec = reinterpret_cast<float*>(ws + ly.rec);
  p.part = reinterpret_cast<float*>(ws + ly.part);
  // warps of the merge, blocks of the drafts' kernel
  const int64_t n = (int64_t)p.units * p.rows;
  if ((n + 2 * (int64_t)p.units * tokens) * 32 / kThreads >= INT32_MAX - 1) return CERTKV_EINVAL;
  int sms = grad_ctas();
  if (sms < 1) return CERTKV_ECUDA;
  sms = std::min(sms, kMaxCtas);
  const bool fused = p.dks && p.rows <= kGradFused;
  p.groups = fused ? sms : std::max(sms / p.nblk, 1);
  // shares that a segment may meet, where segments are few and long (one of 131072 slots)
  p.folded = p.dq.p && p.groups > 8 * (int64_t)p.units && p.st.max_pages > 16;
  // a CTA counts its tiles and blocks of rows in 32 bits
  if ((int64_t)p.units * (p.st.max_pages + 2) / p.groups * ((p.rows + kGradFused - 1) / kGradFused) >= (1 << 29))
    return CERTKV_EINVAL;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  {
    TraceScope ts_("grad_rows", st);
    if (!launch_kernel(false, grad_rows_kernel, warps(((int64_t)p.units * p.padded + 1) / 2) + 1, kThreads, 0, st, p)) return cuda_failed();
  }
  if (p.dks) {
    GradArgs all = p;
    all.groups = sms;
    if (!launch_grad_kv(all, store->format, st)) return cuda_failed();
  }
  if (p.dq.p && !fused && !launch_grad_q(p, store->format, st)) return cuda_failed();
  if (p.folded) {
    TraceScope ts_("grad_fold", st);
    if (!launch_kernel(true, grad_fold_kernel, (unsigned)n, kThreads, 0, st, p)) return cuda_failed();
  }
  if (p.kn.p && (p.dq.p || p.dkn.p)) {
    TraceScope ts_("grad_drafts", st);
    const bool early = p.dks || p.dq.p;
    if (!(tokens <= 16 ? launch_drafts<16>(p, early, st) : launch_drafts<64>(p, early, st))) return cuda_failed();
  }
  const int64_t w = p.kn.p ? (p.dkn.p && p.chunks > 1 ? 2 * (int64_t)p.units * tokens : 0) : p.dq.p ? n : 0;
  if (w > 0) {
    TraceScope ts_("grad_merge", st);
    launch_kernel(true, grad_merge_kernel, warps(w), kThreads, 0, st, p);
  }
  return cudaGetLastError() == cudaSuccess ? CERTKV_OK : CERTKV_ECUDA;
}
