// tree.cu — attention of a tree of drafted tokens over the paged store.
//
// For query row r = (token t, head g of the group) of unit u:
//   out_r = sum_s p_s v_s / sum_s p_s,  p_s = exp(scale <q_r, k_s> - m_r),
// over all counts[u] stored slots and the drafts j whose bit is set in token
// t's mask word.  A draft that a row does not see is never read for it, so a
// NaN there cannot reach it.
//
// Three launches: a scan of the segments' tile counts (the split kernels do it
// themselves for few units), a split kernel over equal shares of all tiles
// (tree_mma.cu for few query rows per unit, else tree_tc.cu: small_max), and the
// merge below, which joins the records of the CTAs that met a unit in the
// log-sum-exp domain and, for few rows, adds the drafts.
#include <math.h>

#include <algorithm>

#include "../../include/certkv.h"
#include "common.cuh"
#include "internal.cuh"
#include "tree.cuh"

namespace certkv {

// One block: first[u] = tiles of the segments before u, first[units] their sum.
// Latency of one launch; only for more segments than kInlineUnits.
__global__ void __launch_bounds__(1024) tree_plan_kernel(Store st, int tile, int with_drafts,
                                                         int64_t* __restrict__ first) {
  __shared__ long long wsum[32];
  __shared__ long long carry;
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  release_next();
  if (threadIdx.x == 0) carry = 0;
  __syncthreads();
  for (int base = 0; base < st.units; base += 1024) {
    const int u = base + threadIdx.x;
    const long long v =
        u < st.units ? (st.count(u) + tile - 1) / tile + with_drafts : 0;
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
    if (u < st.units) first[u] = carry + (warp > 0 ? wsum[warp - 1] : 0) + x - v;
    __syncthreads();
    if (threadIdx.x == 0) carry += wsum[31];
    __syncthreads();
  }
  if (threadIdx.x == 0) first[st.units] = carry;
}

// Bound by the records' bytes where there are many (32 segments of 256 rows, 24 MB
// from DRAM: 13 us) and by the latency of a launch else; four records' loads are in
// flight at a time.
//
// One warp per (unit, row), a lane four dimensions: the records of the CTAs that
// met the row's block, each weighted by its sum 2^C l, and what the split left
// out: the NaN and infinite elements of drafts the row sees.
__global__ void __launch_bounds__(256) tree_merge_kernel(const __grid_constant__ TreeArgs p) {
  const int64_t w = (int64_t)blockIdx.x * 8 + (threadIdx.x >> 5);
  await_previous();
  if (w >= (int64_t)p.units * p.rows) return;
  const int lane = threadIdx.x & 31;
  const int u = (int)(w / p.rows), r = (int)(w - (int64_t)u * p.rows), t = r / p.G, g = r - t * p.G;
  const int bl = u / p.H, h = u - bl * p.H, b = bl / p.L, l = bl - b * p.L;
  const int blk = r / p.rb, br = r - blk * p.rb;
  const int64_t n = p.first[u + 1] - p.first[u];
  float M = -INFINITY, L = 0.f;
  float4 A = make_float4(0.f, 0.f, 0.f, 0.f);
  if (n > 0) {
    const int64_t per = tiles_per_cta(p, p.first), at = p.first[u] * p.nblk + blk * n;
    const int64_t vu = (int64_t)u * p.nblk + blk;
    const int c0 = (int)(at / per), c1 = (int)((at + n - 1) / per);
    if (c0 == c1) {  // one record, as where segments are short: as it is
      const int64_t rec = (c0 + vu) * p.rb + br;
      const float2 ml = p.rec_ml[rec];
      const float4 a = *reinterpret_cast<const float4*>(p.rec_acc + rec * kD + 4 * lane);
      if (ml.y != 0.f) {
        M = ml.x;
        L = ml.y;
        A = make_float4(a.x * L, a.y * L, a.z * L, a.w * L);
      }
    }
    for (int c = c0; c0 < c1 && c <= c1; c += 4) {
      float2 ml[4];
      float4 a[4];
      float m = M;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t rec = (min(c + i, c1) + vu) * p.rb + br;
        ml[i] = p.rec_ml[rec];
        a[i] = *reinterpret_cast<const float4*>(p.rec_acc + rec * kD + 4 * lane);
        if (c + i > c1) ml[i] = make_float2(-INFINITY, 0.f);
        m = fmaxf(m, ml[i].x);
      }
      const float back = M == m ? 1.f : exp2f(M - m);
      M = m;
      L *= back;
      A.x *= back;
      A.y *= back;
      A.z *= back;
      A.w *= back;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (ml[i].y == 0.f) continue;  // this CTA's tiles held nothing the row sees
        const float f = ml[i].y * exp2f(ml[i].x - m);
        L += f;
        A.x = fmaf(a[i].x, f, A.x);
        A.y = fmaf(a[i].y, f, A.y);
        A.z = fmaf(a[i].z, f, A.z);
        A.w = fmaf(a[i].w, f, A.w);
      }
    }
  }
  if (p.small && p.kn.p) {
    // the drafts the row sees, four at a time, four dimensions a lane; a draft it
    // does not see is not read
    const uint2 x = *reinterpret_cast<const uint2*>(p.q.at(b, l, t, h * p.G + g) + 4 * lane);
    const float q[4] = {bf16lo(x.x), bf16hi(x.x), bf16lo(x.y), bf16hi(x.y)};
    const uint64_t see = seen(p, b, t);
    for (int j = 0; j < p.T; j += 4) {
      if (!(see >> j & 15u)) continue;
      uint2 k[4], v[4];
      float z[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        k[i] = v[i] = make_uint2(0u, 0u);
        if (see >> (j + i) & 1u) {
          k[i] = *reinterpret_cast<const uint2*>(p.kn.at(b, l, j + i, h) + 4 * lane);
          v[i] = *reinterpret_cast<const uint2*>(p.vn.at(b, l, j + i, h) + 4 * lane);
        }
        z[i] = q[0] * bf16lo(k[i].x) + q[1] * bf16hi(k[i].x) + q[2] * bf16lo(k[i].y) + q[3] * bf16hi(k[i].y);
      }
#pragma unroll
      for (int o = 16; o >= 1; o >>= 1) {
#pragma unroll
        for (int i = 0; i < 4; ++i) z[i] += __shfl_xor_sync(kFull, z[i], o);
      }
      float m = M;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        z[i] = see >> (j + i) & 1u ? z[i] * p.scale_log2 : -INFINITY;
        m = fmaxf(m, z[i]);
      }
      const float back = M == m ? 1.f : exp2f(M - m);
      M = m;
      L *= back;
      A.x *= back;
      A.y *= back;
      A.z *= back;
      A.w *= back;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        if (!(see >> (j + i) & 1u)) continue;
        const float f = z[i] == -INFINITY ? 0.f : exp2f(z[i] - m);  // a NaN logit stays one
        L += f;
        A.x = fmaf(f, bf16lo(v[i].x), A.x);
        A.y = fmaf(f, bf16hi(v[i].x), A.y);
        A.z = fmaf(f, bf16lo(v[i].y), A.z);
        A.w = fmaf(f, bf16hi(v[i].y), A.w);
      }
    }
  }
  const float inv = L != 0.f ? 1.f / L : 0.f;  // a NaN sum stays a NaN
  A.x *= inv;
  A.y *= inv;
  A.z *= inv;
  A.w *= inv;
  if (!p.small && p.kn.p) {
    for (uint64_t odd = p.odd[u] & seen(p, b, t); odd; odd &= odd - 1) {
      const uint2 x = *reinterpret_cast<const uint2*>(p.vn.at(b, l, __ffsll((long long)odd) - 1, h) + 4 * lane);
      const float v[4] = {bf16lo(x.x), bf16hi(x.x), bf16lo(x.y), bf16hi(x.y)};
      if (!(fabsf(v[0]) < INFINITY)) A.x += v[0];
      if (!(fabsf(v[1]) < INFINITY)) A.y += v[1];
      if (!(fabsf(v[2]) < INFINITY)) A.z += v[2];
      if (!(fabsf(v[3]) < INFINITY)) A.w += v[3];
    }
  }
  const __nv_bfloat162 lo = __floats2bfloat162_rn(A.x, A.y), hi = __floats2bfloat162_rn(A.z, A.w);
  *reinterpret_cast<uint2*>(p.o.at(b, l, t, h * p.G + g) + 4 * lane) =
      make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
  if (p.lse && lane == 0)
    p.lse[((int64_t)bl * p.T + t) * p.H * p.G + h * p.G + g] =
        L != 0.f ? (M + log2f(L)) * kLn2 : -INFINITY;
}

namespace {

int tree_shape(const certkv_shape* s, int32_t tokens) {
  if (!s || s->batch < 1 || s->layers < 1 || s->hq < 1 || s->hkv < 1) return CERTKV_EINVAL;
  if (s->d != kD || s->hq % s->hkv != 0 || s->hq / s->hkv > CERTKV_TREE_MAX_GROUP) return CERTKV_EINVAL;
  if (tokens < 1 || tokens > CERTKV_TREE_MAX_TOKENS) return CERTKV_EINVAL;
  if ((int64_t)s->batch * s->layers > (1 << 24) ||
      (int64_t)s->batch * s->layers * s->hkv > (1 << 24))
    return CERTKV_EINVAL;
  return CERTKV_OK;
}

// Query rows of a unit in blocks, as equal as they come: few rows in blocks of at
// most 16 (mma.sync), more in blocks of at most 256 (tcgen05: up to 128 rows are
// one M = 128 operand, up to 256 two).
void row_blocks(int rows, int format, int* nblk, int* rb) {
  const int most = rows <= small_max(format) ? kSmallRows : 256;
  *nblk = (rows + most - 1) / most;
  *rb = (rows + *nblk - 1) / *nblk;
}

constexpr int kTreeMaxCtas = 1024;  // records are sized for at most this many CTAs

struct TreeLayout {
  size_t first, odd, ml, acc, total;
};
// The same for every format: what the format with the most records takes.
TreeLayout tree_layout(int units, int rows) {
  auto a = [](size_t x) { return (x + 255) / 256 * 256; };
  size_t recs = 0;
  for (int format : {CERTKV_STORE_BF16, CERTKV_STORE_FP8, CERTKV_STORE_FP4}) {
    int nblk, rb;
    row_blocks(rows, format, &nblk, &rb);
    recs = std::max(recs, ((size_t)units * nblk + kTreeMaxCtas) * rb);
  }
  TreeLayout ly;
  ly.first = 0;
  ly.odd = a(((size_t)units + 1) * sizeof(int64_t));
  ly.ml = ly.odd + a((size_t)units * sizeof(uint64_t));
  ly.acc = ly.ml + a(recs * sizeof(float2));
  ly.total = ly.acc + recs * kD * sizeof(float);
  return ly;
}

}  // namespace
}  // namespace certkv

extern "C" size_t certkv_tree_workspace_bytes(const certkv_shape* shape, int32_t tokens) {
  if (certkv::tree_shape(shape, tokens)) return 0;
  return certkv::tree_layout(shape->batch * shape->layers * shape->hkv,
                             tokens * (shape->hq / shape->hkv))
      .total;
}

extern "C" int certkv_tree_attn(const certkv_shape* shape, int32_t tokens, const certkv_rows* q,
                                const certkv_rows* k_new, const certkv_rows* v_new,
                                const uint64_t* mask, const certkv_store* store, float scale,
                                const certkv_rows* out, float* lse, void* workspace,
                                size_t workspace_bytes, void* stream) {
  using namespace certkv;
  int rc = tree_shape(shape, tokens);
  if (rc) return rc;
  const int B = shape->batch, L = shape->layers;
  TreeArgs p;
  if ((rc = store_of(store, &p.st))) return rc;
  if ((int64_t)B * L * shape->hkv != p.st.units) return CERTKV_EINVAL;
  if (!rows_ok(q, B, L, tokens, shape->hq) || !rows_out_ok(out, B, L, tokens, shape->hq))
    return CERTKV_EINVAL;
  if ((k_new == nullptr) != (v_new == nullptr)) return CERTKV_EINVAL;
  if (k_new && (!rows_ok(k_new, B, L, tokens, shape->hkv) || !rows_ok(v_new, B, L, tokens, shape->hkv)))
    return CERTKV_EINVAL;
  if ((uintptr_t)mask % 8 != 0 || (uintptr_t)lse % 4 != 0) return CERTKV_EINVAL;
  if (!(scale >= 0.0f) || !isfinite(scale)) return CERTKV_EINVAL;
  if (!workspace || (uintptr_t)workspace % 256 != 0 ||
      workspace_bytes < certkv_tree_workspace_bytes(shape, tokens))
    return CERTKV_EWORKSPACE;
  p.L = L;
  p.H = shape->hkv;
  p.G = shape->hq / shape->hkv;
  p.T = tokens;
  p.units = p.st.units;
  p.rows = tokens * p.G;
  p.q = rows_of(q);
  p.kn = rows_of(k_new);
  p.vn = rows_of(v_new);
  p.o = rows_of(out);
  p.mask = mask;
  p.lse = lse;
  p.scale_log2 = (float)((scale > 0.0f ? scale : 1.0 / sqrt((double)kD)) * 1.4426950408889634);
  row_blocks(p.rows, store->format, &p.nblk, &p.rb);
  const int64_t merge = ((int64_t)p.units * p.rows + 7) / 8;
  if (merge > INT32_MAX) return CERTKV_EINVAL;
  p.small = p.rows <= small_max(store->format);
  p.ctas = p.small ? tree_mma_ctas(store->format) : tree_ctas();
  p.least = p.small ? 4 : p.rb <= 128 ? 2 : 1;  // consumer warps, streams on tiles of their own
  if (p.ctas < 1) return CERTKV_ECUDA;
  if (p.ctas > kTreeMaxCtas) p.ctas = kTreeMaxCtas;
  // a CTA counts its tiles in 32 bits
  if ((int64_t)p.units * (p.st.max_pages + 2) / p.ctas * p.nblk >= (1 << 29)) return CERTKV_EINVAL;
  const TreeLayout ly = tree_layout(p.units, p.rows);
  char* ws = reinterpret_cast<char*>(workspace);
  int64_t* first = reinterpret_cast<int64_t*>(ws + ly.first);
  p.first = first;
  p.odd = reinterpret_cast<uint64_t*>(ws + ly.odd);
  p.rec_ml = reinterpret_cast<float2*>(ws + ly.ml);
  p.rec_acc = reinterpret_cast<float*>(ws + ly.acc);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  if (p.units > kInlineUnits) {
    TraceScope ts_("tree_plan", st);
    if (!launch_kernel(false, tree_plan_kernel, 1, 1024, 0, st, p.st,
                       p.small ? small_tile(store->format) : kTreeTile, !p.small && p.kn.p ? 1 : 0, first))
      return cuda_failed();
  }
  if (!(p.small ? launch_tree_mma(p, store->format, st) : launch_tree_tc(p, store->format, st)))
    return cuda_failed();
  {
    TraceScope ts_("tree_merge", st);
    launch_kernel(true, tree_merge_kernel, (unsigned)merge, 256, 0, st, p);
  }
  return cudaGetLastError() == cudaSuccess ? CERTKV_OK : CERTKV_ECUDA;
}
