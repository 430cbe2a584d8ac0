// tree.cu — attention of a tree of drafted tokens over the paged store.
//
// For query row r = (token t, head g of the group) of unit u:
//   out_r = sum_s p_s v_s / sum_s p_s,  p_s = exp(scale <q_r, k_s> - m_r),
// over all counts[u] stored slots and the drafts j whose bit is set in token
// t's mask word.  A draft that a row does not see is never read for it, so a
// NaN there cannot reach it.
#include <math.h>

#include "../../include/certkv.h"
#include "common.cuh"
#include "internal.cuh"
#include "rows.cuh"
#include "store.cuh"

namespace certkv {

struct TreeArgs {
  int L, H, G, T;     // layers, KV heads, query heads per KV head, drafted tokens
  int units, rows;    // B L H, T G query rows per unit
  Rows q, kn, vn, o;  // kn.p null: the drafts have no keys of their own
  const uint64_t* mask;
  float* lse;
  float scale_log2;
  Store st;
};

constexpr float kLn2 = 0.69314718055994531f;

// Elements 4 lane .. 4 lane + 3 of pool slot `at` in fp32.
template <int FMT>
__device__ __forceinline__ float4 held4(int lane, int64_t at, const uint8_t* codes,
                                        const uint8_t* group, const float* scale) {
  if (FMT == CERTKV_STORE_BF16) {
    const uint2 x = *reinterpret_cast<const uint2*>(codes + at * 256 + lane * 8);
    return make_float4(bf16lo(x.x), bf16hi(x.x), bf16lo(x.y), bf16hi(x.y));
  }
  const float s = scale[at];
  float2 a, b;
  float f = s;
  if (FMT == CERTKV_STORE_FP8) {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(codes + at * 128 + lane * 4);
    a = f16x2_to_f32(e4m3x2_to_f16x2(w & 0xffffu));
    b = f16x2_to_f32(e4m3x2_to_f16x2(w >> 16));
  } else {
    const uint32_t w = *reinterpret_cast<const uint16_t*>(codes + at * 64 + lane * 2);
    a = f16x2_to_f32(e2m1x2_to_f16x2<0>(w));
    b = f16x2_to_f32(e2m1x2_to_f16x2<1>(w));
    f = s * f16x2_to_f32(e4m3x2_to_f16x2(group[at * kGroups + lane / 4])).x;
  }
  return make_float4(a.x * f, a.y * f, b.x * f, b.y * f);
}

__device__ __forceinline__ float4 row4(const uint16_t* row, int lane) {
  const uint2 x = *reinterpret_cast<const uint2*>(row + 4 * lane);
  return make_float4(bf16lo(x.x), bf16hi(x.x), bf16lo(x.y), bf16hi(x.y));
}

struct RowState {
  float m, l;
  float4 a;
  __device__ __forceinline__ void take(float x, float4 v) {  // log2-domain logit x
    const float nm = fmaxf(m, x);
    const float c = m == nm ? 1.f : exp2f(m - nm);
    const float p = x == -INFINITY ? 0.f : exp2f(x - nm);  // a NaN logit stays one
    m = nm;
    l = l * c + p;
    a.x = fmaf(p, v.x, a.x * c);
    a.y = fmaf(p, v.y, a.y * c);
    a.z = fmaf(p, v.z, a.z * c);
    a.w = fmaf(p, v.w, a.w * c);
  }
};

__device__ __forceinline__ float dot4(float4 a, float4 b) {
  float x = a.x * b.x + a.y * b.y + a.z * b.z + a.w * b.w;
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) x += __shfl_xor_sync(kFull, x, o);
  return x;
}

// One warp per (unit, row); a lane holds four dimensions.
template <int FMT>
__global__ void __launch_bounds__(128) tree_row_kernel(TreeArgs p) {
  const int64_t w = (int64_t)blockIdx.x * 4 + (threadIdx.x >> 5);
  if (w >= (int64_t)p.units * p.rows) return;
  const int lane = threadIdx.x & 31;
  const int64_t u = w / p.rows;
  const int r = (int)(w - u * p.rows), t = r / p.G, g = r - t * p.G;
  const int bl = (int)(u / p.H), h = (int)(u - (int64_t)bl * p.H);
  const int b = bl / p.L, l = bl - b * p.L;
  const float4 q = row4(p.q.at(b, l, t, h * p.G + g), lane);
  RowState s = {-INFINITY, 0.f, make_float4(0.f, 0.f, 0.f, 0.f)};
  const int n = p.st.count(u);
  for (int i = 0; i < n; ++i) {
    const int64_t at = p.st.slot(u, i);
    if (at < 0) {
      if (lane == 0) p.st.raise();
      continue;
    }
    const float x = dot4(q, held4<FMT>(lane, at, p.st.k, p.st.kg, p.st.ks)) * p.scale_log2;
    s.take(x, held4<FMT>(lane, at, p.st.v, p.st.vg, p.st.vs));
  }
  if (p.kn.p) {
    const uint64_t word = p.mask ? p.mask[(int64_t)b * p.T + t] : ~0ull >> (63 - t);
    for (int j = 0; j < p.T; ++j)
      if (word >> j & 1)
        s.take(dot4(q, row4(p.kn.at(b, l, j, h), lane)) * p.scale_log2,
               row4(p.vn.at(b, l, j, h), lane));
  }
  const float inv = s.l != 0.f ? 1.f / s.l : 0.f;  // a NaN sum stays a NaN
  const __nv_bfloat162 lo = __floats2bfloat162_rn(s.a.x * inv, s.a.y * inv);
  const __nv_bfloat162 hi = __floats2bfloat162_rn(s.a.z * inv, s.a.w * inv);
  *reinterpret_cast<uint2*>(p.o.at(b, l, t, h * p.G + g) + 4 * lane) =
      make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
  if (p.lse && lane == 0)
    p.lse[((int64_t)bl * p.T + t) * p.H * p.G + h * p.G + g] =
        s.l != 0.f ? (s.m + log2f(s.l)) * kLn2 : -INFINITY;
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

}  // namespace
}  // namespace certkv

extern "C" size_t certkv_tree_workspace_bytes(const certkv_shape* shape, int32_t tokens) {
  if (certkv::tree_shape(shape, tokens)) return 0;
  return 256;
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
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  const int64_t blocks = ((int64_t)p.units * p.rows + 3) / 4;
  if (blocks > INT32_MAX) return CERTKV_EINVAL;
  TraceScope ts_("tree_row", st);
  if (store->format == CERTKV_STORE_BF16)
    tree_row_kernel<CERTKV_STORE_BF16><<<(unsigned)blocks, 128, 0, st>>>(p);
  else if (store->format == CERTKV_STORE_FP8)
    tree_row_kernel<CERTKV_STORE_FP8><<<(unsigned)blocks, 128, 0, st>>>(p);
  else
    tree_row_kernel<CERTKV_STORE_FP4><<<(unsigned)blocks, 128, 0, st>>>(p);
  return cudaGetLastError() == cudaSuccess ? CERTKV_OK : CERTKV_ECUDA;
}
