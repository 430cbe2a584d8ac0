// grad.cu — gradients of tree attention over the paged store.
//
// For query row r and what it sees, slot or draft s:
//   p = exp(scale <q_r, k_s> - lse_r),  e = scale p (<dout_r, v_s> - delta_r),
//   delta_r = <dout_r, out_r> - dlse_r,
//   dq_r = sum_s e k_s,  dk_s = sum_r e q_r,  dv_s = sum_r p dout_r.
// The simple form: one warp for each row that is summed into.
#include <math.h>

#include "../../include/certkv.h"
#include "common.cuh"
#include "grad.cuh"
#include "internal.cuh"

namespace certkv {
namespace {

constexpr int kThreads = 256;

__device__ __forceinline__ float warp_sum(float x) {
#pragma unroll
  for (int o = 16; o >= 1; o >>= 1) x += __shfl_xor_sync(kFull, x, o);
  return x;
}
__device__ __forceinline__ float4 load4(const uint16_t* row, int lane) {
  const uint2 x = *reinterpret_cast<const uint2*>(row + 4 * lane);
  return make_float4(bf16lo(x.x), bf16hi(x.x), bf16lo(x.y), bf16hi(x.y));
}
__device__ __forceinline__ void store4(uint16_t* row, int lane, float4 a) {
  const __nv_bfloat162 lo = __floats2bfloat162_rn(a.x, a.y), hi = __floats2bfloat162_rn(a.z, a.w);
  *reinterpret_cast<uint2*>(row + 4 * lane) =
      make_uint2(*reinterpret_cast<const uint32_t*>(&lo), *reinterpret_cast<const uint32_t*>(&hi));
}
__device__ __forceinline__ float dot(float4 a, float4 b) {
  return warp_sum(a.x * b.x + a.y * b.y + a.z * b.z + a.w * b.w);
}
__device__ __forceinline__ void axpy(float f, float4 x, float4& a) {
  a.x = fmaf(f, x.x, a.x);
  a.y = fmaf(f, x.y, a.y);
  a.z = fmaf(f, x.z, a.z);
  a.w = fmaf(f, x.w, a.w);
}

// Elements 4 lane .. of pool slot `at`.
template <int FMT>
__device__ __forceinline__ float4 stored4(const uint8_t* codes, const uint8_t* group, const float* scale,
                                          int64_t at, int lane) {
  if (FMT == CERTKV_STORE_BF16) return load4(reinterpret_cast<const uint16_t*>(codes) + at * kD, lane);
  const float s = scale[at];
  uint32_t a, b;
  if (FMT == CERTKV_STORE_FP8) {
    const uint32_t w = *reinterpret_cast<const uint32_t*>(codes + at * 128 + 4 * lane);
    a = e4m3x2_to_f16x2(w);
    b = e4m3x2_to_f16x2(w >> 16);
  } else {
    const uint32_t w = *reinterpret_cast<const uint16_t*>(codes + at * 64 + 2 * lane);
    const uint32_t g = group[at * kGroups + lane / 4];
    const uint32_t g2 = e4m3x2_to_f16x2(g | g << 8);
    a = hmul2(e2m1x2_to_f16x2<0>(w), g2);
    b = hmul2(e2m1x2_to_f16x2<1>(w), g2);
  }
  const float2 x = f16x2_to_f32(a), y = f16x2_to_f32(b);
  return make_float4(x.x * s, x.y * s, y.x * s, y.y * s);
}

// One warp per row: its log-sum-exp and delta.
__global__ void __launch_bounds__(kThreads) grad_rows_kernel(const __grid_constant__ GradArgs p) {
  const int64_t w = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> 5;
  const int lane = threadIdx.x & 31;
  release_next();
  if (w >= (int64_t)p.units * p.rows) return;
  const int u = (int)(w / p.rows), r = (int)(w - (int64_t)u * p.rows), t = r / p.G, g = r - t * p.G;
  const GradUnit x(p, u);
  const int qh = x.h * p.G + g;
  const int64_t at = (((int64_t)x.b * p.L + x.l) * p.T + t) * p.H * p.G + qh;
  const float lse = p.lse[at];
  float delta = 0.f;
  if (lse != -INFINITY) {
    delta = dot(load4(p.go.at(x.b, x.l, t, qh), lane), load4(p.o.at(x.b, x.l, t, qh), lane));
    if (p.dlse) delta -= p.dlse[at];
  }
  if (lane == 0) p.row[w] = make_float2(lse == -INFINITY ? INFINITY : lse * 1.4426950408889634f, delta);
}

template <int FMT>
__global__ void __launch_bounds__(kThreads) grad_q_kernel(const __grid_constant__ GradArgs p) {
  const int64_t w = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> 5;
  const int lane = threadIdx.x & 31;
  await_previous();
  if (w >= (int64_t)p.units * p.rows) return;
  const int u = (int)(w / p.rows), r = (int)(w - (int64_t)u * p.rows), t = r / p.G, g = r - t * p.G;
  const GradUnit x(p, u);
  const int qh = x.h * p.G + g;
  const float2 row = p.row[w];
  float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
  if (row.x != INFINITY) {
    const float4 q = load4(p.q.at(x.b, x.l, t, qh), lane), go = load4(p.go.at(x.b, x.l, t, qh), lane);
    auto add = [&](float4 k, float4 v) {
      const float pr = exp2f(fmaf(dot(q, k), p.scale_log2, -row.x));
      axpy(pr * (dot(go, v) - row.y) * p.scale, k, a);
    };
    const int n = p.st.count(u);
    for (int s = 0; s < n; ++s) {
      const int64_t at = p.st.slot(u, s);
      if (at < 0) {
        if (lane == 0) p.st.raise();
        continue;
      }
      add(stored4<FMT>(p.st.k, p.st.kg, p.st.ks, at, lane), stored4<FMT>(p.st.v, p.st.vg, p.st.vs, at, lane));
    }
    if (p.kn.p)
      for (uint64_t see = grad_seen(p, x.b, t); see; see &= see - 1) {
        const int j = __ffsll((long long)see) - 1;
        add(load4(p.kn.at(x.b, x.l, j, x.h), lane), load4(p.vn.at(x.b, x.l, j, x.h), lane));
      }
  }
  store4(p.dq.at(x.b, x.l, t, qh), lane, a);
}

// What row s of keys and values gets from the rows that see it.
__device__ __forceinline__ void grad_kv(const GradArgs& p, int u, const GradUnit& x, int draft, float4 k, float4 v,
                                        int lane, float4* dk, float4* dv) {
  *dk = *dv = make_float4(0.f, 0.f, 0.f, 0.f);
  for (int r = 0; r < p.rows; ++r) {
    const int t = r / p.G, qh = x.h * p.G + r - t * p.G;
    const float2 row = p.row[(int64_t)u * p.rows + r];
    if (row.x == INFINITY || (draft >= 0 && !(grad_seen(p, x.b, t) >> draft & 1u))) continue;
    const float4 q = load4(p.q.at(x.b, x.l, t, qh), lane), go = load4(p.go.at(x.b, x.l, t, qh), lane);
    const float pr = exp2f(fmaf(dot(q, k), p.scale_log2, -row.x));
    axpy(pr, go, *dv);
    axpy(pr * (dot(go, v) - row.y) * p.scale, q, *dk);
  }
}

template <int FMT>
__global__ void __launch_bounds__(kThreads) grad_store_kernel(const __grid_constant__ GradArgs p) {
  const int u = blockIdx.x, lane = threadIdx.x & 31;
  await_previous();
  const GradUnit x(p, u);
  const int n = p.st.count(u);
  for (int s = threadIdx.x >> 5; s < n; s += kThreads / 32) {
    const int64_t at = p.st.slot(u, s);
    if (at < 0) continue;
    float4 dk, dv;
    grad_kv(p, u, x, -1, stored4<FMT>(p.st.k, p.st.kg, p.st.ks, at, lane),
            stored4<FMT>(p.st.v, p.st.vg, p.st.vs, at, lane), lane, &dk, &dv);
    store4(p.dks + at * kD, lane, dk);
    store4(p.dvs + at * kD, lane, dv);
  }
}

__global__ void __launch_bounds__(kThreads) grad_drafts_kernel(const __grid_constant__ GradArgs p) {
  const int64_t w = ((int64_t)blockIdx.x * kThreads + threadIdx.x) >> 5;
  const int lane = threadIdx.x & 31;
  await_previous();
  if (w >= (int64_t)p.units * p.T) return;
  const int u = (int)(w / p.T), j = (int)(w - (int64_t)u * p.T);
  const GradUnit x(p, u);
  float4 dk, dv;
  grad_kv(p, u, x, j, load4(p.kn.at(x.b, x.l, j, x.h), lane), load4(p.vn.at(x.b, x.l, j, x.h), lane), lane, &dk, &dv);
  store4(p.dkn.at(x.b, x.l, j, x.h), lane, dk);
  store4(p.dvn.at(x.b, x.l, j, x.h), lane, dv);
}

int grad_shape(const certkv_shape* s, int32_t tokens) {
  if (!s || s->batch < 1 || s->layers < 1 || s->hq < 1 || s->hkv < 1) return CERTKV_EINVAL;
  if (s->d != kD || s->hq % s->hkv != 0 || s->hq / s->hkv > CERTKV_TREE_MAX_GROUP) return CERTKV_EINVAL;
  if (tokens < 1 || tokens > CERTKV_TREE_MAX_TOKENS) return CERTKV_EINVAL;
  if ((int64_t)s->batch * s->layers > (1 << 24) || (int64_t)s->batch * s->layers * s->hkv > (1 << 24))
    return CERTKV_EINVAL;
  return CERTKV_OK;
}

unsigned warps(int64_t n) { return (unsigned)((n * 32 + kThreads - 1) / kThreads); }

template <int FMT>
bool launch_store_grads(const GradArgs& p, cudaStream_t st) {
  if (p.dq.p) {
    TraceScope ts_("grad_q", st);
    if (!launch_kernel(true, grad_q_kernel<FMT>, warps((int64_t)p.units * p.rows), kThreads, 0, st, p)) return false;
  }
  if (p.dks) {
    TraceScope ts_("grad_store", st);
    if (!launch_kernel(true, grad_store_kernel<FMT>, p.units, kThreads, 0, st, p)) return false;
  }
  return true;
}

}  // namespace
}  // namespace certkv

extern "C" size_t certkv_tree_grad_workspace_bytes(const certkv_shape* shape, int32_t tokens) {
  if (certkv::grad_shape(shape, tokens)) return 0;
  return (size_t)shape->batch * shape->layers * shape->hq * tokens * sizeof(float2);
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
  p.scale_log2 = (float)((scale > 0.0f ? scale : 1.0 / sqrt((double)kD)) * 1.4426950408889634);
  p.dks = reinterpret_cast<uint16_t*>(dk_store);
  p.dvs = reinterpret_cast<uint16_t*>(dv_store);
  p.row = reinterpret_cast<float2*>(workspace);
  if ((int64_t)p.units * p.rows * 32 / kThreads >= INT32_MAX) return CERTKV_EINVAL;
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  {
    TraceScope ts_("grad_rows", st);
    if (!launch_kernel(false, grad_rows_kernel, warps((int64_t)p.units * p.rows), kThreads, 0, st, p))
      return cuda_failed();
  }
  if (!(store->format == CERTKV_STORE_BF16  ? launch_store_grads<CERTKV_STORE_BF16>(p, st)
        : store->format == CERTKV_STORE_FP8 ? launch_store_grads<CERTKV_STORE_FP8>(p, st)
                                            : launch_store_grads<CERTKV_STORE_FP4>(p, st)))
    return cuda_failed();
  if (p.dkn.p) {
    TraceScope ts_("grad_drafts", st);
    launch_kernel(true, grad_drafts_kernel, warps((int64_t)p.units * p.T), kThreads, 0, st, p);
  }
  return cudaGetLastError() == cudaSuccess ? CERTKV_OK : CERTKV_ECUDA;
}
