// rope.cu — rotary positions of query and key rows.
//
// Pair i of a row at position pos turns by the angle pos theta_i.  The angle is
// formed in turns, pos (theta_i / 2 pi), with theta_i / 2 pi held as the
// unevaluated float sum hi + lo and pos split into two exactly representable
// parts, so the products' whole turns are dropped exactly (an fma gives each
// product's error) and the remainder is good to ~2^-23 turns at any position a
// cache reaches; sincospif then takes half-turns.  A float product pos theta_i
// would be off by 2^-24 of the whole angle: 0.008 rad at position 131072.
//
// The rows are read once and written once; the angles depend on the token only,
// so a warp takes one token, works out the cosines and sines of its lanes' four
// elements once and walks over the rows (layers and heads) of that token, eight
// in flight.  Bound by the rows' bytes: 32749 tokens x 40 heads, half of each head
// turned, 108 us (92 % of the copy bandwidth).
#include <math.h>

#include "../../include/certkv.h"
#include "common.cuh"
#include "internal.cuh"
#include "rows.cuh"

namespace certkv {
namespace {

constexpr int kRopeWarps = 8, kRopeBlocks = 4;
constexpr int kRopeBatch = 8;  // rows loaded before the first of them is stored

struct RopeArgs {
  Rows q, qo, k, ko;
  const int32_t* pos;
  int L, T, hq, hkv;  // hkv = 0: no keys
  int per, chunks;    // rows per warp, warps per token
  int64_t warps;      // B T chunks
  float mag, sgn;     // factor, direction of the turn
};

// Fractional turns of pos * (hi + lo), in [-0.5, 0.5].
__device__ __forceinline__ float turns_of(int pos, float hi, float lo) {
  const float pl = (float)(pos & 4095), ph = (float)(pos - (pos & 4095));  // both exact
  float a = __fmul_rn(ph, hi), b = __fmul_rn(pl, hi);
  const float ea = __fmaf_rn(ph, hi, -a), eb = __fmaf_rn(pl, hi, -b);
  a -= rintf(a);
  b -= rintf(b);
  const float r = (a + b) + (ea + eb + (ph + pl) * lo);
  return r - rintf(r);
}

// The rows of a token in order: layer after layer, its query heads, then its keys.
// A step is one addition; only where heads end is a row's address worked out (from
// its indices every time, the kernel was bound by its instructions: 127 -> 108 us).
template <class E>
struct Walk {
  E* at;
  int64_t step;
  int l, left;  // layer, heads to go until the other kind or the next layer
  bool keys;
  __device__ __forceinline__ void enter(const RopeArgs& p, int h, E* q, E* k, const Rows& rq, const Rows& rk) {
    at = keys ? k + l * rk.sl + h * rk.sh : q + l * rq.sl + h * rq.sh;
    step = keys ? rk.sh : rq.sh;
    left = (keys ? p.hkv : p.hq) - h;
  }
  __device__ __forceinline__ Walk(const RopeArgs& p, int r, E* q, E* k, const Rows& rq, const Rows& rk) {
    const int all = p.hq + p.hkv;
    l = r / all;
    const int h = r - l * all;
    keys = h >= p.hq;
    enter(p, keys ? h - p.hq : h, q, k, rq, rk);
  }
  __device__ __forceinline__ void next(const RopeArgs& p, E* q, E* k, const Rows& rq, const Rows& rk) {
    at += step;
    if (--left == 0) {
      keys = !keys && p.hkv > 0;
      l += !keys;
      enter(p, 0, q, k, rq, rk);
    }
  }
};

// grid x kRopeWarps warps; warp = (token, chunk of rows), lane = elements
// 4 lane .. 4 lane + 3.  MODE 0: interleaved pairs; 1: half layout with
// dim / 2 a multiple of 4 (a lane's partners are the four elements of one
// other lane); 2: half layout otherwise (partners read one by one).
template <int MODE>
__global__ void __launch_bounds__(kRopeWarps * 32, kRopeBlocks) rope_kernel(RopeArgs p,
                                                               const __grid_constant__ certkv_rope_angles ang) {
  const int64_t w = (int64_t)blockIdx.x * kRopeWarps + (threadIdx.x >> 5);
  if (w >= p.warps) return;
  const int lane = threadIdx.x & 31;
  const int64_t bt = w / p.chunks;
  const int b = (int)(bt / p.T), t = (int)(bt - (int64_t)b * p.T);
  const int pos = p.pos[bt];
  const int n = ang.dim >> 1, d0 = 4 * lane;

  // cosine and sine of each of the lane's elements (sine signed so that the
  // result is x cos + partner sin); elements past dim are copied
  float c[4], s[4];
  int turned = 0;  // elements of this lane that turn (0, 2 or 4; the first ones)
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    const int j = d0 + e;
    c[e] = 1.f;
    s[e] = 0.f;
    if (j < ang.dim) {
      turned = e + 1;
      if (MODE != 0 || (e & 1) == 0) {
        const int i = MODE == 0 ? j >> 1 : (j < n ? j : j - n);
        float sn, cs;
        sincospif(2.f * turns_of(pos, ang.turns_hi[i], ang.turns_lo[i]), &sn, &cs);
        c[e] = cs * p.mag;
        s[e] = sn * p.mag * p.sgn;
        if (MODE != 0) {
          if (j < n) s[e] = -s[e];
        }
      } else {
        c[e] = c[e - 1];
        s[e] = s[e - 1];
        s[e - 1] = -s[e];
      }
    }
  }
  int partner = lane;
  if (MODE == 1 && turned) partner = d0 < n ? lane + n / 4 : lane - n / 4;

  const int total = p.L * (p.hq + p.hkv);
  const int r0 = (int)(w - bt * p.chunks) * p.per, r1 = min(total, r0 + p.per);
  const uint16_t *qi = p.q.at(b, 0, t, 0) + d0, *ki = p.k.at(b, 0, t, 0) + d0;
  uint16_t *qo = p.qo.at(b, 0, t, 0) + d0, *ko = p.ko.at(b, 0, t, 0) + d0;
  Walk<const uint16_t> from(p, r0, qi, ki, p.q, p.k);
  Walk<uint16_t> to(p, r0, qo, ko, p.qo, p.ko);
  for (int r = r0; r < r1; r += kRopeBatch) {
    uint2 x[kRopeBatch];
    uint16_t y[MODE == 2 ? kRopeBatch : 1][4];
#pragma unroll
    for (int i = 0; i < kRopeBatch; ++i) {
      x[i] = make_uint2(0u, 0u);
      if (r + i < r1) {
        x[i] = *reinterpret_cast<const uint2*>(from.at);
        if (MODE == 2) {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int j = d0 + e;
            y[i][e] = j < ang.dim ? from.at[e + (j < n ? n : -n)] : (uint16_t)0;
          }
        }
        from.next(p, qi, ki, p.q, p.k);
      }
    }
    __syncwarp();  // in place: every lane has read the rows before any is written
#pragma unroll
    for (int i = 0; i < kRopeBatch; ++i) {
      float v[4] = {bf16lo(x[i].x), bf16hi(x[i].x), bf16lo(x[i].y), bf16hi(x[i].y)};
      float u[4];
      if (MODE == 0) {
        u[0] = v[1];
        u[1] = v[0];
        u[2] = v[3];
        u[3] = v[2];
      } else if (MODE == 1) {
        const uint32_t f = __shfl_sync(kFull, x[i].x, partner), g = __shfl_sync(kFull, x[i].y, partner);
        u[0] = bf16lo(f);
        u[1] = bf16hi(f);
        u[2] = bf16lo(g);
        u[3] = bf16hi(g);
      } else {
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] = __uint_as_float((uint32_t)y[i][e] << 16);
      }
      if (r + i < r1) {
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = fmaf(v[e], c[e], u[e] * s[e]);
        const __nv_bfloat162 lo = __floats2bfloat162_rn(v[0], v[1]), hi = __floats2bfloat162_rn(v[2], v[3]);
        // dim is even: the lane's elements turn in pairs
        *reinterpret_cast<uint2*>(to.at) =
            make_uint2(turned > 0 ? *reinterpret_cast<const uint32_t*>(&lo) : x[i].x,
                       turned > 2 ? *reinterpret_cast<const uint32_t*>(&hi) : x[i].y);
        to.next(p, qo, ko, p.qo, p.ko);
      }
    }
  }
}

}  // namespace
}  // namespace certkv

extern "C" int certkv_rope_plan(int32_t dim, int32_t layout, double base,
                                const certkv_rope_scaling* sc, certkv_rope_angles* out) {
  if (!out || dim < 2 || dim > certkv::kD || dim % 2 != 0) return CERTKV_EINVAL;
  if (layout != CERTKV_ROPE_HALF && layout != CERTKV_ROPE_INTERLEAVED) return CERTKV_EINVAL;
  if (!(base > 1.0) || !isfinite(base)) return CERTKV_EINVAL;
  certkv_rope_scaling none = {CERTKV_ROPE_NONE, 1.0, 1.0, 0.0, 1.0, 1.0};
  if (!sc) sc = &none;
  if (sc->kind < CERTKV_ROPE_NONE || sc->kind > CERTKV_ROPE_RAMP) return CERTKV_EINVAL;
  if (!(sc->magnitude > 0.0) || !isfinite(sc->magnitude)) return CERTKV_EINVAL;
  if (sc->kind != CERTKV_ROPE_NONE && (!(sc->factor > 0.0) || !isfinite(sc->factor)))
    return CERTKV_EINVAL;
  if (sc->kind == CERTKV_ROPE_NTK && dim < 4) return CERTKV_EINVAL;
  if (sc->kind == CERTKV_ROPE_RAMP &&
      (!(sc->original > 0.0) || !isfinite(sc->original) || !(sc->low < sc->high) ||
       !isfinite(sc->low) || !isfinite(sc->high)))
    return CERTKV_EINVAL;
  const double kTwoPi = 6.283185307179586476925;
  if (sc->kind == CERTKV_ROPE_NTK) base *= pow(sc->factor, (double)dim / (dim - 2));
  if (!isfinite(base)) return CERTKV_EINVAL;
  out->dim = dim;
  out->layout = layout;
  out->magnitude = (float)sc->magnitude;
  out->inverse_magnitude = (float)(1.0 / sc->magnitude);
  for (int i = 0; i < 64; ++i) {
    double turns = 0.0;
    if (i < dim / 2) {
      double th = pow(base, -2.0 * i / dim);
      if (sc->kind == CERTKV_ROPE_LINEAR) th /= sc->factor;
      if (sc->kind == CERTKV_ROPE_RAMP) {
        double g = (sc->original * th / kTwoPi - sc->low) / (sc->high - sc->low);
        g = g < 0.0 ? 0.0 : g > 1.0 ? 1.0 : g;
        th = (1.0 - g) * th / sc->factor + g * th;
      }
      turns = th / kTwoPi;
    }
    out->turns_hi[i] = (float)turns;
    out->turns_lo[i] = (float)(turns - (double)out->turns_hi[i]);
  }
  return CERTKV_OK;
}

extern "C" int certkv_rope(int32_t batch, int32_t layers, int32_t tokens, int32_t hq, int32_t hkv,
                           const certkv_rows* q, const certkv_rows* q_out, const certkv_rows* k,
                           const certkv_rows* k_out, const int32_t* positions,
                           const certkv_rope_angles* ang, int32_t inverse, void* stream) {
  using namespace certkv;
  if (batch < 1 || layers < 1 || tokens < 1 || hq < 1 || hkv < 0 || (k && hkv < 1))
    return CERTKV_EINVAL;
  if ((int64_t)batch * tokens > INT32_MAX || hq > 65536 || hkv > 65536 || layers > 65536 ||
      (int64_t)layers * ((int64_t)hq + hkv) > (1 << 24))
    return CERTKV_EINVAL;
  if (!rows_ok(q, batch, layers, tokens, hq) || !rows_out_ok(q_out, batch, layers, tokens, hq))
    return CERTKV_EINVAL;
  if ((k == nullptr) != (k_out == nullptr)) return CERTKV_EINVAL;
  if (k && (!rows_ok(k, batch, layers, tokens, hkv) || !rows_out_ok(k_out, batch, layers, tokens, hkv)))
    return CERTKV_EINVAL;
  if (!positions || (uintptr_t)positions % 4 != 0 || !ang || (inverse != 0 && inverse != 1))
    return CERTKV_EINVAL;
  if (ang->dim < 2 || ang->dim > kD || ang->dim % 2 != 0 ||
      (ang->layout != CERTKV_ROPE_HALF && ang->layout != CERTKV_ROPE_INTERLEAVED))
    return CERTKV_EINVAL;
  RopeArgs p;
  p.q = rows_of(q);
  p.qo = rows_of(q_out);
  p.k = rows_of(k);
  p.ko = rows_of(k_out);
  p.pos = positions;
  p.L = layers;
  p.T = tokens;
  p.hq = hq;
  p.hkv = k ? hkv : 0;
  // Rows per warp: working out a token's angles costs a warp about as much as
  // six rows, so a warp takes many rows where that still leaves every SM its
  // warps, and as few as half a batch of loads where there are few tokens.
  const int total = layers * (p.hq + p.hkv);
  const int64_t bt = (int64_t)batch * tokens;
  int per = 64;
  while (per > kRopeBatch / 2 && bt * ((total + per - 1) / per) < 152 * 48) per >>= 1;
  p.per = per;
  p.chunks = (total + per - 1) / per;
  p.warps = bt * p.chunks;
  if (p.warps / kRopeWarps >= INT32_MAX) return CERTKV_EINVAL;
  p.mag = inverse ? ang->inverse_magnitude : ang->magnitude;
  p.sgn = inverse ? -1.f : 1.f;
  const unsigned grid = (unsigned)((p.warps + kRopeWarps - 1) / kRopeWarps);
  cudaStream_t st = reinterpret_cast<cudaStream_t>(stream);
  TraceScope ts_("rope", st);
  if (ang->layout == CERTKV_ROPE_INTERLEAVED)
    rope_kernel<0><<<grid, kRopeWarps * 32, 0, st>>>(p, *ang);
  else if ((ang->dim / 2) % 4 == 0)
    rope_kernel<1><<<grid, kRopeWarps * 32, 0, st>>>(p, *ang);
  else
    rope_kernel<2><<<grid, kRopeWarps * 32, 0, st>>>(p, *ang);
  return cudaGetLastError() == cudaSuccess ? CERTKV_OK : CERTKV_ECUDA;
}
