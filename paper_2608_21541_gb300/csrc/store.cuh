// store.cuh — the paged store (certkv_store) as the kernels see it.
#pragma once

#include <stdint.h>

#include "../../include/certkv.h"
#include "common.cuh"

namespace certkv {

constexpr int kPage = CERTKV_STORE_PAGE;
constexpr int kGroups = kD / 16;  // FP4 scale groups of a row

struct Store {
  int units, max_pages, pool_pages;
  uint8_t *k, *v, *kg, *vg;
  float *ks, *vs;
  int32_t *table, *counts;
  uint32_t* status;

  __device__ __forceinline__ void raise() const {
    if (status) atomicOr(status, CERTKV_STATUS_STORE);
  }
  // live slots of segment u, clamped to what its table row can address
  __device__ __forceinline__ int count(int64_t u) const {
    return min(max(counts[u], 0), max_pages * kPage);
  }
  // pool slot of slot s (0 <= s < 64 max_pages) of segment u; -1: no page
  __device__ __forceinline__ int64_t slot(int64_t u, int s) const {
    const int page = table[u * max_pages + s / kPage];
    return page >= 0 && page < pool_pages ? (int64_t)page * kPage + s % kPage : -1;
  }
};

// Whether n >= 0 slots from `first` on lie in `capacity` >= 0 slots, for any `first`.
__host__ __device__ constexpr bool lies_in(int64_t first, int64_t n, int64_t capacity) {
  return first >= 0 && n <= capacity && first <= capacity - n;
}

// bytes of a row's codes
__host__ __device__ constexpr int row_bytes(int format) {
  return format == CERTKV_STORE_BF16 ? 2 * kD : format == CERTKV_STORE_FP8 ? kD : kD / 2;
}

// Host checks of the store's fields; fills `out`.
inline int store_of(const certkv_store* s, Store* out) {
  if (!s) return CERTKV_EINVAL;
  if (s->units < 1 || s->units > (1 << 24) || s->max_pages < 1 || s->max_pages > (1 << 18) ||
      s->pool_pages < 1 || s->pool_pages >= (1 << 25))
    return CERTKV_EINVAL;
  if (s->format < CERTKV_STORE_BF16 || s->format > CERTKV_STORE_FP4) return CERTKV_EINVAL;
  if (!s->k || !s->v || !s->table || !s->counts) return CERTKV_EINVAL;
  if (((uintptr_t)s->k | (uintptr_t)s->v) % 128 != 0) return CERTKV_EINVAL;
  if (((uintptr_t)s->table | (uintptr_t)s->counts | (uintptr_t)s->status) % 4 != 0)
    return CERTKV_EINVAL;
  if (s->format != CERTKV_STORE_BF16 &&
      (!s->k_scale || !s->v_scale || ((uintptr_t)s->k_scale | (uintptr_t)s->v_scale) % 16 != 0))
    return CERTKV_EINVAL;
  if (s->format == CERTKV_STORE_FP4 &&
      (!s->k_group || !s->v_group || ((uintptr_t)s->k_group | (uintptr_t)s->v_group) % 16 != 0))
    return CERTKV_EINVAL;
  out->units = s->units;
  out->max_pages = s->max_pages;
  out->pool_pages = s->pool_pages;
  out->k = reinterpret_cast<uint8_t*>(s->k);
  out->v = reinterpret_cast<uint8_t*>(s->v);
  out->kg = reinterpret_cast<uint8_t*>(s->k_group);
  out->vg = reinterpret_cast<uint8_t*>(s->v_group);
  out->ks = s->k_scale;
  out->vs = s->v_scale;
  out->table = s->table;
  out->counts = s->counts;
  out->status = s->status;
  return CERTKV_OK;
}

// ------------------------------------------------------ 8- and 4-bit codes --
// Conversions by the hardware's own instructions: round to nearest, ties to
// even, saturating.
__device__ __forceinline__ uint32_t e4m3x2(float lo, float hi) {  // low byte = lo
  uint16_t r;
  asm("cvt.rn.satfinite.e4m3x2.f32 %0, %1, %2;" : "=h"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t e4m3x2_to_f16x2(uint32_t two) {
  uint32_t r;
  asm("cvt.rn.f16x2.e4m3x2 %0, %1;" : "=r"(r) : "h"((uint16_t)two));
  return r;
}
// eight codes, the first the lowest nibble
__device__ __forceinline__ uint32_t e2m1x8(float2 a, float2 b, float2 c, float2 d) {
  uint32_t r;
  asm("{\n .reg .b8 s, t, u, v;\n"
      " cvt.rn.satfinite.e2m1x2.f32 s, %2, %1;\n cvt.rn.satfinite.e2m1x2.f32 t, %4, %3;\n"
      " cvt.rn.satfinite.e2m1x2.f32 u, %6, %5;\n cvt.rn.satfinite.e2m1x2.f32 v, %8, %7;\n"
      " mov.b32 %0, {s, t, u, v};\n}"
      : "=r"(r)
      : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y), "f"(d.x), "f"(d.y));
  return r;
}
// four of the eight codes of a word: byte `which` (two codes) as f16x2
template <int which>
__device__ __forceinline__ uint32_t e2m1x2_to_f16x2(uint32_t word) {
  uint32_t r;
  if (which == 0)
    asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %1;\n cvt.rn.f16x2.e2m1x2 %0, a;\n}" : "=r"(r) : "r"(word));
  else if (which == 1)
    asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %1;\n cvt.rn.f16x2.e2m1x2 %0, b;\n}" : "=r"(r) : "r"(word));
  else if (which == 2)
    asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %1;\n cvt.rn.f16x2.e2m1x2 %0, c;\n}" : "=r"(r) : "r"(word));
  else
    asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %1;\n cvt.rn.f16x2.e2m1x2 %0, d;\n}" : "=r"(r) : "r"(word));
  return r;
}
__device__ __forceinline__ uint32_t hmul2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ float2 f16x2_to_f32(uint32_t h) {
  float2 f;
  asm("{\n .reg .b16 l, h;\n mov.b32 {l, h}, %2;\n cvt.f32.f16 %0, l;\n cvt.f32.f16 %1, h;\n}"
      : "=f"(f.x), "=f"(f.y)
      : "r"(h));
  return f;
}

}  // namespace certkv
