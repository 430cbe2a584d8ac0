// rows.cuh — strided bf16 row views (certkv_rows): host-side checks and device
// addressing shared by the rotary, store and tree-attention entry points.
#pragma once

#include <stdint.h>

#include "../../include/certkv.h"
#include "common.cuh"

namespace certkv {

// Pointer and strides of a [b][l][t][h] view (certkv_rows by value).
struct Rows {
  uint16_t* p;
  int64_t sb, sl, st, sh;
  __host__ __device__ uint16_t* at(int64_t b, int64_t l, int64_t t, int64_t h) const {
    return p + b * sb + l * sl + t * st + h * sh;
  }
};

inline Rows rows_of(const certkv_rows* r) {
  return r ? Rows{reinterpret_cast<uint16_t*>(r->data), r->stride_b, r->stride_l, r->stride_t,
                  r->stride_h}
           : Rows{nullptr, 0, 0, 0, 0};
}

// Present, 16-byte aligned, strides multiples of 8 elements (rows of 256 B are
// read and written with 16-byte accesses).  A stride of an extent of 1 is not
// used, whatever it is.
inline bool rows_ok(const certkv_rows* r, int64_t b, int64_t l, int64_t t, int64_t h) {
  if (!r || !r->data || (uintptr_t)r->data % 16 != 0) return false;
  const int64_t ext[4] = {b, l, t, h};
  const int64_t str[4] = {r->stride_b, r->stride_l, r->stride_t, r->stride_h};
  for (int i = 0; i < 4; ++i)
    if (ext[i] > 1 && (str[i] % 8 != 0 || str[i] > (INT64_MAX >> 26) || str[i] < -(INT64_MAX >> 26)))
      return false;
  return true;
}

// rows_ok, and no two rows overlap: with the extents taken in the order of
// their strides, each stride clears the span of the ones below it.
inline bool rows_out_ok(const certkv_rows* r, int64_t b, int64_t l, int64_t t, int64_t h) {
  if (!rows_ok(r, b, l, t, h)) return false;
  int64_t ext[4] = {b, l, t, h}, str[4] = {r->stride_b, r->stride_l, r->stride_t, r->stride_h};
  for (int i = 0; i < 4; ++i) str[i] = str[i] < 0 ? -str[i] : str[i];
  bool used[4] = {false, false, false, false};
  double span = kD;  // elements; a double holds any product of the checked sizes closely enough
  for (int k = 0; k < 4; ++k) {
    int m = -1;
    for (int i = 0; i < 4; ++i)
      if (!used[i] && ext[i] > 1 && (m < 0 || str[i] < str[m])) m = i;
    if (m < 0) break;
    used[m] = true;
    if ((double)str[m] < span) return false;
    span += (double)(ext[m] - 1) * (double)str[m];
  }
  return true;
}

}  // namespace certkv
