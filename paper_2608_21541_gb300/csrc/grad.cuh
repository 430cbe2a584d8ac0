// grad.cuh — what the launches of one certkv_tree_attn_grad call share.
#pragma once

#include <cuda.h>
#include <stdint.h>

#include "rows.cuh"
#include "store.cuh"

namespace certkv {

struct GradArgs {
  int L, H, G, T;    // layers, KV heads, query heads per KV head, drafted tokens
  int units, rows;   // B L H, T G query rows per unit
  Rows q, kn, vn, o, go, dq, dkn, dvn;  // kn.p null: the drafts have no keys of their own
  const uint64_t* mask;
  const float *lse, *dlse;
  float scale, scale_log2;
  Store st;
  uint16_t *dks, *dvs;  // the store's gradients (null: not asked for)
  // workspace
  float2* row;  // [units][rows] log-sum-exp (log2 domain; +inf: the row takes no part), delta
};

struct GradUnit {
  int b, l, h;
  __device__ __forceinline__ GradUnit(const GradArgs& p, int u) {
    const int bl = u / p.H;
    h = u - bl * p.H;
    b = bl / p.L;
    l = bl - b * p.L;
  }
};

// Drafts that token t of sequence b sees, as bits.
__device__ __forceinline__ uint64_t grad_seen(const GradArgs& p, int b, int t) {
  const uint64_t all = ~0ull >> (64 - p.T);
  return (p.mask ? p.mask[(int64_t)b * p.T + t] : ~0ull >> (63 - t)) & all;
}

}  // namespace certkv
