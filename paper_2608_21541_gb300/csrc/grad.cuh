// grad.cuh — what the launches of one certkv_tree_attn_grad call share.
#pragma once

#include <cuda.h>
#include <stdint.h>

#include "rows.cuh"
#include "store.cuh"

namespace certkv {

constexpr int kGradTile = 128;    // slots of a tile: two pages
constexpr int kGradRows = 128;    // query rows of a block of the query kernel, at most
constexpr int kGradFused = 64;    // up to this many rows a segment's gradients come from one pass

struct GradArgs {
  int L, H, G, T;    // layers, KV heads, query heads per KV head, drafted tokens
  int units, rows;   // B L H, T G query rows per unit
  int padded;        // rows up to a multiple of 16
  int nblk, rb;      // row blocks of a unit, rows of a block: a multiple of 8 (the last may have fewer)
  int groups;        // shares of the tiles; their CTAs leave records
  int chunks;        // of the drafts' kernel: 128 rows each
  int folded;        // a unit's records have been added up into its first
  Rows q, kn, vn, o, go, dq, dkn, dvn;  // kn.p null: the drafts have no keys of their own
  const uint64_t* mask;
  const float *lse, *dlse;
  float scale, scale_log2;
  Store st;
  uint16_t *dks, *dvs;  // the store's gradients (null: not asked for)
  // workspace
  float2* row;     // [units][rows] log-sum-exp (log2 domain), delta; see grad_rows_kernel
  uint8_t* pack;   // [units][4][padded][128 bytes] both halves of q, then of dout; see grad_pack
  float* neg;      // [units][2][padded] -log-sum-exp, -delta
  int64_t* first;  // [units + 1] tiles of the segments before
  float* rec;      // [groups + units][nblk] records of rb rows: dq / scale over a share's tiles
  float* part;     // [units][chunks][2][T][128] the drafts' dk / scale and dv over 128 rows
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

// Row r of part `part` of unit u's queries and gradients (part 0 and 1: elements 0 .. 63 and 64 ..
// of q, 2 and 3: of dout) as the matrix units take them, 16-byte chunk c at c ^ (r & 7): any
// rows from a multiple of 8 on are one bulk copy.  Rows that take no part, or that hold a NaN or
// infinity, are zeros, so that what is summed over rows and slots stays clean.
__device__ __forceinline__ uint8_t* grad_pack(const GradArgs& p, int u, int part, int r) {
  return p.pack + (((int64_t)u * 4 + part) * p.padded + r) * 128;
}

// Tiles of a share: equal consecutive parts of all tiles.
__device__ __forceinline__ int64_t tiles_per_share(const GradArgs& p) {
  return max((p.first[p.units] + p.groups - 1) / p.groups, (int64_t)1);
}
// Record of the share's part of unit u, row block blk: [16][rb][8], so that a warp whose lanes are
// rows writes whole lines (as [rb][128] it took the queries' kernel 3 us a segment).
__device__ __forceinline__ float* grad_record(const GradArgs& p, int share, int u, int blk) {
  return p.rec + (((int64_t)share + u) * p.nblk + blk) * p.rb * kD;
}
// Element d of row r of a record.
__device__ __forceinline__ int grad_at(const GradArgs& p, int r, int d) { return ((d >> 3) * p.rb + r) * 8 + (d & 7); }

bool launch_grad_q(const GradArgs& p, int format, cudaStream_t st);
bool launch_grad_kv(const GradArgs& p, int format, cudaStream_t st);
int grad_ctas();  // SMs of the current device, with the kernels set up for it (0 on an error)

}  // namespace certkv
