// tree.cuh — what the launches of one tree-attention call share.
#pragma once

#include <cuda.h>
#include <stdint.h>

#include "rows.cuh"
#include "store.cuh"

namespace certkv {

constexpr int kTreeTile = 128;  // slots per tile of the tcgen05 kernel: two pages
constexpr int kSmallRows = 16;  // query rows of a block of the mma.sync kernel
// Up to this many query rows go to that kernel.  The tcgen05 kernel costs the same for 1 to
// 128 rows, the mma.sync kernel in proportion to its blocks of 16: one is always cheaper,
// two are where codes have to be expanded, but not where they only read a bf16 store twice.
// 32 rows, 256 segments of 13107 slots, mma.sync against tcgen05: 8-bit 309 and 312 us, 4-bit
// 322 and 331, bf16 512 and 272; 8 segments of 409 slots: 19.9 and 23.7, 21.8 and 23.7, 16.5
// and 19.8.
__host__ __device__ constexpr int small_max(int format) {
  return format == CERTKV_STORE_BF16 ? kSmallRows : 2 * kSmallRows;
}
// slots per tile of that kernel
__host__ __device__ constexpr int small_tile(int format) {
  return format == CERTKV_STORE_BF16 ? 32 : CERTKV_STORE_PAGE;
}
constexpr float kLn2 = 0.69314718055994531f;

// 8- and 4-bit stores: a weight meets the codes as an f16 operand that carries the scale of
// its value row, 2^(x - E) vs.  The reference E of a row follows the largest of x + log2 vs, so
// that what counts most in the sum is what f16 holds best, however much value rows differ in
// size and whatever weight falls on rows that are zero.
constexpr float kHead = 6.f;  // the largest operand is below 2^kHead when E is taken from it
// log2 of a value scale, low by at most 0.09 (its bits read as a fixed-point number).  Not
// below -74, and that for a scale of 0 (nothing in the row) or NaN (no reference helps): E is
// then within 80 of the largest logit x, and the fp32 sum of 2^(x - E) finite.
__device__ __forceinline__ float log2_scale(float s) {
  const int b = __float_as_int(s);
  return b < 0x7f800000 ? fmaxf(fmaf((float)b, 1.1920929e-7f, -127.f), -74.f) : -74.f;
}
// The store holds a row of zeros with scale 1.  Whether anything of such a row is left: codes
// that are not +0 or -0, of the four bytes each.
template <int FMT>
__device__ __forceinline__ uint32_t nonzero_codes(uint32_t four) {
  return four & (FMT == CERTKV_STORE_FP8 ? 0x7f7f7f7fu : 0x77777777u);
}

struct TreeArgs {
  int L, H, G, T;     // layers, KV heads, query heads per KV head, drafted tokens
  int units, rows;    // B L H, T G query rows per unit
  int nblk, rb;       // row blocks of a unit, rows of a block (the last may have fewer)
  int ctas;           // CTAs the tiles are divided among
  int least;          // tiles a CTA takes at least: what its warps work on side by side
  int small;          // the mma.sync kernel: the merge takes the drafts
  Rows q, kn, vn, o;  // kn.p null: the drafts have no keys of their own
  const uint64_t* mask;
  float* lse;
  float scale_log2;
  Store st;
  // workspace
  int64_t* first;        // [units + 1] tiles of the segments before (one row block)
  uint64_t* odd;         // [units] drafts whose value row holds a NaN or infinity
  float2* rec_ml;        // [records][rb] log2-domain reference and sum
  float* rec_acc;        // [records][rb][128] weighted mean of the values
};

// What the merge reads for a row: its reference and sum, or NaN where a wait ran out, the
// writer's own (`ok`) or one of any role whose part the row may hold (`aborted`, read after the
// barrier at which those parts were handed over).
__host__ __device__ __forceinline__ float2 tree_record(bool ok, bool aborted, float ref, float sum) {
  return ok && !aborted ? make_float2(ref, sum) : make_float2(0.f, nanf(""));
}

// Drafts that token t of sequence b sees, as bits.
__device__ __forceinline__ uint64_t seen(const TreeArgs& p, int b, int t) {
  const uint64_t all = ~0ull >> (64 - p.T);
  return (p.mask ? p.mask[(int64_t)b * p.T + t] : ~0ull >> (63 - t)) & all;
}

// Tiles [g0, g1) of CTA c: the global sequence (unit, row block, tile) in equal
// consecutive shares.
__device__ __forceinline__ int64_t tiles_per_cta(const TreeArgs& p, const int64_t* first) {
  return max((first[p.units] * p.nblk + p.ctas - 1) / p.ctas, (int64_t)p.least);
}

// Up to this many units every CTA of a split kernel scans the tile counts itself,
// which saves the launch of the scan (attention of one token over eight heads: 18
// -> 16 us).
constexpr int kInlineUnits = 256;
// The tiles before each unit, as p.first: read from there, or worked out into
// shared memory by the whole block (and by CTA 0 for the merge as well).
__device__ __forceinline__ const int64_t* tree_first(const TreeArgs& p, int64_t* smem, int tile, int drafts) {
  if (p.units > kInlineUnits) return p.first;
  if (threadIdx.x < 32) {
    const int lane = threadIdx.x;
    int64_t v[kInlineUnits / 32], sum = 0;
#pragma unroll
    for (int i = 0; i < kInlineUnits / 32; ++i) {  // units 8 lane ..
      const int u = lane * (kInlineUnits / 32) + i;
      v[i] = u < p.units ? (p.st.count(u) + tile - 1) / tile + drafts : 0;
      sum += v[i];
    }
    int64_t x = sum;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int64_t y = __shfl_up_sync(kFull, x, o);
      if (lane >= o) x += y;
    }
    x -= sum;
#pragma unroll
    for (int i = 0; i < kInlineUnits / 32; ++i) {
      const int u = lane * (kInlineUnits / 32) + i;
      if (u <= p.units) {
        smem[u] = x;
        if (blockIdx.x == 0) p.first[u] = x;
      }
      x += v[i];
    }
    if (lane == 31 && p.units == kInlineUnits) {
      smem[kInlineUnits] = x;
      if (blockIdx.x == 0) p.first[kInlineUnits] = x;
    }
  }
  __syncthreads();
  return smem;
}

// One (CTA, unit, row block) that meet: their partial results are record
// c + unit nblk + block.
struct Item {
  int u, blk;      // unit, row block
  int ka, kb, n;   // its tiles [ka, kb) of n, the last of them the drafts' own
};

// Walks over the items of a CTA.
struct Items {
  const int64_t* first;
  int64_t g, g1;
  int u;
  __device__ __forceinline__ Items(const TreeArgs& p, const int64_t* first_, int64_t per) : first(first_) {
    const int64_t total = first[p.units] * p.nblk;
    g = per * blockIdx.x;
    g1 = min(total, g + per);
    int lo = 0, hi = p.units;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (first[mid] * p.nblk <= g) lo = mid;
      else hi = mid;
    }
    u = lo;
  }
  __device__ __forceinline__ bool next(const TreeArgs& p, Item* it) {
    if (g >= g1) return false;
    while (first[u + 1] * p.nblk <= g) ++u;
    const int n = (int)(first[u + 1] - first[u]);
    const int64_t in = g - first[u] * p.nblk;
    it->u = u;
    it->blk = (int)(in / n);
    it->ka = (int)(in - (int64_t)it->blk * n);
    it->kb = (int)min((int64_t)n, it->ka + (g1 - g));
    it->n = n;
    g += it->kb - it->ka;
    return true;
  }
};

// CTAs of the split kernels on the current device (0 on an error), and their
// launches (false: nothing launched).
int tree_ctas();
int tree_mma_ctas(int format);
bool launch_tree_tc(const TreeArgs& p, int format, cudaStream_t st);
bool launch_tree_mma(const TreeArgs& p, int format, cudaStream_t st);

}  // namespace certkv
