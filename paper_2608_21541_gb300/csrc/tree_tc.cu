// tree_tc.cu — the split kernel of tree attention on the 5th-generation tensor
// cores (tcgen05 + TMEM).
//
// The T G query rows of a unit read the same keys and values, so both products
// are matrix products: S = Q K^T over a tile of 128 slots and O += P V, with
// the query rows as the M = 128 rows of the MMAs.  Two streams of them are kept
// in flight, so that the tensor cores work on one while the softmax of the
// other runs:
//   more than 128 rows: stream s holds rows 128 s .. of the block, and both
//     take every tile (a tile is loaded once for 256 rows);
//   up to 128 rows: both streams hold the same rows and take alternate tiles,
//     and their sums are joined at the end.
// Tensor memory: S0 | S1 | O0 | O1, 128 columns each; P overwrites S.
//
// Roles per CTA (one per SM, persistent over a share of all tiles):
//   warps 0..7   softmax: warp (stream, lane quadrant), a thread owns a row;
//   warps 8..15  loaders: 8- and 4-bit tiles through registers, expanded to f16
//                in the MMAs' swizzled layout; for every store the drafts' own
//                tile and bf16 tiles that are not whole;
//   warp 16      tensor-memory allocation, and issues the MMAs;
//   warp 17      scout: walks the page table ahead of the loaders and states each
//                tile's facts;
//   warps 17, 18 whole bf16 tiles: keys and values by TMA;
//   warp 18      8- and 4-bit stores: has the pages of later tiles brought into L2.
//
// Precision.  bf16 store: bf16 products, and a weight enters P V as a bf16 part
// plus the bf16 rounding of its remainder (2^-16).  8- and 4-bit stores: codes
// are exact in f16, so are query rows once divided by a power of two (elements
// within 2^-17 of the row's largest; smaller ones to 2^-25 of it); a key's fp32
// scale multiplies its logit, a value's fp32 scale the weight, and that product is
// rounded once to f16 (2^-11).  Logits, sums, and accumulators are fp32.  A weight
// is 2^(x - C) for a reference C that moves to the row's maximum (of the products,
// where they are what is rounded: log2_scale) only when the operand would leave
// its range (f16: 2^15), so that most tiles are formed in one pass over the logits,
// without their maximum and without rescaling.
//
// What bounds it, 256 segments of 13107 slots: a bf16 store of 64 rows 282 us, 90 %
// of the copy bandwidth, of 256 rows 480, 48 % of the tensor rate.  8- and 4-bit
// stores: 33 to 128 rows 318 to 362 us, the expansion of every code into an operand
// by eight warps and the softmax beside it (40 % of the issue slots); 256 rows 615 and
// 599, 37 and 38 % of the tensor rate, the chain softmax, hand-over, products,
// hand-over of each stream: a poll of a barrier queues behind the loaders' stores for
// hundreds of cycles.  Value scales on the weights rather than on the values cost the
// softmax a product a weight (256 rows 588 -> 615 us) and save the loaders one (64
// rows, 4-bit, 382 -> 337).  Slower were half tiles, also with the next half's S issued
// before P V (588 -> 721), an issuing warp per stream, sixteen loader warps, and logits
// loaded a step ahead of their use.
//
// Every wait is bounded; on a timeout the roles stop waiting, the rows in
// question read NaN and the store's status word gets CERTKV_STATUS_TIMEOUT.
#include <cuda.h>
#include <stddef.h>

#include "../../include/certkv.h"
#include "common.cuh"
#include "follow.cuh"
#include "internal.cuh"
#include "tma.cuh"
#include "tree.cuh"
#include "umma.cuh"

namespace certkv {
namespace {

constexpr int kSoftWarps = 8;
constexpr int kGroupWarps = 4, kLoadGroups = 2, kLoadWarps = kGroupWarps * kLoadGroups;
constexpr int kThreads = (kSoftWarps + kLoadWarps + 4) * 32;  // whole warpgroups
// A loader thread's (slot, 16-element) pieces of an operand, kStep slots apart.
constexpr int kPieces = 128 * 8 / (kGroupWarps * 32), kStep = 128 / kPieces;
// Registers a thread: the launch gives 96 (640 threads), which the roles share
// out among themselves.  A spill costs more here than elsewhere: next to 200 KB
// of shared memory the L1 holds hardly any of it.  256 segments of 13107 slots, 256
// rows, 8-bit: 120 / 88 / 64 657 us, 120 / 80 / 80 631, 112 / 88 / 80 618.
constexpr int kSoftRegs = 112, kLoadRegs = 88, kIssueRegs = 80;
static_assert(kSoftWarps * 32 * kSoftRegs + kLoadWarps * 32 * kLoadRegs + 128 * kIssueRegs <= kThreads * 96,
              "a larger split would wait for registers for ever");
constexpr int kHalf = 128 * 128;     // bytes of 128 rows x 64 16-bit elements
constexpr int kOperand = 2 * kHalf;  // 128 rows x 128 elements
constexpr int kAhead = 6;            // tiles the L2 prefetch runs ahead
// Shared memory: the query blocks (two when both streams hold rows of their
// own), then a ring of operands, then Misc.  Operand i is place i % 4.
template <bool PAIR>
struct Plan {
  static constexpr int kRing = 4;
  static constexpr int kRingOff = (PAIR ? 2 : 1) * kOperand;
  static constexpr int kMiscOff = kRingOff + kRing * kOperand;
};
// A waiter for a place's release must itself have waited for the release before
// it (a parity tells only neighbouring phases apart): a place belongs to one group.
static_assert(Plan<true>::kRing % kLoadGroups == 0 && Plan<false>::kRing % kLoadGroups == 0, "one group per place");
// The operands of the n tiles of a CTA pass through the ring in the order K(0),
// then K(t + 1), V(t) for t = 0 .., near the order the MMAs take them in.
__device__ __forceinline__ uint32_t k_seq(uint32_t t) { return t == 0 ? 0u : 2u * t - 1u; }
__device__ __forceinline__ uint32_t v_seq(uint32_t t, uint32_t n) { return min(2u * t + 2u, 2u * n - 1u); }
// Place of operand i in the ring, and the parity of that use.
template <bool PAIR>
struct Place {
  uint32_t slot, phase;
  __device__ __forceinline__ explicit Place(uint32_t i)
      : slot(i % Plan<PAIR>::kRing), phase((i / Plan<PAIR>::kRing) & 1u) {}
};
constexpr uint32_t kColS = 0, kColO = 256;  // + 128 stream

// A tile's facts, stated by the scout ahead of its keys.  Slot t % 8 is written
// again, for tile t + 8, when the loaders and the softmax warps have given it back.
constexpr uint32_t kMeta = 8;
struct alignas(16) Meta {  // its arrays are read and written as float4
  float ks[kTreeTile];  // scale of each slot's key (8- and 4-bit stores)
  float vs[kTreeTile];  // scale of each slot's value, 0 where the row is zero
  float lv[kTreeTile];  // log2_scale of it
  uint32_t live[4];     // slots to take
  int a, b;             // the tile's pages (-1: none)
  int count;            // live slots from the tile's first on
  int whole;            // every slot is live
  int drafts;           // the drafts' own tile: live comes from the row's mask
  int unit, first_block;
};

struct Misc {
  uint64_t full[4], empty[4];                // places of the ring
  uint64_t stated[kMeta], ready[kMeta];      // scout -> loaders, loaders -> softmax
  uint64_t back[kMeta];                      // loaders, softmax -> scout
  uint64_t s_full[2], p_full[2], o_full[2], q_full, done;
  uint64_t group[kLoadGroups];               // barriers of the loader groups
  uint32_t tmem;
  int abort;
  uint32_t walked;  // tiles stated so far (8- and 4-bit stores)
  unsigned long long odd[kLoadGroups];
  float qs[256];                   // per row: scale of its f16 queries
  float cm[128], l[128];           // stream 1's reference and sum
  Meta meta[kMeta];
  int64_t first[kInlineUnits + 1];  // see tree_first
};
static_assert(sizeof(Meta) % 16 == 0 && offsetof(Misc, meta) % 16 == 0, "float4 accesses");
template <bool PAIR>
constexpr int smem_bytes() {
  return Plan<PAIR>::kMiscOff + (int)sizeof(Misc) + 1024;
}
static_assert(smem_bytes<true>() <= 232448 && smem_bytes<false>() <= 232448,
              "over the 227 KB of shared memory a CTA can have");

__device__ __forceinline__ uint32_t bar(const uint64_t* b) { return tc::saddr(b); }
__device__ __forceinline__ void softmax_sync() {
  asm volatile("bar.sync 1, %0;" ::"n"(kSoftWarps * 32) : "memory");
}
__device__ __forceinline__ void sts128(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w)
               : "memory");
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  uint32_t r;
  asm("cvt.rn.f16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
  return r;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ float pow2(int e) { return __int_as_float((e + 127) << 23); }  // |e| < 127

// A loader thread's part of an operand: elements 16 sub .. 16 sub + 15 of the
// rows grp, grp + kStep ..  A quarter warp holds the same half of two
// neighbouring rows, which the swizzle puts into different banks.
struct Piece {
  int grp, sub;
  uint32_t at0, at1;  // its two 16-byte chunks of row grp in a swizzled operand
  __device__ __forceinline__ explicit Piece(int tid) {
    const int lane = tid & 31;
    grp = 4 * (tid >> 5) + 2 * (lane >> 4) + ((lane >> 2) & 1);
    sub = (lane & 3) + 4 * ((lane >> 3) & 1);
    const int c = 2 * (sub & 3), x = grp & 7;
    const uint32_t r = (uint32_t)((sub >> 2) * kHalf + grp * 128);
    at0 = r + (uint32_t)((c ^ x) << 4);
    at1 = r + (uint32_t)(((c + 1) ^ x) << 4);
  }
  // row grp + kStep q of the operand at `to`
  __device__ __forceinline__ void put(uint32_t to, int q, const uint32_t (&w)[8]) const {
    sts128(to + at0 + (uint32_t)(q * kStep * 128), w[0], w[1], w[2], w[3]);
    sts128(to + at1 + (uint32_t)(q * kStep * 128), w[4], w[5], w[6], w[7]);
  }
  // the eight lanes of a row
  __device__ __forceinline__ static uint32_t row_max(uint32_t x) {
    x = max(x, __shfl_xor_sync(kFull, x, 1));
    x = max(x, __shfl_xor_sync(kFull, x, 2));
    return max(x, __shfl_xor_sync(kFull, x, 8));
  }
};

__device__ __forceinline__ void load32g(const void* p, uint32_t (&w)[8]) {
  const uint4* q = reinterpret_cast<const uint4*>(p);
  const uint4 a = __ldg(q), b = __ldg(q + 1);
  w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w;
  w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
}

// Largest magnitude of sixteen bf16 as fp32 bits (a NaN or infinity: >= 0x7f800000).
__device__ __forceinline__ uint32_t top16(const uint32_t (&w)[8]) {
  uint32_t top = 0;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    top = max(top, (w[i] & 0x7fffu) << 16);
    top = max(top, w[i] & 0x7fff0000u);
  }
  return top;
}
// sixteen bf16 times f as f16
__device__ __forceinline__ void to_f16(uint32_t (&w)[8], float f) {
#pragma unroll
  for (int i = 0; i < 8; ++i)
    w[i] = pack_f16(__uint_as_float(w[i] << 16) * f, __uint_as_float(w[i] & 0xffff0000u) * f);
}
// Exponent e with 2^e <= x < 2^(e+1) of a positive normal fp32, else 0.
__device__ __forceinline__ int exponent(float x) {
  const int e = (__float_as_int(x) >> 23) & 255;
  return e == 0 || e == 255 ? 0 : e - 127;
}

// Raw codes of this thread's pieces of one operand.
template <int FMT>
struct Raw {
  static constexpr int kWords = FMT == CERTKV_STORE_FP8 ? 4 : 2;
  uint32_t w[kPieces][kWords];
  uint32_t g[FMT == CERTKV_STORE_FP4 ? kPieces : 1];

  // the tile's pages a, b (-1: none), live slots from its first on
  __device__ __forceinline__ void load(const Piece& pc, int a, int b, int live, const uint8_t* codes,
                                       const uint8_t* group) {
#pragma unroll
    for (int q = 0; q < kPieces; ++q) {
      const int page = q < kPieces / 2 ? a : b, row = pc.grp + kStep * (q % (kPieces / 2));
      const bool on = page >= 0 && pc.grp + kStep * q < live;
      const int64_t at = (int64_t)page * kPage + row;
#pragma unroll
      for (int j = 0; j < kWords; ++j) w[q][j] = 0u;
      if (on) {
        if constexpr (FMT == CERTKV_STORE_FP8) {
          const uint4 x = __ldg(reinterpret_cast<const uint4*>(codes + at * 128 + pc.sub * 16));
          w[q][0] = x.x;
          w[q][1] = x.y;
          w[q][2] = x.z;
          w[q][3] = x.w;
        } else {
          const uint2 x = __ldg(reinterpret_cast<const uint2*>(codes + at * 64 + pc.sub * 8));
          w[q][0] = x.x;
          w[q][1] = x.y;
        }
      }
      if constexpr (FMT == CERTKV_STORE_FP4) g[q] = on ? (uint32_t)__ldg(group + at * kGroups + pc.sub) : 0u;
    }
  }
};

// Piece q as f16: codes, with their group scale (exact).
template <int FMT>
__device__ __forceinline__ void expand(const Raw<FMT>& r, int q, uint32_t (&w)[8]) {
  if constexpr (FMT == CERTKV_STORE_FP8) {
#pragma unroll
    for (int j = 0; j < 8; ++j) w[j] = e4m3x2_to_f16x2(r.w[q][j >> 1] >> (16 * (j & 1)));
  } else {
    const uint32_t f2 = e4m3x2_to_f16x2(r.g[q] | (r.g[q] << 8));
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      w[4 * j] = hmul2(e2m1x2_to_f16x2<0>(r.w[q][j]), f2);
      w[4 * j + 1] = hmul2(e2m1x2_to_f16x2<1>(r.w[q][j]), f2);
      w[4 * j + 2] = hmul2(e2m1x2_to_f16x2<2>(r.w[q][j]), f2);
      w[4 * j + 3] = hmul2(e2m1x2_to_f16x2<3>(r.w[q][j]), f2);
    }
  }
}
// Exponent a draft's value row is divided by: its elements then reach as far as codes do.
template <int FMT>
__device__ __forceinline__ int draft_shift(float largest) {
  return min(max(exponent(largest) - (FMT == CERTKV_STORE_FP8 ? 8 : 11), -120), 120);
}

// ----------------------------------------------------------------- scout --
// One warp walks the CTA's tiles, through the page table, ahead of everybody and
// states their facts; a second one walks with it.  Whole bf16 tiles they copy by
// TMA (keys and values), keeping count of a bf16 store's other operands; for the
// other stores the second brings later pages into L2.
template <int FMT, bool PAIR>
struct Scout {
  static constexpr bool kQuant = FMT != CERTKV_STORE_BF16;
  const TreeArgs& p;
  Misc* m;
  const CUtensorMap *tmK, *tmV;
  uint32_t ring;
  int lane;
  bool ok = true;
  // the walk: tile k of item it, of `stored` tiles of stored slots
  Items items;
  Item it;
  int k = 0, count = 0, stored = 0;
  int at = 0, lo = -1, hi = -1;  // table entries of 64 pages from page `at` on
  int a = -1, b = -1;            // pages of tile k
  float4 ks, vs;                 // its scales, on their way

  __device__ __forceinline__ int entry(int page) const {
    if (page >= p.st.max_pages) return -1;
    const int e = __ldg(p.st.table + (int64_t)it.u * p.st.max_pages + page);
    return e >= 0 && e < p.st.pool_pages ? e : -1;
  }
  __device__ __forceinline__ int page(int i) const {  // at <= i < at + 64
    const int x = __shfl_sync(kFull, lo, (i - at) & 31), y = __shfl_sync(kFull, hi, (i - at) & 31);
    return i - at < 32 ? x : y;
  }
  // Page i of the segment on its way into L2: each lane one of its arrays.
  __device__ __forceinline__ void prefetch_page(int i) const {
    if (i >= 2 * stored) return;
    const int pg = page(i);
    if (pg < 0) return;
    const int64_t s = (int64_t)pg * kPage;
    const void* x = nullptr;
    uint32_t bytes = kPage * row_bytes(FMT);
    if (lane < 2) x = (lane ? p.st.v : p.st.k) + s * row_bytes(FMT);
    if (lane == 2 || lane == 3) {
      x = (lane & 1 ? p.st.vs : p.st.ks) + s;
      bytes = kPage * 4;
    }
    if (FMT == CERTKV_STORE_FP4 && (lane == 4 || lane == 5)) {
      x = (lane & 1 ? p.st.vg : p.st.kg) + s * kGroups;
      bytes = kPage * kGroups;
    }
    if (x)
      asm volatile("cp.async.bulk.prefetch.L2.global [%0], %1;" ::"l"(reinterpret_cast<uint64_t>(x)),
                   "r"(bytes)
                   : "memory");
  }
  // Scales of slots 4 lane .. 4 lane + 3 of a tile (`none` where there is no slot).
  __device__ __forceinline__ float4 scales(const float* s, int live, float none) const {
    const int pg = lane < 16 ? a : b, n = live - 4 * lane;
    float4 x = make_float4(none, none, none, none);
    if (pg >= 0)
      x = __ldg(reinterpret_cast<const float4*>(s + (int64_t)pg * kPage + ((4 * lane) & (kPage - 1))));
    if (n < 1) x.x = none;
    if (n < 2) x.y = none;
    if (n < 3) x.z = none;
    if (n < 4) x.w = none;
    return x;
  }
  __device__ __forceinline__ void advance() {
    if (2 * k >= at + 32) {
      at += 32;
      lo = hi;
      hi = entry(at + 32 + lane);
    }
  }
  // Pages and scales of tile k, asked for a tile before they are stated.
  __device__ __forceinline__ void fetch() {
    if (k >= min(stored, it.kb)) return;
    advance();
    a = page(2 * k);
    b = page(2 * k + 1);
    if (kQuant) {
      const int live = count - k * kTreeTile;
      ks = scales(p.st.ks, live, 1.f);  // finite where there is no slot
      vs = scales(p.st.vs, live, 0.f);
    }
  }
  // The next item (there is one).
  __device__ __forceinline__ void enter() {
    items.next(p, &it);
    k = it.ka;
    count = p.st.count(it.u);
    stored = (count + kTreeTile - 1) / kTreeTile;
    at = 2 * k;
    lo = entry(at + lane);
    hi = entry(at + 32 + lane);
  }
  // Scale 0 for the rows of tile k that are zero.  The four rows of a lane's scales lie
  // behind one another; the warp reads them together, for the lanes that have a scale of 1.
  // Nothing where no scale is 1; a store of zeros alone takes 3.4 times as long.
  __device__ __forceinline__ void find_zeros() {
    constexpr int kLanes = row_bytes(FMT) / 16;  // of a row, 16 bytes each
    uint32_t some = __ballot_sync(kFull, vs.x == 1.f || vs.y == 1.f || vs.z == 1.f || vs.w == 1.f);
    while (some) {  // two lanes' rows at a time: a look takes the way to L2
      uint4 x[2];
      int of[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        of[i] = __ffs(some) - 1;
        const int64_t row = (int64_t)(of[i] < 16 ? a : b) * kPage + (4 * of[i]) % kPage;
        x[i] = make_uint4(0u, 0u, 0u, 0u);
        if (of[i] >= 0 && lane < 4 * kLanes)
          x[i] = __ldg(reinterpret_cast<const uint4*>(p.st.v + row * row_bytes(FMT)) + lane);
        some &= some - 1;
      }
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        const uint32_t on = __ballot_sync(kFull, nonzero_codes<FMT>(x[i].x | x[i].y | x[i].z | x[i].w) != 0u);
        constexpr uint32_t kRow = (1u << kLanes) - 1u;
        if (lane == of[i]) {
          if (vs.x == 1.f && !(on & kRow)) vs.x = 0.f;
          if (vs.y == 1.f && !(on >> kLanes & kRow)) vs.y = 0.f;
          if (vs.z == 1.f && !(on >> 2 * kLanes & kRow)) vs.z = 0.f;
          if (vs.w == 1.f && !(on >> 3 * kLanes & kRow)) vs.w = 0.f;
        }
        __syncwarp();
      }
    }
  }
  // State tile t, the next of the walk.
  __device__ __forceinline__ void state(uint32_t t) {
    if (k == it.kb) {
      enter();
      fetch();
    }
    // a bf16 store's walk is paced by its K places: that of K(t - 4), free by now,
    // held K(t - 6), released by a product issued after P of tile t - 8 was written
    if (kQuant && ok && t >= kMeta)
      ok = tc::mbar_wait(bar(&m->back[t % kMeta]), (t / kMeta - 1) & 1u, &m->abort);
    Meta& mt = m->meta[t % kMeta];
    if (k < stored) {
      const int live = count - k * kTreeTile;
      if constexpr (kQuant) {
        find_zeros();
        *reinterpret_cast<float4*>(&mt.ks[4 * lane]) = ks;
        *reinterpret_cast<float4*>(&mt.vs[4 * lane]) = vs;
        *reinterpret_cast<float4*>(&mt.lv[4 * lane]) =
            make_float4(log2_scale(vs.x), log2_scale(vs.y), log2_scale(vs.z), log2_scale(vs.w));
      }
      if (lane < 4) {
        const int c = min(max(live - 32 * lane, 0), 32);
        mt.live[lane] = (lane < 2 ? a : b) < 0 || c == 0 ? 0u : 0xffffffffu >> (32 - c);
      }
      if (lane == 0) {
        mt.a = a;
        mt.b = b;
        mt.count = live;
        mt.whole = live >= kTreeTile && a >= 0 && b >= 0;
        mt.drafts = 0;
        if (a < 0 || (b < 0 && live > kPage)) p.st.raise();
      }
    } else if (lane == 0) {
      mt.a = mt.b = -1;
      mt.count = 0;
      mt.whole = 0;
      mt.drafts = 1;
      mt.unit = it.u;
      mt.first_block = it.blk == 0;
    }
    __syncwarp();
    if (lane == 0) {
      tc::mbar_arrive(bar(&m->stated[t % kMeta]));
      if (kQuant) *(volatile uint32_t*)&m->walked = t + 1;
    }
    ++k;
    fetch();
  }
  // Operand i, tile t, of a bf16 store: a whole tile by four bulk copies, two
  // pages x two 64-element halves; else the scout's arrival alone.
  __device__ __forceinline__ bool operand(const CUtensorMap* map, uint32_t i, uint32_t t) {
    const Place<PAIR> pl(i);
    if (ok) ok = tc::mbar_wait(bar(&m->empty[pl.slot]), pl.phase ^ 1u, &m->abort);
    const Meta& mt = m->meta[t % kMeta];
    const uint32_t full = bar(&m->full[pl.slot]), to = ring + pl.slot * kOperand;
    const bool copied = ok && mt.whole;
    if (lane == 0) {
      if (copied) {
        const int ya = mt.a * kPage, yb = mt.b * kPage;
        tc::mbar_expect_tx(full, kOperand);
        tc::tma_load_2d(to, map, 0, ya, full);
        tc::tma_load_2d(to + kHalf, map, 64, ya, full);
        tc::tma_load_2d(to + kHalf / 2, map, 0, yb, full);
        tc::tma_load_2d(to + kHalf + kHalf / 2, map, 64, yb, full);
      } else {
        tc::mbar_arrive(full);
      }
    }
    __syncwarp();
    return copied;
  }
  // Bulk copies of the last operands land before the CTA may exit.
  __device__ __forceinline__ void drain(uint32_t n, uint32_t copies) const {
    if (lane != 0) return;
    volatile int dummy = 0;
    for (uint32_t i = 2 * n > Plan<PAIR>::kRing ? 2 * n - Plan<PAIR>::kRing : 0; i < 2 * n; ++i) {
      const Place<PAIR> pl(i);
      if (copies >> pl.slot & 1u) tc::mbar_wait(bar(&m->full[pl.slot]), pl.phase, &dummy);
    }
  }
  __device__ __forceinline__ void run(uint32_t n) {
    it.kb = 0;
    if (kQuant) {
      for (uint32_t t = 0; t < n; ++t) state(t);
      return;
    }
    uint32_t stated = 0, copies = 0;  // places whose last operand this warp copied
    for (; stated < min(n, 4u); ++stated) state(stated);
    for (uint32_t t = 0; t < n; ++t) {
      const uint32_t bit = 1u << Place<PAIR>(k_seq(t)).slot;
      copies = operand(tmK, k_seq(t), t) ? copies | bit : copies & ~bit;
      if (stated < n) state(stated++);
    }
    drain(n, copies);
  }
  // 8- and 4-bit stores, a warp of its own (a bulk prefetch is slow to issue): as
  // tile t is stated, the pages kAhead tiles on are brought into L2.  Only a help: it
  // holds nobody up and never aborts.
  __device__ __forceinline__ void run_ahead(uint32_t n) {
    it.kb = 0;
    for (uint32_t t = 0; t < n && ok; ++t, ++k) {
      if (k == it.kb) {
        enter();
        for (int i = 2; i < 2 * kAhead; ++i) prefetch_page(at + i);
      }
      advance();
      prefetch_page(2 * (k + kAhead));
      prefetch_page(2 * (k + kAhead) + 1);
      // nobody waits for this warp: see follow.cuh
      ok = __all_sync(kFull, follow(
                                 t, tc::kSpinLimit, [&] { return *(volatile uint32_t*)&m->walked; },
                                 [&] { return *(volatile int*)&m->abort != 0; }, [] { __nanosleep(64); }));
    }
  }
  // The values of a bf16 store, by a warp of their own: a poll takes hundreds of
  // cycles, and one warp's polls for keys, facts and values add up to a tile's time.
  __device__ __forceinline__ void run_values(uint32_t n) {
    uint32_t copies = 0;
    for (uint32_t t = 0; t < n; ++t) {
      const uint32_t bit = 1u << Place<PAIR>(v_seq(t, n)).slot;
      if (ok) ok = tc::mbar_wait(bar(&m->stated[t % kMeta]), (t / kMeta) & 1u, &m->abort);
      copies = operand(tmV, v_seq(t, n), t) ? copies | bit : copies & ~bit;
    }
    drain(n, copies);
  }
};

// --------------------------------------------------------------- loaders --
// Two groups of four warps take the operands in turn, so that the latencies of one
// operand (its place, its codes' way from L2, the fence before the MMAs)
// pass under the work on the others.
template <int FMT, bool PAIR>
struct Loader {
  static constexpr bool kQuant = FMT != CERTKV_STORE_BF16;
  static constexpr int kRawFmt = kQuant ? FMT : CERTKV_STORE_FP8;
  const TreeArgs& p;
  Misc* m;
  uint32_t ring;
  int group, tid;  // thread of the group
  Piece pc;
  bool ok = true;         // false after a wait gave up
  uint32_t syncs = 0;     // of the group so far

  // NaN and infinities of sixteen bf16 to 0 (in the product they would reach every
  // row, seen or not; the merge adds them to the rows that see their draft).
  __device__ __forceinline__ bool finite_only(uint32_t (&v)[8]) const {
    bool odd = false;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      if ((v[j] & 0x7f80u) == 0x7f80u) {
        v[j] &= 0xffff0000u;
        odd = true;
      }
      if ((v[j] & 0x7f800000u) == 0x7f800000u) {
        v[j] &= 0xffffu;
        odd = true;
      }
    }
    return odd;
  }
  __device__ __forceinline__ void wait(const uint64_t* b, uint32_t phase) {
    if (ok) ok = __all_sync(kFull, tc::mbar_wait(bar(b), phase, &m->abort));
  }
  // A barrier of the group whose wait is bounded like every other.
  __device__ __forceinline__ void group_sync() {
    __syncwarp();
    if ((tid & 31) == 0) tc::mbar_arrive(bar(&m->group[group]));
    wait(&m->group[group], syncs & 1u);
    ++syncs;
  }
  // Keys of the drafts' own tile and the facts that follow from its rows.
  __device__ __forceinline__ void draft_keys(uint32_t to, Meta& mt) {
    const int u = mt.unit, bl = u / p.H, h = u - bl * p.H, b = bl / p.L, l = bl - b * p.L;
    if (tid == 0) m->odd[group] = 0ull;
    group_sync();
#pragma unroll 1
    for (int q = 0; q < kPieces; ++q) {
      const int s = pc.grp + kStep * q;
      uint32_t k[8] = {}, v[8] = {};
      if (s < p.T) {
        load32g(p.kn.at(b, l, s, h) + pc.sub * 16, k);
        load32g(p.vn.at(b, l, s, h) + pc.sub * 16, v);
      }
      if (finite_only(v)) atomicOr(&m->odd[group], 1ull << (s & 63));
      if (kQuant) {
        const float top = __uint_as_float(Piece::row_max(top16(v)));
        const float f = top > 0.f ? pow2(draft_shift<kRawFmt>(top)) : 0.f;
        if (pc.sub == 0) {
          mt.vs[s] = f;
          mt.lv[s] = log2_scale(f);
        }
        const int e = min(max(exponent(__uint_as_float(Piece::row_max(top16(k)))), -120), 120);
        to_f16(k, pow2(-e));
        if (pc.sub == 0) mt.ks[s] = pow2(e);
      }
      pc.put(to, q, k);
    }
    group_sync();
    if (tid == 0 && mt.first_block) p.odd[u] = m->odd[group];
  }
  __device__ __forceinline__ void draft_values(uint32_t to, const Meta& mt) {
    const int u = mt.unit, bl = u / p.H, h = u - bl * p.H, b = bl / p.L, l = bl - b * p.L;
#pragma unroll 1
    for (int q = 0; q < kPieces; ++q) {
      const int s = pc.grp + kStep * q;
      uint32_t v[8] = {};
      if (s < p.T) {
        load32g(p.vn.at(b, l, s, h) + pc.sub * 16, v);
        finite_only(v);
        if (kQuant) to_f16(v, mt.vs[s] > 0.f ? 1.f / mt.vs[s] : 0.f);  // a power of two
      }
      pc.put(to, q, v);
    }
  }
  // One operand of a bf16 tile that is not whole.
  __device__ __forceinline__ void ragged(uint32_t to, const uint8_t* rows, const Meta& mt) {
#pragma unroll 1
    for (int q = 0; q < kPieces; ++q) {
      const int pg = q < kPieces / 2 ? mt.a : mt.b;
      uint32_t w[8] = {};
      if (pg >= 0 && pc.grp + kStep * q < mt.count)
        load32g(rows + ((int64_t)pg * kPage + pc.grp + kStep * (q % (kPieces / 2))) * 256 + pc.sub * 32, w);
      pc.put(to, q, w);
    }
  }
  __device__ __forceinline__ void run(uint32_t n) {
#pragma unroll 1
    for (uint32_t i = group; i < 2 * n; i += kLoadGroups) {
      // operand i: keys of tile 0, (i + 1) / 2, .. or values of tile i / 2 - 1, .., n - 1
      const bool value = i == 2 * n - 1 || (i > 0 && (i & 1) == 0);
      const uint32_t t = i == 2 * n - 1 ? n - 1 : value ? i / 2 - 1 : (i + 1) / 2;
      Meta& mt = m->meta[t % kMeta];
      wait(&m->stated[t % kMeta], (t / kMeta) & 1u);
      const bool own = mt.drafts;
      Raw<kRawFmt> raw;
      if (kQuant && !own)
        raw.load(pc, mt.a, mt.b, mt.count, value ? p.st.v : p.st.k, value ? p.st.vg : p.st.kg);
      // values of the drafts: their scales come from the group that had the keys
      if (own && value) wait(&m->ready[t % kMeta], (t / kMeta) & 1u);
      const Place<PAIR> pl(i);
      wait(&m->empty[pl.slot], pl.phase ^ 1u);
      if (!ok) break;
      const uint32_t to = ring + pl.slot * kOperand;
      bool wrote = true;
      if (own) {
        if (value) draft_values(to, mt);
        else draft_keys(to, mt);
      } else if (kQuant) {
#pragma unroll
        for (int q = 0; q < kPieces; ++q) {
          uint32_t w[8];
          expand<kRawFmt>(raw, q, w);
          pc.put(to, q, w);
        }
      } else {
        wrote = !mt.whole;
        if (wrote) ragged(to, value ? p.st.v : p.st.k, mt);
      }
      if (wrote) um::fence_async();
      __syncwarp();
      if ((tid & 31) == 0) {
        tc::mbar_arrive(bar(&m->full[pl.slot]));
        if (value) tc::mbar_arrive(bar(&m->back[t % kMeta]));
      }
      if (!value && tid == 0) tc::mbar_arrive(bar(&m->ready[t % kMeta]));
    }
  }
};

// ------------------------------------------------------------ MMA issuer --
// Products per tile: S = Q K^T and O += P V.  Streams on tiles of their own:
// S(0), S(1), then O(i), S(i + 2) with stream i & 1 on tile i; both streams on
// every tile: S0(0), S1(0), then O0(j), S0(j + 1), O1(j), S1(j + 1).  A stream's
// next S overwrites the P that its O has read, which the tensor core's in-order
// execution makes safe, and its completion tells the softmax that O is done.
template <int FMT, bool PAIR>
struct Issuer {
  static constexpr bool kBf16 = FMT == CERTKV_STORE_BF16;
  Misc* m;
  uint32_t tmem;
  uint32_t q, ring;  // shared-memory addresses of the queries and the ring
  uint32_t n;        // tiles of the CTA
  bool ok = true;
  uint32_t odd = 0;  // bit st: parity of the O's of stream st so far

  // The warp runs as one: the values below are the same in every lane, and are made
  // so for the compiler too, which then keeps the MMAs' operands in uniform
  // registers instead of moving them there for every MMA.
  static __device__ __forceinline__ uint32_t uni(uint32_t x) { return __shfl_sync(kFull, x, 0); }
  __device__ __forceinline__ void wait(const uint64_t* b, uint32_t phase) {
    if (ok) ok = __all_sync(kFull, tc::mbar_wait(bar(b), phase, &m->abort));
  }
  // Operand i is in place.  A poll takes hundreds of cycles even of a barrier long
  // complete (it queues behind the loaders' stores), so the operands of O and of
  // the S after it are asked for before the wait for P, which is then the only
  // one between P and both; what is not there yet is waited for when it is due.
  struct Operand {
    uint32_t slot, phase;
    bool there;
  };
  __device__ __forceinline__ Operand operand(uint32_t i) {
    const Place<PAIR> pl(i);
    return {uni(pl.slot), pl.phase, __all_sync(kFull, tc::mbar_test(bar(&m->full[pl.slot]), pl.phase)) != 0};
  }
  __device__ __forceinline__ void due(const Operand& x) {
    if (!x.there) wait(&m->full[x.slot], x.phase);
  }
  // S of stream st with the keys x; `last`: the tile's last S
  __device__ __forceinline__ void s(int st, const Operand& x, bool last) {
    const uint32_t slot = x.slot;
    due(x);
    if (!ok) return;
    um::fence_after();
    um::mma_s(uni(tmem + kColS + 128u * st), uni(um::desc_lo(q, 16) + (PAIR ? (uint32_t)st * (kOperand >> 4) : 0u)),
              uni(um::desc_lo(ring, 16) + slot * (kOperand >> 4)), um::kDescHi, um::idesc(kBf16, false));
    um::commit(uni(bar(&m->s_full[st])));
    if (last) um::commit(uni(bar(&m->empty[slot])));
  }
  // O += P V of stream st with the values x; `first`, `fin`: of the item
  __device__ __forceinline__ void o(int st, const Operand& x, bool last, bool first, bool fin) {
    const uint32_t slot = x.slot;
    const uint32_t d = uni(tmem + kColO + 128u * st), a = uni(tmem + kColS + 128u * st);
    const uint32_t b = uni(um::desc_lo(ring, kHalf) + slot * (kOperand >> 4)), acc = uni(!first);
    due(x);
    wait(&m->p_full[st], odd >> st & 1u);
    odd ^= 1u << st;
    if (!ok) return;
    um::fence_after();
    if (kBf16) um::mma_o2(d, a, b, um::kDescHi, um::idesc(true, true), acc);  // weights and remainders
    else um::mma_o(d, a, b, um::kDescHi, um::idesc(false, true), acc);
    if (last) um::commit(uni(bar(&m->empty[slot])));
    if (fin) um::commit(uni(bar(&m->o_full[st])));
  }

  __device__ __forceinline__ void run(const TreeArgs& p, const int64_t* first, int64_t per) {
    Items items(p, first, per);
    Item it;
    uint32_t t0 = 0, item = 0;  // tiles and items before
    while (ok && items.next(p, &it)) {
      const int c = it.kb - it.ka;
      Operand k = operand(k_seq(t0));
      wait(&m->q_full, item & 1u);
      ++item;
      if (PAIR) {
        s(0, k, false);
        s(1, k, true);
        for (int j = 0; ok && j < c; ++j) {
          const bool more = j + 1 < c;
          const Operand v = operand(v_seq(t0 + j, n));
          if (more) k = operand(k_seq(t0 + j + 1));
          o(0, v, false, j == 0, !more);
          if (more) s(0, k, false);
          o(1, v, true, j == 0, !more);
          if (more) s(1, k, true);
        }
      } else {
        s(0, k, true);
        if (c > 1) s(1, operand(k_seq(t0 + 1)), true);
        for (int i = 0; ok && i < c; ++i) {
          const Operand v = operand(v_seq(t0 + i, n));
          if (i + 2 < c) k = operand(k_seq(t0 + i + 2));
          o(i & 1, v, true, i < 2, i + 2 >= c);
          if (i + 2 < c) s(i & 1, k, true);
        }
      }
      t0 += c;
    }
    um::commit(bar(&m->done));  // everything issued above has finished
    volatile int dummy = 0;
    tc::mbar_wait(bar(&m->done), 0, &dummy);
    __syncwarp();
  }
};

// --------------------------------------------------------------- softmax --
// -inf over the logits of the slots that a row does not take (tiles that are not
// whole), so that the passes below need not ask.
__device__ __forceinline__ void mask_tile(uint32_t tS, const uint32_t (&live)[4]) {
#pragma unroll 1
  for (int c = 0; c < 4; ++c) {
    const uint32_t w = c < 2 ? (c ? live[1] : live[0]) : (c == 2 ? live[2] : live[3]);
    uint32_t r[32];
    um::ld32(tS + 32u * c, r);
#pragma unroll
    for (int j = 0; j < 32; ++j)
      if (!(w >> j & 1u)) r[j] = 0xff800000u;
    um::st32(tS + 32u * c, r);
  }
  um::wait_st();
}

// The largest logit of a row over a tile, from tensor memory (times the scale sl only where
// QUANT: there with log2 of the value's scale added).
template <bool QUANT>
__device__ __forceinline__ float tile_max(uint32_t tS, const Meta& mt, float sl) {
  float m0 = -INFINITY, m1 = -INFINITY, m2 = -INFINITY, m3 = -INFINITY;
  const float2 sl2 = make_float2(sl, sl);
#pragma unroll 1
  for (int c = 0; c < 4; ++c) {
    uint32_t r[32];
    um::ld32(tS + 32u * c, r);
#pragma unroll
    for (int j = 0; j < 32; j += 4) {
      float2 x = make_float2(__uint_as_float(r[j]), __uint_as_float(r[j + 1]));
      float2 y = make_float2(__uint_as_float(r[j + 2]), __uint_as_float(r[j + 3]));
      if (QUANT) {
        const float4 k4 = *reinterpret_cast<const float4*>(&mt.ks[32 * c + j]);
        const float4 l4 = *reinterpret_cast<const float4*>(&mt.lv[32 * c + j]);
        x = ffma2(fmul2(x, make_float2(k4.x, k4.y)), sl2, make_float2(l4.x, l4.y));
        y = ffma2(fmul2(y, make_float2(k4.z, k4.w)), sl2, make_float2(l4.z, l4.w));
      }
      if (j & 4) {
        m0 = um::max3(m0, x.x, x.y);
        m1 = um::max3(m1, y.x, y.y);
      } else {
        m2 = um::max3(m2, x.x, x.y);
        m3 = um::max3(m3, y.x, y.y);
      }
    }
  }
  return fmaxf(fmaxf(m0, m1), fmaxf(m2, m3));
}

// A row's running reference, sum and accumulator over the tiles it has met.
template <bool QUANT>
struct Row {
  float C = -INFINITY;  // reference (an integer; log2 domain)
  float lsum = 0.f;     // sum of the weights relative to it
  float sl;             // scale of the row's logits, > 0

  // Largest sum of 32 weights that needs no new reference: far within fp32's and bf16's
  // range.  QUANT: and the largest f16 operand below 2^15 (kTop, as bits of two).
  static constexpr float kLimit = QUANT ? 1.237940039285380e27f : 1.152921504606847e18f;
  static constexpr uint32_t kTop = 0x78007800u;
  // from what tile_max gives
  __device__ __forceinline__ float reference(float mx) const {
    return ceilf(QUANT ? mx - kHead : mx * sl);  // -inf stays
  }
  __device__ __forceinline__ float offset() const { return C == -INFINITY ? 0.f : -C; }

  // Weights of columns 32 c ..: the packed A operand in hi (and remainders in
  // lo); returns their sum, and in `top` the largest operand of each half (QUANT).  The
  // keys' scales are fetched before the logits, while nothing waits for them.
  __device__ __forceinline__ float chunk(uint32_t tS, int c, const Meta& mt, float off, uint32_t (&hi)[16],
                                         uint32_t (&lo)[16], uint32_t& top) const {
    const float2 sl2 = make_float2(sl, sl), off2 = make_float2(off, off);
    float2 sum0 = make_float2(0.f, 0.f), sum1 = make_float2(0.f, 0.f);
    float4 k4[8], v4;
    if (QUANT) {
#pragma unroll
      for (int j = 0; j < 8; ++j) k4[j] = *reinterpret_cast<const float4*>(&mt.ks[32 * c + 4 * j]);
    }
    uint32_t r[32];
    um::ld32(tS + 32u * c, r);
#pragma unroll
    for (int j = 0; j < 16; ++j) {
      float2 x = make_float2(__uint_as_float(r[2 * j]), __uint_as_float(r[2 * j + 1]));
      if (QUANT)
        x = fmul2(x, j & 1 ? make_float2(k4[j / 2].z, k4[j / 2].w) : make_float2(k4[j / 2].x, k4[j / 2].y));
      x = ffma2(x, sl2, off2);
      x.x = um::ex2(x.x);
      x.y = um::ex2(x.y);
      if (j & 1) sum1 = fadd2(sum1, x);
      else sum0 = fadd2(sum0, x);
      if (QUANT) {
        if (!(j & 1)) v4 = *reinterpret_cast<const float4*>(&mt.vs[32 * c + 2 * j]);
        x = fmul2(x, j & 1 ? make_float2(v4.z, v4.w) : make_float2(v4.x, v4.y));
        hi[j] = pack_f16(x.x, x.y);
        if (j & 1) top = __vimax3_u16x2(top, hi[j - 1], hi[j]);  // none is negative
      } else {
        hi[j] = pack_bf16(x.x, x.y);
        lo[j] = pack_bf16(x.x - bf16lo(hi[j]), x.y - bf16hi(hi[j]));
      }
    }
    return (sum0.x + sum0.y) + (sum1.x + sum1.y);
  }

  // A new reference from columns 32 c .. of the tile for a row that needs one
  // (`over`): its accumulator, its sums and the weights of the tile's earlier
  // columns are scaled to it (by a power of two).  `acc`: there is an accumulator.
  __device__ __forceinline__ void regrow(uint32_t tS, uint32_t tO, int c, const Meta& mt, bool over, bool acc,
                                         float& sum) {
    float mx = -INFINITY;
    um::wait_st();  // earlier columns' weights are read back below
    {
      uint32_t r[32];
      um::ld32(tS + 32u * c, r);
#pragma unroll
      for (int j = 0; j < 32; ++j) {
        const float x = __uint_as_float(r[j]);
        mx = fmaxf(mx, QUANT ? fmaf(x * mt.ks[32 * c + j], sl, mt.lv[32 * c + j]) : x);
      }
    }
    const float nc = reference(mx);
    float f = 1.f;
    if (over && nc > C) {
      // the factor of a step of 2^127 and more is 0, but may leave much of a quantised sum: in two
      const float half = QUANT ? floorf(0.5f * (C - nc)) : 0.f, g = um::ex2(half);
      f = um::ex2(C - nc - half);
      lsum *= g;
      sum *= g;
      lsum *= f;
      sum *= f;
      f *= g;
      C = nc;
    }
    if (acc) {
#pragma unroll 1
      for (int i = 0; i < 4; ++i) {
        uint32_t r[32];
        um::ld32(tO + 32u * i, r);
#pragma unroll
        for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(__uint_as_float(r[j]) * f);
        um::st32(tO + 32u * i, r);
      }
    }
#pragma unroll 1
    for (int i = 0; i < (QUANT ? c : 2 * c); ++i) {  // sixteen columns each
      const uint32_t at = tS + (QUANT ? 32u * i : 16u * i);
      uint32_t r[16];
      um::ld16(at, r);
#pragma unroll
      for (int j = 0; j < 16; ++j) {
        if (QUANT) {
          const float2 x = f16x2_to_f32(r[j]);
          r[j] = pack_f16(x.x * f, x.y * f);
        } else {
          r[j] = pack_bf16(bf16lo(r[j]) * f, bf16hi(r[j]) * f);
        }
      }
      um::st16(at, r);
    }
  }

  // One tile: its weights are written over its logits as the MMAs' A operand, 16
  // columns of every 32 (for bf16 the next 16 hold the remainders).  The
  // reference at hand is tried first: only columns whose weights leave the
  // range have their maximum taken and the reference moved.
  __device__ __forceinline__ void tile(uint32_t tS, uint32_t tO, const Meta& mt, bool acc) {
    if (__any_sync(kFull, C == -INFINITY)) {  // a row that has met nothing yet: no accumulator to scale
      const float mx = tile_max<QUANT>(tS, mt, sl);
      if (C == -INFINITY) C = reference(mx);
    }
    float sum = 0.f;
    bool again = false;
#pragma unroll 1
    for (int c = 0; c < 4;) {
      uint32_t hi[16], lo[16];
      uint32_t top = 0;
      const float x = chunk(tS, c, mt, offset(), hi, lo, top);
      const bool over = !(x < kLimit) || (QUANT && __vmaxu2(top, kTop) != kTop);
      if (!again && __any_sync(kFull, over)) {
        regrow(tS, tO, c, mt, over, acc, sum);
        again = true;
        continue;
      }
      again = false;
      um::st16(tS + 32u * c, hi);
      if (!QUANT) um::st16(tS + 32u * c + 16u, lo);
      sum += x;
      ++c;
    }
    lsum += sum;
  }
};

template <int FMT, bool PAIR>
__device__ __forceinline__ void softmax(const TreeArgs& p, Misc* m, uint32_t base, uint32_t tmem,
                                        int tid, const int64_t* first, int64_t per) {
  constexpr bool kQuant = FMT != CERTKV_STORE_BF16;
  volatile int* ab = &m->abort;
  const int warp = tid >> 5, lane = tid & 31, s = warp >> 2, quad = warp & 3;
  const int lrow = quad * 32 + lane;  // row of the stream, lane of tensor memory
  const int brow = PAIR ? 128 * s + lrow : lrow;  // row of the block
  const bool busy = (PAIR ? 128 * s : 0) + quad * 32 < p.rb;  // some block has a row here
  const uint32_t tS = tmem + kColS + 128u * s + ((uint32_t)(quad * 32) << 16);
  const uint32_t tO = tmem + kColO + 128u * s + ((uint32_t)(quad * 32) << 16);
  uint32_t t0 = 0, uses = 0, finals = 0;  // tiles before; S and final O of this stream so far
  bool ok = true;                         // false after a wait gave up, for good
  Items items(p, first, per);
  Item it;
  while (items.next(p, &it)) {
    const int rows = min(p.rb, p.rows - it.blk * p.rb);  // of the block
    const int bl = it.u / p.H, h = it.u - bl * p.H, b = bl / p.L, l = bl - b * p.L;
    // ---- queries into shared memory: 16 lanes a row, eight rows in flight a thread
#pragma unroll 1
    for (int r0 = tid >> 4; r0 < (PAIR ? 256 : 128); r0 += 128) {
      uint4 x[8];
      const int c = tid & 15;
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = r0 + 16 * i;
        x[i] = make_uint4(0u, 0u, 0u, 0u);
        if (r < rows) {
          const int br = it.blk * p.rb + r, t = br / p.G, g = br - t * p.G;
          x[i] = __ldg(reinterpret_cast<const uint4*>(p.q.at(b, l, t, h * p.G + g)) + c);
        }
      }
#pragma unroll
      for (int i = 0; i < 8; ++i) {
        const int r = r0 + 16 * i;
        uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
        if (kQuant) {
          uint32_t top = 0;
#pragma unroll
          for (int j = 0; j < 4; ++j) top = max(top, max((w[j] & 0x7fffu) << 16, w[j] & 0x7fff0000u));
#pragma unroll
          for (int o = 1; o < 16; o <<= 1) top = max(top, __shfl_xor_sync(kFull, top, o));
          const int e = min(max(exponent(__uint_as_float(top)), -120), 120);
          const float f = pow2(-e);
#pragma unroll
          for (int j = 0; j < 4; ++j)
            w[j] = pack_f16(__uint_as_float(w[j] << 16) * f, __uint_as_float(w[j] & 0xffff0000u) * f);
          if (c == 0) m->qs[r] = pow2(e);
        }
        sts128(base + (uint32_t)((r >> 7) * kOperand + (c >> 3) * kHalf + (r & 127) * 128 +
                                 (((c & 7) ^ (r & 7)) << 4)),
               w[0], w[1], w[2], w[3]);
      }
    }
    um::fence_async();
    softmax_sync();  // also: qs of every row is there
    Row<kQuant> row;
    row.sl = fmaxf(kQuant ? m->qs[brow] * p.scale_log2 : p.scale_log2, 1.1754944e-38f);
    __syncwarp();
    if (lane == 0) tc::mbar_arrive(bar(&m->q_full));  // rows written, qs read by the warp

    const int n = it.kb - it.ka, steps = PAIR ? n : (n - s + 1) / 2;
    const int tok = (it.blk * p.rb + min(brow, rows - 1)) / p.G;
    const uint64_t word = p.kn.p ? seen(p, b, tok) : 0ull;
    for (int i = 0; busy && i < steps; ++i) {
      const uint32_t t = t0 + (uint32_t)(PAIR ? i : 2 * i + s);
      // the tile's facts are there long before its logits: asked for first, the poll
      // and the reads pass while S is awaited
      ok = ok && __all_sync(kFull, tc::mbar_wait(bar(&m->ready[t % kMeta]), (t / kMeta) & 1u, ab));
      const Meta& mt = m->meta[t % kMeta];
      const bool whole = mt.whole, own = mt.drafts;
      ok = ok && __all_sync(kFull, tc::mbar_wait(bar(&m->s_full[s]), uses & 1u, ab));
      ++uses;
      if (!ok) break;
      um::fence_after();
      if (!whole) {
        const uint32_t live[4] = {own ? (uint32_t)word : mt.live[0], own ? (uint32_t)(word >> 32) : mt.live[1],
                                  own ? 0u : mt.live[2], own ? 0u : mt.live[3]};
        mask_tile(tS, live);
      }
      row.tile(tS, tO, mt, i > 0);  // O of the tiles before is done (see Issuer)
      um::wait_st();
      um::fence_before();
      __syncwarp();
      if (lane == 0) {
        tc::mbar_arrive(bar(&m->p_full[s]));
        tc::mbar_arrive(bar(&m->back[t % kMeta]));
      }
    }
    // ---- the item's result: one record per row
    if (ok && busy && steps > 0) {
      ok = __all_sync(kFull, tc::mbar_wait(bar(&m->o_full[s]), finals & 1u, ab));
      ++finals;
    }
    um::fence_after();
    const bool both = !PAIR && n > 1;  // join the streams: stream 0 writes
    if (!PAIR && s == 1 && busy) {
      m->cm[lrow] = row.C;
      m->l[lrow] = row.lsum;
    }
    um::fence_before();
    softmax_sync();  // from here on nothing reads the queries any more either
    um::fence_after();
    if (busy && (PAIR || s == 0)) {
      // sum and accumulator are relative to 2^C; a quantised store's C goes with the values, so
      // the sum's own exponent is taken into the record's reference
      const float C = row.C, lsum = row.lsum, C1 = both ? m->cm[lrow] : -INFINITY, l1 = both ? m->l[lrow] : 0.f;
      const float Cj = fmaxf(C + (kQuant ? (float)exponent(lsum) : 0.f), C1 + (kQuant ? (float)exponent(l1) : 0.f));
      const float f0 = C == -INFINITY ? 0.f : exp2f(C - Cj), f1 = C1 == -INFINITY ? 0.f : exp2f(C1 - Cj);
      const float lj = both ? lsum * f0 + l1 * f1 : C == -INFINITY ? lsum : lsum * f0;
      const float inv = lj != 0.f ? 1.f / lj : 0.f, g0 = f0 * inv, g1 = f1 * inv;
      const int64_t rec = ((int64_t)blockIdx.x + (int64_t)it.u * p.nblk + it.blk) * p.rb + brow;
      const bool mine = brow < rows;
#pragma unroll 1
      for (int c = 0; c < 8; ++c) {
        uint32_t r[16];
        um::ld16(tO + 16u * c, r);
#pragma unroll
        for (int j = 0; j < 16; ++j) r[j] = g0 == 0.f ? 0u : __float_as_uint(__uint_as_float(r[j]) * g0);
        if (both) {
          uint32_t r1[16];
          um::ld16(tO + 128u + 16u * c, r1);
#pragma unroll
          for (int j = 0; j < 16; ++j)
            if (g1 != 0.f) r[j] = __float_as_uint(fmaf(__uint_as_float(r1[j]), g1, __uint_as_float(r[j])));
        }
        if (mine) {
#pragma unroll
          for (int j = 0; j < 16; j += 8)  // whole sectors
            asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(
                             p.rec_acc + rec * kD + 16 * c + j),
                         "r"(r[j]), "r"(r[j + 1]), "r"(r[j + 2]), "r"(r[j + 3]), "r"(r[j + 4]), "r"(r[j + 5]),
                         "r"(r[j + 6]), "r"(r[j + 7])
                         : "memory");
        }
      }
      // a stream that gave up has handed over what it had
      if (mine) p.rec_ml[rec] = tree_record(ok, *ab != 0, Cj, lj);
    }
    um::fence_before();
    t0 += n;
  }
}

template <int N>
__device__ __forceinline__ void regs_up() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void regs_down() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}

// grid = p.ctas (one CTA per SM), block = kThreads; PAIR: blocks of more than
// 128 rows.
template <int FMT, bool PAIR>
__global__ void __launch_bounds__(kThreads, 1) tree_tc_kernel(const __grid_constant__ CUtensorMap tmK,
                                                              const __grid_constant__ CUtensorMap tmV,
                                                              const __grid_constant__ TreeArgs p) {
  extern __shared__ char smem_raw[];
  char* sm = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  Misc* m = reinterpret_cast<Misc*>(sm + Plan<PAIR>::kMiscOff);
  const int warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    for (int i = 0; i < Plan<PAIR>::kRing; ++i) {
      tc::mbar_init(bar(&m->full[i]), kGroupWarps + (FMT == CERTKV_STORE_BF16));  // a group, and the scout
      tc::mbar_init(bar(&m->empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      const int rows = PAIR ? (i ? p.rb - 128 : 128) : p.rb;
      tc::mbar_init(bar(&m->s_full[i]), 1);
      tc::mbar_init(bar(&m->p_full[i]), (rows + 31) / 32);  // the warps with rows
      tc::mbar_init(bar(&m->o_full[i]), 1);
    }
    for (uint32_t i = 0; i < kMeta; ++i) {
      tc::mbar_init(bar(&m->stated[i]), 1);
      tc::mbar_init(bar(&m->ready[i]), 1);
      tc::mbar_init(bar(&m->back[i]), kGroupWarps + (p.rb + 31) / 32);  // the values' group, the softmax warps
    }
    for (int i = 0; i < kLoadGroups; ++i) tc::mbar_init(bar(&m->group[i]), kGroupWarps);
    tc::mbar_init(bar(&m->q_full), kSoftWarps);
    tc::mbar_init(bar(&m->done), 1);
    m->abort = 0;
    m->walked = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  release_next();
  await_previous();
  const int64_t* first = tree_first(p, m->first, kTreeTile, p.kn.p != nullptr);
  const int64_t per = tiles_per_cta(p, first), left = first[p.units] * p.nblk - per * blockIdx.x;
  if (left <= 0) return;  // uniform, before any barrier
  const uint32_t n = (uint32_t)min(left, per);  // tiles of this CTA
  if (warp == kSoftWarps + kLoadWarps) um::alloc(tc::saddr(&m->tmem), 512);
  um::fence_before();
  __syncthreads();
  um::fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&m->tmem);
  const uint32_t base = tc::saddr(sm);
  if (warp < kSoftWarps) {
    regs_up<kSoftRegs>();
    softmax<FMT, PAIR>(p, m, base, tmem, threadIdx.x, first, per);
  } else if (warp < kSoftWarps + kLoadWarps) {
    regs_down<kLoadRegs>();
    const int tid = (int)threadIdx.x - kSoftWarps * 32;
    const int group = tid / (kGroupWarps * 32), gt = tid % (kGroupWarps * 32);
    Loader<FMT, PAIR> ld{p, m, base + Plan<PAIR>::kRingOff, group, gt, Piece(gt)};
    ld.run(n);
  } else {
    regs_down<kIssueRegs>();
    if (warp == kSoftWarps + kLoadWarps) {
      Issuer<FMT, PAIR> is{m, tmem, base, base + Plan<PAIR>::kRingOff, n};
      is.run(p, first, per);
    } else if (warp == kSoftWarps + kLoadWarps + 1) {
      Scout<FMT, PAIR> sc{p, m, &tmK, &tmV, base + Plan<PAIR>::kRingOff, (int)threadIdx.x & 31, true, Items(p, first, per)};
      sc.run(n);
    } else if (warp == kSoftWarps + kLoadWarps + 2) {
      Scout<FMT, PAIR> sc{p, m, &tmK, &tmV, base + Plan<PAIR>::kRingOff, (int)threadIdx.x & 31, true, Items(p, first, per)};
      if (FMT == CERTKV_STORE_BF16) sc.run_values(n);
      else sc.run_ahead(n);
    }
    __syncwarp();
  }
  um::fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && m->abort && p.st.status) atomicOr(p.st.status, CERTKV_STATUS_TIMEOUT);
  if (warp == kSoftWarps + kLoadWarps) {
    um::fence_after();
    um::dealloc(tmem, 512);
  }
}

constexpr int kMaxDevices = 64;

template <int FMT, bool PAIR>
bool opt_in() {
  return cudaFuncSetAttribute(tree_tc_kernel<FMT, PAIR>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              smem_bytes<PAIR>()) == cudaSuccess;
}

// CTAs: one per SM.  Set up once per device: the shared-memory opt-in.
int ctas_of_device() {
  static int cached[kMaxDevices] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return 0;
  if (dev < kMaxDevices && cached[dev] > 0) return cached[dev];
  int sms = 0;
  if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1 ||
      !opt_in<CERTKV_STORE_BF16, true>() || !opt_in<CERTKV_STORE_BF16, false>() ||
      !opt_in<CERTKV_STORE_FP8, true>() || !opt_in<CERTKV_STORE_FP8, false>() ||
      !opt_in<CERTKV_STORE_FP4, true>() || !opt_in<CERTKV_STORE_FP4, false>())
    return 0;
  if (dev < kMaxDevices) cached[dev] = sms;
  return sms;
}

template <int FMT>
bool launch(const CUtensorMap& mk, const CUtensorMap& mv, const TreeArgs& p, cudaStream_t st) {
  return p.rb > 128
             ? launch_kernel(true, tree_tc_kernel<FMT, true>, p.ctas, kThreads, smem_bytes<true>(), st, mk, mv, p)
             : launch_kernel(true, tree_tc_kernel<FMT, false>, p.ctas, kThreads, smem_bytes<false>(), st, mk, mv, p);
}

}  // namespace

int tree_ctas() { return ctas_of_device(); }

bool launch_tree_tc(const TreeArgs& p, int format, cudaStream_t st) {
  CUtensorMap mk = {}, mv = {};
  if (format == CERTKV_STORE_BF16) {
    const uint64_t rows = (uint64_t)p.st.pool_pages * kPage;
    if (!make_row_map(&mk, p.st.k, rows, kPage) || !make_row_map(&mv, p.st.v, rows, kPage)) return false;
  }
  TraceScope ts_("tree_split", st);
  return format == CERTKV_STORE_BF16  ? launch<CERTKV_STORE_BF16>(mk, mv, p, st)
         : format == CERTKV_STORE_FP8 ? launch<CERTKV_STORE_FP8>(mk, mv, p, st)
                                      : launch<CERTKV_STORE_FP4>(mk, mv, p, st);
}

}  // namespace certkv
