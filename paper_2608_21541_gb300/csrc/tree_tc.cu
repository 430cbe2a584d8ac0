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
//   warps 8..15  loaders: bf16 tiles by TMA; 8- and 4-bit tiles through
//                registers, expanded to f16 in the MMAs' swizzled layout; the
//                drafts' own tile in either case;
//   warp 16      tensor-memory allocation, and the thread that issues the MMAs.
//
// Precision.  bf16 store: bf16 products, and a weight enters P V as a bf16 part
// plus the bf16 rounding of its remainder (2^-16).  8- and 4-bit stores: codes
// are exact in f16, so are query rows once divided by a power of two; a key's
// fp32 scale multiplies its logit; a value is rounded once to f16 (2^-11) with
// its scale taken relative to the tile's largest, and a weight once to f16.
// Logits, sums, and accumulators are fp32.  A weight is 2^(x - C) for a
// reference C that follows the row's maximum only when it grows by more than
// 2^8, which keeps weights in f16's range and most tiles free of rescaling.
//
// Every wait is bounded; on a timeout the roles stop waiting, the rows in
// question read NaN and the store's status word gets CERTKV_STATUS_TIMEOUT.
#include <cuda.h>

#include "../../include/certkv.h"
#include "common.cuh"
#include "internal.cuh"
#include "tma.cuh"
#include "tree.cuh"
#include "umma.cuh"

namespace certkv {
namespace {

constexpr int kSoftWarps = 8, kLoadWarps = 8;
constexpr int kThreads = (kSoftWarps + kLoadWarps + 1) * 32;
constexpr int kLoaders = kLoadWarps * 32;
constexpr int kStages = 2;
constexpr int kMeta = 4;  // see Meta
constexpr int kHalf = 128 * 128;           // bytes of 128 rows x 64 16-bit elements
constexpr int kOperand = 2 * kHalf;        // 128 rows x 128 elements
constexpr int kQOff = 0;                   // two row blocks
constexpr int kKVOff = 2 * kOperand;       // stages of K | V
constexpr int kMiscOff = kKVOff + kStages * 2 * kOperand;
constexpr uint32_t kColS = 0, kColO = 256; // + 128 stream
constexpr float kLazy = 8.f;               // growth of the maximum that moves the reference

// Per-tile facts for the softmax.  Slot t % kMeta is written again with tile
// t + kMeta, whose key stage is free only once the products with tile
// t + kMeta - kStages are done; those were issued after P of tile t had been
// written, so the softmax has read slot t by then (kMeta >= kStages + 2).
struct Meta {
  float ks[kTreeTile];  // scale of the key of each slot (8- and 4-bit stores)
  uint32_t live[4];     // slots to take
  int shift;            // exponent the tile's values were divided by
  int whole;            // every slot is live
  int drafts;           // the drafts' own tile: live comes from the row's mask
  int pad;
};

struct Misc {
  uint64_t k_full[kStages], k_empty[kStages], v_full[kStages], v_empty[kStages];
  uint64_t s_full[2], p_full[2], o_full[2], q_full, meta_full[kMeta], done;
  uint32_t tmem;
  int abort;
  unsigned long long odd;
  float red[kLoadWarps];
  float qs[256];                    // per row: scale of its f16 queries
  float cm[128], l[128], sh[128];   // stream 1's reference, sum and shift
  Meta meta[kMeta];
};
constexpr int kSmemBytes = kMiscOff + (int)sizeof(Misc) + 1024;
static_assert(kSmemBytes <= 232448, "over the 227 KB of shared memory a CTA can have");

__device__ __forceinline__ uint32_t bar(const uint64_t* b) { return tc::saddr(b); }
__device__ __forceinline__ void loaders_sync() {
  asm volatile("bar.sync 1, %0;" ::"n"(kLoaders) : "memory");
}
__device__ __forceinline__ void softmax_sync() {
  asm volatile("bar.sync 2, %0;" ::"n"(kSoftWarps * 32) : "memory");
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

// The 32 bytes of elements 16 sub .. 16 sub + 15 of a row into the swizzled
// operand at `base`.  The eight lanes of a row store their two chunks in
// opposite order above and below element 64, so that they meet different banks.
__device__ __forceinline__ void put32(uint32_t base, int row, int sub, const uint32_t (&w)[8]) {
  const uint32_t r = base + (uint32_t)((sub >> 2) * kHalf + row * 128);
  const int c = 2 * (sub & 3), x = row & 7;
  const uint32_t a0 = r + (uint32_t)((c ^ x) << 4), a1 = r + (uint32_t)(((c + 1) ^ x) << 4);
  if (sub < 4) {
    sts128(a0, w[0], w[1], w[2], w[3]);
    sts128(a1, w[4], w[5], w[6], w[7]);
  } else {
    sts128(a1, w[4], w[5], w[6], w[7]);
    sts128(a0, w[0], w[1], w[2], w[3]);
  }
}

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

// Raw codes of this thread's four (slot, 16-element) pieces of one operand.
template <int FMT>
struct Raw {
  uint32_t w[4][FMT == CERTKV_STORE_FP8 ? 4 : 2];
  uint32_t g[FMT == CERTKV_STORE_FP4 ? 4 : 1];
};

template <int FMT>
__device__ __forceinline__ void load_raw(Raw<FMT>& r, const int64_t (&at)[4], int sub,
                                         const uint8_t* codes, const uint8_t* group) {
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    if (FMT == CERTKV_STORE_FP8) {
      uint4 x = make_uint4(0u, 0u, 0u, 0u);
      if (at[i] >= 0) x = __ldg(reinterpret_cast<const uint4*>(codes + at[i] * 128 + sub * 16));
      r.w[i][0] = x.x;
      r.w[i][1] = x.y;
      r.w[i][2 % (FMT == CERTKV_STORE_FP8 ? 4 : 2)] = x.z;
      r.w[i][3 % (FMT == CERTKV_STORE_FP8 ? 4 : 2)] = x.w;
    } else {
      uint2 x = make_uint2(0u, 0u);
      uint32_t g = 0;
      if (at[i] >= 0) {
        x = __ldg(reinterpret_cast<const uint2*>(codes + at[i] * 64 + sub * 8));
        g = __ldg(group + at[i] * kGroups + sub);
      }
      r.w[i][0] = x.x;
      r.w[i][1] = x.y;
      r.g[i % (FMT == CERTKV_STORE_FP4 ? 4 : 1)] = g;
    }
  }
}

// One piece as f16: codes (with their group scale) times f; f unused for keys.
template <int FMT, bool VALUE>
__device__ __forceinline__ void expand(const Raw<FMT>& r, int i, float f, uint32_t (&w)[8]) {
  if (FMT == CERTKV_STORE_FP8) {
    const uint32_t f2 = VALUE ? pack_f16(f, f) : 0u;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      w[j] = e4m3x2_to_f16x2(r.w[i][(j >> 1) % (FMT == CERTKV_STORE_FP8 ? 4 : 2)] >> (16 * (j & 1)));
      if (VALUE) w[j] = hmul2(w[j], f2);
    }
  } else {
    const float gs = f16x2_to_f32(e4m3x2_to_f16x2(r.g[i % (FMT == CERTKV_STORE_FP4 ? 4 : 1)])).x;
    const float x = VALUE ? gs * f : gs;
    const uint32_t f2 = pack_f16(x, x);
#pragma unroll
    for (int j = 0; j < 2; ++j) {
      w[4 * j] = hmul2(e2m1x2_to_f16x2<0>(r.w[i][j]), f2);
      w[4 * j + 1] = hmul2(e2m1x2_to_f16x2<1>(r.w[i][j]), f2);
      w[4 * j + 2] = hmul2(e2m1x2_to_f16x2<2>(r.w[i][j]), f2);
      w[4 * j + 3] = hmul2(e2m1x2_to_f16x2<3>(r.w[i][j]), f2);
    }
  }
}

// --------------------------------------------------------------- loaders --
template <int FMT>
struct Loader {
  static constexpr bool kQuant = FMT != CERTKV_STORE_BF16;
  using Pieces = Raw<kQuant ? FMT : CERTKV_STORE_FP8>;
  const TreeArgs& p;
  Misc* m;
  const CUtensorMap *tmK, *tmV;
  uint32_t kv0;
  int tid, warp, lane, grp, sub;
  volatile int* ab;
  bool ok = true;    // false after a wait gave up; the walk over the tiles goes on (the
                     // loaders' barriers must stay in step) without further copies
  int64_t tile = 0;  // tiles of this CTA so far
  int pages_at = 0, pages_lo = -1, pages_hi = -1;  // table entries of 64 pages from pages_at on
  uint32_t k_copy = 0, v_copy = 0;  // stages whose last tile came by bulk copy

  __device__ __forceinline__ Loader(const TreeArgs& p_, Misc* m_, uint32_t kv, const CUtensorMap* a,
                                    const CUtensorMap* b, int tid_)
      : p(p_), m(m_), tmK(a), tmV(b), kv0(kv), tid(tid_) {
    warp = tid >> 5;
    lane = tid & 31;
    grp = tid >> 3;
    sub = tid & 7;
    ab = &m->abort;
  }

  __device__ __forceinline__ int entry(int u, int page) const {
    if (page >= p.st.max_pages) return -1;
    const int e = __ldg(p.st.table + (int64_t)u * p.st.max_pages + page);
    return e >= 0 && e < p.st.pool_pages ? e : -1;
  }
  // Pages of tile k (-1: none).  Every lane of the warp; k ascends by one after
  // `start`.
  __device__ __forceinline__ void pages(int u, int k, bool start, int& a, int& b) {
    const int page = 2 * k;
    if (start) {
      pages_at = page;
      pages_lo = entry(u, page + lane);
      pages_hi = entry(u, page + 32 + lane);
    } else if (page >= pages_at + 32) {
      pages_at += 32;
      pages_lo = pages_hi;
      pages_hi = entry(u, pages_at + 32 + lane);
    }
    a = __shfl_sync(kFull, pages_lo, page - pages_at);
    b = __shfl_sync(kFull, pages_lo, page + 1 - pages_at);
  }
  // Pool slots of this thread's pieces (slots grp + 32 i of the tile; -1: none).
  __device__ __forceinline__ void pieces(int a, int b, int live, int64_t (&at)[4]) const {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int s = grp + 32 * i, page = i < 2 ? a : b;
      at[i] = s < live && page >= 0 ? (int64_t)page * kPage + (s & (kPage - 1)) : -1;
    }
  }
  // Scales of slots 4 lane .. 4 lane + 3 of the tile (0: no slot).
  __device__ __forceinline__ float4 scales(const float* s, int a, int b, int live) const {
    const int page = lane < 16 ? a : b, n = live - 4 * lane;
    float4 x = make_float4(0.f, 0.f, 0.f, 0.f);
    if (page >= 0)
      x = __ldg(reinterpret_cast<const float4*>(s + (int64_t)page * kPage + ((4 * lane) & (kPage - 1))));
    if (n < 1) x.x = 0.f;
    if (n < 2) x.y = 0.f;
    if (n < 3) x.z = 0.f;
    if (n < 4) x.w = 0.f;
    return x;
  }
  __device__ __forceinline__ void wait(const uint64_t* b) {  // a stage's earlier use
    if (ok && tile >= kStages) ok = tc::mbar_wait(bar(b), (uint32_t)((tile / kStages - 1) & 1), ab);
  }
  __device__ __forceinline__ void arrive(const uint64_t* b) const {
    um::fence_async();
    __syncwarp();
    if (lane == 0) tc::mbar_arrive(bar(b));
  }
  // One operand of a whole bf16 tile: two pages, two 64-element halves.
  __device__ __forceinline__ void copy(const CUtensorMap* map, uint32_t to, const uint64_t* full, int a,
                                       int b) const {
    if (!ok) return;
    if (tid == 0) {
      tc::mbar_expect_tx(bar(full), kOperand);
      tc::tma_load_2d(to, map, 0, a * kPage, bar(full));
      tc::tma_load_2d(to + kHalf, map, 64, a * kPage, bar(full));
      tc::tma_load_2d(to + kHalf / 2, map, 0, b * kPage, bar(full));
      tc::tma_load_2d(to + kHalf + kHalf / 2, map, 64, b * kPage, bar(full));
    } else if (lane == 0) {
      tc::mbar_arrive(bar(full));
    }
  }
  // The exponent that brings the largest magnitude t to 2^13 .. 2^14.
  __device__ __forceinline__ int shift_of(float t) const {
    return t > 0.f && t < INFINITY ? min(max(exponent(t) - 13, -110), 114) : 0;
  }

  // The drafts' own tile: bf16 rows, converted for the 8- and 4-bit stores.
  __device__ __forceinline__ void drafts(int u, bool first_block) {
    const int st = (int)(tile % kStages);
    const uint32_t kb = kv0 + (uint32_t)(st * 2 * kOperand), vb = kb + kOperand;
    wait(&m->k_empty[st]);
    k_copy &= ~(1u << st);
    Meta& mt = m->meta[tile % kMeta];
    const int bl = u / p.H, h = u - bl * p.H, b = bl / p.L, l = bl - b * p.L;
    uint32_t v[2][8], top = 0;
    if (tid == 0) m->odd = 0ull;
    loaders_sync();
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t k[8] = {};
      const int s = grp + 32 * i;
      if (i < 2) {
        // values: a NaN or infinity is left out of the product (it would reach
        // every row, seen or not); the merge adds it to the rows that see its draft
        bool odd = false;
#pragma unroll
        for (int j = 0; j < 8; ++j) v[i & 1][j] = 0u;
        if (s < p.T) {
          load32g(p.kn.at(b, l, s, h) + sub * 16, k);
          load32g(p.vn.at(b, l, s, h) + sub * 16, v[i & 1]);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
          if ((v[i & 1][j] & 0x7f80u) == 0x7f80u) {
            v[i & 1][j] &= 0xffff0000u;
            odd = true;
          }
          if ((v[i & 1][j] & 0x7f800000u) == 0x7f800000u) {
            v[i & 1][j] &= 0xffffu;
            odd = true;
          }
        }
        if (odd) atomicOr(&m->odd, 1ull << s);
        top = max(top, top16(v[i & 1]));
        if (kQuant) {
          uint32_t kt = top16(k);
#pragma unroll
          for (int o = 1; o < 8; o <<= 1) kt = max(kt, __shfl_xor_sync(kFull, kt, o));
          const int e = min(max(exponent(__uint_as_float(kt)), -120), 120);
          to_f16(k, pow2(-e));
          if (sub == 0) mt.ks[s] = pow2(e);
        }
      } else if (kQuant && sub == 0) {
        mt.ks[s] = 0.f;
      }
      put32(kb, s, sub, k);
    }
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) top = max(top, __shfl_xor_sync(kFull, top, o));
    if (lane == 0) m->red[warp] = __uint_as_float(top);
    loaders_sync();
    int shift = 0;
    if (kQuant) {
      float t = 0.f;
#pragma unroll
      for (int i = 0; i < kLoadWarps; ++i) t = fmaxf(t, m->red[i]);
      shift = shift_of(t);
    }
    if (tid == 0) {
      mt.shift = shift;
      mt.whole = 0;
      mt.drafts = 1;
      if (first_block) p.odd[u] = m->odd;
      tc::mbar_arrive(bar(&m->meta_full[tile % kMeta]));
    }
    arrive(&m->k_full[st]);
    wait(&m->v_empty[st]);
    v_copy &= ~(1u << st);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      uint32_t w[8] = {};
      if (i < 2) {
#pragma unroll
        for (int j = 0; j < 8; ++j) w[j] = v[i & 1][j];
        if (kQuant) to_f16(w, pow2(-shift));
      }
      put32(vb, grp + 32 * i, sub, w);
    }
    arrive(&m->v_full[st]);
  }

  // Tiles [ka, ke) of the stored slots of segment u.
  __device__ __forceinline__ void stored(int u, int count, int ka, int ke) {
    Pieces kr, vr;
    float4 ks4 = {}, vs4 = {};
    float vs[4] = {};
    int64_t at[4];
    int a, b;
    pages(u, ka, true, a, b);
    if (kQuant) {
      const int live = count - ka * kTreeTile;
      pieces(a, b, live, at);
      load_raw(kr, at, sub, p.st.k, p.st.kg);
      ks4 = scales(p.st.ks, a, b, live);
      load_raw(vr, at, sub, p.st.v, p.st.vg);
      vs4 = scales(p.st.vs, a, b, live);
#pragma unroll
      for (int i = 0; i < 4; ++i) vs[i] = at[i] >= 0 ? __ldg(p.st.vs + at[i]) : 0.f;
    }
    for (int k = ka; k < ke; ++k, ++tile) {
      const int live = count - k * kTreeTile;
      const int st = (int)(tile % kStages), a0 = a, b0 = b;
      const uint32_t kb = kv0 + (uint32_t)(st * 2 * kOperand), vb = kb + kOperand;
      const bool whole = live >= kTreeTile && a >= 0 && b >= 0;
      int shift = 0;
      if (kQuant) {  // from the tile's largest row maximum, a NaN left out
        float t = fmaxf(fmaxf(vs4.x, vs4.y), fmaxf(vs4.z, vs4.w));
#pragma unroll
        for (int o = 16; o >= 1; o >>= 1) t = fmaxf(t, __shfl_xor_sync(kFull, t, o));
        shift = shift_of(t * (FMT == CERTKV_STORE_FP8 ? 448.f : 2688.f));
      }
      wait(&m->k_empty[st]);
      if (warp == 0) {
        Meta& mt = m->meta[tile % kMeta];
        if (kQuant) *reinterpret_cast<float4*>(&mt.ks[4 * lane]) = ks4;
        if (lane < 4) {
          const int n = min(max(live - 32 * lane, 0), 32);
          mt.live[lane] = (lane < 2 ? a : b) < 0 || n == 0 ? 0u : 0xffffffffu >> (32 - n);
        }
        if (lane == 0) {
          mt.shift = shift;
          mt.whole = whole;
          mt.drafts = 0;
          if (a < 0 || (b < 0 && live > kPage)) p.st.raise();
        }
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(bar(&m->meta_full[tile % kMeta]));
      }
      if (!kQuant && whole) {
        copy(tmK, kb, &m->k_full[st], a, b);
        k_copy |= 1u << st;
      } else {
        if (!kQuant) pieces(a, b, live, at);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t w[8] = {};
          if (kQuant) expand<kQuant ? FMT : CERTKV_STORE_FP8, false>(kr, i, 0.f, w);
          else if (at[i] >= 0) load32g(p.st.k + at[i] * 256 + sub * 32, w);
          put32(kb, grp + 32 * i, sub, w);
        }
        k_copy &= ~(1u << st);
        arrive(&m->k_full[st]);
      }
      const int next = count - (k + 1) * kTreeTile;
      if (k + 1 < ke) {
        pages(u, k + 1, false, a, b);
        if (kQuant) {
          pieces(a, b, next, at);
          load_raw(kr, at, sub, p.st.k, p.st.kg);
          ks4 = scales(p.st.ks, a, b, next);
          vs4 = scales(p.st.vs, a, b, next);
        }
      }
      wait(&m->v_empty[st]);
      if (!kQuant && whole) {
        copy(tmV, vb, &m->v_full[st], a0, b0);
        v_copy |= 1u << st;
      } else {
        if (!kQuant) pieces(a0, b0, live, at);
        const float down = pow2(-shift);
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t w[8] = {};
          if (kQuant) expand<kQuant ? FMT : CERTKV_STORE_FP8, true>(vr, i, vs[i] * down, w);
          else if (at[i] >= 0) load32g(p.st.v + at[i] * 256 + sub * 32, w);
          put32(vb, grp + 32 * i, sub, w);
        }
        v_copy &= ~(1u << st);
        arrive(&m->v_full[st]);
      }
      if (kQuant && k + 1 < ke) {
        load_raw(vr, at, sub, p.st.v, p.st.vg);
#pragma unroll
        for (int i = 0; i < 4; ++i) vs[i] = at[i] >= 0 ? __ldg(p.st.vs + at[i]) : 0.f;
      }
    }
  }

  __device__ __forceinline__ void run(int64_t per) {
    Items items(p, per);
    Item it;
    while (items.next(p, &it)) {
      const int count = p.st.count(it.u);
      const int nst = (count + kTreeTile - 1) / kTreeTile;  // tiles of stored slots
      if (it.ka < nst) stored(it.u, count, it.ka, min(it.kb, nst));
      if (it.kb > nst) {
        drafts(it.u, it.blk == 0);
        ++tile;
      }
    }
    if (!kQuant && tid == 0) {  // bulk copies land before the CTA may exit
      volatile int dummy = 0;
      for (int s = 0; s < kStages; ++s) {
        const int64_t t = (tile - 1 - s) / kStages * kStages + s;  // the last tile of stage s
        const uint32_t phase = (uint32_t)((t / kStages) & 1);
        if (tile > s && (k_copy >> s & 1)) tc::mbar_wait(bar(&m->k_full[s]), phase, &dummy);
        if (tile > s && (v_copy >> s & 1)) tc::mbar_wait(bar(&m->v_full[s]), phase, &dummy);
      }
    }
  }
};

// ------------------------------------------------------------ MMA issuer --
// Per item, products i = 0 .. N - 1 alternate between the streams: product i
// belongs to stream i & 1 and, with both streams on every tile (`pair`), to
// tile i / 2, else to tile i.  Issued in the order S(0), S(1), then O(i),
// S(i + 2): S(i + 2) overwrites what O(i) has read, which the tensor core's
// in-order execution makes safe, and its completion tells the softmax that
// O(i) is done.
template <int FMT>
__device__ __forceinline__ void issue(const TreeArgs& p, Misc* m, uint32_t base, uint32_t tmem,
                                      int64_t per) {
  constexpr bool kBf16 = FMT == CERTKV_STORE_BF16;
  volatile int* ab = &m->abort;
  const bool pair = p.rb > 128;
  const uint64_t qd = um::desc(base + kQOff, 16), kd = um::desc(base + kKVOff, 16);
  const uint64_t vd = um::desc(base + kKVOff + kOperand, kHalf);
  constexpr uint32_t idS = um::idesc(kBf16, false), idO = um::idesc(kBf16, true);
  int64_t tile0 = 0;             // tiles of this CTA before the item
  uint32_t uses[2] = {0u, 0u};   // products of each stream so far
  uint32_t item = 0;
  bool ok = true;
  Items items(p, per);
  Item it;
  auto stage_phase = [](int64_t t) { return (uint32_t)((t / kStages) & 1); };
  while (ok && items.next(p, &it)) {
    ok = tc::mbar_wait(bar(&m->q_full), item & 1, ab);
    if (!ok) break;
    um::fence_after();
    const int n = it.kb - it.ka, N = pair ? 2 * n : n;
    auto issue_s = [&](int i) {
      const int s = i & 1;
      const int64_t t = tile0 + (pair ? i >> 1 : i);
      const int st = (int)(t % kStages);
      if ((!pair || s == 0) && !tc::mbar_wait(bar(&m->k_full[st]), stage_phase(t), ab)) return false;
      um::fence_after();
      const uint64_t a = qd + (uint64_t)((pair && s ? kOperand : 0) >> 4);
      const uint64_t b = kd + (uint64_t)((st * 2 * kOperand) >> 4);
      const uint32_t d = tmem + kColS + 128u * s;
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) {
        const uint64_t o = (uint64_t)(((ks >> 2) * kHalf + (ks & 3) * 32) >> 4);
        um::mma_ss(d, a + o, b + o, idS, ks > 0);
      }
      um::commit(bar(&m->s_full[s]));
      if (!pair || s == 1) um::commit(bar(&m->k_empty[st]));
      return true;
    };
    auto issue_o = [&](int i) {
      const int s = i & 1;
      const int64_t t = tile0 + (pair ? i >> 1 : i);
      const int st = (int)(t % kStages);
      if (!tc::mbar_wait(bar(&m->p_full[s]), uses[s] & 1, ab)) return false;
      ++uses[s];
      if ((!pair || s == 0) && !tc::mbar_wait(bar(&m->v_full[st]), stage_phase(t), ab)) return false;
      um::fence_after();
      const uint64_t b = vd + (uint64_t)((st * 2 * kOperand) >> 4);
      const uint32_t d = tmem + kColO + 128u * s, a = tmem + kColS + 128u * s;
      const bool first = i < 2;
#pragma unroll
      for (int ks = 0; ks < 8; ++ks) {  // 16 slots each: 8 columns of P
        const uint32_t pa = a + (uint32_t)((ks >> 1) * 32 + (ks & 1) * 8);
        const uint64_t bb = b + (uint64_t)((ks * 2048) >> 4);
        um::mma_ts(d, pa, bb, idO, !first || ks > 0);
        if (kBf16) um::mma_ts(d, pa + 16, bb, idO, true);  // the remainders
      }
      if (!pair || s == 1) um::commit(bar(&m->v_empty[st]));
      if (i + 2 >= N) um::commit(bar(&m->o_full[s]));
      return true;
    };
    ok = issue_s(0) && (N < 2 || issue_s(1));
    for (int i = 0; ok && i < N; ++i) ok = issue_o(i) && (i + 2 >= N || issue_s(i + 2));
    tile0 += n;
    ++item;
  }
  um::commit(bar(&m->done));  // everything issued above has finished
  volatile int dummy = 0;
  tc::mbar_wait(bar(&m->done), 0, &dummy);
}

// --------------------------------------------------------------- softmax --
template <int FMT>
__device__ __forceinline__ void softmax(const TreeArgs& p, Misc* m, uint32_t base, uint32_t tmem,
                                        int tid, int64_t per) {
  constexpr bool kQuant = FMT != CERTKV_STORE_BF16;
  volatile int* ab = &m->abort;
  const bool pair = p.rb > 128;
  const int warp = tid >> 5, lane = tid & 31, s = warp >> 2, quad = warp & 3;
  const int lrow = quad * 32 + lane;  // row of the stream, lane of tensor memory
  const uint32_t tS = tmem + kColS + 128u * s + ((uint32_t)(quad * 32) << 16);
  const uint32_t tO = tmem + kColO + 128u * s + ((uint32_t)(quad * 32) << 16);
  int64_t tile0 = 0;
  uint32_t uses = 0, finals = 0;  // S and final O of this stream so far
  bool ok = true;                 // false after a wait gave up, for good
  Items items(p, per);
  Item it;
  while (items.next(p, &it)) {
    const int rows = min(p.rb, p.rows - it.blk * p.rb);  // of the block
    const int bl = it.u / p.H, h = it.u - bl * p.H, b = bl / p.L, l = bl - b * p.L;
    // ---- queries into shared memory: 16 lanes a row
    const int qrows = pair ? 256 : 128;
    for (int r = tid >> 4; r < qrows; r += 16) {
      uint4 x = make_uint4(0u, 0u, 0u, 0u);
      const int c = tid & 15;
      if (r < rows) {
        const int row = it.blk * p.rb + r, t = row / p.G, g = row - t * p.G;
        x = __ldg(reinterpret_cast<const uint4*>(p.q.at(b, l, t, h * p.G + g)) + c);
      }
      if (kQuant) {
        uint32_t w[4] = {x.x, x.y, x.z, x.w}, top = 0;
#pragma unroll
        for (int j = 0; j < 4; ++j) top = max(top, max((w[j] & 0x7fffu) << 16, w[j] & 0x7fff0000u));
#pragma unroll
        for (int o = 1; o < 16; o <<= 1) top = max(top, __shfl_xor_sync(kFull, top, o));
        const int e = min(max(exponent(__uint_as_float(top)), -120), 120);
        const float f = pow2(-e);
#pragma unroll
        for (int j = 0; j < 4; ++j)
          w[j] = pack_f16(__uint_as_float(w[j] << 16) * f, __uint_as_float(w[j] & 0xffff0000u) * f);
        x = make_uint4(w[0], w[1], w[2], w[3]);
        if (c == 0) m->qs[r] = pow2(e);
      }
      const uint32_t at = base + kQOff + (uint32_t)((r >> 7) * kOperand + (c >> 3) * kHalf +
                                                    (r & 127) * 128 + (((c & 7) ^ (r & 7)) << 4));
      sts128(at, x.x, x.y, x.z, x.w);
    }
    um::fence_async();
    softmax_sync();  // also: qs of every row is there

    const int brow = pair ? 128 * s + lrow : lrow;  // row of the block
    const bool mine = brow < rows;
    const bool busy = (pair ? 128 * s + quad * 32 : quad * 32) < rows;  // warp has a row
    const int row = it.blk * p.rb + min(brow, rows - 1), tok = row / p.G;
    const uint64_t word = p.kn.p ? seen(p, b, tok) : 0ull;
    const float sl = fmaxf(kQuant ? m->qs[brow] * p.scale_log2 : p.scale_log2, 1.1754944e-38f);
    __syncwarp();
    if (lane == 0) tc::mbar_arrive(bar(&m->q_full));  // rows written, qs read by the warp
    const int n = it.kb - it.ka;
    // C: reference of the weights (log2 domain, less 6 bits of head room for f16);
    // lsum: their sum; shift0: exponent the accumulator is relative to
    float C = -INFINITY, lsum = 0.f;
    int shift0 = 0;
    const int steps = pair ? n : (n - s + 1) / 2;
    for (int i = 0; i < steps; ++i) {
      const int64_t t = tile0 + (pair ? i : 2 * i + s);
      ok = ok && __all_sync(kFull, tc::mbar_wait(bar(&m->s_full[s]), uses & 1, ab));
      ++uses;
      if (!ok) break;
      if (busy) {
        um::fence_after();
        ok = __all_sync(kFull, tc::mbar_wait(bar(&m->meta_full[t % kMeta]), (uint32_t)((t / kMeta) & 1), ab));
        if (!ok) break;
        const Meta& mt = m->meta[t % kMeta];
        const bool whole = mt.whole;
        uint32_t live[4];
        if (!whole) {
          if (mt.drafts) {
            live[0] = (uint32_t)word;
            live[1] = (uint32_t)(word >> 32);
            live[2] = live[3] = 0u;
          } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) live[j] = mt.live[j];
          }
        }
        if (i == 0) shift0 = mt.shift;
        const float dE = kQuant ? (float)(mt.shift - shift0) : 0.f;
        // the row's maximum
        float mx = -INFINITY;
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t r[32];
          um::ld32(tS + 32u * c, r);
          if (kQuant) {
#pragma unroll
            for (int j = 0; j < 32; j += 4) {
              const float4 k4 = *reinterpret_cast<const float4*>(&mt.ks[32 * c + j]);
              const float2 x0 = fmul2(make_float2(__uint_as_float(r[j]), __uint_as_float(r[j + 1])),
                                      make_float2(k4.x, k4.y));
              const float2 x1 = fmul2(make_float2(__uint_as_float(r[j + 2]), __uint_as_float(r[j + 3])),
                                      make_float2(k4.z, k4.w));
              r[j] = __float_as_uint(x0.x);
              r[j + 1] = __float_as_uint(x0.y);
              r[j + 2] = __float_as_uint(x1.x);
              r[j + 3] = __float_as_uint(x1.y);
            }
          }
          if (!whole) {
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (!(live[c] >> j & 1u)) r[j] = 0xff800000u;
          }
#pragma unroll
          for (int j = 0; j < 32; j += 2) mx = um::max3(mx, __uint_as_float(r[j]), __uint_as_float(r[j + 1]));
        }
        mx = fmaf(mx, sl, dE - (kQuant ? 6.f : 0.f));  // sl > 0; -inf stays
        const bool grow = mx > C + kLazy || C == -INFINITY;
        float f = 1.f;
        if (grow) {
          const float nc = fmaxf(mx, C);
          f = C == -INFINITY ? 1.f : um::ex2(C - nc);
          C = nc;
        }
        if (i > 0 && __any_sync(kFull, f != 1.f)) {  // O of the tiles before is done (see issue)
          lsum *= f;
#pragma unroll
          for (int c = 0; c < 4; ++c) {
            uint32_t r[32];
            um::ld32(tO + 32u * c, r);
#pragma unroll
            for (int j = 0; j < 32; ++j) r[j] = __float_as_uint(__uint_as_float(r[j]) * f);
            um::st32(tO + 32u * c, r);
          }
        }
        // weights
        const float cc = C == -INFINITY ? 0.f : C;
        const float2 sl2 = make_float2(sl, sl), off2 = make_float2(dE - cc, dE - cc);
        float2 sum2 = make_float2(0.f, 0.f);
#pragma unroll
        for (int c = 0; c < 4; ++c) {
          uint32_t r[32];
          um::ld32(tS + 32u * c, r);
          uint32_t hi[16], lo[16];
#pragma unroll
          for (int j = 0; j < 32; j += 4) {
            float2 x0 = make_float2(__uint_as_float(r[j]), __uint_as_float(r[j + 1]));
            float2 x1 = make_float2(__uint_as_float(r[j + 2]), __uint_as_float(r[j + 3]));
            if (kQuant) {
              const float4 k4 = *reinterpret_cast<const float4*>(&mt.ks[32 * c + j]);
              x0 = fmul2(x0, make_float2(k4.x, k4.y));
              x1 = fmul2(x1, make_float2(k4.z, k4.w));
            }
            x0 = ffma2(x0, sl2, off2);
            x1 = ffma2(x1, sl2, off2);
            if (!whole) {
              if (!(live[c] >> j & 1u)) x0.x = -INFINITY;
              if (!(live[c] >> (j + 1) & 1u)) x0.y = -INFINITY;
              if (!(live[c] >> (j + 2) & 1u)) x1.x = -INFINITY;
              if (!(live[c] >> (j + 3) & 1u)) x1.y = -INFINITY;
            }
            x0.x = um::ex2(x0.x);
            x0.y = um::ex2(x0.y);
            x1.x = um::ex2(x1.x);
            x1.y = um::ex2(x1.y);
            sum2 = fadd2(sum2, fadd2(x0, x1));
            if (kQuant) {
              hi[j / 2] = pack_f16(x0.x, x0.y);
              hi[j / 2 + 1] = pack_f16(x1.x, x1.y);
            } else {
              hi[j / 2] = pack_bf16(x0.x, x0.y);
              hi[j / 2 + 1] = pack_bf16(x1.x, x1.y);
              lo[j / 2] = pack_bf16(x0.x - bf16lo(hi[j / 2]), x0.y - bf16hi(hi[j / 2]));
              lo[j / 2 + 1] = pack_bf16(x1.x - bf16lo(hi[j / 2 + 1]), x1.y - bf16hi(hi[j / 2 + 1]));
            }
          }
          um::st16(tS + 32u * c, hi);
          if (!kQuant) um::st16(tS + 32u * c + 16u, lo);
        }
        lsum = fmaf(sum2.x + sum2.y, kQuant ? um::ex2(-dE) : 1.f, lsum);
        um::wait_st();
        um::fence_before();
      }
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(bar(&m->p_full[s]));
    }
    // ---- the item's result: one record per row
    if (ok && steps > 0) {
      ok = __all_sync(kFull, tc::mbar_wait(bar(&m->o_full[s]), finals & 1, ab));
      ++finals;
    }
    um::fence_after();
    const int64_t rec = (int64_t)blockIdx.x + (int64_t)it.u * p.nblk + it.blk;
    // stream s: sum 2^C lsum, accumulator relative to 2^(C + shift0)
    float f0 = 1.f, f1 = 0.f, Cj = C, lj = lsum;
    const bool both = !pair && n > 1;  // join the streams: stream 0 writes
    if (!pair) {
      if (s == 1 && busy) {
        m->cm[lrow] = C;
        m->l[lrow] = lsum;
        m->sh[lrow] = (float)shift0;
      }
      um::fence_before();
      softmax_sync();
      um::fence_after();
    }
    if (pair || s == 0) {
      if (busy) {
        if (both) {
          const float C1 = m->cm[lrow], l1 = m->l[lrow];
          Cj = fmaxf(C, C1);
          f0 = C == -INFINITY ? 0.f : exp2f(C - Cj);
          f1 = C1 == -INFINITY ? 0.f : exp2f(C1 - Cj);
          lj = lsum * f0 + l1 * f1;
          f1 *= kQuant ? exp2f(m->sh[lrow] - (float)shift0) : 1.f;
        }
        const float inv = lj != 0.f ? 1.f / lj : 0.f, up = kQuant ? exp2f((float)shift0) : 1.f;
        const float g0 = f0 == 0.f ? 0.f : f0 * inv * up, g1 = f1 == 0.f ? 0.f : f1 * inv * up;
        float* acc = p.rec_acc + (rec * p.rb + brow) * kD;
#pragma unroll 1
        for (int c = 0; c < 4; ++c) {
          uint32_t r[32];
          um::ld32(tO + 32u * c, r);
#pragma unroll
          for (int j = 0; j < 32; ++j) r[j] = g0 == 0.f ? 0u : __float_as_uint(__uint_as_float(r[j]) * g0);
          if (both) {
            uint32_t r1[32];
            um::ld32(tO + 128u + 32u * c, r1);
#pragma unroll
            for (int j = 0; j < 32; ++j)
              if (g1 != 0.f) r[j] = __float_as_uint(fmaf(__uint_as_float(r1[j]), g1, __uint_as_float(r[j])));
          }
          if (mine) {
#pragma unroll
            for (int j = 0; j < 32; j += 4)
              *reinterpret_cast<float4*>(acc + 32 * c + j) =
                  ok ? make_float4(__uint_as_float(r[j]), __uint_as_float(r[j + 1]), __uint_as_float(r[j + 2]),
                                   __uint_as_float(r[j + 3]))
                     : make_float4(0.f, 0.f, 0.f, 0.f);
          }
        }
        if (mine) p.rec_ml[rec * p.rb + brow] = ok ? make_float2(Cj, lj) : make_float2(0.f, __int_as_float(0x7fc00000));
      }
    }
    um::fence_before();
    tile0 += n;
  }
}

// grid = p.ctas (one CTA per SM), block = kThreads.
template <int FMT>
__global__ void __launch_bounds__(kThreads, 1) tree_tc_kernel(const __grid_constant__ CUtensorMap tmK,
                                                              const __grid_constant__ CUtensorMap tmV,
                                                              const __grid_constant__ TreeArgs p) {
  extern __shared__ char smem_raw[];
  char* sm = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  Misc* m = reinterpret_cast<Misc*>(sm + kMiscOff);
  const int64_t per = tiles_per_cta(p);
  if (per * blockIdx.x >= p.first[p.units] * p.nblk) return;  // uniform, before any barrier
  const int warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    for (int i = 0; i < kStages; ++i) {
      tc::mbar_init(bar(&m->k_full[i]), kLoadWarps);
      tc::mbar_init(bar(&m->k_empty[i]), 1);
      tc::mbar_init(bar(&m->v_full[i]), kLoadWarps);
      tc::mbar_init(bar(&m->v_empty[i]), 1);
    }
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(bar(&m->s_full[i]), 1);
      tc::mbar_init(bar(&m->p_full[i]), 4);
      tc::mbar_init(bar(&m->o_full[i]), 1);
    }
    for (int i = 0; i < kMeta; ++i) tc::mbar_init(bar(&m->meta_full[i]), 1);
    tc::mbar_init(bar(&m->q_full), kSoftWarps);
    tc::mbar_init(bar(&m->done), 1);
    m->abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  if (warp == kSoftWarps + kLoadWarps) um::alloc(tc::saddr(&m->tmem), 512);
  um::fence_before();
  __syncthreads();
  um::fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&m->tmem);
  const uint32_t base = tc::saddr(sm);
  if (warp < kSoftWarps) {
    softmax<FMT>(p, m, base, tmem, threadIdx.x, per);
  } else if (warp < kSoftWarps + kLoadWarps) {
    Loader<FMT> ld(p, m, base + kKVOff, &tmK, &tmV, threadIdx.x - kSoftWarps * 32);
    ld.run(per);
  } else if ((threadIdx.x & 31) == 0) {
    issue<FMT>(p, m, base, tmem, per);
  }
  __syncwarp();
  um::fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && m->abort && p.st.status) atomicOr(p.st.status, CERTKV_STATUS_TIMEOUT);
  if (warp == kSoftWarps + kLoadWarps) {
    um::fence_after();
    um::dealloc(tmem, 512);
  }
}

constexpr int kMaxDevices = 64;

// CTAs: one per SM.  Set up once per device: the shared-memory opt-in.
int ctas_of_device() {
  static int cached[kMaxDevices] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return 0;
  if (dev < kMaxDevices && cached[dev] > 0) return cached[dev];
  int sms = 0;
  if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1 ||
      cudaFuncSetAttribute(tree_tc_kernel<CERTKV_STORE_BF16>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                           kSmemBytes) != cudaSuccess ||
      cudaFuncSetAttribute(tree_tc_kernel<CERTKV_STORE_FP8>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                           kSmemBytes) != cudaSuccess ||
      cudaFuncSetAttribute(tree_tc_kernel<CERTKV_STORE_FP4>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                           kSmemBytes) != cudaSuccess)
    return 0;
  if (dev < kMaxDevices) cached[dev] = sms;
  return sms;
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
  if (format == CERTKV_STORE_BF16)
    tree_tc_kernel<CERTKV_STORE_BF16><<<p.ctas, kThreads, kSmemBytes, st>>>(mk, mv, p);
  else if (format == CERTKV_STORE_FP8)
    tree_tc_kernel<CERTKV_STORE_FP8><<<p.ctas, kThreads, kSmemBytes, st>>>(mk, mv, p);
  else
    tree_tc_kernel<CERTKV_STORE_FP4><<<p.ctas, kThreads, kSmemBytes, st>>>(mk, mv, p);
  return true;
}

}  // namespace certkv
