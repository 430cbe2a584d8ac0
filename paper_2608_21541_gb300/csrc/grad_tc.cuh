// grad_tc.cuh — what the tensor-core kernels of tree attention's gradients share: the walk over
// a share's tiles, and the warps that bring keys and values into operands.
#pragma once

#include <stddef.h>

#include "common.cuh"
#include "follow.cuh"
#include "grad.cuh"
#include "operand.cuh"
#include "tma.cuh"
#include "umma.cuh"

namespace certkv {
namespace gt {

__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// A bounded wait, as tc::mbar_wait, with the abort flag in shared memory: a pointer less to keep.
__device__ __forceinline__ bool aborted(uint32_t flag) {
  int x;
  asm volatile("ld.volatile.shared.b32 %0, [%1];" : "=r"(x) : "r"(flag) : "memory");
  return x != 0;
}
__device__ __forceinline__ bool wait(uint32_t mbar, uint32_t parity, uint32_t flag) {
  return look(
      tc::kSpinLimit, [&] { return tc::mbar_try(mbar, parity); }, [&] { return aborted(flag); },
      [&] { asm volatile("st.volatile.shared.b32 [%0], 1;" ::"r"(flag) : "memory"); });
}
// Looks without a limit of their own: false when the role is to stop.
__device__ __forceinline__ bool patience(uint32_t look, uint32_t flag) {
  if ((look & 255u) == 255u && aborted(flag)) return false;
  if (look < tc::kSpinLimit) return true;
  asm volatile("st.volatile.shared.b32 [%0], 1;" ::"r"(flag) : "memory");
  return false;
}
// The same by a whole warp.
__device__ __forceinline__ bool wait_all(uint32_t mbar, uint32_t parity, uint32_t flag) {
  return __all_sync(kFull, wait(mbar, parity, flag));
}

// Shared memory by its address: generic pointers cost two registers each, and a spill next to
// 200 KB of shared memory costs more than anything else (the L1 holds hardly any of it: 4500
// clocks a tile).
__device__ __forceinline__ float4 lds128(uint32_t a) {
  float4 x;
  asm volatile("ld.shared.v4.f32 {%0, %1, %2, %3}, [%4];" : "=f"(x.x), "=f"(x.y), "=f"(x.z), "=f"(x.w) : "r"(a) : "memory");
  return x;
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t x;
  asm volatile("ld.shared.b32 %0, [%1];" : "=r"(x) : "r"(a) : "memory");
  return x;
}
__device__ __forceinline__ void sts32(uint32_t a, uint32_t x) {
  asm volatile("st.shared.b32 [%0], %1;" ::"r"(a), "r"(x) : "memory");
}
// A role's last wait, for what it has on its way itself: the block's shared memory is another's once
// it has gone, so nobody else's giving up may cut this short.  `own`: a flag that only this role has.
// (With no flag at all the queries' kernel of 8- and 4-bit stores took 720 us for 703.)
__device__ __forceinline__ void finish(uint32_t mbar, uint32_t parity, uint32_t own) {
  sts32(own, 0u);
  wait(mbar, parity, own);
}
// The address of a field of the kernel's Misc, from `base`, Plan P and Misc M of the scope.
#define GRAD_AT(field) (base + (uint32_t)(P::kMiscOff + offsetof(M, field)))

// One segment met by a share: its tiles [ka, kb).
struct Item {
  int u, ka, kb;
};
// Where a share begins: worked out once, by everybody, and walked on from by each role.
struct Walk {
  int u, k, left;  // segment, its next tile, tiles of the share from there on
  static __device__ __forceinline__ Walk of(const GradArgs& p, int share) {
    const int64_t per = tiles_per_share(p), g = per * share;
    Walk w;
    w.left = (int)max(min(p.first[p.units] - g, per), (int64_t)0);
    int lo = 0, hi = p.units;
#pragma unroll 1
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (p.first[mid] <= g) lo = mid;
      else hi = mid;
    }
    w.u = lo;
    w.k = w.left > 0 ? (int)(g - p.first[lo]) : 0;
    return w;
  }
  __device__ __forceinline__ bool next(const GradArgs& p, Item* it) {
    if (left <= 0) return false;
    int n;
#pragma unroll 1
    while ((n = (int)(p.first[u + 1] - p.first[u])) <= k) ++u, k = 0;
    *it = {u, k, min(n, k + left)};
    left -= it->kb - k;
    k = it->kb;
    return true;
  }
};

// The facts of a tile's slots that are read across a row (the query kernel).
struct Facts {
  uint32_t live[4];  // slots to take
};
struct alignas(16) ScaledFacts {  // 8- and 4-bit stores
  uint32_t live[4];
  float ks[kGradTile], vs[kGradTile];  // scales of keys, times the logits', and of values
};
template <int FMT>
struct FactsOf {
  using type = ScaledFacts;
};
template <>
struct FactsOf<CERTKV_STORE_BF16> {
  using type = Facts;
};

// What a code of the operands stands for is the code times its row's scale times this: a
// 4-bit code's product with its group scale is put into bf16 2^-8 times as large (below).
template <int FMT>
constexpr float kCodeScale = FMT == CERTKV_STORE_FP4 ? 256.f : 1.f;

// Sixteen codes as bf16, exactly: their bits are moved into place as the bits of a bf16 whose
// exponent is too small by a constant (subnormal codes become subnormal bf16), and one
// product puts that right.  2^120 for 8 bits; for 4 bits 2^126, of which the group's scale
// (at most 448) leaves room for 2^118 in the same product.
__device__ __forceinline__ void codes_to_bf16(const uint32_t (&c)[4], uint32_t, uint32_t (&w)[8]) {
#pragma unroll
  for (int j = 0; j < 8; ++j) {
    const uint32_t x = __byte_perm(c[j >> 1], 0u, j & 1 ? 0x3424 : 0x1404);
    w[j] = mul_bf16x2((x >> 4 & 0x07f007f0u) | (x & 0x80008000u), 0x7b807b80u);
  }
}
__device__ __forceinline__ void codes_to_bf16(const uint32_t (&c)[2], uint32_t group, uint32_t (&w)[8]) {
  const float2 g = f16x2_to_f32(e4m3x2_to_f16x2(group));
  const uint32_t f = pack2(g.x * 0x1p118f, g.x * 0x1p118f);
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const uint32_t lo = c[i], hi = c[i] >> 4;  // even and odd elements, in the low nibble of each byte
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      // both nibbles to bits 8..11 of their halves
      const uint32_t x = __byte_perm(lo, hi, j == 0 ? 0x4000 : j == 1 ? 0x5010 : j == 2 ? 0x6020 : 0x7030);
      w[4 * i + j] = mul_bf16x2((x >> 2 & 0x01c001c0u) | (x << 4 & 0x80008000u), f);
    }
  }
}

__device__ __forceinline__ void cp16(uint32_t to, const void* from, bool on) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(to), "l"(from), "r"(on ? 16 : 0) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() {
  asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory");
}

// Tiles of a share one after the other, and where the walk stands: the tile's table entries, which
// are looked at a tile later so that nobody waits for them, and its live slots from its first on.
struct Tile {
  int a, b, live;
};
struct Tiles {
  const GradArgs& p;
  Walk walk;
  Item it = {0, 0, 0};  // ka: the next tile
  int count = 0;
  __device__ __forceinline__ Tiles(const GradArgs& p_, const Walk& w) : p(p_), walk(w) {}
  __device__ __forceinline__ bool next(Tile* t) {
    if (it.ka == it.kb) {
      if (!walk.next(p, &it)) return false;
      count = p.st.count(it.u);
    }
    const int32_t* e = p.st.table + (int64_t)it.u * p.st.max_pages + 2 * it.ka;
    t->live = count - it.ka * kGradTile;
    t->a = __ldg(e);
    t->b = t->live > kPage ? __ldg(e + 1) : -1;
    ++it.ka;
    return true;
  }
};
// The entries of a tile that are no page of the pool become -1.
__device__ __forceinline__ void check(const GradArgs& p, Tile& t, bool raise) {
  const bool a = t.a >= 0 && t.a < p.st.pool_pages, b = t.b >= 0 && t.b < p.st.pool_pages;
  if (raise && ((!a && t.live > 0) || (!b && t.live > kPage))) p.st.raise();
  if (!a) t.a = -1;
  if (!b) t.b = -1;
}

// Live rows of a tile's page 0 or 1.
__device__ __forceinline__ int live_rows(const Tile& t, int half) {
  return (half ? t.b : t.a) < 0 ? 0 : max(min(t.live - kPage * half, kPage), 0);
}

constexpr int kLoadThreads = 2 * kGroupWarps * 32;  // of the loaders
// Bytes of the loaders' stretches for the keys, or the values, of a tile.
template <int FMT>
constexpr int kStage = FMT == CERTKV_STORE_BF16 ? 0 : 128 * (row_bytes(FMT) + (FMT == CERTKV_STORE_FP4 ? kGroups : 0));

// Warps that hand an operand over.
template <int FMT>
constexpr int kArrivals = FMT == CERTKV_STORE_BF16 ? kGroupWarps : 2 * kGroupWarps;

// Where the loaders put a tile's keys or values: a ring of operands, and its barriers; addresses
// in shared memory.
struct Ring {
  uint32_t full, empty, at;
};

// A bf16 store: two groups of four warps, one for the keys and one for the values, bring every
// tile into a ring of PLACES operands, rows that are not live as zeros.  Whole tiles are bulk
// copies; other rows are copied 16 bytes at a time, a tile's on their way while the one before
// lands (whole tiles this way took 2000 clocks to ask for).
template <int PLACES, bool FACTS>
struct Copier {
  const CUtensorMap* map;
  const GradArgs& p;
  Ring ring;
  uint32_t facts, abort, own;  // facts [PLACES] (FACTS: written by this group); own: a flag
  const uint8_t* rows;
  int tid;               // of 128
  uint32_t t = 0;
  bool pending = false;  // a tile's copies have not been handed over
  uint32_t bulk = 0;     // places whose last tile came by bulk copies

  // The fence before the tensor core's reads is the issuer's: here it would wait for every load
  // that is on its way (1200 clocks a tile).
  __device__ __forceinline__ void hand_over(uint32_t tile) const {
    __syncwarp();
    if ((tid & 31) == 0) tc::mbar_arrive(ring.full + 8 * (tile % PLACES));
  }
  __device__ __forceinline__ void state(uint32_t place, const Tile& x) const {
    const uint32_t word = __ballot_sync(kFull, (tid < kPage ? x.a : x.b) >= 0 && tid < x.live);
    if ((tid & 31) == 0) sts32(facts + place * (uint32_t)sizeof(Facts) + 4 * (tid >> 5), word);
  }
  __device__ __forceinline__ bool wait_place() const {
    return wait_all(ring.empty + 8 * (t % PLACES), ((t / PLACES) & 1u) ^ 1u, abort);
  }
  // A whole tile by four bulk copies, two pages x two 64-element halves.
  __device__ __forceinline__ bool copy_whole(const Tile& x) {
    const uint32_t place = t % PLACES, to = ring.at + place * kOperand, full = ring.full + 8 * place;
    if (pending) {
      cp_wait<0>();
      hand_over(t - 1);
      pending = false;
    }
    if (!wait_place()) return false;
    if constexpr (FACTS) state(place, x);
    __syncwarp();
    if (tid == 0) {
      tc::mbar_expect_tx(full, kOperand);
      tc::tma_load_2d(to, map, 0, x.a * kPage, full);
      tc::tma_load_2d(to + kHalf, map, 64, x.a * kPage, full);
      tc::tma_load_2d(to + kHalf / 2, map, 0, x.b * kPage, full);
      tc::tma_load_2d(to + kHalf + kHalf / 2, map, 64, x.b * kPage, full);
    } else if ((tid & 31) == 0) {
      tc::mbar_arrive(full);
    }
    bulk |= 1u << place;
    ++t;
    return true;
  }
  __device__ __forceinline__ bool copy(const Tile& x) {
    const uint32_t place = t % PLACES, to = ring.at + place * kOperand;
    if (x.a >= 0 && x.b >= 0 && x.live >= kGradTile) return copy_whole(x);
    // what is on its way is not held up by the wait for a place
    if (pending && !__all_sync(kFull, tc::mbar_test(ring.empty + 8 * place, ((t / PLACES) & 1u) ^ 1u))) {
      cp_wait<0>();
      hand_over(t - 1);
      pending = false;
    }
    if (!wait_place()) return false;
    const int c = tid & 15, r0 = tid >> 4;  // 16 lanes a row, 16 bytes each
#pragma unroll 4
    for (int i = 0; i < 16; ++i) {
      const int r = r0 + 8 * i, pg = i < 8 ? x.a : x.b;
      const bool on = pg >= 0 && r < x.live;
      cp16(to + (uint32_t)((c >> 3) * kHalf + r * 128 + (((c & 7) ^ (r & 7)) << 4)),
           rows + (on ? ((int64_t)pg * kPage + (r & (kPage - 1))) * 256 + c * 16 : 0), on);
    }
    cp_commit();
    if constexpr (FACTS) state(place, x);
    if (pending) {
      cp_wait<1>();
      hand_over(t - 1);
    }
    pending = true;
    bulk &= ~(1u << place);
    ++t;
    return true;
  }
  __device__ __forceinline__ void run(const Walk& walk) {
    Tiles tiles(p, walk);
    Tile x, y;  // the next tile's pages are looked up a tile before
    bool ok = true, more = tiles.next(&x);
#pragma unroll 1
    while (ok && more) {
      more = tiles.next(&y);
      check(p, x, tid == 0);
      ok = copy(x);
      x = y;
    }
    cp_wait<0>();  // nothing lands after the CTA has gone
    if (ok && pending) hand_over(t - 1);
    if (tid == 0)
      for (uint32_t i = t > PLACES ? t - PLACES : 0; i < t; ++i)
        if (bulk >> (i % PLACES) & 1u) finish(ring.full + 8 * (i % PLACES), (i / PLACES) & 1u, own);
  }
};

// 8- and 4-bit stores: the codes of a tile's values and of its keys on their way into a stretch of
// shared memory each, page by page, by one lane's bulk copies; eight warps expand them into the
// rings' operands, rows that are not live as zeros, codes as bf16 without their row's scale.  All
// eight at one operand, since the way from a free place to the next product is what a tile waits
// for (8-bit trees 203 us, 222 with four each for keys and for values), and one body for both: code
// for whole tiles in registers took the instruction caches of an SM more time than all else (395 and
// 700 us).  Codes copied 16 bytes at a time by the expanding warps took 1400 clocks a tile to ask for.
template <int FMT>
struct Stages {
  static constexpr uint32_t kPageCodes = kPage * row_bytes(FMT), kPageGroups = FMT == CERTKV_STORE_FP4 ? kPage * kGroups : 0;
  uint32_t at;           // of the keys' stretch; kStage<FMT> bytes on that of the values
  uint32_t full, empty;  // barriers, of keys and of values
  uint32_t live;         // of either, live rows of each page (int2)
};

template <int FMT>
struct Stager {
  using S = Stages<FMT>;
  const GradArgs& p;
  S st;
  uint32_t abort, own;  // own: a flag

  // Codes of operand `value` of tile number t on their way.
  __device__ __forceinline__ void page(int pg, int half, bool value) const {
    if (pg < 0) return;
    const uint32_t to = st.at + (value ? kStage<FMT> : 0u), full = st.full + 8 * value;
    tc::bulk_load(to + half * S::kPageCodes, (value ? p.st.v : p.st.k) + (int64_t)pg * S::kPageCodes, S::kPageCodes, full);
    if (FMT == CERTKV_STORE_FP4)
      tc::bulk_load(to + 2 * S::kPageCodes + half * S::kPageGroups,
                    (value ? p.st.vg : p.st.kg) + (int64_t)pg * S::kPageGroups, S::kPageGroups, full);
  }
  __device__ __forceinline__ bool stage(const Tile& x, uint32_t t, bool value) const {
    if (!wait(st.empty + 8 * value, (t & 1u) ^ 1u, abort)) return false;
    sts32(st.live + 8 * value, live_rows(x, 0));
    sts32(st.live + 8 * value + 4, live_rows(x, 1));
    tc::mbar_expect_tx(st.full + 8 * value, ((x.a >= 0) + (x.b >= 0)) * (S::kPageCodes + S::kPageGroups));
    page(x.a, 0, value);
    page(x.b, 1, value);
    return true;
  }
  __device__ __forceinline__ void run(const Walk& walk) const {
    Tiles tiles(p, walk);
    Tile x, y;  // x: whose values are next, checked; y: whose keys are
    uint32_t keys = 0, values = 0;  // staged
    bool more = tiles.next(&x);
    check(p, x, true);
    bool ok = stage(x, keys++, false);
#pragma unroll 1
    while (ok && more) {
      more = tiles.next(&y);
      ok = stage(x, values, true);
      values += ok;
      if (!ok || !more) break;
      check(p, y, true);
      ok = stage(y, keys, false);
      keys += ok;
      x = y;
    }
    // nothing lands after the CTA has gone
    if (keys > 0) finish(st.full, (keys - 1) & 1u, own);
    if (values > 0) finish(st.full + 8, (values - 1) & 1u, own);
  }
};

// A warp that states the facts of the tiles' slots in two places of their own: its loads'
// latency is nobody else's (the expanding warps waited 1000 clocks a tile for them).  A place is
// free when the tile before last has given back its keys.
template <int FMT, int KEYS>
struct FactFeeder {
  const GradArgs& p;
  uint32_t full, empty;   // barriers, of the facts [2] and of the keys [KEYS]
  uint32_t facts, abort;  // facts [2]
  int lane;

  __device__ __forceinline__ void put(uint32_t to, float4 x, float f) const {
    sts128(to + 16 * lane, __float_as_uint(x.x * f), __float_as_uint(x.y * f), __float_as_uint(x.z * f),
           __float_as_uint(x.w * f));
  }
  __device__ __forceinline__ void run(const Walk& walk) {
    Tiles tiles(p, walk);
    Tile x, y;
    uint32_t t = 0;
    bool ok = true, more = tiles.next(&x);
#pragma unroll 1
    for (; ok && more; ++t) {
      more = tiles.next(&y);
      check(p, x, false);
      const int pg = lane < 16 ? x.a : x.b;
      float4 ks = {0.f, 0.f, 0.f, 0.f}, vs = ks;
      if (pg >= 0) {  // of four slots a lane; what is not live is masked
        ks = __ldg(reinterpret_cast<const float4*>(p.st.ks + (int64_t)pg * kPage) + (lane & 15));
        vs = __ldg(reinterpret_cast<const float4*>(p.st.vs + (int64_t)pg * kPage) + (lane & 15));
      }
      const uint32_t to = facts + (t & 1u) * (uint32_t)sizeof(ScaledFacts);
      if (t >= 2) ok = wait_all(empty + 8 * ((t - 2) % KEYS), ((t - 2) / KEYS) & 1u, abort);
      if (lane < 4) {
        const int n = max(live_rows(x, lane >> 1) - 32 * (lane & 1), 0);
        sts32(to + 4 * lane, n >= 32 ? kFull : (1u << n) - 1u);
      }
      put(to + (uint32_t)offsetof(ScaledFacts, ks), ks, kCodeScale<FMT> * p.scale_log2);
      put(to + (uint32_t)offsetof(ScaledFacts, vs), vs, kCodeScale<FMT>);
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(full + 8 * (t & 1u));
      x = y;
    }
  }
};

template <int FMT, int KEYS, int VALUES>
struct Expander {
  using S = Stages<FMT>;
  static constexpr int kWords = FMT == CERTKV_STORE_FP8 ? 4 : 2;
  static constexpr int kMine = 128 * 8 / kLoadThreads, kApart = 128 / kMine;  // a thread's pieces, rows apart
  Ring keys, values;
  S st;
  uint32_t abort;
  int tid;  // of 256

  // Codes 16 sub .. of row r of a stretch, of four bits the word with their group's scale too.
  __device__ __forceinline__ void piece(uint32_t from, int r, int sub, uint32_t (&c)[kWords], uint32_t& g) const {
    if constexpr (FMT == CERTKV_STORE_FP8) {
      asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
                   : "=r"(c[0]), "=r"(c[1]), "=r"(c[2]), "=r"(c[3])
                   : "r"(from + 128 * r + 16 * sub));
    } else {
      asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(c[0]), "=r"(c[1]) : "r"(from + 64 * r + 8 * sub));
      asm volatile("ld.shared.b32 %0, [%1];" : "=r"(g) : "r"(from + 2 * S::kPageCodes + 8 * r + (sub & 4)));
    }
  }
  // All operands one after the other, the keys of a tile and then its values.  A thread's codes
  // are read at once, and their stretch given back, before the place that they go to is waited for.
  __device__ __forceinline__ void run(const Walk& walk) const {
    const Piece pc(tid);
#pragma unroll 1
    for (uint32_t i = 0, n = 2 * (uint32_t)walk.left; i < n; ++i) {
      const uint32_t t = i >> 1, value = i & 1u, place = value ? t % VALUES : t % KEYS;
      const Ring& ring = value ? values : keys;
      const uint32_t from = st.at + value * kStage<FMT>, to = ring.at + place * kOperand;
      if (!wait_all(st.full + 8 * value, t & 1u, abort)) break;
      const int la = (int)lds32(st.live + 8 * value), lb = kPage + (int)lds32(st.live + 8 * value + 4);
      uint32_t c[kMine][kWords], g[kMine] = {};
#pragma unroll
      for (int q = 0; q < kMine; ++q) piece(from, pc.grp + kApart * q, pc.sub, c[q], g[q]);
      __syncwarp();
      if ((tid & 31) == 0) tc::mbar_arrive(st.empty + 8 * value);
      if (!wait_all(ring.empty + 8 * place, ((value ? t / VALUES : t / KEYS) & 1u) ^ 1u, abort)) break;
#pragma unroll
      for (int q = 0; q < kMine; ++q) {
        uint32_t w[8];
        codes_to_bf16(c[q], g[q] >> (8 * (pc.sub & 3)) & 255u, w);
        if (pc.grp + kApart * q >= (q < kMine / 2 ? la : lb)) {
#pragma unroll
          for (int j = 0; j < 8; ++j) w[j] = 0u;
        }
        const uint32_t row = to + (uint32_t)(q * kApart * 128);
        sts128(row + pc.at0, w[0], w[1], w[2], w[3]);
        sts128(row + pc.at1, w[4], w[5], w[6], w[7]);
      }
      __syncwarp();
      if ((tid & 31) == 0) tc::mbar_arrive(ring.full + 8 * place);
    }
  }
};

// A warpgroup's registers, from those of the launch up or down; the launch's must cover all.
template <int N, int LAUNCH>
__device__ __forceinline__ void registers() {
  if constexpr (N > LAUNCH) asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
  if constexpr (N < LAUNCH) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}

// The maps of a bf16 store's pools.
inline bool pool_maps(const GradArgs& p, int format, CUtensorMap* k, CUtensorMap* v) {
  const uint64_t rows = (uint64_t)p.st.pool_pages * kPage;
  return format != CERTKV_STORE_BF16 || (make_row_map(k, p.st.k, rows, kPage) && make_row_map(v, p.st.v, rows, kPage));
}

}  // namespace gt
}  // namespace certkv
