// grad_tc.cuh — what the tensor-core kernels of tree attention's gradients share: the walk over
// a share's tiles, and the warps that bring keys and values into operands.
#pragma once

#include "common.cuh"
#include "grad.cuh"
#include "operand.cuh"
#include "tma.cuh"
#include "umma.cuh"

namespace certkv {
namespace gt {

__device__ __forceinline__ uint32_t bar(const uint64_t* b) { return tc::saddr(b); }
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  const __nv_bfloat162 h = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&h);
}
__device__ __forceinline__ uint32_t mul_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}

// One segment met by a share: its tiles [ka, kb).
struct Item {
  int u, ka, kb;
};
struct Walk {
  const GradArgs& p;
  int64_t g, g1;
  int u;
  __device__ __forceinline__ Walk(const GradArgs& p_, int share) : p(p_) {
    const int64_t per = tiles_per_share(p);
    g = per * share;
    g1 = min(p.first[p.units], g + per);
    int lo = 0, hi = p.units;
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (p.first[mid] <= g) lo = mid;
      else hi = mid;
    }
    u = lo;
  }
  __device__ __forceinline__ bool next(Item* it) {
    if (g >= g1) return false;
    while (p.first[u + 1] <= g) ++u;
    it->u = u;
    it->ka = (int)(g - p.first[u]);
    it->kb = (int)(it->ka + min(p.first[u + 1] - g, g1 - g));
    g += it->kb - it->ka;
    return true;
  }
};

// The facts of a tile's slots that are read across a row (the query kernel).
struct Facts {
  uint32_t live[4];  // slots to take
};
struct alignas(16) ScaledFacts {  // 8- and 4-bit stores
  uint32_t live[4];
  float ksl[kGradTile], ks[kGradTile], vs[kGradTile];  // of keys, with and without the logits' scale, and values
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

// A group of four warps that brings the keys, or the values, of every tile into a ring of
// PLACES operands: rows that are not live as zeros, 8- and 4-bit codes as bf16 without their
// row's scale.  The next tile's codes are on their way into registers, and its pages known,
// while a place is waited for; a bf16 store's rows are copied without registers, and one
// tile's are on their way while the one before lands.
template <int FMT, int PLACES, bool FACTS>
struct Feeder {
  using F = typename FactsOf<FMT>::type;
  const GradArgs& p;
  uint64_t *full, *empty;  // [PLACES]
  F* facts;                // [PLACES], FACTS: written by this group
  volatile int* abort;
  uint32_t ring;
  bool value;
  int tid;  // of 128
  uint32_t t = 0;
  bool pending = false;  // a tile's copies have not been handed over

  // The tile's page for slots 64 half ..
  __device__ __forceinline__ int page(int64_t u, int k, int half, int count) const {
    const int s = k * kGradTile + half * kPage;
    if (s >= count) return -1;
    const int e = __ldg(p.st.table + u * p.st.max_pages + s / kPage);
    if (e >= 0 && e < p.st.pool_pages) return e;
    if (tid == 0) p.st.raise();
    return -1;
  }
  __device__ __forceinline__ void hand_over(uint32_t tile) const {
    um::fence_async();
    __syncwarp();
    if ((tid & 31) == 0) tc::mbar_arrive(bar(&full[tile % PLACES]));
  }
  // Slot tid's facts: asked for, and stated once the place is free.
  struct Fact {
    bool on;
    float ks, vs;
  };
  __device__ __forceinline__ Fact fact(int a, int b, int live) const {
    const int pg = tid < kPage ? a : b;
    Fact x = {pg >= 0 && tid < live, 0.f, 0.f};
    if (FMT != CERTKV_STORE_BF16 && x.on) {
      x.ks = __ldg(p.st.ks + (int64_t)pg * kPage + (tid & (kPage - 1)));
      x.vs = __ldg(p.st.vs + (int64_t)pg * kPage + (tid & (kPage - 1)));
    }
    return x;
  }
  __device__ __forceinline__ void state(uint32_t place, const Fact& x) const {
    F& f = facts[place];
    const uint32_t word = __ballot_sync(kFull, x.on);
    if ((tid & 31) == 0) f.live[tid >> 5] = word;
    if constexpr (FMT != CERTKV_STORE_BF16) {
      f.ks[tid] = x.ks * kCodeScale<FMT>;
      f.ksl[tid] = x.ks * (kCodeScale<FMT> * p.scale_log2);
      f.vs[tid] = x.vs * kCodeScale<FMT>;
    }
  }
  __device__ __forceinline__ bool wait_place() {
    const uint32_t place = t % PLACES, phase = ((t / PLACES) & 1u) ^ 1u;
    return __all_sync(kFull, tc::mbar_wait(bar(&empty[place]), phase, abort));
  }
  __device__ __forceinline__ bool tile(int a, int b, int live) {
    const uint32_t place = t % PLACES, to = ring + place * kOperand;
    if constexpr (FMT == CERTKV_STORE_BF16) {
      // what is on its way is not held up by the wait for a place
      if (pending && !__all_sync(kFull, tc::mbar_test(bar(&empty[place]), ((t / PLACES) & 1u) ^ 1u))) {
        cp_wait<0>();
        hand_over(t - 1);
        pending = false;
      }
      if (!wait_place()) return false;
      const uint8_t* rows = value ? p.st.v : p.st.k;
      const int c = tid & 15, r0 = tid >> 4;  // 16 lanes a row, 16 bytes each
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        const int r = r0 + 8 * i, pg = i < 8 ? a : b;
        const bool on = pg >= 0 && r < live;
        cp16(to + (uint32_t)((c >> 3) * kHalf + r * 128 + (((c & 7) ^ (r & 7)) << 4)),
             rows + (on ? ((int64_t)pg * kPage + (r & (kPage - 1))) * 256 + c * 16 : 0), on);
      }
      cp_commit();
      if constexpr (FACTS) state(place, fact(a, b, live));
      if (pending) {
        cp_wait<1>();
        hand_over(t - 1);
      }
      pending = true;
    } else {
      const Piece pc(tid);
      Raw<FMT> raw;
      raw.load(pc, a, b, live, value ? p.st.v : p.st.k, value ? p.st.vg : p.st.kg);
      const Fact x = FACTS ? fact(a, b, live) : Fact{};
      if (!wait_place()) return false;
      if constexpr (FACTS) state(place, x);
#pragma unroll
      for (int q = 0; q < kPieces; ++q) {
        uint32_t w[8];
        codes_to_bf16(raw.w[q], FMT == CERTKV_STORE_FP4 ? raw.g[q % (FMT == CERTKV_STORE_FP4 ? kPieces : 1)] : 0u, w);
        pc.put(to, q, w);
      }
      hand_over(t);
    }
    ++t;
    return true;
  }
  __device__ __forceinline__ void run(Walk walk) {
    Item it;
    bool ok = true;
    while (ok && walk.next(&it)) {
      const int count = p.st.count(it.u);
      int a = page(it.u, it.ka, 0, count), b = page(it.u, it.ka, 1, count);
      for (int k = it.ka; ok && k < it.kb; ++k) {
        const int a1 = k + 1 < it.kb ? page(it.u, k + 1, 0, count) : -1;
        const int b1 = k + 1 < it.kb ? page(it.u, k + 1, 1, count) : -1;
        ok = tile(a, b, count - k * kGradTile);
        a = a1;
        b = b1;
      }
    }
    if constexpr (FMT == CERTKV_STORE_BF16) {
      cp_wait<0>();  // nothing lands after the CTA has gone
      if (ok && pending) hand_over(t - 1);
    }
  }
};

template <int N>
__device__ __forceinline__ void regs_up() {
  asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(N));
}
template <int N>
__device__ __forceinline__ void regs_down() {
  asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(N));
}

}  // namespace gt
}  // namespace certkv
