// tree_mma.cu — the split kernel of tree attention for few query rows per unit
// (decode steps and small trees), in blocks of up to 16.
//
// With so few rows the work is reading the store: a 128-row tcgen05 tile would be
// nearly empty, and expanding 8- and 4-bit codes into its shared-memory operands
// costs as much as for full ones.  Here the codes go from shared memory straight
// into the B fragments of mma.sync m16n8k16 (f16, fp32 accumulate), expanded in
// registers; the rows are the 16 rows of the A fragments.  Orders of the
// contracted and of the free indices are chosen so that a thread's part of a row
// is contiguous:
//   S = Q K^T: thread (row n = lane / 4 of eight slots, quarter qc = lane % 4)
//     holds elements 32 qc .. 32 qc + 31 of its slot's key, four a k-step;
//   O += P V: it holds elements 16 n .. 16 n + 15 of four slots' values; pairs of
//     slots are interleaved bytewise, and column n of block i is element 16 n + i.
// bf16 rows are read with ldmatrix in the usual order.
//
// CTA: a producer warp streams tiles (64 slots, 32 for bf16) into a ring by TMA,
// four consumer warps take them in turn, each with a running reference, sum and
// accumulator per row; where the CTA's share passes into the next unit they are
// joined into one record.  Two CTAs per SM.
//
// Weights 2^(x - C), C following the maximum when it grows by more than 2^8.  bf16
// ones come in two parts (2^-16).  f16 ones carry their value row's scale and are
// rounded once (2^-11), C following the largest of those products (log2_scale);
// codes are exact.
//
// What bounds it, 256 segments of 13107 slots, up to 4 rows: bf16 260 us, the copy
// bandwidth.  8-bit 156 us; the copies alone, with nothing done to the tiles, 138.
// 4-bit 160 and 94: the consumers' expansion and products, which eight warps of 168
// registers on an SM do not overlap further.  Slower were tiles of 32 slots (8-bit
// 198; with three CTAs per SM 169), values in stages of their own (161, 4-bit 192:
// their expansion then no longer fills the softmax's gaps) and five consumers with
// one stage each (4-bit 172).
#include <cuda.h>

#include "../../include/certkv.h"
#include "common.cuh"
#include "internal.cuh"
#include "tma.cuh"
#include "tree.cuh"
#include "umma.cuh"

namespace certkv {
namespace {

constexpr int kConsumers = 4;
constexpr int kThreads = (1 + kConsumers) * 32;
constexpr int kRows = kSmallRows;
constexpr float kLazy = 8.f;

template <int FMT>
struct Geo {
  static constexpr bool kQuant = FMT != CERTKV_STORE_BF16;
  static constexpr int kSlots = small_tile(FMT);
  static constexpr int kCodes = kSlots * row_bytes(FMT);  // bytes of one operand's codes
  static constexpr int kGrp = FMT == CERTKV_STORE_FP4 ? kSlots * kGroups : 0;
  static constexpr int kScl = kQuant ? kSlots * 4 : 0;
  static constexpr int kK = 0, kV = kCodes, kKg = 2 * kCodes, kVg = kKg + kGrp, kKs = kVg + kGrp,
                       kVs = kKs + kScl;
  // the swizzle's period: 1024 bytes for rows of 128, 512 for rows of 64
  static constexpr int kAlign = FMT == CERTKV_STORE_FP4 ? 512 : 1024;
  static constexpr int kStage = (kVs + kScl + kAlign - 1) / kAlign * kAlign;
  // each stage belongs to one consumer warp, which has itself waited for the
  // stage's previous phase: a multiple of the consumers
  static constexpr int kStages = FMT == CERTKV_STORE_FP4 ? 8 : 4;
  static constexpr uint32_t kBytes = 2 * (kCodes + kGrp + kScl);
};
struct Tail {
  uint64_t full[8], empty[8];
  int live[8];  // slots of the stage's tile to take
  int abort;
  float m[kConsumers][kRows], l[kConsumers][kRows], e[kConsumers][kRows];
  int64_t first[kInlineUnits + 1];  // see tree_first
};
template <int FMT>
constexpr int smem_bytes() {
  return Geo<FMT>::kStages * Geo<FMT>::kStage + kConsumers * kRows * kD * 4 + (int)sizeof(Tail) + 1024;
}
static_assert(2 * (smem_bytes<CERTKV_STORE_BF16>() + 1024) <= 228 * 1024 &&
                  2 * (smem_bytes<CERTKV_STORE_FP8>() + 1024) <= 228 * 1024 &&
                  2 * (smem_bytes<CERTKV_STORE_FP4>() + 1024) <= 228 * 1024,
              "two CTAs per SM");

__device__ __forceinline__ void consumers_sync() {
  asm volatile("bar.sync 1, %0;" ::"n"(kConsumers * 32) : "memory");
}
__device__ __forceinline__ uint32_t bar(const uint64_t* b) { return tc::saddr(b); }
__device__ __forceinline__ uint4 lds128(uint32_t a) {
  uint4 x;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];"
               : "=r"(x.x), "=r"(x.y), "=r"(x.z), "=r"(x.w)
               : "r"(a));
  return x;
}
__device__ __forceinline__ uint2 lds64(uint32_t a) {
  uint2 x;
  asm volatile("ld.shared.v2.b32 {%0, %1}, [%2];" : "=r"(x.x), "=r"(x.y) : "r"(a));
  return x;
}
__device__ __forceinline__ float lds32f(uint32_t a) {
  float x;
  asm volatile("ld.shared.f32 %0, [%1];" : "=f"(x) : "r"(a));
  return x;
}
__device__ __forceinline__ void sts32f(uint32_t a, float x) {
  asm volatile("st.shared.f32 [%0], %1;" ::"r"(a), "f"(x) : "memory");
}
__device__ __forceinline__ uint32_t lds32(uint32_t a) {
  uint32_t x;
  asm volatile("ld.shared.u32 %0, [%1];" : "=r"(x) : "r"(a));
  return x;
}
__device__ __forceinline__ uint32_t lds16(uint32_t a) {
  uint16_t x;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(a));
  return x;
}
__device__ __forceinline__ uint32_t lds8(uint32_t a) {
  uint32_t x;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(x) : "r"(a));
  return x;
}
__device__ __forceinline__ void ldsm4(uint32_t a, uint32_t& r0, uint32_t& r1, uint32_t& r2, uint32_t& r3) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3)
               : "r"(a));
}
__device__ __forceinline__ void ldsm4t(uint32_t a, uint32_t& r0, uint32_t& r1, uint32_t& r2, uint32_t& r3) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r0), "=r"(r1), "=r"(r2), "=r"(r3)
               : "r"(a));
}
template <bool BF16>
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  if (BF16)
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
        "{%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
  else
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, "
        "{%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
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
__device__ __forceinline__ int exponent(float x) {
  const int e = (__float_as_int(x) >> 23) & 255;
  return e == 0 || e == 255 ? 0 : e - 127;
}

// Slot (0..7) of column j of an eight-slot block.  4-bit rows are 64 bytes, so
// two share a line of banks: their order makes the four slots that a value read
// touches at once fall into both halves of a line.
template <int FMT>
__device__ __forceinline__ int slot_of(int j) {
  return FMT == CERTKV_STORE_FP4 ? ((j >> 1) & 1) + 2 * (j & 1) + 4 * (j >> 2) : j;
}
// Element held by accumulator (block i, column 2 qc + e) of O.
template <int FMT>
__device__ __forceinline__ int element_of(int i, int qc, int e) {
  return FMT == CERTKV_STORE_BF16 ? 8 * i + 2 * qc + e : 32 * qc + 16 * e + i;
}

// ------------------------------------------------------------- producer --
template <int FMT>
__device__ __forceinline__ void produce(const TreeArgs& p, const CUtensorMap* tmK, const CUtensorMap* tmV,
                                        uint32_t sm, Tail* tl, int lane, const int64_t* first, int64_t per) {
  using G = Geo<FMT>;
  constexpr int kPer = kPage / G::kSlots;  // tiles of a page
  int64_t issued = 0;
  bool ok = true;
  Items items(p, first, per);
  Item it;
  uint32_t copied = 0;  // stages whose last tile came by copies
  while (ok && items.next(p, &it)) {
    const int count = p.st.count(it.u);
    int at = 0, lo = -1, hi = -1;  // table entries of 64 pages from page `at` on
    auto entry = [&](int page) {
      if (page >= p.st.max_pages) return -1;
      const int e = __ldg(p.st.table + (int64_t)it.u * p.st.max_pages + page);
      return e >= 0 && e < p.st.pool_pages ? e : -1;
    };
    for (int k = it.ka; k < it.kb; ++k, ++issued) {
      const int page = k / kPer;
      if (k == it.ka) {
        at = page;
        lo = entry(at + lane);
        hi = entry(at + 32 + lane);
      } else if (page >= at + 32) {
        at += 32;
        lo = hi;
        hi = entry(at + 32 + lane);
      }
      const int e = __shfl_sync(kFull, lo, page - at);
      const int s = (int)(issued % G::kStages);
      if (issued >= G::kStages)
        ok = __all_sync(kFull, tc::mbar_wait(bar(&tl->empty[s]), (uint32_t)((issued / G::kStages - 1) & 1),
                                             &tl->abort));
      if (!ok) break;
      copied = e >= 0 ? copied | 1u << s : copied & ~(1u << s);
      if (lane == 0) {
        const uint32_t full = bar(&tl->full[s]), st = sm + (uint32_t)(s * G::kStage);
        tl->live[s] = e >= 0 ? min(count - k * G::kSlots, G::kSlots) : 0;
        if (e < 0) {
          p.st.raise();
          tc::mbar_arrive(full);
        } else {
          tc::mbar_expect_tx(full, G::kBytes);
          const int64_t row = (int64_t)e * kPage + (k % kPer) * G::kSlots;
          const int y = (int)row;
          if (FMT == CERTKV_STORE_BF16) {
            tc::tma_load_2d(st + G::kK, tmK, 0, y, full);
            tc::tma_load_2d(st + G::kK + G::kCodes / 2, tmK, 64, y, full);
            tc::tma_load_2d(st + G::kV, tmV, 0, y, full);
            tc::tma_load_2d(st + G::kV + G::kCodes / 2, tmV, 64, y, full);
          } else {
            tc::tma_load_2d(st + G::kK, tmK, 0, y, full);
            tc::tma_load_2d(st + G::kV, tmV, 0, y, full);
            tc::bulk_load(st + G::kKs, p.st.ks + row, G::kScl, full);
            tc::bulk_load(st + G::kVs, p.st.vs + row, G::kScl, full);
          }
          if (FMT == CERTKV_STORE_FP4) {
            tc::bulk_load(st + G::kKg, p.st.kg + row * kGroups, G::kGrp, full);
            tc::bulk_load(st + G::kVg, p.st.vg + row * kGroups, G::kGrp, full);
          }
        }
      }
    }
  }
  if (lane == 0) {  // the last copies land before the CTA may exit
    volatile int dummy = 0;
    for (int64_t i = issued > G::kStages ? issued - G::kStages : 0; i < issued; ++i)
      if (copied >> (i % G::kStages) & 1u)
        tc::mbar_wait(bar(&tl->full[i % G::kStages]), (uint32_t)((i / G::kStages) & 1), &dummy);
  }
  __syncwarp();
}

// ------------------------------------------------------------ consumers --
template <int FMT>
__device__ __forceinline__ void consume(const TreeArgs& p, char* smem, float* wacc, Tail* tl, int tid,
                                        const int64_t* first, int64_t per) {
  using G = Geo<FMT>;
  constexpr bool kQuant = G::kQuant;
  constexpr int kNb = G::kSlots / 8;  // eight-slot blocks of a tile
  const int cw = tid >> 5, lane = tid & 31, qr = lane >> 2, qc = lane & 3;
  const uint32_t sm = tc::saddr(smem);
  int64_t tile = 0;  // tiles of this CTA before the item
  bool ok = true;
  Items items(p, first, per);
  Item it;
  while (items.next(p, &it)) {
    const int bl = it.u / p.H, h = it.u - bl * p.H, b = bl / p.L, l = bl - b * p.L;
    const int row0 = it.blk * p.rb, rows = min(p.rb, p.rows - row0);  // of the block
    // ---- queries as A fragments; for an 8-bit store kept where the warp's sums go
    // at the end, which makes room for four blocks' keys at a time (161 -> 156 us;
    // a 4-bit store's keys are half the registers: 155 -> 167)
    uint32_t qa[8][4];
    float sl[2];  // per row: scale of its logits (log2 domain)
#pragma unroll
    for (int rr = 0; rr < 2; ++rr) {
      const int r = row0 + qr + 8 * rr, t = r / p.G, g = r - t * p.G;
      const uint16_t* row = qr + 8 * rr < rows ? p.q.at(b, l, t, h * p.G + g) : nullptr;
      if (kQuant) {
        uint32_t w[16], top = 0;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const uint4 x = row ? __ldg(reinterpret_cast<const uint4*>(row + 32 * qc) + i) : make_uint4(0u, 0u, 0u, 0u);
          w[4 * i] = x.x;
          w[4 * i + 1] = x.y;
          w[4 * i + 2] = x.z;
          w[4 * i + 3] = x.w;
        }
#pragma unroll
        for (int i = 0; i < 16; ++i) top = max(top, max((w[i] & 0x7fffu) << 16, w[i] & 0x7fff0000u));
        top = max(top, __shfl_xor_sync(kFull, top, 1));
        top = max(top, __shfl_xor_sync(kFull, top, 2));
        const int e = min(max(exponent(__uint_as_float(top)), -120), 120);
        const float f = pow2(-e);
        sl[rr] = fmaxf(pow2(e) * p.scale_log2, 1.1754944e-38f);
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
#pragma unroll
          for (int z = 0; z < 2; ++z) {
            const uint32_t x = w[2 * ks + z];
            qa[ks][rr + 2 * z] = pack_f16(__uint_as_float(x << 16) * f, __uint_as_float(x & 0xffff0000u) * f);
          }
        }
      } else {
        sl[rr] = fmaxf(p.scale_log2, 1.1754944e-38f);
#pragma unroll
        for (int ks = 0; ks < 8; ++ks) {
          const uint32_t* x = reinterpret_cast<const uint32_t*>(row) + 8 * ks + qc;
          qa[ks][rr] = row ? __ldg(x) : 0u;
          qa[ks][rr + 2] = row ? __ldg(x + 4) : 0u;
        }
      }
    }
    float* acc = wacc + cw * kRows * kD;  // this warp's
    const uint32_t qf = tc::saddr(acc) + (uint32_t)(lane * 16);
    const uint32_t lv = tc::saddr(acc) + kRows * kD * 2;  // a tile's log2_scale, behind the queries
    if (FMT == CERTKV_STORE_FP8) {
#pragma unroll
      for (int ks = 0; ks < 8; ++ks)
        *reinterpret_cast<uint4*>(acc + (ks * 32 + lane) * 4) = make_uint4(qa[ks][0], qa[ks][1], qa[ks][2], qa[ks][3]);
      __syncwarp();
    }
    float C[2] = {-INFINITY, -INFINITY}, ls[2] = {0.f, 0.f};
    float o[16][4];
#pragma unroll
    for (int i = 0; i < 16; ++i) o[i][0] = o[i][1] = o[i][2] = o[i][3] = 0.f;
    const int n = it.kb - it.ka;
    for (int k = (int)((cw - tile % kConsumers + kConsumers) % kConsumers); k < n; k += kConsumers) {
      const int64_t ti = tile + k;
      const int s = (int)(ti % G::kStages);
      ok = ok && __all_sync(kFull, tc::mbar_wait(bar(&tl->full[s]), (uint32_t)((ti / G::kStages) & 1), &tl->abort));
      if (!ok) break;
      const uint32_t st = sm + (uint32_t)(s * G::kStage);
      const int live = tl->live[s];
      if (live > 0) {
        if (live < G::kSlots) {
          // values past the live slots may hold anything: a weight of 0 would not
          // silence a NaN
          char* v = smem + s * G::kStage + G::kV;
          constexpr int kRow = FMT == CERTKV_STORE_BF16 ? 128 : row_bytes(FMT);  // bytes of a row (half)
          for (int i = live * kRow + lane * 16; i < G::kSlots * kRow; i += 512) {
            *reinterpret_cast<uint4*>(v + i) = make_uint4(0u, 0u, 0u, 0u);
            if (FMT == CERTKV_STORE_BF16)
              *reinterpret_cast<uint4*>(v + G::kCodes / 2 + i) = make_uint4(0u, 0u, 0u, 0u);
          }
          if (FMT == CERTKV_STORE_FP4)
            for (int i = live * kGroups + lane; i < G::kSlots * kGroups; i += 32) smem[s * G::kStage + G::kVg + i] = 0;
          __syncwarp();
        }
        // ---- logarithms of the value scales (see tree.cuh)
        bool zeroed = live < G::kSlots;
        if (kQuant) {
          uint32_t one[G::kSlots / 32];  // slots of scale 1: whether they are zero
#pragma unroll
          for (int i = 0; i < G::kSlots / 32; ++i) {
            const uint32_t at = 4u * (lane + 32 * i);
            const float x = lane + 32 * i < live ? lds32f(st + G::kVs + at) : 0.f;
            if (lane + 32 * i >= live) sts32f(st + G::kVs + at, 0.f);
            sts32f(lv + at, log2_scale(x));
            one[i] = __ballot_sync(kFull, x == 1.f);
          }
#pragma unroll
          for (int i = 0; i < G::kSlots / 32; ++i) {
            for (; one[i]; one[i] &= one[i] - 1) {
              const int r = 32 * i + __ffs(one[i]) - 1;
              constexpr int kRow = row_bytes(FMT);
              const uint32_t c = 4 * lane < kRow ? lds32(st + (uint32_t)(G::kV + r * kRow + 4 * lane)) : 0u;
              if (__any_sync(kFull, nonzero_codes<FMT>(c) != 0u)) continue;
              zeroed = true;
              if (lane == (r & 31)) {
                sts32f(st + G::kVs + 4u * r, 0.f);
                sts32f(lv + 4u * r, log2_scale(0.f));
              }
            }
          }
          __syncwarp();
        }
        // ---- S = Q K^T
        float sc[kNb][4];
#pragma unroll
        for (int nb = 0; nb < kNb; ++nb) sc[nb][0] = sc[nb][1] = sc[nb][2] = sc[nb][3] = 0.f;
        if constexpr (FMT == CERTKV_STORE_BF16) {
          const int mi = lane >> 3, mr = lane & 7;
#pragma unroll
          for (int ks = 0; ks < 8; ++ks) {
#pragma unroll
            for (int np = 0; np < kNb / 2; ++np) {
              uint32_t b0, b1, b2, b3;
              const int row = 8 * (2 * np + (mi >> 1)) + mr, c = 2 * ks + (mi & 1);
              ldsm4(st + G::kK + (uint32_t)((c >> 3) * (G::kCodes / 2) + row * 128 + (((c & 7) ^ (row & 7)) << 4)),
                    b0, b1, b2, b3);
              mma<true>(sc[2 * np], qa[ks], b0, b1);
              mma<true>(sc[2 * np + 1], qa[ks], b2, b3);
            }
          }
        } else if constexpr (FMT == CERTKV_STORE_FP8) {
          // four blocks at a time: a block's products depend on one another
#pragma unroll
          for (int nb = 0; nb < kNb; nb += 4) {
#pragma unroll
            for (int c = 0; c < 2; ++c) {
              uint32_t w[4][4];
#pragma unroll
              for (int y = 0; y < 4; ++y) {
                const int row = 8 * (nb + y) + qr;
                const uint4 x = lds128(st + G::kK + (uint32_t)(row * 128 + (((2 * qc + c) ^ (row & 7)) << 4)));
                w[y][0] = x.x;
                w[y][1] = x.y;
                w[y][2] = x.z;
                w[y][3] = x.w;
              }
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const uint4 q = lds128(qf + (uint32_t)((4 * c + i) * 512));
                const uint32_t a[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
                for (int y = 0; y < 4; ++y)
                  mma<false>(sc[nb + y], a, e4m3x2_to_f16x2(w[y][i] & 0xffffu),
                             e4m3x2_to_f16x2(w[y][i] >> 16));
              }
            }
          }
        } else {
#pragma unroll
          for (int nb = 0; nb < kNb; nb += 4) {
            uint32_t w[4][4], ga[4], gb[4];
#pragma unroll
            for (int y = 0; y < 4; ++y) {
              const int row = 8 * (nb + y) + slot_of<FMT>(qr);
              const uint4 x = lds128(st + G::kK + (uint32_t)(row * 64 + ((qc ^ ((row >> 1) & 3)) << 4)));
              const uint32_t g2 = e4m3x2_to_f16x2(lds16(st + G::kKg + (uint32_t)(row * kGroups + 2 * qc)));
              w[y][0] = x.x;
              w[y][1] = x.y;
              w[y][2] = x.z;
              w[y][3] = x.w;
              ga[y] = __byte_perm(g2, g2, 0x1010);
              gb[y] = __byte_perm(g2, g2, 0x3232);
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
#pragma unroll
              for (int y = 0; y < 4; ++y) {
                const uint32_t g = i < 2 ? ga[y] : gb[y];
                mma<false>(sc[nb + y], qa[2 * i], hmul2(e2m1x2_to_f16x2<0>(w[y][i]), g),
                           hmul2(e2m1x2_to_f16x2<1>(w[y][i]), g));
              }
#pragma unroll
              for (int y = 0; y < 4; ++y) {
                const uint32_t g = i < 2 ? ga[y] : gb[y];
                mma<false>(sc[nb + y], qa[2 * i + 1], hmul2(e2m1x2_to_f16x2<2>(w[y][i]), g),
                           hmul2(e2m1x2_to_f16x2<3>(w[y][i]), g));
              }
            }
          }
        }
        // ---- weights; this thread's slots of block nb: columns 2 qc, 2 qc + 1
        const int c0 = slot_of<FMT>(2 * qc), c1 = slot_of<FMT>(2 * qc + 1);
        float mx[2] = {-INFINITY, -INFINITY};  // of the products, or of x + log2 vs
#pragma unroll
        for (int nb = 0; nb < kNb; ++nb) {
          if (kQuant) {
            const float k0 = lds32f(st + G::kKs + 4 * (8 * nb + c0)), k1 = lds32f(st + G::kKs + 4 * (8 * nb + c1));
            sc[nb][0] *= k0;
            sc[nb][1] *= k1;
            sc[nb][2] *= k0;
            sc[nb][3] *= k1;
          }
          if (live < G::kSlots) {
            if (8 * nb + c0 >= live) sc[nb][0] = sc[nb][2] = -INFINITY;
            if (8 * nb + c1 >= live) sc[nb][1] = sc[nb][3] = -INFINITY;
          }
          if (kQuant) {
            const float l0 = lds32f(lv + 4 * (8 * nb + c0)), l1 = lds32f(lv + 4 * (8 * nb + c1));
            mx[0] = um::max3(mx[0], fmaf(sc[nb][0], sl[0], l0), fmaf(sc[nb][1], sl[0], l1));
            mx[1] = um::max3(mx[1], fmaf(sc[nb][2], sl[1], l0), fmaf(sc[nb][3], sl[1], l1));
          } else {
            mx[0] = um::max3(mx[0], sc[nb][0], sc[nb][1]);
            mx[1] = um::max3(mx[1], sc[nb][2], sc[nb][3]);
          }
        }
        float f[2], off[2];
#pragma unroll
        for (int rr = 0; rr < 2; ++rr) {
          mx[rr] = fmaxf(mx[rr], __shfl_xor_sync(kFull, mx[rr], 1));
          mx[rr] = fmaxf(mx[rr], __shfl_xor_sync(kFull, mx[rr], 2));
          const float x = kQuant ? ceilf(mx[rr] - kHead) : mx[rr] * sl[rr];
          f[rr] = 1.f;
          if (x > C[rr] + kLazy || C[rr] == -INFINITY) {
            const float nc = fmaxf(x, C[rr]);
            // quantised: of half the step, as a step of 2^127 and more, whose factor is 0, may
            // leave much of a sum
            if (C[rr] > -INFINITY) f[rr] = um::ex2((kQuant ? 0.5f : 1.f) * (C[rr] - nc));
            C[rr] = nc;
          }
          off[rr] = C[rr] == -INFINITY ? 0.f : -C[rr];
        }
        if (__any_sync(kFull, f[0] != 1.f || f[1] != 1.f)) {
          ls[0] *= f[0];
          ls[1] *= f[1];
          if (kQuant) {
            ls[0] *= f[0];
            ls[1] *= f[1];
            f[0] *= f[0];
            f[1] *= f[1];
          }
#pragma unroll
          for (int i = 0; i < 16; ++i) {
            o[i][0] *= f[0];
            o[i][1] *= f[0];
            o[i][2] *= f[1];
            o[i][3] *= f[1];
          }
        }
        float sum0 = 0.f, sum1 = 0.f;
#pragma unroll
        for (int nb = 0; nb < kNb; ++nb) {
          sc[nb][0] = um::ex2(fmaf(sc[nb][0], sl[0], off[0]));
          sc[nb][1] = um::ex2(fmaf(sc[nb][1], sl[0], off[0]));
          sc[nb][2] = um::ex2(fmaf(sc[nb][2], sl[1], off[1]));
          sc[nb][3] = um::ex2(fmaf(sc[nb][3], sl[1], off[1]));
          sum0 += sc[nb][0] + sc[nb][1];
          sum1 += sc[nb][2] + sc[nb][3];
          if (kQuant) {
            const float v0 = lds32f(st + G::kVs + 4 * (8 * nb + c0)), v1 = lds32f(st + G::kVs + 4 * (8 * nb + c1));
            sc[nb][0] *= v0;
            sc[nb][1] *= v1;
            sc[nb][2] *= v0;
            sc[nb][3] *= v1;
          }
        }
        ls[0] += sum0;
        ls[1] += sum1;
        // ---- O += P V, sixteen slots a k-step
#pragma unroll
        for (int kb = 0; kb < kNb / 2; ++kb) {
          const float(&x)[4] = sc[2 * kb];
          const float(&y)[4] = sc[2 * kb + 1];
          uint32_t pa[4];
          if (kQuant) {
            pa[0] = pack_f16(x[0], x[1]);
            pa[1] = pack_f16(x[2], x[3]);
            pa[2] = pack_f16(y[0], y[1]);
            pa[3] = pack_f16(y[2], y[3]);
          } else {
            pa[0] = pack_bf16(x[0], x[1]);
            pa[1] = pack_bf16(x[2], x[3]);
            pa[2] = pack_bf16(y[0], y[1]);
            pa[3] = pack_bf16(y[2], y[3]);
          }
          if constexpr (FMT == CERTKV_STORE_BF16) {
            const uint32_t pl[4] = {pack_bf16(x[0] - bf16lo(pa[0]), x[1] - bf16hi(pa[0])),
                                    pack_bf16(x[2] - bf16lo(pa[1]), x[3] - bf16hi(pa[1])),
                                    pack_bf16(y[0] - bf16lo(pa[2]), y[1] - bf16hi(pa[2])),
                                    pack_bf16(y[2] - bf16lo(pa[3]), y[3] - bf16hi(pa[3]))};
            const int mi = lane >> 3, mr = lane & 7;
#pragma unroll
            for (int np = 0; np < 8; ++np) {
              uint32_t b0, b1, b2, b3;
              const int row = 16 * kb + 8 * (mi & 1) + mr, c = 2 * np + (mi >> 1);
              ldsm4t(st + G::kV + (uint32_t)((c >> 3) * (G::kCodes / 2) + row * 128 + (((c & 7) ^ (row & 7)) << 4)),
                     b0, b1, b2, b3);
              mma<true>(o[2 * np], pa, b0, b1);
              mma<true>(o[2 * np + 1], pa, b2, b3);
              mma<true>(o[2 * np], pl, b0, b1);
              mma<true>(o[2 * np + 1], pl, b2, b3);
            }
          } else if constexpr (FMT == CERTKV_STORE_FP8) {
            uint32_t w[4][4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int row = 16 * kb + 8 * (i >> 1) + 2 * qc + (i & 1);
              const uint4 v = lds128(st + G::kV + (uint32_t)(row * 128 + ((qr ^ (row & 7)) << 4)));
              w[i][0] = v.x;
              w[i][1] = v.y;
              w[i][2] = v.z;
              w[i][3] = v.w;
            }
#pragma unroll
            for (int j = 0; j < 4; ++j) {
              const uint32_t a0 = __byte_perm(w[0][j], w[1][j], 0x5140), a1 = __byte_perm(w[0][j], w[1][j], 0x7362);
              const uint32_t b0 = __byte_perm(w[2][j], w[3][j], 0x5140), b1 = __byte_perm(w[2][j], w[3][j], 0x7362);
              mma<false>(o[4 * j], pa, e4m3x2_to_f16x2(a0 & 0xffffu), e4m3x2_to_f16x2(b0 & 0xffffu));
              mma<false>(o[4 * j + 1], pa, e4m3x2_to_f16x2(a0 >> 16), e4m3x2_to_f16x2(b0 >> 16));
              mma<false>(o[4 * j + 2], pa, e4m3x2_to_f16x2(a1 & 0xffffu), e4m3x2_to_f16x2(b1 & 0xffffu));
              mma<false>(o[4 * j + 3], pa, e4m3x2_to_f16x2(a1 >> 16), e4m3x2_to_f16x2(b1 >> 16));
            }
          } else {
            uint32_t w[4][2], g[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const int row = 16 * kb + 8 * (i >> 1) + slot_of<FMT>(2 * qc + (i & 1));
              const uint2 v =
                  lds64(st + G::kV + (uint32_t)(row * 64 + (((qr >> 1) ^ ((row >> 1) & 3)) << 4) + (qr & 1) * 8));
              w[i][0] = v.x;
              w[i][1] = v.y;
              g[i] = lds8(st + G::kVg + (uint32_t)(row * kGroups + qr));
            }
            const uint32_t ga = e4m3x2_to_f16x2(g[0] | (g[1] << 8)), gb = e4m3x2_to_f16x2(g[2] | (g[3] << 8));
#pragma unroll
            for (int j = 0; j < 2; ++j) {
#define CERTKV_PAIR(B)                                                                               \
  {                                                                                                  \
    const uint32_t x0 = e2m1x2_to_f16x2<B>(w[0][j]), x1 = e2m1x2_to_f16x2<B>(w[1][j]);               \
    const uint32_t y0 = e2m1x2_to_f16x2<B>(w[2][j]), y1 = e2m1x2_to_f16x2<B>(w[3][j]);               \
    mma<false>(o[8 * j + 2 * B], pa, hmul2(__byte_perm(x0, x1, 0x5410), ga),                         \
               hmul2(__byte_perm(y0, y1, 0x5410), gb));                                              \
    mma<false>(o[8 * j + 2 * B + 1], pa, hmul2(__byte_perm(x0, x1, 0x7632), ga),                     \
               hmul2(__byte_perm(y0, y1, 0x7632), gb));                                              \
  }
              CERTKV_PAIR(0)
              CERTKV_PAIR(1)
              CERTKV_PAIR(2)
              CERTKV_PAIR(3)
#undef CERTKV_PAIR
            }
          }
        }
        // zeros written above come before the next copy into the stage
        if (zeroed) um::fence_async();
      }
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(bar(&tl->empty[s]));
    }
    // ---- join the consumers: sums and accumulators relative to 2^C; a quantised store's C
    // goes with the values, so a sum's own exponent is taken into its reference
#pragma unroll
    for (int rr = 0; rr < 2; ++rr) {
      ls[rr] += __shfl_xor_sync(kFull, ls[rr], 1);
      ls[rr] += __shfl_xor_sync(kFull, ls[rr], 2);
      const int r = qr + 8 * rr;
      if (r >= rows) continue;
      if (qc == 0) {
        const int e = kQuant ? exponent(ls[rr]) : 0;
        tl->m[cw][r] = C[rr] + (float)e;
        tl->l[cw][r] = ls[rr] * pow2(-e);
        tl->e[cw][r] = (float)e;
      }
#pragma unroll
      for (int i = 0; i < 16; ++i) {
        float* a = acc + r * kD;
        a[element_of<FMT>(i, qc, 0)] = o[i][2 * rr];
        a[element_of<FMT>(i, qc, 1)] = o[i][2 * rr + 1];
      }
    }
    consumers_sync();
    const int64_t rec = (int64_t)blockIdx.x + (int64_t)it.u * p.nblk + it.blk;
    const bool failed = tl->abort != 0;
    for (int i = tid; i < rows * (kD / 4); i += kConsumers * 32) {
      const int r = i / (kD / 4), d = 4 * (i - r * (kD / 4));
      float M = -INFINITY, L = 0.f;
#pragma unroll
      for (int w = 0; w < kConsumers; ++w) M = fmaxf(M, tl->m[w][r]);
      float4 A = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int w = 0; w < kConsumers; ++w) {
        if (tl->l[w][r] == 0.f) continue;
        const float x = tl->m[w][r] - M, f = exp2f(x), g = kQuant ? exp2f(x - tl->e[w][r]) : f;
        const float4 a = *reinterpret_cast<const float4*>(wacc + (w * kRows + r) * kD + d);
        L = fmaf(tl->l[w][r], f, L);
        A.x = fmaf(a.x, g, A.x);
        A.y = fmaf(a.y, g, A.y);
        A.z = fmaf(a.z, g, A.z);
        A.w = fmaf(a.w, g, A.w);
      }
      const float inv = L != 0.f ? 1.f / L : 0.f;
      *reinterpret_cast<float4*>(p.rec_acc + (rec * p.rb + r) * kD + d) =
          make_float4(A.x * inv, A.y * inv, A.z * inv, A.w * inv);
      if (d == 0)
        p.rec_ml[rec * p.rb + r] = tree_record(true, failed, M, L);
    }
    consumers_sync();
    tile += n;
  }
}

// grid = p.ctas, block = kThreads.
template <int FMT>
__global__ void __launch_bounds__(kThreads, 2) tree_mma_kernel(const __grid_constant__ CUtensorMap tmK,
                                                               const __grid_constant__ CUtensorMap tmV,
                                                               const __grid_constant__ TreeArgs p) {
  using G = Geo<FMT>;
  extern __shared__ char smem_raw[];
  char* sm = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  float* wacc = reinterpret_cast<float*>(sm + G::kStages * G::kStage);
  Tail* tl = reinterpret_cast<Tail*>(wacc + kConsumers * kRows * kD);
  if (threadIdx.x == 0) {
    for (int i = 0; i < G::kStages; ++i) {
      tc::mbar_init(bar(&tl->full[i]), 1);
      tc::mbar_init(bar(&tl->empty[i]), 1);
    }
    tl->abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  release_next();
  await_previous();
  const int64_t* first = tree_first(p, tl->first, small_tile(FMT), false);
  const int64_t per = tiles_per_cta(p, first);
  if (per * blockIdx.x >= first[p.units] * p.nblk) return;  // uniform, before any barrier
  __syncthreads();
  if (threadIdx.x < 32) produce<FMT>(p, &tmK, &tmV, tc::saddr(sm), tl, threadIdx.x, first, per);
  else consume<FMT>(p, sm, wacc, tl, threadIdx.x - 32, first, per);
  __syncthreads();
  if (threadIdx.x == 0 && tl->abort && p.st.status) atomicOr(p.st.status, CERTKV_STATUS_TIMEOUT);
}

constexpr int kMaxDevices = 64;
template <int FMT>
int ctas_of_device() {
  static int cached[kMaxDevices] = {};
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return 0;
  if (dev < kMaxDevices && cached[dev] > 0) return cached[dev];
  int sms = 0, per_sm = 0;
  if (cudaFuncSetAttribute(tree_mma_kernel<FMT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes<FMT>()) !=
          cudaSuccess ||
      cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
      cudaOccupancyMaxActiveBlocksPerMultiprocessor(&per_sm, tree_mma_kernel<FMT>, kThreads, smem_bytes<FMT>()) !=
          cudaSuccess ||
      per_sm < 1 || sms < 1)
    return 0;
  if (dev < kMaxDevices) cached[dev] = sms * per_sm;
  return sms * per_sm;
}

template <int FMT>
bool launch(const TreeArgs& p, cudaStream_t st) {
  CUtensorMap mk, mv;
  const uint64_t rows = (uint64_t)p.st.pool_pages * kPage;
  if (FMT == CERTKV_STORE_BF16) {
    if (!make_row_map(&mk, p.st.k, rows, Geo<FMT>::kSlots) || !make_row_map(&mv, p.st.v, rows, Geo<FMT>::kSlots))
      return false;
  } else if (!make_code_map(&mk, p.st.k, row_bytes(FMT), rows, Geo<FMT>::kSlots) ||
             !make_code_map(&mv, p.st.v, row_bytes(FMT), rows, Geo<FMT>::kSlots)) {
    return false;
  }
  return launch_kernel(true, tree_mma_kernel<FMT>, p.ctas, kThreads, smem_bytes<FMT>(), st, mk, mv, p);
}

}  // namespace

int tree_mma_ctas(int format) {
  return format == CERTKV_STORE_BF16  ? ctas_of_device<CERTKV_STORE_BF16>()
         : format == CERTKV_STORE_FP8 ? ctas_of_device<CERTKV_STORE_FP8>()
                                      : ctas_of_device<CERTKV_STORE_FP4>();
}

bool launch_tree_mma(const TreeArgs& p, int format, cudaStream_t st) {
  TraceScope ts_("tree_split", st);
  return format == CERTKV_STORE_BF16  ? launch<CERTKV_STORE_BF16>(p, st)
         : format == CERTKV_STORE_FP8 ? launch<CERTKV_STORE_FP8>(p, st)
                                      : launch<CERTKV_STORE_FP4>(p, st);
}

}  // namespace certkv
