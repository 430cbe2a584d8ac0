// grad_kv.cu — the stored slots' gradients on the 5th-generation tensor cores, and with few query
// rows those of the queries in the same pass.
//
// A CTA walks a share of all tiles of 128 slots, which are the M = 128 rows of the MMAs, and for
// each the unit's query rows in blocks of at most 64, the N columns:
//   S = K Q^T,  R = V dO^T,  p = 2^(S - lse),  e = p (R - delta),
//   dV += p dO,  dK += e Q,
// p and e handed over in tensor memory as two bf16 parts each, the first over S and the second
// over R (2^-14 at most; one part each took 225 us for 279 with 1024 rows over 32768 slots, and left
// 1.4 to 1.5 times the error).  Blocks of 64 columns leave room in tensor memory for two of them
// beside dV and dK, so that one block's S and R are made while p and e of the other are:
// S, R | S, R (64 columns each) | dV | dK (128 each).  Each block reads K and V from shared memory
// again, which with the rows and their coming takes 1500 clocks of the 2270 a block's step has.
//
// Up to 64 rows (FUSED) a segment is one block, whose rows stay in shared memory, and
// dQ^T += K^T e (M = 128 elements of a row) is summed over the share's tiles in the columns of
// the second block; e times the key's scale is handed over in shared memory for it, in two parts
// too.  The store is then read once for all gradients, and over bf16 the time is that of its bytes
// (64 rows over 13107 slots of 256 segments: 3.4 GB in 530 us, 96 % of a copy's rate; 8- and 4-bit
// 589 and 586 us, the pace of writing two and four times the bytes read).  Reading it again for
// the queries' kernel would cost as much as reading it here.
//
// Every wait is bounded; on a timeout the roles stop waiting, the rows and slots in question get
// NaN and the store's status word CERTKV_STATUS_TIMEOUT.
#include <atomic>

#include "../../include/certkv.h"
#include "grad_tc.cuh"
#include "internal.cuh"

namespace certkv {
namespace {

// Warps: softmax, loaders, four that write the slots' gradients (a whole warpgroup each: a warp
// reaches the quarter of tensor memory that its number mod 4 says), the issuer and a lane each that
// asks for rows and for codes.
constexpr int kSoftWarps = 8, kLoadWarps = 2 * kGroupWarps, kDrainWarps = 4;
constexpr int kDrain = kSoftWarps + kLoadWarps, kIssue = kDrain + kDrainWarps;
constexpr int kThreads = (kIssue + 4) * 32;
// Registers a thread: the launch gives 80, which the roles share out among themselves.
constexpr int kLaunchRegs = 80;
constexpr int kSoftRegs = 104, kLoadRegs = 64, kDrainRegs = 72, kIssueRegs = 72;
static_assert(kSoftWarps * 32 * kSoftRegs + kLoadWarps * 32 * kLoadRegs + kDrainWarps * 32 * kDrainRegs + 128 * kIssueRegs <=
                  kThreads * kLaunchRegs,
              "a larger split would wait for registers for ever");
constexpr int kCols = kGradFused;       // query rows of a block
constexpr int kRowHalf = kCols * 128;   // bytes of a block's 64 rows x 64 elements
constexpr int kBlock = 4 * kRowHalf;    // a block: its rows, then their gradients
constexpr uint32_t kColV = 256, kColK = 384, kColQ = 128;  // S of block i: column 128 (i & 1), R 64 on

template <int FMT, bool FUSED>
struct Plan {
  // More than 64 rows: blocks of rows on their way are worth more than a second place for keys or
  // values (1024 rows over 32768 slots: 279 us with 1 + 1 + 4 blocks, 282 with 1 + 2 + 3, 287 with
  // 2 + 1 + 3, 387 with 2 + 2 + 2).
  static constexpr int kKeys = FUSED ? 2 : 1;  // places of the rings: keys are read again for dQ
  static constexpr int kValues = FUSED && FMT == CERTKV_STORE_BF16 ? 2 : 1;
  static constexpr int kBlocks = FUSED ? (FMT == CERTKV_STORE_BF16 ? 2 : 1) : FMT == CERTKV_STORE_BF16 ? 4 : 3;
  static constexpr int kValueOff = kKeys * kOperand;
  static constexpr int kBlockOff = kValueOff + kValues * kOperand;
  static constexpr int kEOff = kBlockOff + kBlocks * kBlock;  // e, FUSED: two parts [128 slots][64 rows]
  static constexpr int kStageOff = kEOff + (FUSED ? 2 * kHalf : 0);  // of keys, then of values
  // Slots' gradients are written by lines through shared memory, half a row of 32 slots a warp (over
  // 13107 slots of 256 segments, 8 bits, 64 rows 589 us, 645 by sectors; 4 bits 586 and 603), but by
  // sectors where a bf16 store's bytes bound the pass (64 rows 530 us, and by lines, which leave room
  // for one block of rows only, 553; 4 rows 573 and 553).
  static constexpr bool kLines = !FUSED || FMT != CERTKV_STORE_BF16;
  static constexpr int kDrainOff = kStageOff + 2 * gt::kStage<FMT>;
  static constexpr int kMiscOff = kDrainOff + (kLines ? kDrainWarps * 4096 : 0);
};
template <int FMT, bool FUSED>
struct Misc {
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2];
  uint64_t b_full[4], b_empty[4];
  uint64_t s_full[2], p_full[2], o_full[2], drained[2], done;  // o_full, drained: dV, dK
  uint64_t st_full[2], st_empty[2];  // stretches of codes, keys' and values'
  int2 live[2];  // of the stretches
  uint32_t tmem;
  int abort, own[5];  // own: flags of the issuer, the feeder of rows, the copiers of keys and values, the stager
  alignas(16) float nlse[Plan<FMT, FUSED>::kBlocks][kCols], ndelta[Plan<FMT, FUSED>::kBlocks][kCols];  // negated
};
template <int FMT, bool FUSED>
constexpr int smem_bytes() {
  static_assert(Plan<FMT, FUSED>::kMiscOff + sizeof(Misc<FMT, FUSED>) <= 232448,
                "over the 227 KB of shared memory a CTA can have");
  return Plan<FMT, FUSED>::kMiscOff + (int)sizeof(Misc<FMT, FUSED>);
}

// Blocks of 64 rows of a unit, and the rows of block j.
__device__ __forceinline__ int blocks_of(const GradArgs& p) { return (p.rows + kCols - 1) / kCols; }
__device__ __forceinline__ int rows_of_block(const GradArgs& p, int j) { return min(kCols, p.rows - j * kCols); }
__device__ __forceinline__ uint32_t up16(int n) { return (uint32_t)(n + 15) & ~15u; }

// Where in the walk a block stands: block j of tile t, number i of all.
struct Step {
  uint32_t i, t, blk;  // blk: number of the block in shared memory
  int j, n;            // its place among the tile's n
  bool first, last;    // FUSED: the item's first and last tile
};
template <bool FUSED>
struct Steps {
  const GradArgs& p;
  gt::Walk walk;
  gt::Item it;
  int k, j, n;
  uint32_t i = 0, t = 0, item = 0;
  __device__ __forceinline__ Steps(const GradArgs& p_, const gt::Walk& w) : p(p_), walk(w) {
    it = {0, 0, 0};
    k = j = 0;
    n = blocks_of(p_);
  }
  __device__ __forceinline__ bool next(Step* s) {
    if (k == it.kb) {
      if (!walk.next(p, &it)) return false;
      k = it.ka;
      ++item;
    }
    *s = {i, t, FUSED ? item - 1 : i, j, n, k == it.ka, k + 1 == it.kb};
    ++i;
    if (++j == n) {
      j = 0;
      ++k;
      ++t;
    }
    return true;
  }
};

// A lane that brings blocks of rows and their gradients into shared memory, each for a tile
// (FUSED: for an item), by bulk copies.
template <int FMT, bool FUSED>
struct RowFeeder {
  using P = Plan<FMT, FUSED>;
  using M = Misc<FMT, FUSED>;
  const GradArgs& p;
  uint32_t base;
  uint32_t n = 0;

  __device__ __forceinline__ bool block(int u, int j) {
    const uint32_t place = n % P::kBlocks, full = GRAD_AT(b_full) + 8u * place, rows = up16(rows_of_block(p, j));
    if (!gt::wait(GRAD_AT(b_empty) + 8u * place, ((n / P::kBlocks) & 1u) ^ 1u, GRAD_AT(abort))) return false;
    tc::mbar_expect_tx(full, rows * (4u * 128u + 2u * 4u));
#pragma unroll 1
    for (int part = 0; part < 4; ++part)
      tc::bulk_load(base + P::kBlockOff + place * kBlock + part * kRowHalf, grad_pack(p, u, part, j * kCols), rows * 128u, full);
    const float* neg = p.neg + (int64_t)u * 2 * p.padded + j * kCols;
    tc::bulk_load(GRAD_AT(nlse) + place * kCols * 4u, neg, rows * 4u, full);
    tc::bulk_load(GRAD_AT(ndelta) + place * kCols * 4u, neg + p.padded, rows * 4u, full);
    ++n;
    return true;
  }
  __device__ __forceinline__ void run(gt::Walk walk) {
    gt::Item it;
    bool ok = true;
#pragma unroll 1
    while (ok && walk.next(p, &it)) {
#pragma unroll 1
      for (int k = it.ka; ok && k < (FUSED ? it.ka + 1 : it.kb); ++k)
#pragma unroll 1
        for (int j = 0; ok && j < blocks_of(p); ++j) ok = block(it.u, j);
    }
    for (uint32_t i = n > P::kBlocks ? n - P::kBlocks : 0; i < n; ++i)  // nothing lands after the CTA has gone
      gt::finish(GRAD_AT(b_full) + 8u * (i % P::kBlocks), (i / P::kBlocks) & 1u, GRAD_AT(own) + 4u);
  }
};

// Issues the MMAs; the whole warp runs, one lane issues.
template <int FMT, bool FUSED>
struct Issuer {
  using P = Plan<FMT, FUSED>;
  using M = Misc<FMT, FUSED>;
  const GradArgs& p;
  uint32_t tmem, base;
  bool ok = true;
  uint32_t tiles = 0;  // whose products have been begun
  uint32_t odd = 0;    // parities of p_full
  __device__ __forceinline__ void wait(uint32_t mbar, uint32_t phase) {
    if (ok) ok = gt::wait_all(mbar, phase & 1u, GRAD_AT(abort));
  }
  __device__ __forceinline__ uint32_t buffer(const Step& s) const { return FUSED ? 0u : s.i & 1u; }
  __device__ __forceinline__ uint32_t columns(const Step& s) const { return up16(rows_of_block(p, s.j)); }
  // S and R of a block
  __device__ __forceinline__ void logits(const Step& s) {
    if (s.j == 0) {
      wait(GRAD_AT(k_full) + 8u * (s.t % P::kKeys), s.t / P::kKeys);
      wait(GRAD_AT(v_full) + 8u * (s.t % P::kValues), s.t / P::kValues);
    }
    if (!FUSED || s.first) wait(GRAD_AT(b_full) + 8u * (s.blk % P::kBlocks), s.blk / P::kBlocks);
    if (!ok) return;
    if (s.j == 0) um::fence_async();  // the loaders' writes, before the tensor core's reads
    um::fence_after();
    const uint32_t d = tmem + 128u * buffer(s), id = um::idesc_n(columns(s), false, false);
    const uint32_t q = um::desc_lo(base + P::kBlockOff, 16) + (s.blk % P::kBlocks) * (kBlock >> 4);
    um::mma_s64(d, um::desc_lo(base, 16) + (s.t % P::kKeys) * (kOperand >> 4), q, um::kDescHi, id, 0u);
    um::mma_s64(d + 64, um::desc_lo(base + P::kValueOff, 16) + (s.t % P::kValues) * (kOperand >> 4),
                q + (2 * kRowHalf >> 4), um::kDescHi, id, 0u);
    um::commit(GRAD_AT(s_full) + 8u * buffer(s));
    if (s.j + 1 == s.n) {
      um::commit(GRAD_AT(v_empty) + 8u * (s.t % P::kValues));
      if (!FUSED) um::commit(GRAD_AT(k_empty) + 8u * (s.t % P::kKeys));
    }
  }
  // what p and e of a block go into
  __device__ __forceinline__ void products(const Step& s) {
    const uint32_t x = buffer(s);
    wait(GRAD_AT(p_full) + 8u * (x), odd >> x & 1u);
    odd ^= 1u << x;
    const bool begins = s.j == 0 && tiles++ > 0;  // those of the tile before are written first
    if (begins) wait(GRAD_AT(drained), tiles - 2);
    if (!ok) return;
    if (FUSED) um::fence_async();
    um::fence_after();
    const uint32_t a = tmem + 128u * x, steps = columns(s) / 16, acc = s.j > 0;
    const uint32_t q = um::desc_lo(base + P::kBlockOff, kRowHalf) + (s.blk % P::kBlocks) * (kBlock >> 4);
    constexpr uint32_t id = um::idesc_n(128, false, true);
    um::mma_p64<8, 32, 40>(tmem + kColV, a, q + (2 * kRowHalf >> 4), um::kDescHi, id, acc, steps);
    um::mma_p64<16, 32, 48>(tmem + kColV, a + 64, q + (2 * kRowHalf >> 4), um::kDescHi, id, 1u, steps);
    if (s.j + 1 == s.n) um::commit(GRAD_AT(o_full));
    if (begins) wait(GRAD_AT(drained) + 8u, tiles - 2);
    if (!ok) return;
    um::fence_after();
    um::mma_p64<8, 32, 40>(tmem + kColK, a + 16, q, um::kDescHi, id, acc, steps);
    um::mma_p64<16, 32, 48>(tmem + kColK, a + 72, q, um::kDescHi, id, 1u, steps);
    if (FUSED) {
      const uint32_t keys = um::desc_lo(base, kHalf) + (s.t % P::kKeys) * (kOperand >> 4), idq = um::idesc_n(columns(s), true, true);
      um::mma_mn(tmem + kColQ, keys, um::desc_lo(base + P::kEOff, 16), um::kDescHi, idq, !s.first);
      um::mma_mn(tmem + kColQ, keys, um::desc_lo(base + P::kEOff + kHalf, 16), um::kDescHi, idq, 1u);
    }
    if (FUSED) um::commit(GRAD_AT(k_empty) + 8u * (s.t % P::kKeys));
    if (!FUSED || s.last) um::commit(GRAD_AT(b_empty) + 8u * (s.blk % P::kBlocks));
    if (s.j + 1 == s.n) um::commit(GRAD_AT(o_full) + 8u);
  }
  __device__ __forceinline__ void run(const gt::Walk& walk) {
    Steps<FUSED> steps(p, walk);
    Step cur, nxt;
    bool more = steps.next(&cur);
    if (more) logits(cur);
#pragma unroll 1
    while (ok && more) {
      more = steps.next(&nxt);
      // behind a tile's last block the next tile may still be on its way; FUSED: there is one
      // buffer, and e of this tile is read by its products before it is written again
      const bool ahead = !FUSED && cur.j + 1 < cur.n;
      if (more && ahead) logits(nxt);
      products(cur);
      if (more && !ahead) logits(nxt);
      cur = nxt;
    }
    um::commit(GRAD_AT(done));  // everything issued above has finished
    gt::finish(GRAD_AT(done), 0, GRAD_AT(own));
    __syncwarp();
  }
};

// The slot of a softmax thread.  Its table entry is looked up a tile before its scales, and these
// a tile before they are used, so that neither load is waited for.
template <int FMT>
struct Slot {
  bool live;
  float ks, vs;  // scales of its key and value
  static __device__ __forceinline__ int entry(const GradArgs& p, int u, int s, int count) {
    return s < count ? __ldg(p.st.table + (int64_t)u * p.st.max_pages + s / kPage) : -1;
  }
  __device__ __forceinline__ void load(const GradArgs& p, int page, int s) {
    live = page >= 0 && page < p.st.pool_pages;
    ks = vs = 1.f;
    if (FMT != CERTKV_STORE_BF16 && live) {
      const int64_t at = (int64_t)page * kPage + s % kPage;
      ks = __ldg(p.st.ks + at);
      vs = __ldg(p.st.vs + at);
    }
  }
};

// Two values as bf16 parts, the upper halves as they are and those of what that leaves: neither
// takes a conversion (2^-14 together, towards 0).
__device__ __forceinline__ void split(float2 x, uint32_t& hi, uint32_t& lo) {
  const float2 y = fadd2(x, make_float2(-__uint_as_float(__float_as_uint(x.x) & 0xffff0000u),
                                        -__uint_as_float(__float_as_uint(x.y) & 0xffff0000u)));
  hi = __byte_perm(__float_as_uint(x.x), __float_as_uint(x.y), 0x7632);
  lo = __byte_perm(__float_as_uint(y.x), __float_as_uint(y.y), 0x7632);
}

__device__ __forceinline__ void store_sector(uint16_t* to, const uint32_t (&w)[8]) {
  asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to), "r"(w[0]), "r"(w[1]), "r"(w[2]),
               "r"(w[3]), "r"(w[4]), "r"(w[5]), "r"(w[6]), "r"(w[7])
               : "memory");
}

template <int FMT, bool FUSED>
__device__ __forceinline__ void softmax(const GradArgs& p, uint32_t base, uint32_t tmem, int tid, int share,
                                        gt::Walk walk) {
  using P = Plan<FMT, FUSED>;
  using M = Misc<FMT, FUSED>;
  constexpr bool kQuant = FMT != CERTKV_STORE_BF16;
  extern __shared__ __align__(1024) char smem[];
  const int warp = tid >> 5, lane = tid & 31, quad = warp & 3, half = warp >> 2;
  const int row = quad * 32 + lane;  // slot of the tile
  const uint32_t at = (uint32_t)(quad * 32) << 16;
  const int blocks = FUSED ? 1 : blocks_of(p);
  uint32_t i = 0, t = 0, item = 0;
  bool ok = true;
  gt::Item it;
#pragma unroll 1
  while (walk.next(p, &it)) {
    const gt::Item now = it;
    const int count = p.st.count(now.u);
    Slot<FMT> next;
    int page = Slot<FMT>::entry(p, now.u, now.ka * kGradTile + row, count);
    if (kQuant) {
      next.load(p, page, row);
      page = Slot<FMT>::entry(p, now.u, (now.ka + 1) * kGradTile + row, count);
    }
#pragma unroll 1
    for (int k = now.ka; k < now.kb; ++k, ++t) {
      Slot<FMT> slot = next;
      (kQuant ? next : slot).load(p, page, row);
      page = Slot<FMT>::entry(p, now.u, (k + 1 + kQuant) * kGradTile + row, count);
      const bool live = slot.live;
      const float key = slot.ks * gt::kCodeScale<FMT>, value = slot.vs * gt::kCodeScale<FMT>;
      const float2 ksl = make_float2(key * p.scale_log2, key * p.scale_log2);
      const float2 vs = make_float2(value, value), ks = make_float2(key, key);
#pragma unroll 1
      for (int j = 0; ok && j < blocks; ++j, ++i) {
        const uint32_t x = FUSED ? 0u : i & 1u, use = FUSED ? i : i >> 1, blk = FUSED ? item : i;
        const uint32_t place = blk % P::kBlocks;
        if (!FUSED || k == now.ka)
          ok = gt::wait_all(GRAD_AT(b_full) + 8u * place, (blk / P::kBlocks) & 1u, GRAD_AT(abort));
        ok = ok && gt::wait_all(GRAD_AT(s_full) + 8u * x, use & 1u, GRAD_AT(abort));
        if (!ok) break;
        um::fence_after();
        if (32 * half < rows_of_block(p, j)) {
          const uint32_t tS = tmem + at + 128u * x + 32u * half;
          const float* nlse = &reinterpret_cast<const M*>(smem + P::kMiscOff)->nlse[place][32 * half];
          const float* ndelta = &reinterpret_cast<const M*>(smem + P::kMiscOff)->ndelta[place][32 * half];
          uint32_t s[32];
          um::ld32(tS, s);
#pragma unroll
          for (int h = 0; h < 2; ++h) {  // 16 rows; the logits are all read before any is written over
            uint32_t r[16];
            um::ld16(tS + 64u + 16u * h, r);
#pragma unroll
            for (int c = 0; c < 2; ++c) {  // eight of them
              uint32_t p1[4], p2[4], e1[4], e2[4], q1[4], q2[4];
#pragma unroll
              for (int i = 0; i < 4; ++i) {
                const int q = 8 * c + 2 * i;
                const float2 l = *reinterpret_cast<const float2*>(nlse + 16 * h + q);
                float2 e = make_float2(__uint_as_float(s[16 * h + q]), __uint_as_float(s[16 * h + q + 1]));
                float2 d = make_float2(__uint_as_float(r[q]), __uint_as_float(r[q + 1]));
                const float2 nd = *reinterpret_cast<const float2*>(ndelta + 16 * h + q);
                e = ffma2(e, ksl, l);
                d = kQuant ? ffma2(d, vs, nd) : fadd2(d, nd);
                e.x = live ? um::ex2(e.x) : 0.f;
                e.y = live ? um::ex2(e.y) : 0.f;
                d = live ? fmul2(e, d) : make_float2(0.f, 0.f);
                split(e, p1[i], p2[i]);
                split(d, e1[i], e2[i]);
                if (FUSED && kQuant) split(fmul2(d, ks), q1[i], q2[i]);
              }
              um::st4(tS + 8u * h + 4u * c, p1);
              um::st4(tS + 16u + 8u * h + 4u * c, e1);
              um::st4(tS + 64u + 16u * h + 4u * c, p2);
              um::st4(tS + 72u + 16u * h + 4u * c, e2);
              if (FUSED) {
                const uint32_t to = base + P::kEOff + (uint32_t)(row * 128 + (((4 * half + 2 * h + c) ^ (row & 7)) << 4));
                const uint32_t *a = kQuant ? q1 : e1, *b = kQuant ? q2 : e2;
                sts128(to, a[0], a[1], a[2], a[3]);
                sts128(to + kHalf, b[0], b[1], b[2], b[3]);
              }
            }
          }
          um::wait_st();
        }
        um::fence_before();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(GRAD_AT(p_full) + 8u * (x));
      }
    }
    ++item;
  }
}

// Whether some row of unit u takes part; by a whole warp.
__device__ __forceinline__ bool takes_part(const GradArgs& p, int u, int lane) {
  const float* nlse = p.neg + (int64_t)u * 2 * p.padded;
  bool any = false;
#pragma unroll 1
  for (int r = 0; !any && r < p.rows; r += 32) any = __any_sync(kFull, r + lane < p.rows && nlse[r + lane] != -INFINITY);
  return any;
}

// The four warps that write a tile's gradients, a slot a thread, while the softmax goes on with
// the next tile; at an item's end (FUSED) its queries' too.  Where no row of the segment takes part
// they are zeros, which the products, of zeros with a slot's NaN or infinity, need not be.
template <int FMT, bool FUSED>
__device__ __forceinline__ void drain(const GradArgs& p, uint32_t base, uint32_t tmem, int tid, int share,
                                        gt::Walk walk) {
  using P = Plan<FMT, FUSED>;
  using M = Misc<FMT, FUSED>;
  const int lane = tid & 31, quad = tid >> 5;
  const uint32_t at = (uint32_t)(quad * 32) << 16;
  const uint32_t mine = base + P::kDrainOff + (uint32_t)quad * 4096u;
  uint32_t t = 0;
  bool ok = true;
  gt::Item it;
#pragma unroll 1
  while (walk.next(p, &it)) {
    const gt::Item now = it;
    const int count = p.st.count(now.u);
    const bool any = takes_part(p, now.u, lane);
#pragma unroll 1
    for (int k = now.ka; k < now.kb; ++k, ++t) {
      // a warp's slots are half a page's
      const int s = k * kGradTile + quad * 32;
      const int page = s < count ? __ldg(p.st.table + (int64_t)now.u * p.st.max_pages + s / kPage) : -1;
      const int rows = page >= 0 && page < p.st.pool_pages ? min(count - s, 32) : 0;
      const int64_t first = ((int64_t)page * kPage + s % kPage) * kD;
#pragma unroll 1
      for (int key = 0; key < 2; ++key) {  // dV, then dK
        ok = ok && gt::wait_all(GRAD_AT(o_full) + 8u * key, t & 1u, GRAD_AT(abort));
        um::fence_after();
        const bool good = ok && !gt::aborted(GRAD_AT(abort)), plain = good && any;
        const uint32_t other = good ? 0u : 0x7fc07fc0u;
        const uint32_t from = tmem + at + (key ? kColK : kColV);
        uint16_t* to = (key ? p.dks : p.dvs) + first;
        const float f = key ? p.scale : 1.f;
        if constexpr (P::kLines) {
#pragma unroll 1
          for (int d0 = 0; d0 < kD; d0 += 64) {  // half a row: written by slot, read by line
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              uint32_t r[32];
              um::ld32(from + (uint32_t)(d0 + 32 * h), r);
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                uint32_t w[4];
#pragma unroll
                for (int q = 0; q < 4; ++q)
                  w[q] = plain ? gt::pack2(__uint_as_float(r[8 * x + 2 * q]) * f, __uint_as_float(r[8 * x + 2 * q + 1]) * f)
                               : other;
                sts128(mine + (uint32_t)(lane * 128 + (((4 * h + x) ^ (lane & 7)) << 4)), w[0], w[1], w[2], w[3]);
              }
            }
            __syncwarp();
            uint16_t* out = to + d0 + 8 * (lane & 7);
#pragma unroll 4
            for (int x = 0; x < 8; ++x) {
              const int row = 4 * x + (lane >> 3);
              const float4 v = gt::lds128(mine + (uint32_t)(row * 128 + (((lane & 7) ^ (row & 7)) << 4)));
              if (row < rows) *reinterpret_cast<float4*>(out + row * kD) = v;
            }
            __syncwarp();
          }
        } else {
#pragma unroll 1
          for (int d0 = 0; d0 < kD; d0 += 16) {  // a sector of a slot a thread
            uint32_t r[16], w[8];
            um::ld16(from + (uint32_t)d0, r);
#pragma unroll
            for (int q = 0; q < 8; ++q)
              w[q] = plain ? gt::pack2(__uint_as_float(r[2 * q]) * f, __uint_as_float(r[2 * q + 1]) * f) : other;
            if (lane < rows) store_sector(to + lane * kD + d0, w);
          }
        }
        if (FUSED && key && p.dq.p && k + 1 == now.kb) {  // element tid of every row
          float* out = grad_record(p, share, now.u, 0) + grad_at(p, 0, tid);
#pragma unroll 1
          for (int r0 = 0; r0 < p.rows; r0 += 16) {
            uint32_t r[16];
            um::ld16(tmem + at + kColQ + (uint32_t)r0, r);
#pragma unroll
            for (int q = 0; q < 16; ++q)
              if (r0 + q < p.rows) out[(r0 + q) * 8] = plain ? __uint_as_float(r[q]) : __uint_as_float(other);
          }
        }
        um::fence_before();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(GRAD_AT(drained) + 8u * key);
      }
    }
  }
}

// grid = groups (one CTA per SM), block = kThreads.
template <int FMT, bool FUSED>
__global__ void __launch_bounds__(kThreads, 1) grad_kv_kernel(const __grid_constant__ CUtensorMap tmK,
                                                              const __grid_constant__ CUtensorMap tmV,
                                                              const __grid_constant__ GradArgs p) {
  using P = Plan<FMT, FUSED>;
  using M = Misc<FMT, FUSED>;
  extern __shared__ __align__(1024) char smem[];
  const uint32_t base = tc::saddr(smem);
  const int warp = __shfl_sync(kFull, (int)threadIdx.x >> 5, 0);  // so that the compiler, too, knows it uniform
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(GRAD_AT(k_full) + 8u * (i), gt::kArrivals<FMT>);
      tc::mbar_init(GRAD_AT(k_empty) + 8u * (i), 1);
      tc::mbar_init(GRAD_AT(v_full) + 8u * (i), gt::kArrivals<FMT>);
      tc::mbar_init(GRAD_AT(v_empty) + 8u * (i), 1);
      tc::mbar_init(GRAD_AT(s_full) + 8u * (i), 1);
      tc::mbar_init(GRAD_AT(p_full) + 8u * (i), kSoftWarps);
      tc::mbar_init(GRAD_AT(st_full) + 8u * i, 1);
      tc::mbar_init(GRAD_AT(st_empty) + 8u * i, kLoadWarps);
    }
    for (int i = 0; i < 4; ++i) {
      tc::mbar_init(GRAD_AT(b_full) + 8u * (i), 1);
      tc::mbar_init(GRAD_AT(b_empty) + 8u * (i), 1);
    }
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(GRAD_AT(o_full) + 8u * i, 1);
      tc::mbar_init(GRAD_AT(drained) + 8u * i, kDrainWarps);
    }
    tc::mbar_init(GRAD_AT(done), 1);
    gt::sts32(GRAD_AT(abort), 0u);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  await_previous();
  release_next();  // behind the wait: what it starts reads what was waited for here
  const int share = blockIdx.x;
  const gt::Walk walk = gt::Walk::of(p, share);
  if (walk.left == 0) return;  // uniform, before any barrier
  if (warp == kIssue) um::alloc(GRAD_AT(tmem), 512);
  um::fence_before();
  __syncthreads();
  um::fence_after();
  const uint32_t tmem = gt::lds32(GRAD_AT(tmem));
  const gt::Stages<FMT> stages = {base + P::kStageOff, GRAD_AT(st_full), GRAD_AT(st_empty), GRAD_AT(live)};
  if (warp < kSoftWarps) {
    gt::registers<kSoftRegs, kLaunchRegs>();
    softmax<FMT, FUSED>(p, base, tmem, threadIdx.x, share, walk);
  } else if (warp < kSoftWarps + kLoadWarps) {
    gt::registers<kLoadRegs, kLaunchRegs>();
    const int tid = (int)threadIdx.x - kSoftWarps * 32;
    const gt::Ring keys = {GRAD_AT(k_full), GRAD_AT(k_empty), base};
    const gt::Ring values = {GRAD_AT(v_full), GRAD_AT(v_empty), base + P::kValueOff};
    if constexpr (FMT != CERTKV_STORE_BF16) {
      gt::Expander<FMT, P::kKeys, P::kValues> f{keys, values, stages, GRAD_AT(abort), tid};
      f.run(walk);
    } else if (tid < kGroupWarps * 32) {
      gt::Copier<P::kKeys, false> f{&tmK, p, keys, 0u, GRAD_AT(abort), GRAD_AT(own) + 8u, p.st.k, tid};
      f.run(walk);
    } else {
      gt::Copier<P::kValues, false> f{&tmV, p, values, 0u, GRAD_AT(abort), GRAD_AT(own) + 12u, p.st.v, tid - kGroupWarps * 32};
      f.run(walk);
    }
  } else if (warp < kIssue) {
    gt::registers<kDrainRegs, kLaunchRegs>();
    drain<FMT, FUSED>(p, base, tmem, (int)threadIdx.x - kDrain * 32, share, walk);
  } else {
    gt::registers<kIssueRegs, kLaunchRegs>();
    if (warp == kIssue) {
      Issuer<FMT, FUSED> is{p, tmem, base};
      is.run(walk);
    } else if (warp == kIssue + 1 && threadIdx.x % 32 == 0) {
      RowFeeder<FMT, FUSED> f{p, base};
      f.run(walk);
    } else if (FMT != CERTKV_STORE_BF16 && warp == kIssue + 2 && threadIdx.x % 32 == 0) {
      gt::Stager<FMT> f{p, stages, GRAD_AT(abort), GRAD_AT(own) + 16u};
      f.run(walk);
    }
  }
  um::fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && p.st.status && gt::aborted(GRAD_AT(abort))) atomicOr(p.st.status, CERTKV_STATUS_TIMEOUT);
  if (warp == kIssue) {
    um::fence_after();
    um::dealloc(tmem, 512);
  }
}

template <int FMT, bool FUSED>
bool launch(const CUtensorMap& mk, const CUtensorMap& mv, const GradArgs& p, cudaStream_t st) {
  static std::atomic<uint64_t> ready{0};  // devices on which the shared memory is opted in to
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  if (dev > 63 || !(ready.load() >> dev & 1u)) {
    if (cudaFuncSetAttribute(grad_kv_kernel<FMT, FUSED>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             smem_bytes<FMT, FUSED>()) != cudaSuccess)
      return false;
    if (dev < 64) ready.fetch_or(1ull << dev);
  }
  return launch_kernel(true, grad_kv_kernel<FMT, FUSED>, (unsigned)p.groups, kThreads, smem_bytes<FMT, FUSED>(), st, mk,
                       mv, p);
}
template <int FMT>
bool launch_rows(const CUtensorMap& mk, const CUtensorMap& mv, const GradArgs& p, cudaStream_t st) {
  return p.rows <= kGradFused ? launch<FMT, true>(mk, mv, p, st) : launch<FMT, false>(mk, mv, p, st);
}

}  // namespace

bool launch_grad_kv(const GradArgs& p, int format, cudaStream_t st) {
  CUtensorMap mk = {}, mv = {};
  if (!gt::pool_maps(p, format, &mk, &mv)) return false;
  TraceScope ts_("grad_kv", st);
  return format == CERTKV_STORE_BF16  ? launch_rows<CERTKV_STORE_BF16>(mk, mv, p, st)
         : format == CERTKV_STORE_FP8 ? launch_rows<CERTKV_STORE_FP8>(mk, mv, p, st)
                                      : launch_rows<CERTKV_STORE_FP4>(mk, mv, p, st);
}

int grad_ctas() {
  static std::atomic<int> cached[64];
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || dev < 0) return 0;
  if (dev < 64 && (sms = cached[dev].load()) > 0) return sms;
  if (cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess || sms < 1) return 0;
  if (dev < 64) cached[dev].store(sms);
  return sms;
}

}  // namespace certkv
