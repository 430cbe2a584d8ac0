// grad_kv.cu — the stored slots' gradients on the 5th-generation tensor cores, and with few query
// rows those of the queries in the same pass.
//
// A CTA walks a share of all tiles of 128 slots, which are the M = 128 rows of the MMAs, and for
// each the unit's query rows in blocks of at most 64, the N columns:
//   S = K Q^T,  R = V dO^T,  p = 2^(S - lse),  e = p (R - delta),
//   dV += p dO,  dK += e Q,
// p and e rounded once to bf16 and handed over in tensor memory, over S.  Blocks of 64 columns
// leave room in tensor memory for two of them beside dV and dK, so that one block's S and R are
// made while p and e of the other are: S, R | S, R (64 columns each) | dV | dK (128 each).
//
// Up to 64 rows (FUSED) a segment is one block, whose rows stay in shared memory, and
// dQ^T += K^T e (M = 128 elements of a row) is summed over the share's tiles in the columns of
// the second block; e times the key's scale is handed over in shared memory for it.  The store
// is then read once for all gradients: with 64 rows or less the time is that of its bytes.
// Reading it again for the queries' kernel would cost as much as reading it here.
//
// Every wait is bounded; on a timeout the roles stop waiting, the rows and slots in question get
// NaN and the store's status word CERTKV_STATUS_TIMEOUT.
#include <atomic>

#include "../../include/certkv.h"
#include "grad_tc.cuh"
#include "internal.cuh"

namespace certkv {
namespace {

using gt::bar;
constexpr int kSoftWarps = 8, kLoadWarps = 2 * kGroupWarps, kRowWarps = 2;
constexpr int kThreads = (kSoftWarps + kLoadWarps + 4) * 32;  // whole warpgroups
constexpr int kSoftRegs = 112, kLoadRegs = 88, kIssueRegs = 80;
static_assert(kSoftWarps * 32 * kSoftRegs + kLoadWarps * 32 * kLoadRegs + 128 * kIssueRegs <= kThreads * 96,
              "a larger split would wait for registers for ever");
constexpr int kCols = kGradFused;       // query rows of a block
constexpr int kRowHalf = kCols * 128;   // bytes of a block's 64 rows x 64 elements
constexpr int kBlock = 4 * kRowHalf;    // a block: its rows, then their gradients
constexpr uint32_t kColV = 256, kColK = 384, kColQ = 128;  // S of block i: column 128 (i & 1), R 64 on

template <bool FUSED>
struct Plan {
  static constexpr int kKeys = FUSED ? 2 : 1, kValues = FUSED ? 2 : 1;  // places of the rings
  static constexpr int kBlocks = FUSED ? 2 : 4;
  static constexpr int kValueOff = kKeys * kOperand;
  static constexpr int kBlockOff = kValueOff + kValues * kOperand;
  static constexpr int kEOff = kBlockOff + kBlocks * kBlock;  // e, FUSED: [128 slots][64 rows]
  static constexpr int kMiscOff = kEOff + (FUSED ? kHalf : 0);
};
template <bool FUSED>
struct Misc {
  uint64_t k_full[2], k_empty[2], v_full[2], v_empty[2];
  uint64_t b_full[4], b_empty[4];
  uint64_t s_full[2], p_full[2], o_full, drained, done;
  uint32_t tmem;
  int abort;
  alignas(16) float nlse[Plan<FUSED>::kBlocks][kCols], ndelta[Plan<FUSED>::kBlocks][kCols];  // negated
};
template <bool FUSED>
constexpr int smem_bytes() {
  return Plan<FUSED>::kMiscOff + (int)sizeof(Misc<FUSED>) + 1024;
}
static_assert(smem_bytes<true>() <= 232448 && smem_bytes<false>() <= 232448,
              "over the 227 KB of shared memory a CTA can have");

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
  __device__ __forceinline__ Steps(const GradArgs& p_, int share) : p(p_), walk(p_, share) {
    it.ka = it.kb = k = j = 0;
    n = blocks_of(p_);
  }
  __device__ __forceinline__ bool next(Step* s) {
    if (k == it.kb) {
      if (!walk.next(&it)) return false;
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

// Two warps bring blocks of rows and their gradients into shared memory, each for a tile
// (FUSED: for an item).  A row that takes no part, or that holds a NaN or infinity, comes as
// zeros.
template <bool FUSED>
struct RowFeeder {
  const GradArgs& p;
  Misc<FUSED>* m;
  uint32_t ring;
  int tid;  // of 64
  uint32_t n = 0;
  bool pending = false;

  __device__ __forceinline__ void hand_over(uint32_t i) const {
    um::fence_async();
    __syncwarp();
    if ((tid & 31) == 0) tc::mbar_arrive(bar(&m->b_full[i % Plan<FUSED>::kBlocks]));
  }
  __device__ __forceinline__ bool block(int u, int j) {
    constexpr uint32_t kPlaces = Plan<FUSED>::kBlocks;
    const uint32_t place = n % kPlaces, phase = ((n / kPlaces) & 1u) ^ 1u;
    if (pending && !__all_sync(kFull, tc::mbar_test(bar(&m->b_empty[place]), phase))) {
      gt::cp_wait<0>();
      hand_over(n - 1);
      pending = false;
    }
    if (!__all_sync(kFull, tc::mbar_wait(bar(&m->b_empty[place]), phase, &m->abort))) return false;
    const GradUnit x(p, u);
    const int rows = rows_of_block(p, j);
    const float2* info = p.row + (int64_t)u * p.rows + j * kCols;
    const float2 mine = tid < rows ? info[tid] : make_float2(INFINITY, 0.f);
    m->nlse[place][tid] = -mine.x;
    m->ndelta[place][tid] = -mine.y;
    const uint32_t to = ring + place * kBlock;
    const int c = tid & 15;
#pragma unroll 4
    for (int i = 0; i < 16; ++i) {
      const int r = (tid >> 4) + 4 * i;
      const bool on = r < rows && fabsf(info[min(r, rows - 1)].x) < INFINITY;
      const int br = j * kCols + min(r, rows - 1), tok = br / p.G, qh = x.h * p.G + br - tok * p.G;
      const uint32_t at = to + (uint32_t)((c >> 3) * kRowHalf + r * 128 + (((c & 7) ^ (r & 7)) << 4));
      gt::cp16(at, p.q.at(x.b, x.l, tok, qh) + 8 * c, on);
      gt::cp16(at + 2 * kRowHalf, p.go.at(x.b, x.l, tok, qh) + 8 * c, on);
    }
    gt::cp_commit();
    if (pending) {
      gt::cp_wait<1>();
      hand_over(n - 1);
    }
    pending = true;
    ++n;
    return true;
  }
  __device__ __forceinline__ void run(int share) {
    gt::Walk walk(p, share);
    gt::Item it;
    bool ok = true;
    while (ok && walk.next(&it)) {
      for (int k = it.ka; ok && k < (FUSED ? it.ka + 1 : it.kb); ++k)
        for (int j = 0; ok && j < blocks_of(p); ++j) ok = block(it.u, j);
    }
    gt::cp_wait<0>();  // nothing lands after the CTA has gone
    if (ok && pending) hand_over(n - 1);
  }
};

// Issues the MMAs; the whole warp runs, one lane issues.
template <bool FUSED>
struct Issuer {
  using P = Plan<FUSED>;
  const GradArgs& p;
  Misc<FUSED>* m;
  uint32_t tmem, base;
  bool ok = true;
  uint32_t tiles = 0;  // whose products have been begun
  uint32_t odd = 0;    // parities of p_full
  __device__ __forceinline__ void wait(const uint64_t* b, uint32_t phase) {
    if (ok) ok = __all_sync(kFull, tc::mbar_wait(bar(b), phase & 1u, &m->abort));
  }
  __device__ __forceinline__ uint32_t buffer(const Step& s) const { return FUSED ? 0u : s.i & 1u; }
  __device__ __forceinline__ uint32_t columns(const Step& s) const { return up16(rows_of_block(p, s.j)); }
  // S and R of a block
  __device__ __forceinline__ void logits(const Step& s) {
    if (s.j == 0) {
      wait(&m->k_full[s.t % P::kKeys], s.t / P::kKeys);
      wait(&m->v_full[s.t % P::kValues], s.t / P::kValues);
    }
    if (!FUSED || s.first) wait(&m->b_full[s.blk % P::kBlocks], s.blk / P::kBlocks);
    if (!ok) return;
    um::fence_after();
    if (um::elected()) {
      const uint32_t d = tmem + 128u * buffer(s), id = um::idesc_n(columns(s), false, false);
      const uint32_t k = um::desc_lo(base + (s.t % P::kKeys) * kOperand, 16);
      const uint32_t v = um::desc_lo(base + P::kValueOff + (s.t % P::kValues) * kOperand, 16);
      const uint32_t q = um::desc_lo(base + P::kBlockOff + (s.blk % P::kBlocks) * kBlock, 16);
#pragma unroll
      for (uint32_t i = 0; i < 8; ++i)
        um::mma_ss(d, k + 2 * (i & 3) + (i >> 2) * (kHalf >> 4), q + 2 * (i & 3) + (i >> 2) * (kRowHalf >> 4),
                   um::kDescHi, id, i > 0);
#pragma unroll
      for (uint32_t i = 0; i < 8; ++i)
        um::mma_ss(d + 64, v + 2 * (i & 3) + (i >> 2) * (kHalf >> 4),
                   q + (2 * kRowHalf >> 4) + 2 * (i & 3) + (i >> 2) * (kRowHalf >> 4), um::kDescHi, id, i > 0);
    }
    __syncwarp();
    um::commit(bar(&m->s_full[buffer(s)]));
    if (s.j + 1 == s.n) {
      um::commit(bar(&m->v_empty[s.t % P::kValues]));
      if (!FUSED) um::commit(bar(&m->k_empty[s.t % P::kKeys]));
    }
  }
  // what p and e of a block go into
  __device__ __forceinline__ void products(const Step& s) {
    const uint32_t x = buffer(s);
    wait(&m->p_full[x], odd >> x & 1u);
    odd ^= 1u << x;
    if (s.j == 0 && tiles++ > 0) wait(&m->drained, tiles - 2);
    if (!ok) return;
    um::fence_after();
    if (um::elected()) {
      const uint32_t a = tmem + 128u * x, steps = columns(s) / 16;
      const uint32_t q = um::desc_lo(base + P::kBlockOff + (s.blk % P::kBlocks) * kBlock, kRowHalf);
      constexpr uint32_t id = um::idesc_n(128, false, true);
      // 16 rows a step: 8 columns of every 32 for p, 16 on for e; 2048 bytes of the block
      for (uint32_t i = 0; i < steps; ++i)
        um::mma_ts(tmem + kColV, a + 32 * (i >> 1) + 8 * (i & 1), q + (2 * kRowHalf >> 4) + 128 * i, um::kDescHi, id,
                   s.j > 0 || i > 0);
      for (uint32_t i = 0; i < steps; ++i)
        um::mma_ts(tmem + kColK, a + 16 + 32 * (i >> 1) + 8 * (i & 1), q + 128 * i, um::kDescHi, id, s.j > 0 || i > 0);
      if (FUSED) {
        const uint32_t k = um::desc_lo(base + (s.t % P::kKeys) * kOperand, kHalf);
        const uint32_t e = um::desc_lo(base + P::kEOff, 16), idq = um::idesc_n(columns(s), true, true);
#pragma unroll
        for (uint32_t i = 0; i < 8; ++i)
          um::mma_ss(tmem + kColQ, k + 128 * i, e + 128 * i, um::kDescHi, idq, !s.first || i > 0);
      }
    }
    __syncwarp();
    if (FUSED) um::commit(bar(&m->k_empty[s.t % P::kKeys]));
    if (!FUSED || s.last) um::commit(bar(&m->b_empty[s.blk % P::kBlocks]));
    if (s.j + 1 == s.n) um::commit(bar(&m->o_full));
  }
  __device__ __forceinline__ void run(int share) {
    Steps<FUSED> steps(p, share);
    Step cur, nxt;
    bool more = steps.next(&cur);
    if (more) logits(cur);
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
    um::commit(bar(&m->done));  // everything issued above has finished
    volatile int dummy = 0;
    tc::mbar_wait(bar(&m->done), 0, &dummy);
    __syncwarp();
  }
};

// The slot of a softmax thread.
template <int FMT>
struct Slot {
  int64_t at;        // of the pool, -1: none
  float ks, vs;      // scales of its key and value
  __device__ __forceinline__ void load(const GradArgs& p, int u, int s, int count) {
    at = s < count ? p.st.slot(u, s) : -1;
    ks = vs = gt::kCodeScale<FMT>;
    if (FMT != CERTKV_STORE_BF16 && at >= 0) {
      ks *= __ldg(p.st.ks + at);
      vs *= __ldg(p.st.vs + at);
    }
  }
};

__device__ __forceinline__ void store_row_part(uint16_t* to, const uint32_t (&w)[16]) {
#pragma unroll
  for (int j = 0; j < 16; j += 8)  // whole sectors
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(to + 2 * j), "r"(w[j]), "r"(w[j + 1]),
                 "r"(w[j + 2]), "r"(w[j + 3]), "r"(w[j + 4]), "r"(w[j + 5]), "r"(w[j + 6]), "r"(w[j + 7])
                 : "memory");
}

template <int FMT, bool FUSED>
__device__ __forceinline__ void softmax(const GradArgs& p, Misc<FUSED>* m, uint32_t base, uint32_t tmem, int tid,
                                        int share) {
  using P = Plan<FUSED>;
  constexpr bool kQuant = FMT != CERTKV_STORE_BF16;
  volatile int* ab = &m->abort;
  const int warp = tid >> 5, lane = tid & 31, quad = warp & 3, half = warp >> 2;
  const int row = quad * 32 + lane;  // slot of the tile
  const uint32_t at = (uint32_t)(quad * 32) << 16;
  const int blocks = blocks_of(p);
  const bool want_q = FUSED && p.dq.p;
  uint32_t i = 0, t = 0, item = 0;
  bool ok = true;
  gt::Walk walk(p, share);
  gt::Item it;
  while (walk.next(&it)) {
    const gt::Item now = it;
    const int count = p.st.count(now.u);
    Slot<FMT> next;
    next.load(p, now.u, now.ka * kGradTile + row, count);
    for (int k = now.ka; k < now.kb; ++k, ++t) {
      const Slot<FMT> slot = next;
      if (k + 1 < now.kb) next.load(p, now.u, (k + 1) * kGradTile + row, count);
      const bool live = slot.at >= 0;
      const float2 ksl = make_float2(slot.ks * p.scale_log2, slot.ks * p.scale_log2);
      const float2 vs = make_float2(slot.vs, slot.vs), ks = make_float2(slot.ks, slot.ks);
      for (int j = 0; ok && j < blocks; ++j, ++i) {
        const uint32_t x = FUSED ? 0u : i & 1u, use = FUSED ? i : i >> 1, blk = FUSED ? item : i;
        const uint32_t place = blk % P::kBlocks;
        if (!FUSED || k == now.ka)
          ok = __all_sync(kFull, tc::mbar_wait(bar(&m->b_full[place]), (blk / P::kBlocks) & 1u, ab));
        ok = ok && __all_sync(kFull, tc::mbar_wait(bar(&m->s_full[x]), use & 1u, ab));
        if (!ok) break;
        um::fence_after();
        if (32 * half < rows_of_block(p, j)) {
          const uint32_t tS = tmem + at + 128u * x + 32u * half;
          uint32_t s[32], r[32], pw[16], ew[16], qw[16];
          um::ld32(tS, s);
          um::ld32(tS + 64u, r);
          const float* nlse = &m->nlse[place][32 * half];
          const float* ndelta = &m->ndelta[place][32 * half];
#pragma unroll
          for (int c = 0; c < 8; ++c) {
            const float4 l4 = *reinterpret_cast<const float4*>(nlse + 4 * c);
            const float4 d4 = *reinterpret_cast<const float4*>(ndelta + 4 * c);
#pragma unroll
            for (int h = 0; h < 2; ++h) {
              const int q = 4 * c + 2 * h;
              float2 e = make_float2(__uint_as_float(s[q]), __uint_as_float(s[q + 1]));
              float2 d = make_float2(__uint_as_float(r[q]), __uint_as_float(r[q + 1]));
              e = ffma2(e, ksl, h ? make_float2(l4.z, l4.w) : make_float2(l4.x, l4.y));
              d = kQuant ? ffma2(d, vs, h ? make_float2(d4.z, d4.w) : make_float2(d4.x, d4.y))
                         : fadd2(d, h ? make_float2(d4.z, d4.w) : make_float2(d4.x, d4.y));
              e.x = um::ex2(e.x);
              e.y = um::ex2(e.y);
              d = fmul2(e, d);
              pw[2 * c + h] = live ? gt::pack2(e.x, e.y) : 0u;
              ew[2 * c + h] = live ? gt::pack2(d.x, d.y) : 0u;
              if (FUSED && kQuant) {
                d = fmul2(d, ks);
                qw[2 * c + h] = live ? gt::pack2(d.x, d.y) : 0u;
              }
            }
          }
          um::st16(tS, pw);
          um::st16(tS + 16u, ew);
          if (FUSED) {
            const uint32_t to = base + P::kEOff + (uint32_t)row * 128u;
#pragma unroll
            for (int c = 0; c < 4; ++c) {
              const uint32_t* w = kQuant ? &qw[4 * c] : &ew[4 * c];
              sts128(to + (uint32_t)(((4 * half + c) ^ (row & 7)) << 4), w[0], w[1], w[2], w[3]);
            }
            um::fence_async();
          }
          um::wait_st();
        }
        um::fence_before();
        __syncwarp();
        if (lane == 0) tc::mbar_arrive(bar(&m->p_full[x]));
      }
      // ---- the tile's gradients, 64 elements a thread
      if (ok) ok = __all_sync(kFull, tc::mbar_wait(bar(&m->o_full), t & 1u, ab));
      um::fence_after();
      const bool good = ok && *ab == 0;
#pragma unroll 1
      for (int c = 0; c < 4; ++c) {
        const bool key = c >= 2;
        const int d0 = 64 * half + 32 * (c & 1);
        uint32_t r[32], w[16];
        um::ld32(tmem + at + (key ? kColK : kColV) + (uint32_t)d0, r);
        const float f = key ? p.scale : 1.f;
#pragma unroll
        for (int q = 0; q < 16; ++q)
          w[q] = good ? gt::pack2(__uint_as_float(r[2 * q]) * f, __uint_as_float(r[2 * q + 1]) * f) : 0x7fc07fc0u;
        if (live) store_row_part((key ? p.dks : p.dvs) + slot.at * kD + d0, w);
      }
      if (want_q && k + 1 == now.kb) {
        float* out = p.rec + grad_record(p, share, now.u, 0) * kD + row;
        const int r0 = 32 * half, rows = min(p.rows - r0, 32);
        if (rows > 0) {
          uint32_t r[32];
          um::ld32(tmem + at + kColQ + (uint32_t)r0, r);
#pragma unroll
          for (int q = 0; q < 32; ++q)
            if (q < rows) out[(int64_t)(r0 + q) * kD] = good ? __uint_as_float(r[q]) : nanf("");
        }
      }
      um::fence_before();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(bar(&m->drained));
    }
    ++item;
  }
}

// grid = groups (one CTA per SM), block = kThreads.
template <int FMT, bool FUSED>
__global__ void __launch_bounds__(kThreads, 1) grad_kv_kernel(const __grid_constant__ GradArgs p) {
  using P = Plan<FUSED>;
  extern __shared__ char smem_raw[];
  char* sm = reinterpret_cast<char*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~(uintptr_t)1023);
  Misc<FUSED>* m = reinterpret_cast<Misc<FUSED>*>(sm + P::kMiscOff);
  const int warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(bar(&m->k_full[i]), kGroupWarps);
      tc::mbar_init(bar(&m->k_empty[i]), 1);
      tc::mbar_init(bar(&m->v_full[i]), kGroupWarps);
      tc::mbar_init(bar(&m->v_empty[i]), 1);
      tc::mbar_init(bar(&m->s_full[i]), 1);
      tc::mbar_init(bar(&m->p_full[i]), kSoftWarps);
    }
    for (int i = 0; i < 4; ++i) {
      tc::mbar_init(bar(&m->b_full[i]), kRowWarps);
      tc::mbar_init(bar(&m->b_empty[i]), 1);
    }
    tc::mbar_init(bar(&m->o_full), 1);
    tc::mbar_init(bar(&m->drained), kSoftWarps);
    tc::mbar_init(bar(&m->done), 1);
    m->abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  release_next();
  await_previous();
  const int share = blockIdx.x;
  if (tiles_per_share(p) * share >= p.first[p.units]) return;  // uniform, before any barrier
  if (warp == kSoftWarps + kLoadWarps) um::alloc(tc::saddr(&m->tmem), 512);
  um::fence_before();
  __syncthreads();
  um::fence_after();
  const uint32_t tmem = *reinterpret_cast<volatile uint32_t*>(&m->tmem);
  const uint32_t base = tc::saddr(sm);
  if (warp < kSoftWarps) {
    gt::regs_up<kSoftRegs>();
    softmax<FMT, FUSED>(p, m, base, tmem, threadIdx.x, share);
  } else if (warp < kSoftWarps + kLoadWarps) {
    gt::regs_down<kLoadRegs>();
    const int tid = (int)threadIdx.x - kSoftWarps * 32;
    if (tid < kGroupWarps * 32) {
      gt::Feeder<FMT, P::kKeys, false> f{p, m->k_full, m->k_empty, nullptr, &m->abort, base, false, tid};
      f.run(gt::Walk(p, share));
    } else {
      gt::Feeder<FMT, P::kValues, false> f{p,  m->v_full, m->v_empty, nullptr, &m->abort, base + P::kValueOff,
                                           true, tid - kGroupWarps * 32};
      f.run(gt::Walk(p, share));
    }
  } else {
    gt::regs_down<kIssueRegs>();
    if (warp == kSoftWarps + kLoadWarps) {
      Issuer<FUSED> is{p, m, tmem, base};
      is.run(share);
    } else if (warp <= kSoftWarps + kLoadWarps + kRowWarps) {
      RowFeeder<FUSED> f{p, m, base + P::kBlockOff, (int)threadIdx.x - (kSoftWarps + kLoadWarps + 1) * 32};
      f.run(share);
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

template <int FMT, bool FUSED>
bool launch(const GradArgs& p, cudaStream_t st) {
  static std::atomic<uint64_t> ready{0};  // devices on which the shared memory is opted in to
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  if (dev > 63 || !(ready.load() >> dev & 1u)) {
    if (cudaFuncSetAttribute(grad_kv_kernel<FMT, FUSED>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                             smem_bytes<FUSED>()) != cudaSuccess)
      return false;
    if (dev < 64) ready.fetch_or(1ull << dev);
  }
  return launch_kernel(true, grad_kv_kernel<FMT, FUSED>, (unsigned)p.groups, kThreads, smem_bytes<FUSED>(), st, p);
}
template <int FMT>
bool launch_rows(const GradArgs& p, cudaStream_t st) {
  return p.rows <= kGradFused ? launch<FMT, true>(p, st) : launch<FMT, false>(p, st);
}

}  // namespace

bool launch_grad_kv(const GradArgs& p, int format, cudaStream_t st) {
  TraceScope ts_("grad_kv", st);
  return format == CERTKV_STORE_BF16  ? launch_rows<CERTKV_STORE_BF16>(p, st)
         : format == CERTKV_STORE_FP8 ? launch_rows<CERTKV_STORE_FP8>(p, st)
                                      : launch_rows<CERTKV_STORE_FP4>(p, st);
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
