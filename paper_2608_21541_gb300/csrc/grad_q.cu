// grad_q.cu — the queries' gradients over the stored slots on the 5th-generation tensor cores.
//
// A CTA holds up to 128 query rows of a unit, and their output's gradients, as the M = 128 rows
// of the MMAs, and walks a share of all tiles of 128 slots:
//   S = Q K^T,  R = dO V^T,  e = 2^(S - lse) (R - delta),  dQ += e K,
// with e handed over in tensor memory, over S, as a bf16 part and one of its remainder (2^-14).
// Neither a maximum nor a rescaling is needed, the log-sum-exp is known, so a tile is formed in
// one pass.
// Tensor memory: S of even tiles | S of odd tiles | R | dQ, 128 columns each.  S of the next
// tile is made while e of this one is, R of the next as soon as this one's is in registers,
// dQ of this one under e of the next.
//
// bf16 stores are bound by their bytes (64 rows over 13107 slots of 256 segments: 1.72 GB in
// 281 us, 90 % of a copy's rate), 8- and 4-bit ones by what a tile goes through, expanding of codes,
// S and R, softmax, dQ, with no unit full (317 and 326 us; the products of 128 rows, half of them
// empty there, take 235, and 4 rows as long as 64: 309 and 327).
//
// 8- and 4-bit stores: codes are exact in bf16 (gt::codes_to_bf16); a key's fp32 scale multiplies
// its logit and its e, a value's its R, all in fp32.  The scale comes times that of the logits,
// which is taken out of dQ again at the end.
//
// CTAs of the same share and different row blocks are neighbours: they read the same tiles at
// about the same time, so all but the first find them in L2.
//
// Every wait is bounded; on a timeout the roles stop waiting, the rows in question read NaN and
// the store's status word gets CERTKV_STATUS_TIMEOUT.
#include <atomic>

#include "../../include/certkv.h"
#include "grad_tc.cuh"
#include "internal.cuh"

namespace certkv {
namespace {

// Warps, whole warpgroups of them: softmax, 64 columns of a row a thread where codes are expanded
// beside it and 32 else (1024 rows over 32768 slots, bf16: 196 us with eight warps, 158 with
// sixteen, 150 since; 8-bit trees 204 and 208, 152 since with eight), loaders, and
// the issuer beside the warps that ask for codes and state scales.
constexpr int kLoadWarps = 2 * kGroupWarps;
template <int FMT>
struct Warps {
  static constexpr int kSoft = FMT == CERTKV_STORE_BF16 ? 16 : 8, kColumns = 512 / kSoft;
  static constexpr int kLoad = kSoft, kIssue = kSoft + kLoadWarps, kThreads = (kIssue + 4) * 32;
  // registers a thread: those of the launch, which the roles share out among themselves
  static constexpr int kLaunch = FMT == CERTKV_STORE_BF16 ? 72 : 96;
  static constexpr int kSoftRegs = FMT == CERTKV_STORE_BF16 ? 72 : 104;
  static constexpr int kLoadRegs = FMT == CERTKV_STORE_BF16 ? 72 : 88;
  static constexpr int kIssueRegs = FMT == CERTKV_STORE_BF16 ? 72 : 96;
  static_assert(kSoft * 32 * kSoftRegs + kLoadWarps * 32 * kLoadRegs + 128 * kIssueRegs <= kThreads * kLaunch,
                "a larger split would wait for registers for ever");
};
constexpr uint32_t kColR = 256, kColQ = 384;  // S of tile t: column 128 (t & 1)

template <int FMT>
struct Plan {
  // Places of the rings.  The keys' are held from S of a tile to its dQ, the values' for R alone
  // (8 bits, 64 rows over 13107 slots of 256 segments: 396 us with 2 + 2 places, 357 with 3 + 1;
  // 317 since).
  static constexpr int kKeys = 3;
  static constexpr int kValues = FMT == CERTKV_STORE_BF16 ? 2 : 1;
  static constexpr int kFacts = FMT == CERTKV_STORE_BF16 ? kKeys : 2;  // bf16: the copying warps state them
  static constexpr int kKeyOff = 2 * kOperand;  // behind the rows and their gradients
  static constexpr int kValueOff = kKeyOff + kKeys * kOperand;
  static constexpr int kStageOff = kValueOff + kValues * kOperand;  // of keys, then of values
  static constexpr int kMiscOff = kStageOff + 2 * gt::kStage<FMT>;
};
template <int FMT>
struct Misc {
  uint64_t k_full[3], k_empty[3], v_full[2], v_empty[2];
  uint64_t q_full, q_empty, s_full, r_free, p_full, o_full, o_free, done;
  uint64_t f_full[2];                // facts (8- and 4-bit stores)
  uint64_t st_full[2], st_empty[2];  // stretches of codes, keys' and values'
  int2 live[2];  // of the stretches
  uint32_t tmem;
  int abort, own[5];  // own: flags of the issuer, the feeder of rows, the copiers of keys and values, the stager
  alignas(16) typename gt::FactsOf<FMT>::type facts[Plan<FMT>::kFacts];
};
template <int FMT>
constexpr int smem_bytes() {
  return Plan<FMT>::kMiscOff + (int)sizeof(Misc<FMT>);
}
static_assert(smem_bytes<CERTKV_STORE_BF16>() <= 232448 && smem_bytes<CERTKV_STORE_FP8>() <= 232448 &&
                  smem_bytes<CERTKV_STORE_FP4>() <= 232448,
              "over the 227 KB of shared memory a CTA can have");

// A lane that brings an item's rows and their gradients, by bulk copies, as soon as the products
// of the item before are done with theirs.
template <int FMT>
struct RowFeeder {
  using P = Plan<FMT>;
  using M = Misc<FMT>;
  const GradArgs& p;
  uint32_t base;
  int blk;
  __device__ __forceinline__ void run(gt::Walk walk) const {
    const uint32_t bytes = 128u * min(p.rb, p.padded - blk * p.rb);
    gt::Item it;
    uint32_t n = 0;
#pragma unroll 1
    while (walk.next(p, &it) && gt::wait(GRAD_AT(q_empty), (n & 1u) ^ 1u, GRAD_AT(abort))) {
      tc::mbar_expect_tx(GRAD_AT(q_full), 4u * bytes);
#pragma unroll 1
      for (int part = 0; part < 4; ++part)
        tc::bulk_load(base + part * kHalf, grad_pack(p, it.u, part, blk * p.rb), bytes, GRAD_AT(q_full));
      ++n;
    }
    if (n > 0) gt::finish(GRAD_AT(q_full), (n - 1) & 1u, GRAD_AT(own) + 4u);  // nothing lands after the CTA has gone
  }
};

// Issues the MMAs of the share's tiles; the whole warp runs, one lane issues.
template <int FMT>
struct Issuer {
  using P = Plan<FMT>;
  using M = Misc<FMT>;
  uint32_t tmem, base;
  bool ok = true;
  __device__ __forceinline__ void wait(uint32_t mbar, uint32_t phase) {
    if (ok) ok = gt::wait_all(mbar, phase, GRAD_AT(abort));
  }
  // A place of a ring and the parity of its use.
  template <int N>
  struct Place {
    uint32_t slot = 0, phase = 0;
    __device__ __forceinline__ void operator++() {
      if (++slot == N) slot = 0, phase ^= 1u;
    }
  };
  Place<P::kKeys> sk, qk;  // of the next S, of the next dQ
  Place<P::kValues> rv;    // of the next R
  static __device__ __forceinline__ bool test(uint32_t mbar, uint32_t phase) {
    return __all_sync(kFull, tc::mbar_test(mbar, phase));
  }
  __device__ __forceinline__ void await_keys() { wait(GRAD_AT(k_full) + 8u * sk.slot, sk.phase); }
  __device__ __forceinline__ void await_values() { wait(GRAD_AT(v_full) + 8u * rv.slot, rv.phase); }
  // S of tile t, whose keys are there, and its R, whose values are; last: nothing reads the item's
  // rows behind it
  __device__ __forceinline__ void s(uint32_t t) {
    if (!ok) return;
    um::fence_async();  // the loaders' writes, before the tensor core's reads
    um::fence_after();
    um::mma_s(tmem + 128u * (t & 1u), um::desc_lo(base, 16), um::desc_lo(base + P::kKeyOff, 16) + sk.slot * (kOperand >> 4),
              um::kDescHi, um::idesc(true, false));
    ++sk;
  }
  __device__ __forceinline__ void r(bool last) {
    if (!ok) return;
    um::fence_async();
    um::fence_after();
    um::mma_s(tmem + kColR, um::desc_lo(base + kOperand, 16),
              um::desc_lo(base + P::kValueOff, 16) + rv.slot * (kOperand >> 4), um::kDescHi, um::idesc(true, false));
    um::commit(GRAD_AT(s_full));
    um::commit(GRAD_AT(v_empty) + 8u * rv.slot);
    if (last) um::commit(GRAD_AT(q_empty));
    ++rv;
  }
  __device__ __forceinline__ void run(const GradArgs& p, gt::Walk walk) {
    gt::Item it;
    uint32_t t = 0, item = 0;
#pragma unroll 1
    while (ok && walk.next(p, &it)) {
      const int n = it.kb - it.ka;
      wait(GRAD_AT(q_full), item & 1u);
      await_keys();
      s(t);
      await_values();
      if (t > 0) wait(GRAD_AT(r_free), (t - 1) & 1u);
      r(n == 1);
#pragma unroll 1
      for (int i = 0; ok && i < n; ++i, ++t) {
        // S of the next tile goes when its keys and values are there, R when this tile's has been
        // read, dQ of this tile when e is there, in whatever order these come: each gives back
        // what another role waits for.
        const bool more = i + 1 < n;
        bool has_s = !more, has_r = !more;
#pragma unroll 1
        for (uint32_t look = 0; ok; ++look) {
          if (!has_s && test(GRAD_AT(k_full) + 8u * sk.slot, sk.phase)) {
            s(t + 1);
            has_s = true;
          }
          if (has_s && !has_r && test(GRAD_AT(r_free), t & 1u) && test(GRAD_AT(v_full) + 8u * rv.slot, rv.phase)) {
            r(i + 2 == n);
            has_r = true;
          }
          if (test(GRAD_AT(p_full), t & 1u)) break;
          ok = gt::patience(look, GRAD_AT(abort));
        }
        if (i == 0 && item > 0) wait(GRAD_AT(o_free), (item - 1) & 1u);  // dQ of the item before has been read
        if (!ok) break;
        um::fence_after();
        um::mma_e2(tmem + kColQ, tmem + 128u * (t & 1u), um::desc_lo(base + P::kKeyOff, kHalf) + qk.slot * (kOperand >> 4),
                   um::kDescHi, um::idesc(true, true), i > 0);
        um::commit(GRAD_AT(k_empty) + 8u * qk.slot);
        ++qk;
        if (!more) um::commit(GRAD_AT(o_full));
        if (!has_s) {
          await_keys();
          s(t + 1);
        }
        if (!has_r) {
          await_values();
          r(i + 2 == n);
        }
      }
      ++item;
    }
    um::commit(GRAD_AT(done));  // everything issued above has finished
    gt::finish(GRAD_AT(done), 0, GRAD_AT(own));
    __syncwarp();
  }
};

// e of 16 columns of a row, from the first column c on, over its logits: eight columns of bf16
// and eight of what they leave.
template <int FMT>
__device__ __forceinline__ void columns(uint32_t tS, const uint32_t* r, const typename gt::FactsOf<FMT>::type& f, int c,
                                        float sl, float nlse, float ndelta) {
  constexpr bool kQuant = FMT != CERTKV_STORE_BF16;
  const float2 nl = make_float2(nlse, nlse), nd = make_float2(ndelta, ndelta), sl2 = make_float2(sl, sl);
  uint32_t s[16], e[16];
  um::ld16(tS, s);
#pragma unroll
  for (int j = 0; j < 4; ++j) {
    float4 ks, vs;
    if constexpr (kQuant) {
      ks = *reinterpret_cast<const float4*>(&f.ks[c + 4 * j]);
      vs = *reinterpret_cast<const float4*>(&f.vs[c + 4 * j]);
    }
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const int at = 4 * j + 2 * i;
      float2 x = make_float2(__uint_as_float(s[at]), __uint_as_float(s[at + 1]));
      float2 y = make_float2(__uint_as_float(r[at]), __uint_as_float(r[at + 1]));
      const float2 k2 = i ? make_float2(ks.z, ks.w) : make_float2(ks.x, ks.y);
      if constexpr (kQuant) {
        x = ffma2(x, k2, nl);
        y = ffma2(y, i ? make_float2(vs.z, vs.w) : make_float2(vs.x, vs.y), nd);
      } else {
        x = ffma2(x, sl2, nl);
        y = fadd2(y, nd);
      }
      x.x = um::ex2(x.x);
      x.y = um::ex2(x.y);
      x = fmul2(x, y);
      if constexpr (kQuant) x = fmul2(x, k2);
      // the upper halves as they are, then the upper halves of what that leaves: neither takes a
      // conversion (2^-14 together, towards 0)
      y = fadd2(x, make_float2(-__uint_as_float(__float_as_uint(x.x) & 0xffff0000u),
                               -__uint_as_float(__float_as_uint(x.y) & 0xffff0000u)));
      e[at / 2] = __byte_perm(__float_as_uint(x.x), __float_as_uint(x.y), 0x7632);
      e[8 + at / 2] = __byte_perm(__float_as_uint(y.x), __float_as_uint(y.y), 0x7632);
    }
  }
  const uint32_t live = f.live[c / 32] >> (c & 31) & 0xffffu;
  if (live != 0xffffu) {
#pragma unroll
    for (int j = 0; j < 8; ++j) {
      const uint32_t keep = (live >> (2 * j) & 1u ? 0xffffu : 0u) | (live >> (2 * j + 1) & 1u ? 0xffff0000u : 0u);
      e[j] &= keep;
      e[8 + j] &= keep;
    }
  }
  um::st16(tS, e);
}

template <int FMT>
__device__ __forceinline__ void softmax(const GradArgs& p, uint32_t base, uint32_t tmem, int tid, int share, int blk,
                                        gt::Walk walk) {
  using P = Plan<FMT>;
  using M = Misc<FMT>;
  using W = Warps<FMT>;
  extern __shared__ __align__(1024) char smem[];
  const int warp = tid >> 5, lane = tid & 31, quad = warp & 3, col = (warp >> 2) * W::kColumns;
  const int row = quad * 32 + lane;
  const uint32_t at = (uint32_t)(quad * 32) << 16;  // this warp's lanes of tensor memory
  const int rows = min(p.rb, p.rows - blk * p.rb);
  const bool busy = quad * 32 < p.rb;  // some block has a row here
  uint32_t t = 0, item = 0;
  bool ok = true;
  gt::Item it;
#pragma unroll 1
  while (walk.next(p, &it)) {
    const gt::Item now = it;
    const float2 mine = row < rows ? p.row[(int64_t)now.u * p.rows + blk * p.rb + row] : make_float2(INFINITY, 0.f);
#pragma unroll 1
    for (int k = now.ka; ok && busy && k < now.kb; ++k, ++t) {
      const uint32_t place = t % P::kFacts;
      ok = gt::wait_all((FMT == CERTKV_STORE_BF16 ? GRAD_AT(k_full) : GRAD_AT(f_full)) + 8u * place,
                        (t / P::kFacts) & 1u, GRAD_AT(abort)) &&
           gt::wait_all(GRAD_AT(s_full), t & 1u, GRAD_AT(abort));
      if (!ok) break;
      um::fence_after();
      uint32_t r[W::kColumns];
#pragma unroll
      for (int c = 0; c < W::kColumns; c += 32)
        um::ld32(tmem + at + kColR + col + c, *reinterpret_cast<uint32_t(*)[32]>(r + c));
      um::fence_before();  // this warp's part of R has been read
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(GRAD_AT(r_free));
#pragma unroll
      for (int c = 0; c < W::kColumns; c += 16)
        columns<FMT>(tmem + at + 128u * (t & 1u) + col + c, r + c,
                     reinterpret_cast<const M*>(smem + P::kMiscOff)->facts[place], col + c, p.scale_log2, -mine.x, -mine.y);
      um::wait_st();
      um::fence_before();
      __syncwarp();
      if (lane == 0) tc::mbar_arrive(GRAD_AT(p_full));
    }
    if (ok) ok = gt::wait_all(GRAD_AT(o_full), item & 1u, GRAD_AT(abort));
    ++item;
    um::fence_after();
    float* out = grad_record(p, share, now.u, blk) + grad_at(p, row, col);
    const bool good = ok && !gt::aborted(GRAD_AT(abort));
    const float unscale = FMT == CERTKV_STORE_BF16 ? 1.f : 1.f / p.scale_log2;
#pragma unroll 1
    for (int c = 0; c < W::kColumns / 16; ++c) {
      uint32_t r[16];
      um::ld16(tmem + at + kColQ + col + 16u * c, r);
      if (row < rows) {
#pragma unroll
        for (int j = 0; j < 16; ++j)
          r[j] = good ? __float_as_uint(__uint_as_float(r[j]) * unscale) : 0x7fc00000u;
#pragma unroll
        for (int j = 0; j < 16; j += 8)  // whole lines of a warp
          asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"l"(out + (2 * c + j / 8) * p.rb * 8), "r"(r[j]),
                       "r"(r[j + 1]), "r"(r[j + 2]), "r"(r[j + 3]), "r"(r[j + 4]), "r"(r[j + 5]), "r"(r[j + 6]),
                       "r"(r[j + 7])
                       : "memory");
      }
    }
    um::fence_before();  // this warp's part of dQ has been read
    __syncwarp();
    if (lane == 0) tc::mbar_arrive(GRAD_AT(o_free));
  }
}

// grid = groups nblk (one CTA per SM), block = Warps<FMT>::kThreads.
template <int FMT>
__global__ void __launch_bounds__(Warps<FMT>::kThreads, 1) grad_q_kernel(const __grid_constant__ CUtensorMap tmK,
                                                             const __grid_constant__ CUtensorMap tmV,
                                                             const __grid_constant__ GradArgs p) {
  extern __shared__ __align__(1024) char smem[];
  using P = Plan<FMT>;
  using M = Misc<FMT>;
  using W = Warps<FMT>;
  const uint32_t base = tc::saddr(smem);
  const int warp = __shfl_sync(kFull, (int)threadIdx.x >> 5, 0);  // so that the compiler, too, knows it uniform
  if (threadIdx.x == 0) {
    for (int i = 0; i < 3; ++i) {
      tc::mbar_init(GRAD_AT(k_full) + 8u * (i), gt::kArrivals<FMT>);
      tc::mbar_init(GRAD_AT(k_empty) + 8u * (i), 1);
    }
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(GRAD_AT(v_full) + 8u * (i), gt::kArrivals<FMT>);
      tc::mbar_init(GRAD_AT(v_empty) + 8u * (i), 1);
    }
    for (int i = 0; i < 2; ++i) {
      tc::mbar_init(GRAD_AT(f_full) + 8u * i, 1);
      tc::mbar_init(GRAD_AT(st_full) + 8u * i, 1);
      tc::mbar_init(GRAD_AT(st_empty) + 8u * i, kLoadWarps);
    }
    tc::mbar_init(GRAD_AT(q_full), 1);
    tc::mbar_init(GRAD_AT(q_empty), 1);
    tc::mbar_init(GRAD_AT(o_free), W::kSoft);
    tc::mbar_init(GRAD_AT(s_full), 1);
    tc::mbar_init(GRAD_AT(r_free), W::kSoft / 4 * ((p.rb + 31) / 32));
    tc::mbar_init(GRAD_AT(p_full), W::kSoft / 4 * ((p.rb + 31) / 32));  // the warps with rows
    tc::mbar_init(GRAD_AT(o_full), 1);
    tc::mbar_init(GRAD_AT(done), 1);
    gt::sts32(GRAD_AT(abort), 0u);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
  }
  await_previous();
  release_next();  // behind the wait: what it starts reads what was waited for here
  const int share = blockIdx.x / p.nblk, blk = blockIdx.x - share * p.nblk;
  const gt::Walk walk = gt::Walk::of(p, share);
  if (walk.left == 0) return;  // uniform, before any barrier
  if (warp == W::kIssue) um::alloc(GRAD_AT(tmem), 512);
  um::fence_before();
  __syncthreads();
  um::fence_after();
  const uint32_t tmem = gt::lds32(GRAD_AT(tmem));
  const gt::Stages<FMT> stages = {base + P::kStageOff, GRAD_AT(st_full), GRAD_AT(st_empty), GRAD_AT(live)};
  if (warp < W::kSoft) {
    gt::registers<W::kSoftRegs, W::kLaunch>();
    softmax<FMT>(p, base, tmem, threadIdx.x, share, blk, walk);
  } else if (warp < W::kIssue) {
    gt::registers<W::kLoadRegs, W::kLaunch>();
    const int tid = (int)threadIdx.x - W::kLoad * 32;
    const gt::Ring keys = {GRAD_AT(k_full), GRAD_AT(k_empty), base + P::kKeyOff};
    const gt::Ring values = {GRAD_AT(v_full), GRAD_AT(v_empty), base + P::kValueOff};
    if constexpr (FMT != CERTKV_STORE_BF16) {
      gt::Expander<FMT, P::kKeys, P::kValues> f{keys, values, stages, GRAD_AT(abort), tid};
      f.run(walk);
    } else if (tid < kGroupWarps * 32) {
      gt::Copier<P::kKeys, true> f{&tmK, p, keys, GRAD_AT(facts), GRAD_AT(abort), GRAD_AT(own) + 8u, p.st.k, tid};
      f.run(walk);
    } else {
      gt::Copier<P::kValues, false> f{&tmV, p, values, 0u, GRAD_AT(abort), GRAD_AT(own) + 12u, p.st.v, tid - kGroupWarps * 32};
      f.run(walk);
    }
  } else {
    gt::registers<W::kIssueRegs, W::kLaunch>();
    if (warp == W::kIssue) {
      Issuer<FMT> is{tmem, base};
      is.run(p, walk);
    } else if (FMT != CERTKV_STORE_BF16 && warp == W::kIssue + 1 && threadIdx.x % 32 == 0) {
      gt::Stager<FMT> f{p, stages, GRAD_AT(abort), GRAD_AT(own) + 16u};
      f.run(walk);
    } else if (FMT != CERTKV_STORE_BF16 && warp == W::kIssue + 2) {
      gt::FactFeeder<FMT, P::kKeys> f{p, GRAD_AT(f_full), GRAD_AT(k_empty), GRAD_AT(facts), GRAD_AT(abort), (int)threadIdx.x & 31};
      f.run(walk);
    } else if (warp == W::kIssue + 3 && threadIdx.x % 32 == 0) {
      RowFeeder<FMT>{p, base, blk}.run(walk);
    }
  }
  um::fence_before();
  __syncthreads();
  if (threadIdx.x == 0 && p.st.status && gt::aborted(GRAD_AT(abort))) atomicOr(p.st.status, CERTKV_STATUS_TIMEOUT);
  if (warp == W::kIssue) {
    um::fence_after();
    um::dealloc(tmem, 512);
  }
}

template <int FMT>
bool launch(const CUtensorMap& mk, const CUtensorMap& mv, const GradArgs& p, cudaStream_t st) {
  static std::atomic<uint64_t> ready{0};  // devices on which the shared memory is opted in to
  int dev = 0;
  if (cudaGetDevice(&dev) != cudaSuccess) return false;
  if (dev > 63 || !(ready.load() >> dev & 1u)) {
    if (cudaFuncSetAttribute(grad_q_kernel<FMT>, cudaFuncAttributeMaxDynamicSharedMemorySize, smem_bytes<FMT>()) !=
        cudaSuccess)
      return false;
    if (dev < 64) ready.fetch_or(1ull << dev);
  }
  return launch_kernel(true, grad_q_kernel<FMT>, (unsigned)(p.groups * p.nblk), Warps<FMT>::kThreads, smem_bytes<FMT>(), st, mk, mv,
                       p);
}

}  // namespace

bool launch_grad_q(const GradArgs& p, int format, cudaStream_t st) {
  CUtensorMap mk = {}, mv = {};
  if (!gt::pool_maps(p, format, &mk, &mv)) return false;
  TraceScope ts_("grad_q", st);
  return format == CERTKV_STORE_BF16  ? launch<CERTKV_STORE_BF16>(mk, mv, p, st)
         : format == CERTKV_STORE_FP8 ? launch<CERTKV_STORE_FP8>(mk, mv, p, st)
                                      : launch<CERTKV_STORE_FP4>(mk, mv, p, st);
}

}  // namespace certkv
