// umma.cuh — tcgen05 primitives (inline PTX for sm_103a) of the tree-attention
// kernel: descriptors, tensor-memory loads and stores, commits and fences.
#pragma once

#include <stdint.h>

namespace certkv {
namespace um {

// Shared-memory matrix descriptors of 128-byte swizzled operands: rows of 128 B,
// atoms of 8 rows (1024 B).  K-major: a row holds 64 consecutive k of one m or
// n; atoms follow each other along m or n.  MN-major: a row holds 64 consecutive
// n of one k; atoms follow each other along k, and the next 64 n lie `lbo`
// bytes on.
__device__ __forceinline__ uint32_t desc_lo(uint32_t smem, uint32_t lbo) {
  return ((smem >> 4) & 0x3FFFu) | (((lbo >> 4) & 0x3FFFu) << 16);
}
// high word: 1024 bytes between atoms, descriptor version, 128-byte swizzle
constexpr uint32_t kDescHi = (1024u >> 4) | (1u << 14) | (2u << 29);

// Instruction descriptor of kind::f16: fp32 accumulate, M = 128, N = 128; A and
// B both bf16 or both f16; B K-major or MN-major.
__host__ __device__ constexpr uint32_t idesc(bool bf16, bool b_mn) {
  return (1u << 4) | (bf16 ? (1u << 7) | (1u << 10) : 0u) | (b_mn ? 1u << 16 : 0u) |
         ((128u >> 3) << 17) | ((128u >> 4) << 24);
}

// The eight k-steps of S = Q K^T over a 128 x 128 x 128 tile, both operands
// K-major in two 64-element halves; a, b: low words of their descriptors.  The
// whole warp calls (uniform operands); one elected lane issues.
__device__ __forceinline__ void mma_s(uint32_t d, uint32_t a, uint32_t b, uint32_t hi, uint32_t id) {
  asm volatile(
      "{\n"
      ".reg .pred pe, pz, po;\n"
      ".reg .b32 x, y;\n"
      ".reg .b64 da, db;\n"
      "elect.sync _|pe, 0xffffffff;\n"
      "setp.ne.b32 po, %4, 0;\n"
      "setp.eq.b32 pz, %4, 0;\n"
      "add.u32 x, %1, 0;\n"
      "mov.b64 da, {x, %3};\n"
      "add.u32 y, %2, 0;\n"
      "mov.b64 db, {y, %3};\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, pz;\n"
      "add.u32 x, %1, 2;\n"
      "mov.b64 da, {x, %3};\n"
      "add.u32 y, %2, 2;\n"
      "mov.b64 db, {y, %3};\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, po;\n"
      "add.u32 x, %1, 4;\n"
      "mov.b64 da, {x, %3};\n"
      "add.u32 y, %2, 4;\n"
      "mov.b64 db, {y, %3};\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, po;\n"
      "add.u32 x, %1, 6;\n"
      "mov.b64 da, {x, %3};\n"
      "add.u32 y, %2, 6;\n"
      "mov.b64 db, {y, %3};\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, po;\n"
      "add.u32 x, %1, 1024;\n"
      "mov.b64 da, {x, %3};\n"
      "add.u32 y, %2, 1024;\n"
      "mov.b64 db, {y, %3};\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, po;\n"
      "add.u32 x, %1, 1026;\n"
      "mov.b64 da, {x, %3};\n"
      "add.u32 y, %2, 1026;\n"
      "mov.b64 db, {y, %3};\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, po;\n"
      "add.u32 x, %1, 1028;\n"
      "mov.b64 da, {x, %3};\n"
      "add.u32 y, %2, 1028;\n"
      "mov.b64 db, {y, %3};\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, po;\n"
      "add.u32 x, %1, 1030;\n"
      "mov.b64 da, {x, %3};\n"
      "add.u32 y, %2, 1030;\n"
      "mov.b64 db, {y, %3};\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %4, po;\n"
      "}\n"
      ::"r"(d), "r"(a), "r"(b), "r"(hi), "r"(id)
      : "memory");
}
// The eight k-steps of O (+)= P V: P in tensor memory, 16 slots in each 8 columns
// of every 32; V MN-major, 2048 bytes a k-step.  acc = 0: O is overwritten.
__device__ __forceinline__ void mma_o(uint32_t d, uint32_t a, uint32_t b, uint32_t hi, uint32_t id, uint32_t acc) {
  asm volatile(
      "{\n"
      ".reg .pred pe, p0, po;\n"
      ".reg .b32 x, y;\n"
      ".reg .b64 db;\n"
      "elect.sync _|pe, 0xffffffff;\n"
      "setp.ne.b32 p0, %5, 0;\n"
      "setp.ne.b32 po, %4, 0;\n"
      "add.u32 x, %1, 0;\n"
      "add.u32 y, %2, 0;\n"
      "mov.b64 db, {y, %3};\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %4, p0;\n"
      "add.u32 x, %1, 8;\n"
      "add.u32 y, %2, 128;\n"
      "mov.b64 db, {y, %3};\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %4, po;\n"
      "add.u32 x, %1, 32;\n"
      "add.u32 y, %2, 256;\n"
      "mov.b64 db, {y, %3};\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %4, po;\n"
      "add.u32 x, %1, 40;\n"
      "add.u32 y, %2, 384;\n"
      "mov.b64 db, {y, %3};\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %4, po;\n"
      "add.u32 x, %1, 64;\n"
      "add.u32 y, %2, 512;\n"
      "mov.b64 db, {y, %3};\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %4, po;\n"
      "add.u32 x, %1, 72;\n"
      "add.u32 y, %2, 640;\n"
      "mov.b64 db, {y, %3};\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %4, po;\n"
      "add.u32 x, %1, 96;\n"
      "add.u32 y, %2, 768;\n"
      "mov.b64 db, {y, %3};\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %4, po;\n"
      "add.u32 x, %1, 104;\n"
      "add.u32 y, %2, 896;\n"
      "mov.b64 db, {y, %3};\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %4, po;\n"
      "}\n"
      ::"r"(d), "r"(a), "r"(b), "r"(hi), "r"(id), "r"(acc)
      : "memory");
}
// The same with a second P, 16 columns on, added to the first.
__device__ __forceinline__ void mma_o2(uint32_t d, uint32_t a, uint32_t b, uint32_t hi, uint32_t id, uint32_t acc) {
  asm volatile(
      "{\n"
      ".reg .pred pe, p0, po;\n"
      ".reg .b32 x, y;\n"
      ".reg .b64 db;\n"
      "elect.sync _|pe, 0xffffffff;\n"
      "setp.ne.b32 p0, %5, 0;\n"
      "setp.ne.b32 po, %4, 0;\n"
      "add.u32 x, %1, 0;\n"
      "add.u32 y, %2, 0;\n"
      "mov.b64 db, {y, %3};\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %4, p0;\n"
      "add.u32 x, x, 16;\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %4, po;\n"
      "add.u32 x, %1, 8;\n"
      "add.u32 y, %2, 128;\n"
      "mov.b64 db, {y, %3};\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %4, po;\n"
      "add.u32 x, x, 16;\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %4, po;\n"
      "add.u32 x, %1, 32;\n"
      "add.u32 y, %2, 256;\n"
      "mov.b64 db, {y, %3};\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %4, po;\n"
      "add.u32 x, x, 16;\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %4, po;\n"
      "add.u32 x, %1, 40;\n"
      "add.u32 y, %2, 384;\n"
      "mov.b64 db, {y, %3};\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %4, po;\n"
      "add.u32 x, x, 16;\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %4, po;\n"
      "add.u32 x, %1, 64;\n"
      "add.u32 y, %2, 512;\n"
      "mov.b64 db, {y, %3};\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %4, po;\n"
      "add.u32 x, x, 16;\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %4, po;\n"
      "add.u32 x, %1, 72;\n"
      "add.u32 y, %2, 640;\n"
      "mov.b64 db, {y, %3};\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %4, po;\n"
      "add.u32 x, x, 16;\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %4, po;\n"
      "add.u32 x, %1, 96;\n"
      "add.u32 y, %2, 768;\n"
      "mov.b64 db, {y, %3};\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %4, po;\n"
      "add.u32 x, x, 16;\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %4, po;\n"
      "add.u32 x, %1, 104;\n"
      "add.u32 y, %2, 896;\n"
      "mov.b64 db, {y, %3};\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %4, po;\n"
      "add.u32 x, x, 16;\n"
      "@pe tcgen05.mma.cta_group::1.kind::f16 [%0], [x], db, %4, po;\n"
      "}\n"
      ::"r"(d), "r"(a), "r"(b), "r"(hi), "r"(id), "r"(acc)
      : "memory");
}
// The whole warp calls; the lane that issues the MMAs commits them.
__device__ __forceinline__ void commit(uint32_t mbar) {
  asm volatile(
      "{\n .reg .pred pe;\n elect.sync _|pe, 0xffffffff;\n"
      " @pe tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n}" ::"r"(mbar)
      : "memory");
}
__device__ __forceinline__ void fence_before() {
  asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory");
}
__device__ __forceinline__ void fence_after() {
  asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory");
}
// generic-proxy shared-memory writes before the tensor core's (async-proxy) reads
__device__ __forceinline__ void fence_async() {
  asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
}

// 16 or 32 consecutive columns of this warp's 32 lanes, one lane per thread; the
// wait is part of the statement, so no use can be scheduled before it.
__device__ __forceinline__ void ld32(uint32_t a, uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31}, [%32];\n"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(a + 0u)
      : "memory");
}
__device__ __forceinline__ void ld16(uint32_t a, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n"
      "tcgen05.wait::ld.sync.aligned;"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(a)
      : "memory");
}
__device__ __forceinline__ void st32(uint32_t a, const uint32_t (&r)[32]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,"
      "%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,%24,%25,%26,%27,%28,%29,%30,%31,%32};" ::"r"(a),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
      "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
      "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]),
      "r"(r[23]), "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]),
      "r"(r[30]), "r"(r[31])
      : "memory");
}
__device__ __forceinline__ void st16(uint32_t a, const uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,"
      "%14,%15,%16};" ::"r"(a),
      "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
      "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15])
      : "memory");
}
__device__ __forceinline__ void wait_st() {
  asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory");
}
// the whole warp; columns: a power of two >= 32
__device__ __forceinline__ void alloc(uint32_t slot, uint32_t columns) {
  asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot),
               "r"(columns)
               : "memory");
  asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void dealloc(uint32_t base, uint32_t columns) {
  asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(base), "r"(columns)
               : "memory");
}
// Hardware base-2 exponential, flush to zero, relative error ~2^-22; -inf -> 0.
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// max(a, b, c); a NaN operand is ignored
__device__ __forceinline__ float max3(float a, float b, float c) {
  float r;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(r) : "f"(a), "f"(b), "f"(c));
  return r;
}

}  // namespace um
}  // namespace certkv
