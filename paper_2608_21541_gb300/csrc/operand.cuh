// operand.cuh — a tile of 128 rows of the store on its way into a swizzled operand of the
// tensor cores: which of its elements a loader thread takes and where they go.
#pragma once

#include <stdint.h>

#include "common.cuh"
#include "store.cuh"

namespace certkv {

constexpr int kGroupWarps = 4;       // warps that load an operand together
constexpr int kHalf = 128 * 128;     // bytes of 128 rows x 64 16-bit elements
constexpr int kOperand = 2 * kHalf;  // 128 rows x 128 elements
// A loader thread's (slot, 16-element) pieces of an operand, kStep slots apart.
constexpr int kPieces = 128 * 8 / (kGroupWarps * 32), kStep = 128 / kPieces;

__device__ __forceinline__ void sts128(uint32_t a, uint32_t x, uint32_t y, uint32_t z, uint32_t w) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" ::"r"(a), "r"(x), "r"(y), "r"(z), "r"(w)
               : "memory");
}

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

}  // namespace certkv
