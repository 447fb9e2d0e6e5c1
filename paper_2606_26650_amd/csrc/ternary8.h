// Packed-ternary codes and 8-bit activations as matrix operands, shared by the products on them.
//
// Codes to operands.  Word w of 16 codes (code i in bits 2i) gives four operand words:
// the codes j, 4 + j, 8 + j, 12 + j are the bytes of (w >> 2j) & 0x03030303, and one byte
// permute looks their values T up (0 -> -1, 1 -> 0, 2 -> 1, 3 -> 0): 11 instructions for
// 16 codes, where bf16 operands take 22.  The contraction order inside 16 values is thus
// 0 4 8 12 1 5 9 13 ..., and the activations are brought into the same order, a 4 x 4
// transposition of bytes.
#pragma once

#include "catq_internal.h"

namespace catq {

typedef __attribute__((ext_vector_type(4))) int i32x4;

constexpr uint32_t kTernTab = 0x000100FFu;   // bytes by code: -1, 0, 1, 0

__device__ __forceinline__ u32x4 decode16_i8(uint32_t w) {
  u32x4 r;
#pragma unroll
  for (int j = 0; j < 4; ++j)
    r[j] = __builtin_amdgcn_perm(0u, kTernTab, (w >> (2 * j)) & 0x03030303u);
  return r;
}

// 16 bytes x0 .. x15 -> words {x0 x4 x8 x12} {x1 x5 x9 x13} ...
__device__ __forceinline__ u32x4 transpose16(u32x4 x) {
  const uint32_t a = __builtin_amdgcn_perm(x[1], x[0], 0x05010400u);   // x0 x4 x1 x5
  const uint32_t b = __builtin_amdgcn_perm(x[1], x[0], 0x07030602u);   // x2 x6 x3 x7
  const uint32_t c = __builtin_amdgcn_perm(x[3], x[2], 0x05010400u);   // x8 x12 x9 x13
  const uint32_t d = __builtin_amdgcn_perm(x[3], x[2], 0x07030602u);
  u32x4 r;
  r[0] = __builtin_amdgcn_perm(c, a, 0x05040100u);
  r[1] = __builtin_amdgcn_perm(c, a, 0x07060302u);
  r[2] = __builtin_amdgcn_perm(d, b, 0x05040100u);
  r[3] = __builtin_amdgcn_perm(d, b, 0x07060302u);
  return r;
}

__device__ __forceinline__ i32x4 mfma_i8(u32x4 a, u32x4 b, i32x4 c) {
  return __builtin_amdgcn_mfma_i32_16x16x64_i8(__builtin_bit_cast(i32x4, a), __builtin_bit_cast(i32x4, b), c,
                                               0, 0, 0);
}

// the LDS reads of this wave have returned
__device__ __forceinline__ void wait_lds() {
#if defined(__HIP_DEVICE_COMPILE__)
  asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#endif
}

}  // namespace catq
