// Microscaled 4-bit floating point (MXFP4): blocks of 32 values along a row, each value an e2m1 code (0, 0.5, 1, 1.5, 2, 3,
// 4, 6 and their negatives) times the block's power of two, an e8m0 byte (2^(byte - 127); 255: not a number).
#pragma once

#include "dense_gemm.h"

namespace hire {

typedef __bf16 bf16x2v __attribute__((ext_vector_type(2)));

constexpr int kMxBlock = 32;

// A scale byte as the conversions take it: in the exponent of an fp32.  They read nothing else of it, so that byte 0 is 2^-127
// and 255 makes NaN of every code.
__device__ __forceinline__ float mx_scale(uint32_t byte) { return __uint_as_float(byte << 23); }
// The same of byte J of a word.
template <int J>
__device__ __forceinline__ float mx_scale_of(uint32_t word) {
  return __uint_as_float((J == 3 ? word >> 1 : word << (23 - 8 * J)) & 0x7F800000u);
}

// Eight codes (one dword) times a scale as bf16 pairs: exact (two bits of significand) but for magnitudes beyond the type's
// largest, which become infinite.
__device__ __forceinline__ uint4 mx_to_bf16(uint32_t codes, float scale) {
  const bf16x2v v[4] = {
      __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1),
      __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2), __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3)};
  uint4 u;
  __builtin_memcpy(&u, v, 16);
  return u;
}

}  // namespace hire
