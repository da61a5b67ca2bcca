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

// Lane (row r, q = lane / 16) has sixteen bytes of codes, block q of four; afterwards word j of it is word q of block j.
template <int RU>
__device__ __forceinline__ void exchange_blocks(uint4 (&c)[RU]) {
#pragma unroll
  for (int r = 0; r < RU; ++r) {
    const auto a = __builtin_amdgcn_permlane32_swap(c[r].x, c[r].z, false, false);
    const auto b = __builtin_amdgcn_permlane32_swap(c[r].y, c[r].w, false, false);
    const auto lo = __builtin_amdgcn_permlane16_swap(a[0], b[0], false, false);
    const auto hi = __builtin_amdgcn_permlane16_swap(a[1], b[1], false, false);
    c[r] = make_uint4(lo[0], lo[1], hi[0], hi[1]);
  }
}

// Four neighbouring rows' results of a token, as far as they are there.
__device__ __forceinline__ void store_rows(void* __restrict__ y, int y_bf16, int T, int rows, int token, int row, const f32x4v& v) {
  if (token >= T || row >= rows) return;
  const size_t at = (size_t)token * rows + row;
  if (rows % 4 != 0) {
    for (int e = 0; e < 4 && row + e < rows; ++e) {
      if (y_bf16)
        static_cast<__bf16*>(y)[at + e] = (__bf16)v[e];
      else
        static_cast<float*>(y)[at + e] = v[e];
    }
  } else if (y_bf16) {
    *reinterpret_cast<uint2*>(static_cast<uint16_t*>(y) + at) = make_uint2(bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]));
  } else {
    *reinterpret_cast<float4*>(static_cast<float*>(y) + at) = make_float4(v[0], v[1], v[2], v[3]);
  }
}

}  // namespace hire
