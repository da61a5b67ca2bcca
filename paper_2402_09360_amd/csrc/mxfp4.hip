// Microscaled 4-bit floating point: packing, reading back, and the product of packed rows with tokens in bf16 or packed
// themselves.  Layout: codes [rows, cols / 2], the lower column in the low nibble; scale bytes [rows, cols / 32].
#include "mxfp4.h"

#include "dense_epilogue.h"

namespace hire {
namespace {

// ---- packing ----------------------------------------------------------------
// A block is eight values in each of four lanes.  Its power of two is that of its largest magnitude, less two (6 = 1.5 2^2 is
// the largest code), so only magnitudes in (6, 8) 2^e saturate; e is at least -127.  The quotients are exact, and the
// conversion rounds half steps to the even code.
__global__ __launch_bounds__(256) void k_pack_mxfp4(const uint4* __restrict__ w, long long eights, uint32_t* __restrict__ codes,
                                                    uint8_t* __restrict__ scales) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < eights; i += (long long)gridDim.x * 256) {
    const uint4 v = w[i];
    const uint32_t d[4] = {v.x, v.y, v.z, v.w};
    u16x2 m = {0, 0};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      u16x2 a;
      const uint32_t magnitude = d[q] & 0x7FFF7FFFu;
      __builtin_memcpy(&a, &magnitude, 4);
      m = __builtin_elementwise_max(m, a);
    }
    uint32_t top = m[0] > m[1] ? m[0] : m[1];
    top = max(top, dpp_move<0xB1, 0xF>(0u, top));  // lanes 1 0 3 2 of every four
    top = max(top, dpp_move<0x4E, 0xF>(0u, top));  // lanes 2 3 0 1
    const uint32_t exponent = top >> 7;
    uint32_t byte = exponent > 2u ? exponent - 2u : 0u;
    if (top == 0u) byte = 127u;
    const bool finite = top < 0x7F80u;
    const float scale = mx_scale(byte);
    uint32_t c = 0u;
    bf16x2v pair[4];
    __builtin_memcpy(pair, d, 16);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, pair[0], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, pair[1], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, pair[2], scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, pair[3], scale, 3);
    codes[i] = finite ? c : 0u;
    if ((i & 3) == 0) scales[i >> 2] = finite ? (uint8_t)byte : (uint8_t)255;
  }
}

__global__ __launch_bounds__(256) void k_unpack_mxfp4(const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                      long long eights, uint4* __restrict__ w) {
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < eights; i += (long long)gridDim.x * 256)
    w[i] = mx_to_bf16(codes[i], mx_scale(scales[i >> 2]));
}

// ---- few tokens -----------------------------------------------------------------
// A wave multiplies RU times sixteen rows with NT times sixteen tokens; the waves of a workgroup take the steps of 128 columns
// in turn and their sums are added in LDS in a fixed order.  A lane holds one block (32 codes) of one row per step.
constexpr int kFewWaves = 4;

template <bool PACKED_TOKENS, int NT, int RU>
__global__ __launch_bounds__(64 * kFewWaves) void k_mx_few(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                           const void* __restrict__ x, const uint8_t* __restrict__ x_scales,
                                                           int T, int rows, int cols, void* __restrict__ y, int y_bf16) {
  __shared__ float sums[kFewWaves][RU * NT * 256];
  const int lane = lane_id(), wave = wave_id(), kq = lane >> 4, blocks = cols / kMxBlock;
  const int row0 = blockIdx.x * 16 * RU;
  const uint8_t *row[RU], *row_scale[RU];
#pragma unroll
  for (int r = 0; r < RU; ++r) {
    const int at = min(row0 + 16 * r + (lane & 15), rows - 1);
    row[r] = codes + (size_t)at * (cols / 2);
    row_scale[r] = scales + (size_t)at * blocks;
  }
  size_t token[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) token[t] = (size_t)min(16 * t + (lane & 15), T - 1);

  f32x4v acc[RU][NT] = {};
  const int steps = (blocks + 3) / 4;
  for (int s = wave; s < steps; s += kFewWaves) {
    const int block = 4 * s + kq;
    const bool there = block < blocks;
    const int b = there ? block : blocks - 1;
    uint4 c[RU];
    uint32_t sc[RU];
#pragma unroll
    for (int r = 0; r < RU; ++r) {
      c[r] = load_streaming(reinterpret_cast<const uint4*>(row[r]) + b);
      sc[r] = row_scale[r][b];
    }
    if constexpr (PACKED_TOKENS) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        uint4 xc = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(x) + token[t] * (cols / 2))[b];
        const uint32_t xs = there ? x_scales[token[t] * blocks + b] : 127u;
        if (!there) xc = make_uint4(0u, 0u, 0u, 0u);
        const i32x8v xv = {(int)xc.x, (int)xc.y, (int)xc.z, (int)xc.w, 0, 0, 0, 0};
#pragma unroll
        for (int r = 0; r < RU; ++r) {
          const i32x8v cv = {(int)c[r].x, (int)c[r].y, (int)c[r].z, (int)c[r].w, 0, 0, 0, 0};
          acc[r][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(cv, xv, acc[r][t], 4, 4, 0, there ? (int)sc[r] : 127, 0,
                                                                       (int)xs);
        }
      }
    } else {
      uint4 xv[NT][4];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const uint4* p = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(x) + token[t] * cols) + 4 * b;
#pragma unroll
        for (int j = 0; j < 4; ++j) xv[t][j] = there ? p[j] : make_uint4(0u, 0u, 0u, 0u);
      }
#pragma unroll
      for (int r = 0; r < RU; ++r) {
        const float scale = mx_scale(there ? sc[r] : 127u);
        const uint32_t cd[4] = {c[r].x, c[r].y, c[r].z, c[r].w};
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const uint4 w4 = mx_to_bf16(there ? cd[j] : 0u, scale);
          bf16x8v wv;
          __builtin_memcpy(&wv, &w4, 16);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            bf16x8v xf;
            __builtin_memcpy(&xf, &xv[t][j], 16);
            acc[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv, xf, acc[r][t], 0, 0, 0);
          }
        }
      }
    }
  }
  // acc[r][t]: token 16 t + lane % 16, rows 16 r + 4 (lane / 16) ... of this wave's columns
#pragma unroll
  for (int r = 0; r < RU; ++r)
#pragma unroll
    for (int t = 0; t < NT; ++t)
      *reinterpret_cast<f32x4v*>(&sums[wave][((r * NT + t) * 64 + lane) * 4]) = acc[r][t];
  __syncthreads();
  for (int i = threadIdx.x; i < RU * NT * 256; i += 64 * kFewWaves) {
    // neighbouring threads: neighbouring rows of one token
    const int n = i % (16 * RU), tok = i / (16 * RU), at = ((n / 16 * NT + tok / 16) * 64 + (n % 16 / 4) * 16 + tok % 16) * 4 + n % 4;
    float v = sums[0][at];
#pragma unroll
    for (int q = 1; q < kFewWaves; ++q) v += sums[q][at];
    if (tok < T && row0 + n < rows) {
      const size_t o = (size_t)tok * rows + row0 + n;
      if (y_bf16)
        static_cast<__bf16*>(y)[o] = (__bf16)v;
      else
        static_cast<float*>(y)[o] = v;
    }
  }
}

// ---- many tokens, packed ----------------------------------------------------------
// y's rows out of the sums: whole vectors where the row length admits them.
struct StoreProduct {
  void* y;
  int bf16;
  template <int MB, int NB>
  __device__ __forceinline__ void store(const f32x16v (&acc)[MB][NB], char* smem, int m0, int n0, int M, int N, int, int) const {
    for_rows<false>(acc, smem, m0, n0, M, N, [&](int m, int n, const float (&v)[1][8]) {
      const size_t at = (size_t)m * N + n;
      if (N % 8 != 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (n + e < N) {
            if (bf16)
              static_cast<__bf16*>(y)[at + e] = (__bf16)v[0][e];
            else
              static_cast<float*>(y)[at + e] = v[0][e];
          }
      } else if (bf16) {
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(y) + at) = pack8(v[0]);
      } else {
        float4* to = reinterpret_cast<float4*>(static_cast<float*>(y) + at);
        to[0] = make_float4(v[0][0], v[0][1], v[0][2], v[0][3]);
        to[1] = make_float4(v[0][4], v[0][5], v[0][6], v[0][7]);
      }
    });
  }
};

// Scale bytes in rows of whole words, 127 behind the last block: what the product reads where the columns are no multiple of
// 128 (or the caller's bytes start between words).
__global__ __launch_bounds__(256) void k_pad_scales(const uint8_t* __restrict__ scales, long long rows, int blocks, int words,
                                                    uint32_t* __restrict__ out) {
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < rows * words; i += (long long)gridDim.x * 256) {
    const long long row = i / words;
    const int b = (int)(i - row * words) * 4;
    uint32_t v = 0u;
#pragma unroll
    for (int e = 0; e < 4; ++e) v |= (b + e < blocks ? (uint32_t)scales[row * blocks + b + e] : 127u) << (8 * e);
    out[i] = v;
  }
}

template <bool PACKED, int NT, int RU>
hipError_t launch_few(const MxProduct& p, hipStream_t s) {
  return launch(&k_mx_few<PACKED, NT, RU>, dim3((unsigned)((p.rows + 16 * RU - 1) / (16 * RU))), dim3(64 * kFewWaves), 0, s,
                p.codes, p.scales, p.x, p.x_scales, p.T, p.rows, p.cols, p.y, p.y_bf16);
}
template <bool PACKED>
hipError_t launch_few_tokens(const MxProduct& p, hipStream_t s) {
  const int nt = (p.T + 15) / 16;
  if (nt == 1) return p.rows >= 32768 ? launch_few<PACKED, 1, 4>(p, s) : launch_few<PACKED, 1, 2>(p, s);
  if (nt == 2) return launch_few<PACKED, 2, 2>(p, s);
  return launch_few<PACKED, 4, 2>(p, s);
}

}  // namespace

hipError_t launch_pack_mxfp4(const uint16_t* w, int rows, int cols, uint8_t* codes, uint8_t* scales, hipStream_t s) {
  const long long eights = (long long)rows * cols / 8, groups = (eights + 255) / 256;
  return launch(&k_pack_mxfp4, dim3((unsigned)(groups < 16384 ? groups : 16384)), dim3(256), 0, s, reinterpret_cast<const uint4*>(w),
                eights, reinterpret_cast<uint32_t*>(codes), scales);
}

hipError_t launch_unpack_mxfp4(const uint8_t* codes, const uint8_t* scales, int rows, int cols, uint16_t* w, hipStream_t s) {
  const long long eights = (long long)rows * cols / 8, groups = (eights + 255) / 256;
  return launch(&k_unpack_mxfp4, dim3((unsigned)(groups < 16384 ? groups : 16384)), dim3(256), 0, s,
                reinterpret_cast<const uint32_t*>(codes), scales, eights, reinterpret_cast<uint4*>(w));
}

namespace {
bool mx_pads_scales(const MxProduct& p) {
  return p.cols % 128 != 0 || reinterpret_cast<uintptr_t>(p.x_scales) % 4 != 0 || reinterpret_cast<uintptr_t>(p.scales) % 4 != 0;
}
}  // namespace

// Room for the padded scale bytes, whether this call's pointers need them or not.
size_t mx_workspace_bytes(int T, int rows, int cols) {
  return T <= kMxFewTokens ? 0 : ((size_t)T + rows) * ((cols / kMxBlock + 3) / 4) * 4;
}

hipError_t launch_mx_product(const MxProduct& p, hipStream_t s) {
  if (p.T <= kMxFewTokens) return p.x_scales ? launch_few_tokens<true>(p, s) : launch_few_tokens<false>(p, s);
  const int blocks = p.cols / kMxBlock, words = (blocks + 3) / 4;
  GemmArgs g{};
  g.a[0] = p.x, g.b[0] = p.codes;
  g.M = p.T, g.N = p.rows, g.K = p.cols / 4, g.lda = g.ldb = (uint32_t)p.cols / 2;
  g.segments = g.products = g.splits = 1;
  g.a_scales = p.x_scales, g.b_scales = p.scales, g.scale_ld = 4u * words;
  if (mx_pads_scales(p)) {
    uint32_t* padded = static_cast<uint32_t*>(p.workspace);
    auto pad = [&](const uint8_t* from, int rows, uint32_t* to) {
      const long long groups = ((long long)rows * words + 255) / 256;
      return launch(&k_pad_scales, dim3((unsigned)(groups < 4096 ? groups : 4096)), dim3(256), 0, s, from, (long long)rows, blocks,
                    words, to);
    };
    hipError_t e = pad(p.x_scales, p.T, padded);
    if (e == hipSuccess) e = pad(p.scales, p.rows, padded + (size_t)p.T * words);
    if (e != hipSuccess) return e;
    g.a_scales = reinterpret_cast<const uint8_t*>(padded);
    g.b_scales = reinterpret_cast<const uint8_t*>(padded + (size_t)p.T * words);
  }
  return launch_product<true, true, false, true>(g, StoreProduct{p.y, p.y_bf16}, s);
}

}  // namespace hire
