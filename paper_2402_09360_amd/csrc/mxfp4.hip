// Microscaled 4-bit floating point: packing, reading back, and the product of packed rows with tokens in bf16 or packed
// themselves.  Layout: codes [rows, cols / 2], the lower column in the low nibble; scale bytes [rows, cols / 32].
#include "mxfp4.h"

#include "dense_gemm.h"
#include "kernels.h"

#include <type_traits>

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
// Tiles as in the product of bf16 matrices: 128 bytes of a row are a stage of 256 columns, 16 of them a block and what a lane
// holds of the matrix instruction.  A row's eight scale bytes of a stage come straight into registers of the lanes that
// need them, requested with the stage.
constexpr int kMxStage = 256;

__device__ __forceinline__ uint2 stage_scales(const uint8_t* row, int block, int blocks) {
  uint2 v;
  if (block + 8 <= blocks) {
    __builtin_memcpy(&v, row + block, 8);
    return v;
  }
  uint32_t d[2] = {0x7F7F7F7Fu, 0x7F7F7F7Fu};  // 1 behind the end, where the codes are 0
  for (int i = 0; i < 8; ++i)
    if (block + i < blocks) d[i / 4] = (d[i / 4] & ~(0xFFu << (8 * (i % 4)))) | (uint32_t)row[block + i] << (8 * (i % 4));
  return make_uint2(d[0], d[1]);
}

template <int KS>
__device__ __forceinline__ f32x16v mx_mfma(const i32x8v& a, const i32x8v& b, const f32x16v& c, uint32_t sa, uint32_t sb) {
  return __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(a, b, c, 4, 4, KS, (int)sa, KS, (int)sb);
}

template <int MT, int NT, int MW, int NW>
__global__ __launch_bounds__(64 * MW * NW) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_mx_product(
    const uint8_t* __restrict__ x, const uint8_t* __restrict__ x_scales, int T, const uint8_t* __restrict__ codes,
    const uint8_t* __restrict__ scales, int rows, int cols, void* __restrict__ y, int y_bf16) {
  constexpr int kWaves = MW * NW, kMB = MT / MW / 32, kNB = NT / NW / 32;
  using TA = GemmTile<MT, kWaves, true, false>;
  using TB = GemmTile<NT, kWaves, true, false>;
  constexpr int kStage = TA::kBytes + TB::kBytes;
  __shared__ __align__(1024) char smem[2 * kStage];

  const int tiles_m = (T + MT - 1) / MT, tiles_n = (rows + NT - 1) / NT, blocks = cols / kMxBlock;
  const int t = gemm_place((int)blockIdx.x, (int)gridDim.x);
  const int group = t / (8 * tiles_n), in = t % (8 * tiles_n), gm = min(8, tiles_m - 8 * group);
  const int m0 = (8 * group + in % gm) * MT, n0 = in / gm * NT;
  const uint32_t ld = (uint32_t)cols / 2;
  const int steps = (cols + kMxStage - 1) / kMxStage;

  TA ta;
  TB tb;
  ta.init(m0, T, ld);
  tb.init(n0, rows, ld);
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(gemm_lds_offset(smem));
  const int wave = wave_id(), lane = lane_id(), wm = wave / NW * (MT / MW), wn = wave % NW * (NT / NW);
  const uint8_t *xs[kMB], *ws[kNB];
#pragma unroll
  for (int i = 0; i < kMB; ++i) xs[i] = x_scales + (size_t)min(m0 + wm + 32 * i + (lane & 31), T - 1) * blocks;
#pragma unroll
  for (int j = 0; j < kNB; ++j) ws[j] = scales + (size_t)min(n0 + wn + 32 * j + (lane & 31), rows - 1) * blocks;
  uint2 nx[kMB], nw[kNB];
  auto request = [&](int s) {
    const uint32_t lds = lds0 + (uint32_t)(s & 1) * kStage;
    const int left = (cols - s * kMxStage) / 4;  // the tile counts two bytes as one of 64
    ta.load(reinterpret_cast<const char*>(x) + (size_t)m0 * ld + (size_t)s * 128, nullptr, left, lds);
    tb.load(reinterpret_cast<const char*>(codes) + (size_t)n0 * ld + (size_t)s * 128, nullptr, left, lds + TA::kBytes);
#pragma unroll
    for (int i = 0; i < kMB; ++i) nx[i] = stage_scales(xs[i], 8 * s, blocks);
#pragma unroll
    for (int j = 0; j < kNB; ++j) nw[j] = stage_scales(ws[j], 8 * s, blocks);
  };
  // bytes of the blocks 0 2 4 6 for the lower half of the wave, 1 3 5 7 for the upper one
  const uint32_t pick = lane < 32 ? 0x06040200u : 0x07050301u;

  f32x16v acc[kMB][kNB] = {};
  request(0);
  for (int s = 0; s < steps; ++s) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    uint32_t sx[kMB], sw[kNB];
#pragma unroll
    for (int i = 0; i < kMB; ++i) {
      sx[i] = __builtin_amdgcn_perm(nx[i].y, nx[i].x, pick);
      asm volatile("" : "+v"(sx[i]));  // before the next stage's requests: behind them the compiler would wait for those
    }
#pragma unroll
    for (int j = 0; j < kNB; ++j) {
      sw[j] = __builtin_amdgcn_perm(nw[j].y, nw[j].x, pick);
      asm volatile("" : "+v"(sw[j]));
    }
    if (s + 1 < steps) request(s + 1);
    const char* sa = smem + (s & 1) * kStage;
    const char* sb = sa + TA::kBytes;
    auto multiply = [&](auto ks) {
      constexpr int KS = decltype(ks)::value;
      i32x8v fa[kMB] = {}, fb[kNB] = {};
#pragma unroll
      for (int i = 0; i < kMB; ++i) {
        const bf16x8v v = TA::fragment(sa, wm + 32 * i, KS);
        __builtin_memcpy(&fa[i], &v, 16);
      }
#pragma unroll
      for (int j = 0; j < kNB; ++j) {
        const bf16x8v v = TB::fragment(sb, wn + 32 * j, KS);
        __builtin_memcpy(&fb[j], &v, 16);
      }
#pragma unroll
      for (int i = 0; i < kMB; ++i)
#pragma unroll
        for (int j = 0; j < kNB; ++j) acc[i][j] = mx_mfma<KS>(fb[j], fa[i], acc[i][j], sw[j], sx[i]);
    };
    multiply(std::integral_constant<int, 0>{});
    multiply(std::integral_constant<int, 1>{});
    multiply(std::integral_constant<int, 2>{});
    multiply(std::integral_constant<int, 3>{});
  }
#pragma unroll
  for (int i = 0; i < kMB; ++i) {
    const int m = m0 + wm + 32 * i + (lane & 31);
#pragma unroll
    for (int j = 0; j < kNB; ++j)
#pragma unroll
      for (int r = 0; r < 16; ++r) {
        const int n = n0 + wn + 32 * j + 8 * (r / 4) + 4 * (lane >> 5) + r % 4;
        if (m < T && n < rows) {
          const size_t o = (size_t)m * rows + n;
          if (y_bf16)
            static_cast<__bf16*>(y)[o] = (__bf16)acc[i][j][r];
          else
            static_cast<float*>(y)[o] = acc[i][j][r];
        }
      }
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

hipError_t launch_mx_product(const MxProduct& p, hipStream_t s) {
  if (p.T <= kMxFewTokens) return p.x_scales ? launch_few_tokens<true>(p, s) : launch_few_tokens<false>(p, s);
  const long long tiles = (long long)((p.T + 255) / 256) * ((p.rows + 255) / 256);
  return launch(&k_mx_product<256, 256, 2, 4>, dim3((unsigned)tiles), dim3(512), 0, s, static_cast<const uint8_t*>(p.x), p.x_scales,
                p.T, p.codes, p.scales, p.rows, p.cols, p.y, p.y_bf16);
}

}  // namespace hire
