// What the kernels of the dense gated FFN share: the activation and its derivative, and the planes kept for the backward pass.
#pragma once

#include "dense_epilogue.h"

namespace hire {

// Activation a(g) and its derivative.  silu and the tanh form of gelu are both g s(z) with the logistic function s:
// z = g, or 2 sqrt(2/pi) (g + 0.044715 g^3).  a' = s + g s (1 - s) z'.
constexpr float kGelu = 1.5957691216057308f, kGeluCube = 0.044715f, kLog2E = 1.4426950408889634f;
template <int ACT>
__device__ __forceinline__ float activation(float g, float* slope) {
  if constexpr (ACT == kActRelu) {
    *slope = g <= 0.0f ? 0.0f : 1.0f;  // a NaN stays one
    return g <= 0.0f ? 0.0f : g;
  } else {
    const float z = ACT == kActSilu ? g : kGelu * (g + kGeluCube * g * g * g);
    const float dz = ACT == kActSilu ? 1.0f : kGelu * (1.0f + 3.0f * kGeluCube * g * g);
    const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2E * z));
    const float both = s * (1.0f - s);
    *slope = s + (both == 0.0f ? 0.0f : g * both * dz);  // far out dz may be infinite
    return g * s;
  }
}

// The same where few values of a kernel go through it.
__device__ __forceinline__ float activation_of(int act, float g, float* slope) {
  if (act == kActRelu) return activation<kActRelu>(g, slope);
  if (act == kActSilu) return activation<kActSilu>(g, slope);
  return activation<kActGelu>(g, slope);
}

// What the forward call keeps for the backward one: planes of 16 bits per unit and token.  h is rounded to bf16 as the second
// product reads it.  g and u keep 24 bits of their fp32 (15 of the significand), the upper 16 in planes of their own and the
// lower 8 of both in a third (GatedKept): rounded to bf16 they would add their error to that of dg and du, 0.0030 relative to
// dwg instead of 0.0024 (0.0017 is the rounding of dwg itself).
__device__ __forceinline__ uint32_t upper_pair(float a, float b) {
  return __builtin_amdgcn_perm(__float_as_uint(b), __float_as_uint(a), 0x07060302u);
}
// The second bytes of a g pair and a u pair: g0 u0 g1 u1.
__device__ __forceinline__ uint32_t lower_pair(float g0, float u0, float g1, float u1) {
  const uint32_t a = __builtin_amdgcn_perm(__float_as_uint(u0), __float_as_uint(g0), 0x0C0C0501u);
  return a | __builtin_amdgcn_perm(__float_as_uint(u1), __float_as_uint(g1), 0x05010C0Cu);
}
__device__ __forceinline__ void unpack_kept(const uint4& g, const uint4& u, const uint4& low, float (&gv)[8], float (&uv)[8]) {
  const uint32_t gd[4] = {g.x, g.y, g.z, g.w}, ud[4] = {u.x, u.y, u.z, u.w}, ld[4] = {low.x, low.y, low.z, low.w};
#pragma unroll
  for (int q = 0; q < 4; ++q) {  // bytes 0 to 3 of a selector: the second operand's, 4 to 7: the first one's
    gv[2 * q] = __uint_as_float(__builtin_amdgcn_perm(gd[q], ld[q], 0x0504000Cu));
    uv[2 * q] = __uint_as_float(__builtin_amdgcn_perm(ud[q], ld[q], 0x0504010Cu));
    gv[2 * q + 1] = __uint_as_float(__builtin_amdgcn_perm(gd[q], ld[q], 0x0706020Cu));
    uv[2 * q + 1] = __uint_as_float(__builtin_amdgcn_perm(ud[q], ld[q], 0x0706030Cu));
  }
}

// Values in two bf16 terms (kGatedRestTokens).  What the rounding leaves: 0 where the rounded value is no number or infinite.
constexpr float kLargestFloat = 3.4028234663852886e38f;
__device__ __forceinline__ float rest_of(float v, float rounded) {
  const float rest = v - rounded;
  return fabsf(rest) <= kLargestFloat ? rest : 0.0f;
}
__device__ __forceinline__ float bf16_rest(float v) { return rest_of(v, (float)(__bf16)v); }
// A sum of both terms' products that is not finite is to be that of the first terms alone: the second terms' may be infinite on the
// other side, or no number where an infinite factor meets a rest of 0.
__device__ __forceinline__ float first_term(float both, float first) { return fabsf(both) <= kLargestFloat ? both : first; }
template <int N>
__device__ __forceinline__ bool all_finite(const float (&v)[N]) {
  float zero = 0.0f;  // 0 times an infinity, or no number, is no number
#pragma unroll
  for (int e = 0; e < N; ++e) zero = fmaf(v[e], 0.0f, zero);
  return zero == 0.0f;
}

// h = a(g) u of eight units, and what the backward pass needs (kept.g null: h only).
template <int ACT, bool REST = false>
__device__ __forceinline__ void store_gated(const GatedKept& kept, size_t at, const float (&g)[8], const float (&u)[8]) {
  float hv[8], slope;
#pragma unroll
  for (int e = 0; e < 8; ++e) hv[e] = activation<ACT>(g[e], &slope) * u[e];
  *reinterpret_cast<uint4*>(kept.h + at) = pack8(hv);
  if constexpr (REST)
    if (kept.rest) {
#pragma unroll
      for (int e = 0; e < 8; ++e) hv[e] = bf16_rest(hv[e]);
      *reinterpret_cast<uint4*>(kept.rest + at) = pack8(hv);
    }
  if (kept.g) {
    uint32_t gd[4], ud[4], low[4];
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      gd[q] = upper_pair(g[2 * q], g[2 * q + 1]);
      ud[q] = upper_pair(u[2 * q], u[2 * q + 1]);
      low[q] = lower_pair(g[2 * q], u[2 * q], g[2 * q + 1], u[2 * q + 1]);
    }
    *reinterpret_cast<uint4*>(kept.g + at) = make_uint4(gd[0], gd[1], gd[2], gd[3]);
    *reinterpret_cast<uint4*>(kept.u + at) = make_uint4(ud[0], ud[1], ud[2], ud[3]);
    *reinterpret_cast<uint4*>(kept.low + at) = make_uint4(low[0], low[1], low[2], low[3]);
  }
}
// The same from parts of k (StorePart<true>'s order).
template <int ACT>
__global__ __launch_bounds__(256) void k_join_gated(const float* __restrict__ part, int parts, long long values, GatedKept kept) {
  for (long long i = ((long long)blockIdx.x * 256 + threadIdx.x) * 8; i < values; i += (long long)gridDim.x * 2048) {
    float g[8], u[8];
    join_eight(part + i, parts, 2 * (size_t)values, g);
    join_eight(part + values + i, parts, 2 * (size_t)values, u);
    store_gated<ACT, true>(kept, (size_t)i, g, u);
  }
}

// dg = dh u a'(g), du = dh a(g) of eight units, rounded to bf16 for the products that follow.
struct KeptEight {
  uint4 g, u, low;
};
__device__ __forceinline__ KeptEight load_kept(const GatedKept& kept, size_t at) {
  return KeptEight{*reinterpret_cast<const uint4*>(kept.g + at), *reinterpret_cast<const uint4*>(kept.u + at),
                   *reinterpret_cast<const uint4*>(kept.low + at)};
}
template <int ACT>
__device__ __forceinline__ void store_slopes(const KeptEight& k, const float (&dh)[8], uint16_t* dg, uint16_t* du) {
  float gv[8], uv[8], dgv[8], duv[8];
  unpack_kept(k.g, k.u, k.low, gv, uv);
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    float slope;
    const float a = activation<ACT>(gv[e], &slope);
    dgv[e] = dh[e] * uv[e] * slope;
    duv[e] = dh[e] * a;
  }
  *reinterpret_cast<uint4*>(dg) = pack8(dgv);
  *reinterpret_cast<uint4*>(du) = pack8(duv);
}
template <int ACT>
__global__ __launch_bounds__(256) void k_join_slopes(const float* __restrict__ part, int parts, long long values, GatedKept kept,
                                                     uint16_t* __restrict__ dg, uint16_t* __restrict__ du) {
  for (long long i = ((long long)blockIdx.x * 256 + threadIdx.x) * 8; i < values; i += (long long)gridDim.x * 2048) {
    const KeptEight k = load_kept(kept, (size_t)i);
    float dh[8];
    join_eight(part + i, parts, (size_t)values, dh);
    store_slopes<ACT>(k, dh, dg + i, du + i);
  }
}

// Rows of up to three products in bf16.  STREAMING: past the caches, for the weights' gradients, whose writing is what the products
// of few tokens are bound by (d = 2048, 16384 units, one token: 60 -> 36 us, a plain fill 34).
template <bool STREAMING>
struct StoreBf16 {
  uint16_t* c[3];
  template <int MB, int NB>
  __device__ __forceinline__ void store(const f32x16v (&acc)[MB][NB], char* smem, int m0, int n0, int M, int N, int product,
                                        int) const {
    for_rows<false>(acc, smem, m0, n0, M, N, NoFetch{}, [&](int m, int n, const float (&v)[1][8], int) {
      uint16_t* to = c[product] + (size_t)m * N + n;
      if constexpr (STREAMING)
        store_streaming(to, pack8(v[0]));
      else
        *reinterpret_cast<uint4*>(to) = pack8(v[0]);
    });
  }
};
// gated_few.hip: K up to 64; rest: of the products' first operands (null: none)
struct GatedRests {
  const uint16_t* of[3];
};
hipError_t launch_gated_few_weights(const GemmArgs& g, const GatedRests& rest, const StoreBf16<true>& out, hipStream_t s);
hipError_t launch_gated_rest(const GatedLayer& L, int T, const GatedKept& kept, uint16_t* rest, hipStream_t s);  // of the kept h

// Calls f with the activation as a type.
template <typename F>
hipError_t with_activation(int act, F f) {
  if (act == kActRelu) return f(std::integral_constant<int, kActRelu>{});
  if (act == kActSilu) return f(std::integral_constant<int, kActSilu>{});
  return f(std::integral_constant<int, kActGelu>{});
}

}  // namespace hire
