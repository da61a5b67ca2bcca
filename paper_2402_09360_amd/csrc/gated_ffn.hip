// The dense gated FFN, forward and backward, for any number of tokens.
#include "dense_gemm.h"
#include "kernels.h"

#include <type_traits>

namespace hire {
namespace {

// Activation a(g) and its derivative.  silu and the tanh form of gelu are both g s(z) with the logistic function s:
// z = g, or 2 sqrt(2/pi) (g + 0.044715 g^3).  a' = s + g s (1 - s) z'.
constexpr float kGelu = 1.5957691216057308f, kGeluCube = 0.044715f, kLog2E = 1.4426950408889634f;
template <int ACT>
__device__ __forceinline__ float activation(float g, float* slope) {
  if constexpr (ACT == kActRelu) {
    *slope = g > 0.0f ? 1.0f : 0.0f;
    return g > 0.0f ? g : 0.0f;
  } else {
    const float z = ACT == kActSilu ? g : kGelu * (g + kGeluCube * g * g * g);
    const float dz = ACT == kActSilu ? 1.0f : kGelu * (1.0f + 3.0f * kGeluCube * g * g);
    const float s = __builtin_amdgcn_rcpf(1.0f + __builtin_amdgcn_exp2f(-kLog2E * z));
    const float both = s * (1.0f - s);
    *slope = s + (both == 0.0f ? 0.0f : g * both * dz);  // far out dz may be infinite
    return g * s;
  }
}

__device__ __forceinline__ void unpack4(const uint2& v, float (&f)[4]) {
  f[0] = bf16_lo(v.x), f[1] = bf16_hi(v.x), f[2] = bf16_lo(v.y), f[3] = bf16_hi(v.y);
}
__device__ __forceinline__ uint2 pack4(const float (&f)[4]) { return make_uint2(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3])); }

// Four neighbouring columns at a time of a wave's sums: f(row m, column n, quarter of the block, block row, block column).
template <int MB, int NB, typename F>
__device__ __forceinline__ void for_quads(int m0, int n0, int M, int N, F f) {
  const int lane = lane_id();
#pragma unroll
  for (int i = 0; i < MB; ++i) {
    const int m = m0 + 32 * i + (lane & 31);
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q) {
        const int n = n0 + 32 * j + 8 * q + 4 * (lane >> 5);
        if (m < M && n < N) f(m, n, q, i, j);
      }
  }
}

struct StoreBf16 {
  uint16_t* c[3];
  template <int MB, int NB>
  __device__ __forceinline__ void store(const f32x16v (&acc)[MB][NB], int m0, int n0, int M, int N, int product, int) const {
    for_quads<MB, NB>(m0, n0, M, N, [&](int m, int n, int q, int i, int j) {
      const float v[4] = {acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]};
      *reinterpret_cast<uint2*>(c[product] + (size_t)m * N + n) = pack4(v);
    });
  }
};

struct StorePart {  // fp32 sums of one part of k
  float* part;
  template <int MB, int NB>
  __device__ __forceinline__ void store(const f32x16v (&acc)[MB][NB], int m0, int n0, int M, int N, int, int split) const {
    for_quads<MB, NB>(m0, n0, M, N, [&](int m, int n, int q, int i, int j) {
      *reinterpret_cast<float4*>(part + ((size_t)split * M + m) * N + n) =
          make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
    });
  }
};

// h = a(g) u; g and u are kept for the backward pass if asked for, rounded to bf16 like h: the matrix cores take no more.
template <int ACT>
struct StoreGated {
  uint16_t *h, *g, *u;
  template <int MB, int NB>
  __device__ __forceinline__ void store(const f32x16v (&acc)[MB][NB], int m0, int n0, int M, int N, int, int) const {
    static_assert(NB == 2, "the gate's block and the other matrix's");
    for_quads<MB, 1>(m0, n0, M, N, [&](int m, int n, int q, int i, int) {
      float gv[4], uv[4], hv[4], slope;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        gv[e] = acc[i][0][4 * q + e], uv[e] = acc[i][1][4 * q + e];
        hv[e] = activation<ACT>(gv[e], &slope) * uv[e];
      }
      const size_t at = (size_t)m * N + n;
      *reinterpret_cast<uint2*>(h + at) = pack4(hv);
      if (g) {
        *reinterpret_cast<uint2*>(g + at) = pack4(gv);
        *reinterpret_cast<uint2*>(u + at) = pack4(uv);
      }
    });
  }
};

// The sums are dh: dg = dh u a'(g), du = dh a(g), rounded to bf16 for the products that follow.
template <int ACT>
struct StoreGateSlopes {
  const uint16_t *g, *u;
  uint16_t *dg, *du;
  template <int MB, int NB>
  __device__ __forceinline__ void store(const f32x16v (&acc)[MB][NB], int m0, int n0, int M, int N, int, int) const {
    for_quads<MB, NB>(m0, n0, M, N, [&](int m, int n, int q, int i, int j) {
      const size_t at = (size_t)m * N + n;
      float gv[4], uv[4], dgv[4], duv[4];
      unpack4(*reinterpret_cast<const uint2*>(g + at), gv);
      unpack4(*reinterpret_cast<const uint2*>(u + at), uv);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        float slope;
        const float a = activation<ACT>(gv[e], &slope), dh = acc[i][j][4 * q + e];
        dgv[e] = dh * uv[e] * slope;
        duv[e] = dh * a;
      }
      *reinterpret_cast<uint2*>(dg + at) = pack4(dgv);
      *reinterpret_cast<uint2*>(du + at) = pack4(duv);
    });
  }
};

// Sum of the parts in their order, rounded once.
__global__ __launch_bounds__(256) void k_join_parts(const float* __restrict__ part, uint16_t* __restrict__ out, int parts,
                                                    long long quads) {
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < quads; i += (long long)gridDim.x * 256) {
    const float4* p = reinterpret_cast<const float4*>(part) + i;
    float4 s = p[0];
    for (int r = 1; r < parts; ++r) {
      const float4 v = p[(size_t)r * quads];
      s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
    }
    const float f[4] = {s.x, s.y, s.z, s.w};
    reinterpret_cast<uint2*>(out)[i] = pack4(f);
  }
}

constexpr int kTile = 256;

template <bool AK, bool BK, bool PAIR, class Epilogue>
hipError_t launch_product(const GemmArgs& g, const Epilogue& epi, hipStream_t s) {
  auto* kernel = &k_dense_product<kTile, kTile, 2, 4, AK, BK, PAIR, Epilogue>;
  const int n_tile = PAIR ? kTile / 2 : kTile;
  const long long tiles = (long long)((g.M + kTile - 1) / kTile) * ((g.N + n_tile - 1) / n_tile);
  return launch(kernel, dim3((unsigned)(tiles * g.products * g.splits)), dim3(512), 0, s, g, epi);
}

// Parts of k for a product of one M x N matrix: as many as fill the chip, each at least eight stages long.
int product_splits(int M, int N, int steps) {
  const long long tiles = (long long)((M + kTile - 1) / kTile) * ((N + kTile - 1) / kTile);
  int s = (int)(256 / tiles);
  s = s < 1 ? 1 : s;
  const int most = steps / 8 < 1 ? 1 : steps / 8;
  return s < most ? s : most;
}

hipError_t launch_join(const float* part, uint16_t* out, int parts, long long values, hipStream_t s) {
  const long long quads = values / 4, blocks = (quads + 255) / 256;
  return launch(&k_join_parts, dim3((unsigned)(blocks < 4096 ? blocks : 4096)), dim3(256), 0, s, part, out, parts, quads);
}

// One product with an M x N bf16 result, split over k where the tiles are few.
template <bool AK, bool BK>
hipError_t launch_split_product(GemmArgs g, uint16_t* out, float* part, hipStream_t s) {
  g.products = 1;
  g.splits = product_splits(g.M, g.N, g.segments * ((g.K + kGemmStep - 1) / kGemmStep));
  if (g.splits == 1) return launch_product<AK, BK, false>(g, StoreBf16{{out, nullptr, nullptr}}, s);
  const hipError_t e = launch_product<AK, BK, false>(g, StorePart{part}, s);
  return e != hipSuccess ? e : launch_join(part, out, g.splits, (long long)g.M * g.N, s);
}

template <typename F>
hipError_t with_activation(int act, F f) {
  if (act == kActRelu) return f(std::integral_constant<int, kActRelu>{});
  if (act == kActSilu) return f(std::integral_constant<int, kActSilu>{});
  return f(std::integral_constant<int, kActGelu>{});
}

}  // namespace

size_t gated_part_bytes(int T, int d, int d_ff, int segments) {
  const int s = product_splits(T, d, segments * ((d_ff + kGemmStep - 1) / kGemmStep));
  return s > 1 ? (size_t)s * T * d * sizeof(float) : 0;
}

hipError_t launch_gated_forward(const GatedLayer& L, const uint16_t* x, int T, uint16_t* y, uint16_t* h, uint16_t* g,
                                uint16_t* u, float* part, hipStream_t s) {
  GemmArgs up{};
  up.a[0] = x, up.b[0] = L.wg, up.b[1] = L.wu;
  up.M = T, up.N = L.d_ff, up.K = L.d, up.lda = up.ldb = 2u * L.d;
  up.segments = up.products = up.splits = 1;
  const hipError_t e = with_activation(L.act, [&](auto act) {
    return launch_product<true, true, true>(up, StoreGated<decltype(act)::value>{h, g, u}, s);
  });
  if (e != hipSuccess) return e;
  GemmArgs down{};
  down.a[0] = h, down.b[0] = L.w2u;
  down.M = T, down.N = L.d, down.K = L.d_ff, down.lda = 2u * L.d_ff, down.ldb = 2u * L.d;
  down.segments = 1;
  return launch_split_product<true, false>(down, y, part, s);
}

hipError_t launch_gated_backward(const GatedLayer& L, const uint16_t* x, int T, const uint16_t* g, const uint16_t* u,
                                 const uint16_t* h, const uint16_t* dy, uint16_t* dx, uint16_t* dwg, uint16_t* dwu,
                                 uint16_t* dw2u, uint16_t* dg, uint16_t* du, float* part, hipStream_t s) {
  hipError_t e = hipSuccess;
  if (dx || dwg || dwu) {
    GemmArgs a{};
    a.a[0] = dy, a.b[0] = L.w2u;
    a.M = T, a.N = L.d_ff, a.K = L.d, a.lda = a.ldb = 2u * L.d;
    a.segments = a.products = a.splits = 1;
    e = with_activation(L.act, [&](auto act) {
      return launch_product<true, true, false>(a, StoreGateSlopes<decltype(act)::value>{g, u, dg, du}, s);
    });
    if (e != hipSuccess) return e;
  }
  GemmArgs w{};
  StoreBf16 out{};
  auto add = [&](const uint16_t* a, const uint16_t* b, uint16_t* c) {
    if (c) w.a[w.products] = a, w.b[w.products] = b, out.c[w.products++] = c;
  };
  add(dg, x, dwg);
  add(du, x, dwu);
  add(h, dy, dw2u);
  if (w.products > 0) {
    w.M = L.d_ff, w.N = L.d, w.K = T, w.lda = 2u * L.d_ff, w.ldb = 2u * L.d;
    w.segments = w.splits = 1;
    e = launch_product<false, false, false>(w, out, s);
    if (e != hipSuccess) return e;
  }
  if (dx) {
    GemmArgs a{};
    a.a[0] = dg, a.a[1] = du, a.b[0] = L.wg, a.b[1] = L.wu;
    a.M = T, a.N = L.d, a.K = L.d_ff, a.lda = 2u * L.d_ff, a.ldb = 2u * L.d;
    a.segments = 2;
    e = launch_split_product<true, false>(a, dx, part, s);
  }
  return e;
}

}  // namespace hire
