// The dense gated FFN, forward and backward, for any number of tokens.
#include "gated.h"

namespace hire {
namespace {

struct StoreBf16 {
  uint16_t* c[3];
  template <int MB, int NB>
  __device__ __forceinline__ void store(const f32x16v (&acc)[MB][NB], char* smem, int m0, int n0, int M, int N, int product,
                                        int) const {
    for_rows<false>(acc, smem, m0, n0, M, N, NoFetch{}, [&](int m, int n, const float (&v)[1][8], int) {
      *reinterpret_cast<uint4*>(c[product] + (size_t)m * N + n) = pack8(v[0]);
    });
  }
};

// h = a(g) u.
template <int ACT>
struct StoreGated {
  GatedKept kept;  // g null: h only
  template <int MB, int NB>
  __device__ __forceinline__ void store(const f32x16v (&acc)[MB][NB], char* smem, int m0, int n0, int M, int N, int, int) const {
    for_rows<true>(acc, smem, m0, n0, M, N, NoFetch{}, [&](int m, int n, const float (&v)[2][8], int) {
      const size_t at = (size_t)m * N + n;
      float hv[8], slope;
#pragma unroll
      for (int e = 0; e < 8; ++e) hv[e] = activation<ACT>(v[0][e], &slope) * v[1][e];
      *reinterpret_cast<uint4*>(kept.h + at) = pack8(hv);
      if (kept.g) {
        uint32_t g[4], u[4], low[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
          g[q] = upper_pair(v[0][2 * q], v[0][2 * q + 1]);
          u[q] = upper_pair(v[1][2 * q], v[1][2 * q + 1]);
          low[q] = lower_pair(v[0][2 * q], v[1][2 * q], v[0][2 * q + 1], v[1][2 * q + 1]);
        }
        *reinterpret_cast<uint4*>(kept.g + at) = make_uint4(g[0], g[1], g[2], g[3]);
        *reinterpret_cast<uint4*>(kept.u + at) = make_uint4(u[0], u[1], u[2], u[3]);
        *reinterpret_cast<uint4*>(kept.low + at) = make_uint4(low[0], low[1], low[2], low[3]);
      }
    });
  }
};

// The sums are dh: dg = dh u a'(g), du = dh a(g), rounded to bf16 for the products that follow.
template <int ACT>
struct StoreGateSlopes {
  GatedKept kept;
  uint16_t *dg, *du;
  template <int MB, int NB>
  __device__ __forceinline__ void store(const f32x16v (&acc)[MB][NB], char* smem, int m0, int n0, int M, int N, int, int) const {
    struct Planes {
      uint4 g, u, low;
    };
    auto fetch = [&](int m, int n) {
      const size_t at = (size_t)m * N + n;
      return Planes{*reinterpret_cast<const uint4*>(kept.g + at), *reinterpret_cast<const uint4*>(kept.u + at),
                    *reinterpret_cast<const uint4*>(kept.low + at)};
    };
    for_rows<false>(acc, smem, m0, n0, M, N, fetch, [&](int m, int n, const float (&v)[1][8], const Planes& k) {
      const size_t at = (size_t)m * N + n;
      float gv[8], uv[8], dgv[8], duv[8];
      unpack_kept(k.g, k.u, k.low, gv, uv);
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        float slope;
        const float a = activation<ACT>(gv[e], &slope), dh = v[0][e];
        dgv[e] = dh * uv[e] * slope;
        duv[e] = dh * a;
      }
      *reinterpret_cast<uint4*>(dg + at) = pack8(dgv);
      *reinterpret_cast<uint4*>(du + at) = pack8(duv);
    });
  }
};

constexpr int kMostSplits = 32;
int k_steps(int k) { return (k + kGemmStep - 1) / kGemmStep; }
ProductShape split_shape(int M, int N, int K, int segments) {
  return product_shape(M, N, segments * k_steps(K), 1, kMostSplits);
}

// One product with an M x N bf16 result, split over k where the tiles are few.
template <bool AK, bool BK>
hipError_t launch_split_product(GemmArgs g, uint16_t* out, float* part, hipStream_t s) {
  g.products = 1;
  const ProductShape shape = split_shape(g.M, g.N, g.K, g.segments);
  g.splits = shape.splits;
  if (g.splits == 1) return launch_product<AK, BK, false, false>(g, shape.tile, StoreBf16{{out, nullptr, nullptr}}, s);
  const hipError_t e = launch_product<AK, BK, false, false>(g, shape.tile, StorePart{part}, s);
  return e != hipSuccess ? e : launch_join_parts(part, out, true, g.splits, (long long)g.M * g.N, s);
}

}  // namespace

size_t gated_part_bytes(int T, int d, int d_ff, int segments) {
  if (T <= kGatedFewTokens) return gated_few_part_bytes(T, d, d_ff, segments);
  const int s = split_shape(T, d, d_ff, segments).splits;
  return s > 1 ? (size_t)s * T * d * sizeof(float) : 0;
}

hipError_t launch_gated_forward(const GatedLayer& L, const uint16_t* x, int T, uint16_t* y, const GatedKept& kept, float* part,
                                hipStream_t s) {
  if (T <= kGatedFewTokens) return launch_gated_few(L, x, T, y, kept, part, s);
  GemmArgs up{};
  up.a[0] = x, up.b[0] = L.wg, up.b[1] = L.wu;
  up.M = T, up.N = L.d_ff, up.K = L.d, up.lda = up.ldb = 2u * L.d;
  up.segments = up.products = up.splits = 1;
  const hipError_t e = with_activation(L.act, [&](auto act) {
    return launch_product<true, true, true, false>(up, product_shape(T, 2 * L.d_ff, k_steps(L.d), 1, 1).tile, StoreGated<decltype(act)::value>{kept}, s);
  });
  if (e != hipSuccess) return e;
  GemmArgs down{};
  down.a[0] = kept.h, down.b[0] = L.w2u;
  down.M = T, down.N = L.d, down.K = L.d_ff, down.lda = 2u * L.d_ff, down.ldb = 2u * L.d;
  down.segments = 1;
  return launch_split_product<true, false>(down, y, part, s);
}

hipError_t launch_gated_backward(const GatedLayer& L, const uint16_t* x, int T, const GatedKept& kept, const uint16_t* dy,
                                 uint16_t* dx, uint16_t* dwg, uint16_t* dwu, uint16_t* dw2u, uint16_t* dg, uint16_t* du,
                                 float* part, hipStream_t s) {
  hipError_t e = hipSuccess;
  const bool few = T <= kGatedFewTokens;
  if (few && (dx || dwg || dwu)) {
    e = launch_gated_few_slopes(L, dy, T, kept, dg, du, s);
    if (e != hipSuccess) return e;
  } else if (dx || dwg || dwu) {
    GemmArgs a{};
    a.a[0] = dy, a.b[0] = L.w2u;
    a.M = T, a.N = L.d_ff, a.K = L.d, a.lda = a.ldb = 2u * L.d;
    a.segments = a.products = a.splits = 1;
    e = with_activation(L.act, [&](auto act) {
      return launch_product<true, true, false, false>(a, product_shape(T, L.d_ff, k_steps(L.d), 1, 1).tile, StoreGateSlopes<decltype(act)::value>{kept, dg, du}, s);
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
  add(kept.h, dy, dw2u);
  if (w.products > 0) {
    w.M = L.d_ff, w.N = L.d, w.K = T, w.lda = 2u * L.d_ff, w.ldb = 2u * L.d;
    w.segments = w.splits = 1;
    e = launch_product<false, false, false, false>(w, product_shape(L.d_ff, L.d, k_steps(T), w.products, 1).tile, out, s);
    if (e != hipSuccess) return e;
  }
  if (dx && few) return launch_gated_few_dx(L, T, dg, du, dx, part, s);
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
