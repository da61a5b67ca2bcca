// The dense gated FFN, forward and backward, for any number of tokens.
#include "gated.h"

namespace hire {
namespace {

// h = a(g) u.
template <int ACT>
struct StoreGated {
  GatedKept kept;
  template <int MB, int NB>
  __device__ __forceinline__ void store(const f32x16v (&acc)[MB][NB], char* smem, int m0, int n0, int M, int N, int, int) const {
    for_rows<true>(acc, smem, m0, n0, M, N, NoFetch{}, [&](int m, int n, const float (&v)[2][8], int) {
      store_gated<ACT>(kept, (size_t)m * N + n, v[0], v[1]);
    });
  }
};
// The sums are dh.
template <int ACT>
struct StoreGateSlopes {
  GatedKept kept;
  uint16_t *dg, *du;
  template <int MB, int NB>
  __device__ __forceinline__ void store(const f32x16v (&acc)[MB][NB], char* smem, int m0, int n0, int M, int N, int, int) const {
    auto fetch = [&](int m, int n) { return load_kept(kept, (size_t)m * N + n); };
    for_rows<false>(acc, smem, m0, n0, M, N, fetch, [&](int m, int n, const float (&v)[1][8], const KeptEight& k) {
      store_slopes<ACT>(k, v[0], dg + (size_t)m * N + n, du + (size_t)m * N + n);
    });
  }
};
constexpr int kMostSplits = 32;
int k_steps(int k) { return (k + kGemmStep - 1) / kGemmStep; }
ProductShape up_shape(int T, int d, int d_ff) { return product_shape(T, 2 * d_ff, k_steps(d), 1, kMostSplits); }
ProductShape slopes_shape(int T, int d, int d_ff) { return product_shape(T, d_ff, k_steps(d), 1, kMostSplits); }
ProductShape weights_shape(int T, int d, int d_ff, int products) {
  return product_shape(d_ff, d, k_steps(T), products, kMostSplits);
}
ProductShape units_shape(int T, int d, int d_ff, int segments) {
  return product_shape(T, d, segments * k_steps(d_ff), 1, kMostSplits);
}
size_t split_bytes(const ProductShape& shape, size_t values) { return shape.splits > 1 ? shape.splits * values * sizeof(float) : 0; }

// Up to three products of one shape with bf16 results, split over k where their tiles are few.
template <bool AK, bool BK, bool STREAMING>
hipError_t launch_split_products(GemmArgs g, const ProductShape& shape, const StoreBf16<STREAMING>& out, float* part, hipStream_t s) {
  g.splits = shape.splits;
  if (g.splits == 1) return launch_product<AK, BK, false, false>(g, shape.tile, out, s);
  const hipError_t e = launch_product<AK, BK, false, false>(g, shape.tile, StorePart<false>{part, g.splits}, s);
  if (e != hipSuccess) return e;
  return launch_join_products(part, JoinOutputs{{out.c[0], out.c[1], out.c[2]}}, g.products, true, g.splits,
                              (long long)g.M * g.N, s);
}

}  // namespace

size_t gated_forward_part_bytes(int T, int d, int d_ff) {
  if (T <= kGatedFewTokens) return gated_few_part_bytes(T, d, d_ff, 1);
  const size_t up = split_bytes(up_shape(T, d, d_ff), 2 * (size_t)T * d_ff);
  const size_t down = split_bytes(units_shape(T, d, d_ff, 1), (size_t)T * d);
  return up > down ? up : down;
}

size_t gated_backward_part_bytes(int T, int d, int d_ff) {
  const bool few = T <= kGatedFewTokens;
  size_t weights = 0;
  for (int products = 1; products <= 3 && !few; ++products) {
    const size_t bytes = split_bytes(weights_shape(T, d, d_ff, products), products * (size_t)d_ff * d);
    if (bytes > weights) weights = bytes;
  }
  const size_t slopes = few ? 0 : split_bytes(slopes_shape(T, d, d_ff), (size_t)T * d_ff);
  const size_t dx = few ? gated_few_part_bytes(T, d, d_ff, 2) : split_bytes(units_shape(T, d, d_ff, 2), (size_t)T * d);
  const size_t most = weights > slopes ? weights : slopes;
  return most > dx ? most : dx;
}

hipError_t launch_gated_forward(const GatedLayer& L, const uint16_t* x, int T, uint16_t* y, const GatedKept& kept, float* part,
                                hipStream_t s) {
  if (T <= kGatedFewTokens) return launch_gated_few(L, x, T, y, kept, part, s);
  GemmArgs up{};
  up.a[0] = x, up.b[0] = L.wg, up.b[1] = L.wu;
  up.M = T, up.N = L.d_ff, up.K = L.d, up.lda = up.ldb = 2u * L.d;
  up.segments = up.products = 1;
  const ProductShape shape = up_shape(T, L.d, L.d_ff);
  up.splits = shape.splits;
  const long long units = (long long)T * L.d_ff;
  hipError_t e = hipSuccess;
  if (shape.splits > 1) e = launch_product<true, true, true, false>(up, shape.tile, StorePart<true>{part, shape.splits}, s);
  if (e != hipSuccess) return e;
  e = with_activation(L.act, [&](auto act) {
    constexpr int ACT = decltype(act)::value;
    if (shape.splits > 1)
      return launch(&k_join_gated<ACT>, dim3(join_blocks(units / 8)), dim3(256), 0, s, part, shape.splits, units, kept);
    return launch_product<true, true, true, false>(up, shape.tile, StoreGated<ACT>{kept}, s);
  });
  if (e != hipSuccess) return e;
  GemmArgs down{};
  down.a[0] = kept.h, down.b[0] = L.w2u;
  down.M = T, down.N = L.d, down.K = L.d_ff, down.lda = 2u * L.d_ff, down.ldb = 2u * L.d;
  down.segments = down.products = 1;
  return launch_split_products<true, false>(down, units_shape(T, L.d, L.d_ff, 1), StoreBf16<false>{{y, nullptr, nullptr}}, part, s);
}

hipError_t launch_gated_backward(const GatedLayer& L, const uint16_t* x, int T, const GatedKept& kept, const uint16_t* dy,
                                 uint16_t* dx, uint16_t* dwg, uint16_t* dwu, uint16_t* dw2u, const GatedSlopes& slopes, float* part,
                                 hipStream_t s) {
  uint16_t *const dg = slopes.dg, *const du = slopes.du;
  hipError_t e = hipSuccess;
  const bool few = T <= kGatedFewTokens;
  if (few && (dx || dwg || dwu)) {
    e = launch_gated_few_slopes(L, dy, T, kept, slopes, part, s);
  } else if (dx || dwg || dwu) {
    GemmArgs a{};
    a.a[0] = dy, a.b[0] = L.w2u;
    a.M = T, a.N = L.d_ff, a.K = L.d, a.lda = a.ldb = 2u * L.d;
    a.segments = a.products = 1;
    const ProductShape shape = slopes_shape(T, L.d, L.d_ff);
    a.splits = shape.splits;
    const long long units = (long long)T * L.d_ff;
    if (shape.splits > 1) e = launch_product<true, true, false, false>(a, shape.tile, StorePart<false>{part, shape.splits}, s);
    if (e != hipSuccess) return e;
    e = with_activation(L.act, [&](auto act) {
      constexpr int ACT = decltype(act)::value;
      if (shape.splits > 1)
        return launch(&k_join_slopes<ACT>, dim3(join_blocks(units / 8)), dim3(256), 0, s, part, shape.splits, units, kept, dg, du);
      return launch_product<true, true, false, false>(a, shape.tile, StoreGateSlopes<ACT>{kept, dg, du}, s);
    });
  } else if (slopes.h_rest) {
    e = launch_gated_rest(L, T, kept, slopes.h_rest, s);
  }
  if (e != hipSuccess) return e;
  GemmArgs w{};
  GatedRests rest{};
  StoreBf16<true> out{};
  auto add = [&](const uint16_t* a, const uint16_t* a_rest, const uint16_t* b, uint16_t* c) {
    if (c) w.a[w.products] = a, rest.of[w.products] = a_rest, w.b[w.products] = b, out.c[w.products++] = c;
  };
  add(dg, slopes.dg_rest, x, dwg);
  add(du, slopes.du_rest, x, dwu);
  add(kept.h, slopes.h_rest, dy, dw2u);
  if (w.products > 0) {
    w.M = L.d_ff, w.N = L.d, w.K = T, w.lda = 2u * L.d_ff, w.ldb = 2u * L.d;
    w.segments = w.splits = 1;
    e = few ? launch_gated_few_weights(w, rest, out, s)
            : launch_split_products<false, false>(w, weights_shape(T, L.d, L.d_ff, w.products), out, part, s);
    if (e != hipSuccess) return e;
  }
  if (dx && few) return launch_gated_few_dx(L, T, slopes, dx, part, s);
  if (dx) {
    GemmArgs a{};
    a.a[0] = dg, a.a[1] = du, a.b[0] = L.wg, a.b[1] = L.wu;
    a.M = T, a.N = L.d, a.K = L.d_ff, a.lda = 2u * L.d_ff, a.ldb = 2u * L.d;
    a.segments = 2, a.products = 1;
    e = launch_split_products<true, false>(a, units_shape(T, L.d, L.d_ff, 2), StoreBf16<false>{{dx, nullptr, nullptr}}, part, s);
  }
  return e;
}

}  // namespace hire
