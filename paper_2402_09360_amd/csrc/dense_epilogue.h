// What follows the sums of a dense product: rows out of the matrix instruction's layout, stores, parts of k and their join, and
// the launch.
#pragma once

#include "dense_gemm.h"
#include "kernels.h"

namespace hire {

__device__ __forceinline__ uint2 pack4(const float (&f)[4]) { return make_uint2(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3])); }
__device__ __forceinline__ uint4 pack8(const float (&f)[8]) {
  return make_uint4(bf16_pair(f[0], f[1]), bf16_pair(f[2], f[3]), bf16_pair(f[4], f[5]), bf16_pair(f[6], f[7]));
}

// A wave's sums in rows: one block of 32 rows after the other goes through LDS (a place per wave, fp32), from where a lane gets
// eight neighbouring columns of every one of NB blocks that share their columns (PAIRED: all of them), or of one.  Straight
// from the matrix instruction's layout a lane has four columns of a row: with 8-byte accesses, 32 rows each, the product
// behind dy took 740 us instead of the 200 of its arithmetic (4096 tokens of d = 2048, 16384 units).
constexpr int kRowFloats = 68;  // 64 columns and a gap that moves the rows over the banks

// f(row m, column n of the first of eight, values, fetched): values[8] of a block column, or [2][8] of both (PAIRED).
// fetch(m, n): what an epilogue reads from memory for these eight, asked for a block of 32 rows ahead; for rows and columns that
// are not there at the last ones.
struct NoFetch {
  __device__ __forceinline__ int operator()(int, int) const { return 0; }
};
template <bool PAIRED, int MB, int NB, typename Fetch, typename F>
__device__ __forceinline__ void for_rows(const f32x16v (&acc)[MB][NB], char* smem, int m0, int n0, int M, int N, Fetch fetch, F f) {
  static_assert(NB == 2, "64 columns");
  const int lane = lane_id();
  float* tile = reinterpret_cast<float*>(smem) + wave_id() * 32 * kRowFloats;
  constexpr int kLanes = PAIRED ? 4 : 8, kPasses = 32 * kLanes / 64;  // lanes of a row
  const int col = lane % kLanes * 8, row = lane / kLanes;
  using Fetched = decltype(fetch(0, 0));
  Fetched here[kPasses], ahead[kPasses];
  auto request = [&](int i, Fetched (&to)[kPasses]) __attribute__((always_inline)) {
#pragma unroll
    for (int r = 0; r < kPasses; ++r) to[r] = fetch(min(m0 + 32 * i + r * (64 / kLanes) + row, M - 1), min(n0 + col, N - 8));
  };
  request(0, ahead);
#pragma unroll
  for (int i = 0; i < MB; ++i) {
#pragma unroll
    for (int r = 0; r < kPasses; ++r) here[r] = ahead[r];
    if (i + 1 < MB) request(i + 1, ahead);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");  // the wave's own reads of the block before
#pragma unroll
    for (int j = 0; j < NB; ++j)
#pragma unroll
      for (int q = 0; q < 4; ++q)
        *reinterpret_cast<float4*>(tile + (lane & 31) * kRowFloats + 32 * j + 8 * q + 4 * (lane >> 5)) =
            make_float4(acc[i][j][4 * q], acc[i][j][4 * q + 1], acc[i][j][4 * q + 2], acc[i][j][4 * q + 3]);
    asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
#pragma unroll
    for (int pass = 0; pass < kPasses; ++pass) {
      const int r = pass * (64 / kLanes) + row, m = m0 + 32 * i + r, n = n0 + col;
      float v[PAIRED ? 2 : 1][8];
#pragma unroll
      for (int j = 0; j < (PAIRED ? 2 : 1); ++j) {
        *reinterpret_cast<float4*>(&v[j][0]) = *reinterpret_cast<const float4*>(tile + r * kRowFloats + 32 * j + col);
        *reinterpret_cast<float4*>(&v[j][4]) = *reinterpret_cast<const float4*>(tile + r * kRowFloats + 32 * j + col + 4);
      }
      if (m < M && n < N) f(m, n, v, here[pass]);
    }
  }
}

// fp32 sums of one part of k; N a multiple of 8.  In order: products, parts, both matrices (PAIRED), rows.
template <bool PAIRED>
struct StorePart {
  float* part;
  int splits;
  template <int MB, int NB>
  __device__ __forceinline__ void store(const f32x16v (&acc)[MB][NB], char* smem, int m0, int n0, int M, int N, int product,
                                        int split) const {
    constexpr int kMatrices = PAIRED ? 2 : 1;
    float* mine = part + (size_t)(product * splits + split) * kMatrices * M * N;
    for_rows<PAIRED>(acc, smem, m0, n0, M, N, NoFetch{}, [&](int m, int n, const float (&v)[kMatrices][8], int) {
#pragma unroll
      for (int j = 0; j < kMatrices; ++j) {
        float4* to = reinterpret_cast<float4*>(mine + ((size_t)j * M + m) * N + n);
        to[0] = make_float4(v[j][0], v[j][1], v[j][2], v[j][3]);
        to[1] = make_float4(v[j][4], v[j][5], v[j][6], v[j][7]);
      }
    });
  }
};
// Eight values of a plane, added over the parts in their order; `stride` values from part to part.
__device__ __forceinline__ void join_eight(const float* part, int parts, size_t stride, float (&v)[8]) {
  const float4 a = reinterpret_cast<const float4*>(part)[0], b = reinterpret_cast<const float4*>(part)[1];
  v[0] = a.x, v[1] = a.y, v[2] = a.z, v[3] = a.w, v[4] = b.x, v[5] = b.y, v[6] = b.z, v[7] = b.w;
#pragma unroll 4
  for (int r = 1; r < parts; ++r) {
    const float4* p = reinterpret_cast<const float4*>(part + r * stride);
    const float4 c = p[0], d = p[1];
    v[0] += c.x, v[1] += c.y, v[2] += c.z, v[3] += c.w, v[4] += d.x, v[5] += d.y, v[6] += d.z, v[7] += d.w;
  }
}
inline unsigned join_blocks(long long threads) {
  const long long blocks = (threads + 255) / 256;
  return (unsigned)(blocks < 4096 ? blocks : 4096);
}

// Sum of the parts in their order, rounded once to bf16 or left in fp32, of products blockIdx.y; values beyond whole fours
// one by one.
struct JoinOutputs {
  void* out[3];
};
template <bool BF16>
__global__ __launch_bounds__(256) void k_join_parts(const float* __restrict__ part, JoinOutputs outputs, int parts,
                                                    long long values) {
  void* out = outputs.out[blockIdx.y];
  part += (size_t)blockIdx.y * parts * values;
  if (values % 4 != 0) {
    for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < values; i += (long long)gridDim.x * 256) {
      float s = part[i];
#pragma unroll 8
      for (int r = 1; r < parts; ++r) s += part[(size_t)r * values + i];
      if constexpr (BF16)
        static_cast<__bf16*>(out)[i] = (__bf16)s;
      else
        static_cast<float*>(out)[i] = s;
    }
    return;
  }
  const long long quads = values / 4;
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < quads; i += (long long)gridDim.x * 256) {
    const float4* p = reinterpret_cast<const float4*>(part) + i;
    float4 s = p[0];
#pragma unroll 8
    for (int r = 1; r < parts; ++r) {
      const float4 v = p[(size_t)r * quads];
      s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
    }
    if constexpr (BF16) {
      const float f[4] = {s.x, s.y, s.z, s.w};
      static_cast<uint2*>(out)[i] = pack4(f);
    } else {
      static_cast<float4*>(out)[i] = s;
    }
  }
}
inline hipError_t launch_join_products(const float* part, const JoinOutputs& out, int products, bool bf16, int parts,
                                       long long values, hipStream_t s) {
  return launch(bf16 ? &k_join_parts<true> : &k_join_parts<false>, dim3(join_blocks(values / 4 + 1), (unsigned)products), dim3(256),
                0, s, part, out, parts, values);
}
inline hipError_t launch_join_parts(const float* part, void* out, bool bf16, int parts, long long values, hipStream_t s) {
  return launch_join_products(part, JoinOutputs{{out, nullptr, nullptr}}, 1, bf16, parts, values, s);
}

// How a product is cut up: the tile and the parts of k.  In units of a 256 x 256 x 32 stage (about 0.45 us): a tile of 256 takes
// a compute unit, of 128 half of one, which then yields 0.7 of the rate, or 0.4 of it where it has the unit for itself and waits
// for memory; a round of tiles has about eight stages' worth of start and epilogue; parts are written and read again, from
// caches for the most part (8 TB/s), and their join is a kernel (8).  Forward and backward pass, us with no parts of the first
// layer's products and the weights' gradients / with parts: 128 tokens of d = 4096, 4096 units 63 / 46, 101 / 77; 500, 4096, 512
// 57 / 32, 75 / 44; 8192, 512, 2048 84 / 78, 189 / 160; 8192, 256, 512 24 / 23, 117 / 50.  Every other choice of one product's
// tile and parts was timed for 15 such sizes: at most 4 % of a pass better.
struct ProductShape {
  int tile, splits;
};
inline ProductShape product_shape(int M, int N, int steps, int products, int most_splits) {
  ProductShape best{256, 1};
  double least = 0.0;
  for (int tile = 256; tile >= 128; tile /= 2)
    for (int splits = 1; splits <= most_splits; ++splits) {
      if (splits > 1 && steps / splits < 8) break;
      const double tiles = (double)((M + tile - 1) / tile) * ((N + tile - 1) / tile) * products * splits;
      const double slots = tile == 256 ? 256.0 : 512.0, rounds = (double)(long long)((tiles + slots - 1.0) / slots);
      const double stage = tile == 256 ? 1.0 : (tiles <= 256.0 ? 0.6 : 0.72);
      double cost = rounds * (((steps + splits - 1) / splits) * stage + 8.0);
      if (splits > 1) cost += 8.0 + 8.0 * splits * products * M * N / 8e6 / 0.45;
      if (least == 0.0 || cost < least) least = cost, best = ProductShape{tile, splits};
    }
  return best;
}

template <bool AK, bool BK, bool PAIR, bool MX, class Epilogue>
hipError_t launch_product(const GemmArgs& g, int tile, const Epilogue& epi, hipStream_t s) {
  const int n_tile = PAIR ? tile / 2 : tile;
  const long long tiles = (long long)((g.M + tile - 1) / tile) * ((g.N + n_tile - 1) / n_tile);
  return launch(tile == 256 ? &k_dense_product<256, AK, BK, PAIR, MX, Epilogue> : &k_dense_product<128, AK, BK, PAIR, MX, Epilogue>,
                dim3((unsigned)(tiles * g.products * g.splits)), dim3((unsigned)(2 * tile)), 0, s, g, epi);
}

}  // namespace hire
