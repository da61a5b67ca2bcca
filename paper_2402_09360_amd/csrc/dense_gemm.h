// Products of bf16 matrices on the matrix cores with a fused epilogue: C[m, n] = sum_k A[m, k] B[n, k], fp32 sums.
// Either operand may lie k-contiguous ("k-major": row m or n is one run of k) or the other way round (row k is one run of m
// or n), so that the products of a layer's forward and backward pass read every matrix as it is stored.
#pragma once

#include "device_utils.h"

namespace hire {

typedef float f32x4v __attribute__((ext_vector_type(4)));
typedef float f32x16v __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4v __attribute__((ext_vector_type(4)));
typedef short s16x4v __attribute__((ext_vector_type(4)));

constexpr int kGemmStep = 64;  // k of one stage: 128 bytes of a k-major row

// What loads of a stage that lie behind the end of k read instead.
__device__ __align__(16) const uint32_t kGemmZeros[4] = {0u, 0u, 0u, 0u};

__device__ __forceinline__ uint32_t gemm_lds_offset(const void* p) {
  return (uint32_t)(uintptr_t)(__attribute__((address_space(3))) const void*)p;
}
// Asynchronous load of 16 bytes per lane into LDS, lane l's to lds + 16 l (uniform).  Not tracked by the compiler: the
// barriers of the loop wait for it.
__device__ __forceinline__ void gemm_load(const char* base, uint32_t off, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %2\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(off), "s"(base), "s"(lds) : "memory", "m0");
}
__device__ __forceinline__ void gemm_load_at(const void* address, uint32_t lds) {
  asm volatile("s_mov_b32 m0, %1\n\ts_nop 0\n\tglobal_load_lds_dwordx4 %0, off" ::"v"(address), "s"(lds) : "memory", "m0");
}

__device__ __forceinline__ uint32_t bf16_pair(float lo, float hi) {
  const __bf16 v[2] = {(__bf16)lo, (__bf16)hi};  // nearest even
  uint32_t u;
  __builtin_memcpy(&u, v, 4);
  return u;
}

// One operand's tile of ROWS m (or n) by kGemmStep k in LDS.
//   k-major:  [row][128 bytes]; the 16-byte chunk c of row r lies at c ^ (r & 7), so that the rows of a fragment, read at one
//             chunk, are spread over all banks.
//   else:     [k][2 ROWS bytes]; the 32-byte unit u of row k lies at u ^ f(k), f taking its values from the bits of k in which
//             the rows of one transposing read differ.
// The loads write LDS in order, so the permutation is in the global address.
// PAIR: rows of two matrices in turn, 32 of the first, 32 of the second (the same rows).
template <int ROWS, int WAVES, bool KMAJOR, bool PAIR>
struct GemmTile {
  static constexpr int kLoads = ROWS * 2 * kGemmStep / (WAVES * 1024);
  static constexpr int kUnits = ROWS / 16;  // 32-byte units of a row of k
  static constexpr int kBytes = ROWS * 2 * kGemmStep;
  static_assert(ROWS % 64 == 0 && kLoads * WAVES * 1024 == kBytes, "whole loads");
  uint32_t off[kLoads];

  static __device__ __forceinline__ int f_of_k(int k) { return ((k & 3) | (((k >> 3) & 3) << 2)) & (kUnits - 1); }

  // origin: first row of the tile inside a matrix of `extent` rows (PAIR: counts one of the two); ld in bytes.
  __device__ __forceinline__ void init(int origin, int extent, uint32_t ld) {
    const int wave = wave_id(), lane = lane_id();
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int at = i * WAVES + wave;  // 1 KB pieces of the tile
      if constexpr (KMAJOR) {
        int r = at * 8 + lane / 8;
        if constexpr (PAIR) r = r / 64 * 32 + r % 32;
        r = min(r, extent - 1 - origin);
        off[i] = (uint32_t)r * ld + (uint32_t)(((lane & 7) ^ (lane >> 3)) * 16);
      } else {
        constexpr int kLanes = ROWS / 8;  // lanes of a row
        const int k = at * (64 / kLanes) + lane / kLanes, pos = lane % kLanes;
        int chunk = (((pos >> 1) ^ f_of_k(k)) << 1) | (pos & 1);
        chunk = min(chunk, (extent - 1 - origin) / 8);
        off[i] = (uint32_t)k * ld + (uint32_t)(chunk * 16);
      }
    }
  }
  // Loads one stage; base: where the tile's first row and k lie (second: of the second matrix, PAIR); left: k from there on.
  __device__ __forceinline__ void load(const char* base, const char* second, int left, uint32_t lds) const {
    const int wave = __builtin_amdgcn_readfirstlane(wave_id()), lane = lane_id();
    if (left >= kGemmStep) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int at = i * WAVES + wave;
        gemm_load(PAIR && ((at * 8 / 32) & 1) ? second : base, off[i], lds + at * 1024);
      }
    } else {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int at = i * WAVES + wave;
        const char* b = PAIR && ((at * 8 / 32) & 1) ? second : base;
        const int k = KMAJOR ? ((lane & 7) ^ (lane >> 3)) * 8 : at * (64 / (ROWS / 8)) + lane / (ROWS / 8);
        gemm_load_at(k < left ? (const void*)(b + off[i]) : (const void*)kGemmZeros, lds + at * 1024);
      }
    }
  }
  // Eight k (16 ks + 8 (lane / 32) ...) of row `row` + lane % 32 of the tile at `lds` (byte offset).
  static __device__ __forceinline__ bf16x8v fragment(const char* tile, int row, int ks) {
    const int lane = lane_id();
    if constexpr (KMAJOR) {
      const int r = row + (lane & 31), chunk = 2 * ks + (lane >> 5);
      return *reinterpret_cast<const bf16x8v*>(tile + r * 128 + ((chunk ^ (r & 7)) << 4));
    } else {
      // sixteen lanes read four rows of k by sixteen columns and get four k of one column each
      const int k = 16 * ks + 8 * (lane >> 5) + ((lane & 15) >> 2), unit = row / 16 + ((lane >> 4) & 1);
      const char* p = tile + k * (2 * ROWS) + ((unit ^ f_of_k(k)) << 5) + ((lane & 3) << 3);
      const char* q = tile + (k + 4) * (2 * ROWS) + ((unit ^ f_of_k(k + 4)) << 5) + ((lane & 3) << 3);
      using Lds = __attribute__((address_space(3))) s16x4v*;
      const s16x4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)p), hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)q);
      bf16x8v v;
      __builtin_memcpy(&v, &lo, 8);
      __builtin_memcpy(reinterpret_cast<char*>(&v) + 8, &hi, 8);
      return v;
    }
  }
};

struct GemmArgs {
  const void* a[3];  // by segment of k, or by product
  const void* b[3];  // likewise; PAIR: the two matrices
  int M, N, K;       // N counts units with PAIR; K of one segment
  uint32_t lda, ldb; // bytes
  int segments;      // > 1: k runs over a[0] b[0], then a[1] b[1], ...
  int products;      // > 1: so many products of one shape
  int splits;        // parts of k, whose sums the epilogue gets apart
};

// Place of workgroup `w` of `total`: consecutive places on one die (workgroups go to the eight dies in turn), so that the
// tiles that share operands share an L2.
__device__ __forceinline__ int gemm_place(int w, int total) {
  const int die = w & 7, each = total >> 3, rest = total & 7;
  return die * each + min(die, rest) + (w >> 3);
}

// The tile of MT x NT by MW x NW waves; two stages in LDS: while one is multiplied the next one is on its way.
// An epilogue gets a wave's sums: acc[i][j], rows m of block i at lane % 32, columns n of block j: register r is column
// 8 (r / 4) + 4 (lane / 32) + r % 4.
template <int MT, int NT, int MW, int NW, bool AK, bool BK, bool PAIR, class Epilogue>
__global__ __launch_bounds__(64 * MW * NW) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_dense_product(GemmArgs g, Epilogue epi) {
  constexpr int kWaves = MW * NW, kMB = MT / MW / 32, kNB = NT / NW / 32;
  using TA = GemmTile<MT, kWaves, AK, false>;
  using TB = GemmTile<NT, kWaves, BK, PAIR>;
  constexpr int kStage = TA::kBytes + TB::kBytes;
  __shared__ __align__(1024) char smem[2 * kStage];

  const int n_tile = PAIR ? NT / 2 : NT;
  const int tiles_m = (g.M + MT - 1) / MT, tiles_n = (g.N + n_tile - 1) / n_tile, tiles = tiles_m * tiles_n;
  const int w = gemm_place((int)blockIdx.x, (int)gridDim.x), z = w / tiles, t = w % tiles;
  const int product = z / g.splits, split = z % g.splits;
  // groups of eight tiles of m, so that the 32 workgroups of a die form a patch
  const int group = t / (8 * tiles_n), in = t % (8 * tiles_n), gm = min(8, tiles_m - 8 * group);
  const int m0 = (8 * group + in % gm) * MT, n0 = in / gm * n_tile;

  const int seg_steps = (g.K + kGemmStep - 1) / kGemmStep, steps = seg_steps * g.segments;
  const int s0 = (int)((long long)steps * split / g.splits), s1 = (int)((long long)steps * (split + 1) / g.splits);

  TA ta;
  TB tb;
  ta.init(m0, g.M, g.lda);
  tb.init(n0, g.N, g.ldb);
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(gemm_lds_offset(smem));
  auto request = [&](int s) {
    const int seg = s / seg_steps, k = (s - seg * seg_steps) * kGemmStep, left = g.K - k;
    const int which = g.segments > 1 ? seg : product;
    const size_t ka = AK ? (size_t)m0 * g.lda + 2 * (size_t)k : (size_t)k * g.lda + 2 * (size_t)m0;
    const size_t kb = BK ? (size_t)n0 * g.ldb + 2 * (size_t)k : (size_t)k * g.ldb + 2 * (size_t)n0;
    const uint32_t lds = lds0 + (uint32_t)((s - s0) & 1) * kStage;
    ta.load(static_cast<const char*>(g.a[which]) + ka, nullptr, left, lds);
    if constexpr (PAIR)
      tb.load(static_cast<const char*>(g.b[0]) + kb, static_cast<const char*>(g.b[1]) + kb, left, lds + TA::kBytes);
    else
      tb.load(static_cast<const char*>(g.b[which]) + kb, nullptr, left, lds + TA::kBytes);
  };

  const int wave = wave_id(), wm = wave / NW * (MT / MW), wn = wave % NW * (NT / NW);
  f32x16v acc[kMB][kNB] = {};
  if (s0 < s1) request(s0);
  for (int s = s0; s < s1; ++s) {
    // this stage has arrived for every wave, and nobody reads the other one any more
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    if (s + 1 < s1) request(s + 1);
    const char* sa = smem + ((s - s0) & 1) * kStage;
    const char* sb = sa + TA::kBytes;
#pragma unroll
    for (int ks = 0; ks < kGemmStep / 16; ++ks) {
      bf16x8v fa[kMB], fb[kNB];
#pragma unroll
      for (int i = 0; i < kMB; ++i) fa[i] = TA::fragment(sa, wm + 32 * i, ks);
#pragma unroll
      for (int j = 0; j < kNB; ++j) fb[j] = TB::fragment(sb, wn + 32 * j, ks);
#pragma unroll
      for (int i = 0; i < kMB; ++i)
#pragma unroll
        for (int j = 0; j < kNB; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[j], fa[i], acc[i][j], 0, 0, 0);
    }
  }
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // LDS is the epilogue's
  epi.store(acc, smem, m0 + wm, n0 + (PAIR ? wn / 2 : wn), g.M, g.N, product, split);
}

}  // namespace hire
