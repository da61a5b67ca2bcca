// Products of bf16 matrices on the matrix cores with a fused epilogue: C[m, n] = sum_k A[m, k] B[n, k], fp32 sums.
// Either operand may lie k-contiguous ("k-major": row m or n is one run of k) or the other way round (row k is one run of m
// or n), so that the products of a layer's forward and backward pass read every matrix as it is stored.
#pragma once

#include "device_utils.h"

#include <type_traits>

namespace hire {

typedef float f32x4v __attribute__((ext_vector_type(4)));
typedef float f32x16v __attribute__((ext_vector_type(16)));
typedef __bf16 bf16x8v __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x4v __attribute__((ext_vector_type(4)));
typedef short s16x4v __attribute__((ext_vector_type(4)));

constexpr int kGemmStep = 32;    // k of one stage: 64 bytes of a k-major row
constexpr int kGemmStages = 4;   // in LDS: three on their way or there while one is multiplied

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
//   k-major:  [row][64 bytes]; the 16-byte chunk c of row r lies at c ^ (r / 4 % 4), so that the sixteen rows that a cycle
//             reads at one chunk are spread over all banks.
//   else:     [k][2 ROWS bytes]; the 32-byte unit u of row k lies at u ^ 2 (k % 4): half a wave reads four rows of k by two
//             units.
// The loads write LDS in order, so the permutation is in the global address.
// PAIR: rows of two matrices in turn, 32 of the first, 32 of the second (the same rows).
template <int ROWS, int WAVES, bool KMAJOR, bool PAIR>
struct GemmTile {
  static constexpr int kBytes = ROWS * 2 * kGemmStep;
  static constexpr int kLoads = kBytes / (WAVES * 1024);
  static constexpr int kUnits = ROWS / 16;  // 32-byte units of a row of k
  static_assert(ROWS % 128 == 0 && kLoads * WAVES * 1024 == kBytes, "whole loads");
  uint32_t off[kLoads];

  static __device__ __forceinline__ int unit_of_k(int k) { return (k & 3) << 1; }
  // The piece (1 KB) of the tile that load i of a wave fills; what of k a lane's 16 bytes of it are.
  static __device__ __forceinline__ int k_of_lane(int piece) {
    const int lane = lane_id();
    return KMAJOR ? ((lane & 3) ^ ((lane >> 4) & 3)) * 8 : piece * (64 / (ROWS / 8)) + lane / (ROWS / 8);
  }
  static __device__ __forceinline__ bool second(int piece) { return PAIR && ((piece * 16 / 32) & 1) != 0; }

  // origin: first row of the tile inside a matrix of `extent` rows (PAIR: counts one of the two); ld in bytes.  Rows behind
  // the last one repeat it.
  __device__ __forceinline__ void init(int origin, int extent, uint32_t ld) {
    const int wave = wave_id(), lane = lane_id();
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      const int piece = i * WAVES + wave;
      if constexpr (KMAJOR) {
        int r = piece * 16 + lane / 4;
        if constexpr (PAIR) r = r / 64 * 32 + r % 32;
        r = min(r, extent - 1 - origin);
        off[i] = (uint32_t)r * ld + (uint32_t)(k_of_lane(piece) * 2);
      } else {
        const int k = k_of_lane(piece), pos = lane % (ROWS / 8);
        const int chunk = (((pos >> 1) ^ unit_of_k(k)) << 1) | (pos & 1);
        off[i] = (uint32_t)k * ld + (uint32_t)(min(chunk, (extent - 1 - origin) / 8) * 16);
      }
    }
  }
  // Requests one stage; base: where the tile's first row and k lie (other: of the second matrix, PAIR); left: k from there on.
  __device__ __forceinline__ void request(const char* base, const char* other, int left, uint32_t lds, int wave) const {
    if (left >= kGemmStep) {
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int piece = i * WAVES + wave;
        gemm_load(second(piece) ? other : base, off[i], lds + piece * 1024);
      }
    } else {  // the last stage of k
#pragma unroll
      for (int i = 0; i < kLoads; ++i) {
        const int piece = i * WAVES + wave;
        const char* b = second(piece) ? other : base;
        gemm_load_at(k_of_lane(piece) < left ? (const void*)(b + off[i]) : (const void*)kGemmZeros, lds + piece * 1024);
      }
    }
  }
  // Eight k (16 ks + 8 (lane / 32) ...) of row `row` + lane % 32 of the tile in LDS.
  static __device__ __forceinline__ bf16x8v fragment(const char* tile, int row, int ks) {
    const int lane = lane_id();
    if constexpr (KMAJOR) {
      const int r = row + (lane & 31), chunk = 2 * ks + (lane >> 5);
      return *reinterpret_cast<const bf16x8v*>(tile + r * 64 + ((chunk ^ ((r >> 2) & 3)) << 4));
    } else {
      // sixteen lanes read four rows of k by sixteen columns and get four k of one column each
      const int k = 16 * ks + 8 * (lane >> 5) + ((lane & 15) >> 2), unit = row / 16 + ((lane >> 4) & 1);
      const char* p = tile + k * (2 * ROWS) + ((unit ^ unit_of_k(k)) << 5) + ((lane & 3) << 3);
      using Lds = __attribute__((address_space(3))) s16x4v*;
      const s16x4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)p);
      const s16x4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(p + 4 * (2 * ROWS)));  // unit_of_k repeats every four
      bf16x8v v;
      __builtin_memcpy(&v, &lo, 8);
      __builtin_memcpy(reinterpret_cast<char*>(&v) + 8, &hi, 8);
      return v;
    }
  }
};

// A block of 32 codes as the matrix instruction takes it.
typedef int i32x8v __attribute__((ext_vector_type(8)));
__device__ __forceinline__ i32x8v mx_codes(const bf16x8v& block) {
  int d[4];
  __builtin_memcpy(d, &block, 16);
  return i32x8v{d[0], d[1], d[2], d[3], 0, 0, 0, 0};
}

struct GemmArgs {
  const void* a[3];  // by segment of k, or by product
  const void* b[3];  // likewise; PAIR: the two matrices
  int M, N, K;       // N counts units with PAIR; K of one segment
  uint32_t lda, ldb; // bytes
  int segments;      // > 1: k runs over a[0] b[0], then a[1] b[1], ...
  int products;      // > 1: so many products of one shape
  int splits;        // parts of k, whose sums the epilogue gets apart
  // microscaled operands only (a[0], b[0]: 4-bit codes, K in quarters of a column): scale bytes [M, scale_ld], [N, scale_ld],
  // scale_ld a multiple of 16 (bytes behind the last block: 127)
  const uint8_t *a_scales, *b_scales;
  uint32_t scale_ld;
};

// Place of workgroup `w` of `total`: consecutive places on one die (workgroups go to the eight dies in turn), so that the
// tiles that share operands share an L2.
__device__ __forceinline__ int gemm_place(int w, int total) {
  const int die = w & 7, each = total >> 3, rest = total & 7;
  return die * each + min(die, rest) + (w >> 3);
}

// Workgroup barriers that no instruction is moved across.
__device__ __forceinline__ void gemm_barrier() {
  __builtin_amdgcn_sched_barrier(0);
  __builtin_amdgcn_s_barrier();
  __builtin_amdgcn_sched_barrier(0);
}

// A tile of 256 x 256 by eight waves of 128 x 64, two on every SIMD.  The waves work in two groups half a stage apart: while one
// group's matrix instructions run, the other reads its fragments of a whole stage, requests the stage three ahead and waits;
// then they change places.  Per stage of 32 k a wave reads 12 KB of LDS and issues 16 matrix instructions of 32 cycles, so the
// reads of four waves (48 KB at 256 bytes a cycle) hide behind the others' 512 cycles.
//   Places in LDS: stage s lies in place s % 4.  The stage requested while s is read, s + 3, goes where s - 1 was, whose last
// reader is the second group one barrier earlier.  Before a wave passes the barrier behind its reads of stage s, its own loads
// of stage s + 1 have arrived (two younger stages may be on their way), and the group that reads s + 1 first does so behind a
// barrier that all waves passed with that wait done.
//   Measured against a double buffer of 64 k whose waves run freely (4096 x 4096 x 8192, normal values): 1019 -> 1222
// TFLOP/s; 79 % of the cycles are the matrix cores' (56 %), and with these values the clock drops to about 1.6 GHz: with
// zeros the same kernel does 1665.
//   With one group the only barrier of a stage is the one behind its reads: a wave that requests s + 3 has passed that of s - 1,
// in front of which every wave's reads of s - 1 were done.
// An epilogue gets a wave's sums: acc[i][j], rows m of block i at lane % 32, columns n of block j: register r is column
// 8 (r / 4) + 4 (lane / 32) + r % 4.
// MX: microscaled operands.  A stage's 64 bytes of a row are 128 columns, four blocks; every fourth stage brings the scale bytes
// of four, sixteen for each row of both tiles (a word per row and stage would touch as many lines as the codes do).  A lane's sixteen
// bytes of a fragment are one block, whose scale byte the matrix instruction picks from the row's word, shifted by a byte in the
// upper half of the wave.
// TILE 128, where there are too few tiles of 256 for the chip: four waves of 64 x 64 in one group; two workgroups of a compute unit
// fill each other's waits.
template <int TILE, bool AK, bool BK, bool PAIR, bool MX, class Epilogue>
__global__ __launch_bounds__(2 * TILE) __attribute__((amdgpu_waves_per_eu(2, 2))) void k_dense_product(GemmArgs g, Epilogue epi) {
  constexpr int kWaves = TILE / 32, kNW = TILE / 64, kMB = TILE / 64, kNB = 2;
  constexpr bool kGroups = TILE == 256;
  static_assert(TILE == 256 || TILE == 128, "two waves of m, the rest of n");
  using TA = GemmTile<TILE, kWaves, AK, false>;
  using TB = GemmTile<TILE, kWaves, BK, PAIR>;
  static_assert(!MX || (AK && BK && !PAIR), "rows of codes");
  constexpr int kCodes = TA::kBytes + TB::kBytes, kScales = MX ? 2 * TILE * 16 : 0, kStage = kCodes;
  // loads of the two younger stages; with scale bytes among them the wait is for one of those loads too
  constexpr int kYounger = (kGemmStages - 2) * (TA::kLoads + TB::kLoads);
  __shared__ __align__(1024) char smem[kGemmStages * kStage + 2 * kScales];

  const int n_tile = PAIR ? TILE / 2 : TILE;
  const int tiles_m = (g.M + TILE - 1) / TILE, tiles_n = (g.N + n_tile - 1) / n_tile, tiles = tiles_m * tiles_n;
  const int w = gemm_place((int)blockIdx.x, (int)gridDim.x), z = w / tiles, t = w % tiles;
  const int product = z / g.splits, split = z % g.splits;
  // groups of eight tiles of m, so that the 32 workgroups of a die form a patch
  const int group = t / (8 * tiles_n), in = t % (8 * tiles_n), gm = min(8, tiles_m - 8 * group);
  const int m0 = (8 * group + in % gm) * TILE, n0 = in / gm * n_tile;

  const int seg_steps = (g.K + kGemmStep - 1) / kGemmStep, steps = seg_steps * g.segments;
  constexpr int kTurn = MX ? 4 : 1;  // stages that share a load of scale bytes stay together
  const int turns = (steps + kTurn - 1) / kTurn;
  const int s0 = kTurn * (int)((long long)turns * split / g.splits);
  const int n = min(steps, kTurn * (int)((long long)turns * (split + 1) / g.splits)) - s0;

  TA ta;
  TB tb;
  ta.init(m0, g.M, g.lda);
  tb.init(n0, g.N, g.ldb);
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(gemm_lds_offset(smem));
  const int wave = __builtin_amdgcn_readfirstlane(wave_id());
  const char* scales = nullptr;  // MX: the first half of the waves those of the first tile's rows, the others of the second's
  uint32_t scale_off = 0;
  if constexpr (MX) {
    const bool of_a = wave < kWaves / 2;
    const int row0 = of_a ? m0 : n0, last = (of_a ? g.M : g.N) - 1 - row0;
    scales = reinterpret_cast<const char*>(of_a ? g.a_scales : g.b_scales) + (size_t)row0 * g.scale_ld + 4 * s0;
    scale_off = (uint32_t)min(wave % (kWaves / 2) * 64 + lane_id(), last) * g.scale_ld;
  }
  // the next stage to request: its place, addresses and what is left of its segment of k
  int requested = 0, place = 0, left = 0;
  const char *pa = nullptr, *pb = nullptr, *pb2 = nullptr;
  auto locate = [&](int s) {
    const int seg = s / seg_steps, k = (s - seg * seg_steps) * kGemmStep, which = g.segments > 1 ? seg : product;
    left = g.K - k;
    pa = static_cast<const char*>(g.a[which]) + (AK ? (size_t)m0 * g.lda + 2 * (size_t)k : (size_t)k * g.lda + 2 * (size_t)m0);
    const size_t at = BK ? (size_t)n0 * g.ldb + 2 * (size_t)k : (size_t)k * g.ldb + 2 * (size_t)n0;
    pb = static_cast<const char*>(g.b[PAIR ? 0 : which]) + at;
    if constexpr (PAIR) pb2 = static_cast<const char*>(g.b[1]) + at;
  };
  auto request = [&]() {
    const uint32_t lds = lds0 + (uint32_t)place * kStage;
    if constexpr (MX) {
      if (requested % 4 == 0) {
        gemm_load(scales, scale_off, lds0 + kGemmStages * kStage + (uint32_t)(requested / 4 % 2) * kScales + wave * 1024);
        scales += 16;
      }
    }
    ta.request(pa, nullptr, left, lds, wave);
    tb.request(pb, pb2, left, lds + TA::kBytes, wave);
    place = place + 1 == kGemmStages ? 0 : place + 1;
    left -= kGemmStep;
    pa += AK ? 2 * kGemmStep : (size_t)kGemmStep * g.lda;
    const size_t next = BK ? 2 * kGemmStep : (size_t)kGemmStep * g.ldb;
    pb += next;
    if constexpr (PAIR) pb2 += next;
    if (++requested < n && left <= 0) locate(s0 + requested);
  };

  const int wm = wave / kNW * (TILE / 2), wn = wave % kNW * 64;
  f32x16v acc[kMB][kNB] = {};
  if (n > 0) locate(s0);
  for (int i = 0; i < kGemmStages - 1 && i < n; ++i) request();
  if (n >= kGemmStages - 1)
    asm volatile("s_waitcnt vmcnt(%0)\n\ts_barrier" ::"n"(kYounger) : "memory");
  else
    asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
  if (kGroups && wave >= 4) gemm_barrier();  // the second group: half a stage later
  int cur = 0;
  for (int s = 0; s < n; ++s) {
    const char* sa = smem + cur * kStage;
    const char* sb = sa + TA::kBytes;
    cur = cur + 1 == kGemmStages ? 0 : cur + 1;
    bf16x8v fa[2][kMB], fb[2][kNB];
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
#pragma unroll
      for (int j = 0; j < kNB; ++j) fb[ks][j] = TB::fragment(sb, wn + 32 * j, ks);
#pragma unroll
      for (int i = 0; i < kMB; ++i) fa[ks][i] = TA::fragment(sa, wm + 32 * i, ks);
    }
    uint32_t xa[kMB], xb[kNB];  // MX: bytes 0 and 2 are the scales of this lane's blocks
    if constexpr (MX) {
      const uint32_t* words = reinterpret_cast<const uint32_t*>(smem + kGemmStages * kStage + (s / 4 % 2) * kScales) +
                              4 * (lane_id() & 31) + s % 4;
      const int shift = lane_id() >> 5 << 3;
#pragma unroll
      for (int i = 0; i < kMB; ++i) xa[i] = words[4 * (wm + 32 * i)] >> shift;
#pragma unroll
      for (int j = 0; j < kNB; ++j) xb[j] = words[4 * (TILE + wn + 32 * j)] >> shift;
    }
    __builtin_amdgcn_sched_barrier(0);
    if (requested < n) {
      request();
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kYounger) : "memory");
    } else {
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    }
    gemm_barrier();
    if constexpr (kGroups) __builtin_amdgcn_s_setprio(1);
    auto multiply = [&](auto half) {
      constexpr int KS = decltype(half)::value;
#pragma unroll
      for (int i = 0; i < kMB; ++i)
#pragma unroll
        for (int j = 0; j < kNB; ++j) {
          if constexpr (MX)
            acc[i][j] = __builtin_amdgcn_mfma_scale_f32_32x32x64_f8f6f4(mx_codes(fb[KS][j]), mx_codes(fa[KS][i]), acc[i][j], 4, 4,
                                                                        2 * KS, (int)xb[j], 2 * KS, (int)xa[i]);
          else
            acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[KS][j], fa[KS][i], acc[i][j], 0, 0, 0);
        }
    };
    multiply(std::integral_constant<int, 0>{});
    multiply(std::integral_constant<int, 1>{});
    if constexpr (kGroups) {
      __builtin_amdgcn_s_setprio(0);
      gemm_barrier();
    }
  }
  if (kGroups && wave < 4) gemm_barrier();
  asm volatile("s_waitcnt lgkmcnt(0)\n\ts_barrier" ::: "memory");  // LDS is the epilogue's
  epi.store(acc, smem, m0 + wm, n0 + (PAIR ? wn / 2 : wn), g.M, g.N, product, split);
}

}  // namespace hire
