// The dense gated FFN's first layer for 17 to 64 tokens: bound by reading both matrices once.
//   A wave keeps 512 columns of the tokens in registers for as long as it lives and works on sixteen units after the other.  Their
// rows come to LDS by asynchronous loads of runs of 512 bytes: a place holds 256 columns of sixteen rows of one matrix, three
// places are on their way while one is multiplied (96 KB for the four waves of a compute unit), and as every wave has its own, no
// barrier is among them.  SPAN waves share units whose rows have up to 512 SPAN columns and add their sums; longer rows are split
// into parts.
#include "gated.h"

namespace hire {
namespace {

constexpr int kStreamWaves = 4, kStreamCols = 512, kStreamHalf = kStreamCols / 2, kStreamPlaces = 4;
constexpr int kStreamPlace = 16 * kStreamHalf * 2, kStreamLoads = kStreamPlace / 1024;

// part null: h and what is kept; else the sums of columns blockIdx.y, in StorePart<true>'s order.
template <int ACT, int NT, int SPAN>
__global__ __launch_bounds__(64 * kStreamWaves) __attribute__((amdgpu_waves_per_eu(1, 1))) void k_gated_stream(
    GatedLayer L, const uint16_t* __restrict__ x, int T, int part_cols, GatedKept kept, float* __restrict__ part) {
  constexpr int kGroups = kStreamWaves / SPAN, kSteps = kStreamHalf / 32;
  __shared__ __align__(1024) char smem[kStreamWaves * kStreamPlaces * kStreamPlace];
  __shared__ f32x4v join[SPAN > 1 ? kStreamWaves * 2 * NT * 64 : 1];
  const int wave = __builtin_amdgcn_readfirstlane(wave_id()), lane = lane_id(), r = lane & 15, q = lane >> 4;
  const int in_span = wave % SPAN, col_end = min(((int)blockIdx.y + 1) * part_cols, L.d);
  const int col0 = (int)blockIdx.y * part_cols + in_span * kStreamCols, there = max(col_end - col0, 0) / 8;  // chunks of eight

  uint4 xv[NT][2 * kSteps];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const uint4* token = reinterpret_cast<const uint4*>(x + (size_t)min(16 * t + r, T - 1) * L.d);
#pragma unroll
    for (int s = 0; s < 2 * kSteps; ++s) {
      const bool in = 4 * s + q < there;
      const uint4 v = token[in ? col0 / 8 + 4 * s + q : 0];
      xv[t][s] = in ? v : make_uint4(0u, 0u, 0u, 0u);
    }
  }

  const int sixteens = (L.d_ff + 15) / 16, batches = (sixteens + kGroups - 1) / kGroups;
  const int n = (batches - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x;  // at least one
  auto unit_of = [&](int i) { return (((int)blockIdx.x + i * (int)gridDim.x) * kGroups + wave / SPAN) * 16; };
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(gemm_lds_offset(smem)) + (uint32_t)wave * kStreamPlaces * kStreamPlace;
  const uint32_t ld = 2u * L.d;
  // Place p of units i: the gate's first and second 256 columns, then the other matrix's.  A load is two rows; chunk c of row r lies
  // at c ^ r.
  auto request = [&](int i, int p) __attribute__((always_inline)) {
    const int unit0 = min(unit_of(i), L.d_ff - 1), last = L.d_ff - 1 - unit0, ahead = p % 2 * (kStreamHalf / 8);
    const char* base = reinterpret_cast<const char*>(p < 2 ? L.wg : L.wu) + (size_t)unit0 * ld + 2 * (size_t)col0 + 16 * ahead;
    const uint32_t lds = lds0 + (uint32_t)p * kStreamPlace;
#pragma unroll
    for (int k = 0; k < kStreamLoads; ++k) {
      const int row = 2 * k + (lane >> 5), chunk = (lane & 31) ^ row;
      const uint32_t off = (uint32_t)min(row, last) * ld + (uint32_t)chunk * 16;
      if (there >= kStreamCols / 8)
        gemm_load(base, off, lds + k * 1024);
      else
        gemm_load_at(ahead + chunk < there ? (const void*)(base + off) : (const void*)kGemmZeros, lds + k * 1024);
    }
  };
  static_assert(kStreamPlaces == 4, "the places of sixteen units");
#pragma unroll
  for (int p = 0; p < kStreamPlaces - 1; ++p) request(0, p);
  for (int i = 0; i < n; ++i) {
    f32x4v acc[2][NT] = {};
#pragma unroll
    for (int p = 0; p < kStreamPlaces; ++p) {
      if (p < 2 || i + 1 < n)
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(2 * kStreamLoads) : "memory");
      else if (p == 2)
        asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kStreamLoads) : "memory");
      else
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
      if (p == 0)
        request(i, 3);  // where the units before had theirs
      else if (i + 1 < n)
        request(i + 1, p - 1);
      const char* place = smem + (wave * kStreamPlaces + p) * kStreamPlace;
#pragma unroll
      for (int s = 0; s < kSteps; ++s) {
        const bf16x8v w = *reinterpret_cast<const bf16x8v*>(place + r * (2 * kStreamHalf) + (((4 * s + q) ^ r) << 4));
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          bf16x8v xf;
          __builtin_memcpy(&xf, &xv[t][p % 2 * kSteps + s], 16);
          acc[p / 2][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w, xf, acc[p / 2][t], 0, 0, 0);
        }
      }
    }
    // Every lane takes part in the instructions above, also those that store nothing below.
#pragma unroll
    for (int m = 0; m < 2; ++m)
#pragma unroll
      for (int t = 0; t < NT; ++t) asm volatile("" : "+v"(acc[m][t]));
    // token 16 t + lane % 16, units 4 q ... of the sixteen
    auto store = [&](int t, const f32x4v& g, const f32x4v& u) __attribute__((always_inline)) {
      const int token = 16 * t + r, unit = unit_of(i) + 4 * q;
      if (token >= T || unit >= L.d_ff) return;  // d_ff is a multiple of 8
      const size_t at = (size_t)token * L.d_ff + unit, units = (size_t)T * L.d_ff;
      if (part) {
        float* to = part + 2 * blockIdx.y * units + at;
        *reinterpret_cast<f32x4v*>(to) = g;
        *reinterpret_cast<f32x4v*>(to + units) = u;
        return;
      }
      float h[4], slope;
#pragma unroll
      for (int e = 0; e < 4; ++e) h[e] = activation<ACT>(g[e], &slope) * u[e];
      *reinterpret_cast<uint2*>(kept.h + at) = pack4(h);
      if (kept.g) {
        *reinterpret_cast<uint2*>(kept.g + at) = make_uint2(upper_pair(g[0], g[1]), upper_pair(g[2], g[3]));
        *reinterpret_cast<uint2*>(kept.u + at) = make_uint2(upper_pair(u[0], u[1]), upper_pair(u[2], u[3]));
        *reinterpret_cast<uint2*>(kept.low + at) = make_uint2(lower_pair(g[0], u[0], g[1], u[1]), lower_pair(g[2], u[2], g[3], u[3]));
      }
    };
    if constexpr (SPAN == 1) {
#pragma unroll
      for (int t = 0; t < NT; ++t) store(t, acc[0][t], acc[1][t]);
    } else {
      if (i > 0) lds_barrier();  // the sums before are read
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int t = 0; t < NT; ++t) join[((wave * 2 + m) * NT + t) * 64 + lane] = acc[m][t];
      lds_barrier();
      for (int t = in_span; t < NT; t += SPAN) {
        const f32x4v* first = join + ((wave - in_span) * 2 * NT + t) * 64 + lane;
        f32x4v g = first[0], u = first[NT * 64];
#pragma unroll
        for (int w = 1; w < SPAN; ++w) g += first[w * 2 * NT * 64], u += first[(w * 2 + 1) * NT * 64];
        store(t, g, u);
      }
    }
  }
}

template <int ACT, int NT, int SPAN>
hipError_t launch_span(const GatedLayer& L, const uint16_t* x, int T, int parts, int part_cols, const GatedKept& kept, float* part,
                       hipStream_t s) {
  constexpr int kUnits = 16 * (kStreamWaves / SPAN);
  const int batches = (L.d_ff + kUnits - 1) / kUnits, each = 256 / parts;
  const hipError_t e = launch(&k_gated_stream<ACT, NT, SPAN>, dim3((unsigned)(batches < each ? batches : each), (unsigned)parts),
                              dim3(64 * kStreamWaves), 0, s, L, x, T, part_cols, kept, parts > 1 ? part : nullptr);
  if (e != hipSuccess || parts == 1) return e;
  const long long units = (long long)T * L.d_ff;
  return launch(&k_join_gated<ACT>, dim3(join_blocks(units / 8)), dim3(256), 0, s, part, parts, units, kept);
}

template <int ACT, int NT>
hipError_t launch_tiles(const GatedLayer& L, const uint16_t* x, int T, const GatedKept& kept, float* part, hipStream_t s) {
  const int parts = gated_stream_parts(L.d), part_cols = (L.d / 8 + parts - 1) / parts * 8;
  if (part_cols <= kStreamCols) return launch_span<ACT, NT, 1>(L, x, T, parts, part_cols, kept, part, s);
  if (part_cols <= 2 * kStreamCols) return launch_span<ACT, NT, 2>(L, x, T, parts, part_cols, kept, part, s);
  return launch_span<ACT, NT, 4>(L, x, T, parts, part_cols, kept, part, s);
}

// ---- the second layer, and dx -------------------------------------------------------------
// Columns 128 blockIdx.x ..., rows of part blockIdx.y of the matrix (of two matrices one behind the other: dx): the waves take
// blocks of 32 rows in turn, which come to LDS with the tokens' values that go with them, kPlaces - 1 blocks ahead.  The columns'
// operands are read transposed (four rows of sixteen columns by sixteen lanes); unit u (32 bytes) of row k lies at u ^ (k % 4 + 4
// (k / 8 % 2)), so that what half a wave reads lies in different banks.
constexpr int kDownRows = 32, kDownCols = 128, kDownMatrix = kDownRows * kDownCols * 2, kDownLoads = kDownMatrix / 1024;

template <int NT>
__global__ __launch_bounds__(64 * kStreamWaves) __attribute__((amdgpu_waves_per_eu(1, 1))) void k_gated_down_stream(
    GatedDown from, int T, int d, int d_ff, float* __restrict__ part, uint16_t* __restrict__ y) {
  constexpr int kPlaces = NT <= 2 ? 4 : 3, kPlace = kDownMatrix + NT * 1024, kBlocks = kDownCols / 16;
  __shared__ __align__(1024) char smem[kStreamWaves * kPlaces * kPlace];
  static_assert(sizeof(smem) >= kStreamWaves * NT * 16 * kDownCols * 4, "the sums");
  const int wave = __builtin_amdgcn_readfirstlane(wave_id()), lane = lane_id(), r = lane & 15, q = lane >> 4;
  const int parts = gridDim.y, each = (d_ff + kDownRows - 1) / kDownRows, blocks = each * from.pairs;
  const int b0 = (int)((long long)blocks * blockIdx.y / parts) + wave, b1 = (int)((long long)blocks * (blockIdx.y + 1) / parts);
  const int n = b0 < b1 ? (b1 - b0 + kStreamWaves - 1) / kStreamWaves : 0;
  const int col0 = (int)blockIdx.x * kDownCols, chunks = min((d - col0) / 8, kDownCols / 8);
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(gemm_lds_offset(smem)) + (uint32_t)wave * kPlaces * kPlace;
  auto request = [&](int i) __attribute__((always_inline)) {
    const int block = b0 + i * kStreamWaves, pair = block >= each ? 1 : 0, k0 = (block - pair * each) * kDownRows;
    const uint32_t lds = lds0 + (uint32_t)(i % kPlaces) * kPlace;
    const char* w = reinterpret_cast<const char*>(from.w[pair] + (size_t)k0 * d + col0);
    const bool whole = k0 + kDownRows <= d_ff && chunks == kDownCols / 8;
#pragma unroll
    for (int p = 0; p < kDownLoads; ++p) {  // four rows each
      const int k = 4 * p + q, chunk = ((r >> 1) ^ ((k & 3) + 4 * (k >> 3 & 1))) * 2 + (r & 1);
      const uint32_t off = (uint32_t)k * 2u * d + (uint32_t)chunk * 16;
      if (whole)
        gemm_load(w, off, lds + p * 1024);
      else
        gemm_load_at(k0 + k < d_ff && chunk < chunks ? (const void*)(w + off) : (const void*)kGemmZeros, lds + p * 1024);
    }
#pragma unroll
    for (int t = 0; t < NT; ++t) {  // sixteen tokens; chunk c of token m lies at c ^ (m / 4 % 4)
      const int token = lane >> 2, chunk = (lane & 3) ^ (token >> 2);
      const uint16_t* h = from.h[pair] + (size_t)min(16 * t + token, T - 1) * d_ff + k0 + 8 * chunk;
      gemm_load_at(k0 + 8 * chunk < d_ff ? (const void*)h : (const void*)kGemmZeros, lds + kDownMatrix + t * 1024);
    }
  };
  constexpr int kLoads = kDownLoads + NT;
  for (int i = 0; i < kPlaces - 1 && i < n; ++i) request(i);
  f32x4v acc[NT][kBlocks] = {};
  for (int i = 0; i < n; ++i) {
    if (i + kPlaces - 2 < n)
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((kPlaces - 2) * kLoads) : "memory");
    else if (kPlaces == 4 && i + 1 < n)
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kLoads) : "memory");
    else
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    if (i + kPlaces - 1 < n) request(i + kPlaces - 1);  // where the block before was
    const char* place = smem + (wave * kPlaces + i % kPlaces) * kPlace;
    bf16x8v hf[NT];
#pragma unroll
    for (int t = 0; t < NT; ++t)
      hf[t] = *reinterpret_cast<const bf16x8v*>(place + kDownMatrix + t * 1024 + r * 64 + ((q ^ (r >> 2)) << 4));
#pragma unroll
    for (int c = 0; c < kBlocks; ++c) {
      using Lds = __attribute__((address_space(3))) s16x4v*;
      const int k = 8 * q + (r >> 2);  // and four behind
      const char* at = place + k * (2 * kDownCols) + ((c ^ ((k & 3) + 4 * (k >> 3 & 1))) << 5) + ((r & 3) << 3);
      const s16x4v lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)at);
      const s16x4v hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((Lds)(at + 4 * (2 * kDownCols)));
      bf16x8v col;
      __builtin_memcpy(&col, &lo, 8);
      __builtin_memcpy(reinterpret_cast<char*>(&col) + 8, &hi, 8);
#pragma unroll
      for (int t = 0; t < NT; ++t) acc[t][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(col, hf[t], acc[t][c], 0, 0, 0);
    }
  }
  // acc[t][c]: token 16 t + lane % 16, columns 16 c + 4 q ...; the waves' sums are added in their order
  __syncthreads();
  f32x4v* sums = reinterpret_cast<f32x4v*>(smem);
#pragma unroll
  for (int t = 0; t < NT; ++t)
#pragma unroll
    for (int c = 0; c < kBlocks; ++c) sums[((wave * NT + t) * kBlocks + c) * 64 + lane] = acc[t][c];
  __syncthreads();
  for (int j = wave; j < NT * kBlocks; j += kStreamWaves) {
    f32x4v v = sums[j * 64 + lane];
#pragma unroll
    for (int w = 1; w < kStreamWaves; ++w) v += sums[(w * NT * kBlocks + j) * 64 + lane];
    const int token = j / kBlocks * 16 + r, col = col0 + j % kBlocks * 16 + 4 * q;
    if (token >= T || col >= d) continue;  // d is a multiple of 8
    const size_t at = (size_t)token * d + col;
    if (parts > 1) {
      *reinterpret_cast<f32x4v*>(part + (size_t)blockIdx.y * T * d + at) = v;
    } else {
      const float f[4] = {v[0], v[1], v[2], v[3]};
      *reinterpret_cast<uint2*>(y + at) = pack4(f);
    }
  }
}

}  // namespace

hipError_t launch_gated_down_stream(const GatedDown& from, int T, int d, int d_ff, int parts, uint16_t* out, float* part,
                                    hipStream_t s) {
  const dim3 grid((unsigned)((d + kDownCols - 1) / kDownCols), (unsigned)parts), block(64 * kStreamWaves);
  switch ((T + 15) / 16) {
    case 1: return launch(&k_gated_down_stream<1>, grid, block, 0, s, from, T, d, d_ff, part, out);
    case 2: return launch(&k_gated_down_stream<2>, grid, block, 0, s, from, T, d, d_ff, part, out);
    case 3: return launch(&k_gated_down_stream<3>, grid, block, 0, s, from, T, d, d_ff, part, out);
    default: return launch(&k_gated_down_stream<4>, grid, block, 0, s, from, T, d, d_ff, part, out);
  }
}

int gated_stream_parts(int d) { return (d + 4 * kStreamCols - 1) / (4 * kStreamCols); }

hipError_t launch_gated_stream(const GatedLayer& L, const uint16_t* x, int T, const GatedKept& kept, float* part, hipStream_t s) {
  return with_activation(L.act, [&](auto act) {
    constexpr int ACT = decltype(act)::value;
    switch ((T + 15) / 16) {
      case 1: return launch_tiles<ACT, 1>(L, x, T, kept, part, s);
      case 2: return launch_tiles<ACT, 2>(L, x, T, kept, part, s);
      case 3: return launch_tiles<ACT, 3>(L, x, T, kept, part, s);
      default: return launch_tiles<ACT, 4>(L, x, T, kept, part, s);
    }
  });
}

}  // namespace hire
