// The dense gated FFN for few tokens with large layers: bound by reading the matrices once.  Rows come to LDS by asynchronous loads
// of runs of 512 bytes (256 in the second layer), three places ahead (about 96 KB on their way for the four waves of a compute
// unit); every wave has its own places, so that no barrier is among them.  d = 2048, 16384 units, 48 tokens, us against rows that
// come to registers a step or two ahead: first layer 37 -> 30, second 21 -> 18, dh 30 -> 22.
#include "gated.h"

namespace hire {
namespace {

constexpr int kStreamWaves = 4, kStreamCols = 512, kStreamHalf = kStreamCols / 2, kStreamPlaces = 4;
constexpr int kStreamPlace = 16 * kStreamHalf * 2, kStreamLoads = kStreamPlace / 1024;

// ---- the first layer, and dh ------------------------------------------------------------------
// A wave keeps 512 columns of the tokens in registers for as long as it lives and works on sixteen units after the other.  A place
// holds 256 columns of sixteen rows of one matrix.  SPAN waves share units whose rows have up to 512 SPAN columns and add their
// sums; longer rows are split into parts.
//   part null: h and what is kept; else the sums of columns blockIdx.y, in StorePart's order.
// SLOPES: x is dy and the one matrix is the second layer's, 32 units at a time; dg and du instead of h.
template <bool SLOPES, int NT, int SPAN>
__global__ __launch_bounds__(64 * kStreamWaves) __attribute__((amdgpu_waves_per_eu(1, 1))) void k_gated_stream(
    GatedLayer L, const uint16_t* __restrict__ x, int T, int part_cols, GatedKept kept, uint16_t* __restrict__ dg,
    uint16_t* __restrict__ du, float* __restrict__ part) {
  constexpr int kGroups = kStreamWaves / SPAN, kUnits = SLOPES ? 32 : 16, kSteps = kStreamHalf / 32;
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

  const int batches = (L.d_ff + kUnits * kGroups - 1) / (kUnits * kGroups);
  const int n = (batches - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x;  // at least one
  auto unit_of = [&](int i) { return (((int)blockIdx.x + i * (int)gridDim.x) * kGroups + wave / SPAN) * kUnits; };
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(gemm_lds_offset(smem)) + (uint32_t)wave * kStreamPlaces * kStreamPlace;
  const uint32_t ld = 2u * L.d;
  // Place p of units i: the gate's first and second 256 columns, then the other matrix's (SLOPES: the other units').  A load is two
  // rows; chunk c of row r lies at c ^ r.
  auto request = [&](int i, int p) __attribute__((always_inline)) {
    const int unit0 = min(unit_of(i) + (SLOPES ? p / 2 * 16 : 0), L.d_ff - 1), last = L.d_ff - 1 - unit0, ahead = p % 2 * (kStreamHalf / 8);
    const char* base = reinterpret_cast<const char*>(SLOPES ? L.w2u : (p < 2 ? L.wg : L.wu)) + (size_t)unit0 * ld + 2 * (size_t)col0 + 16 * ahead;
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
    // token 16 t + lane % 16, units 4 q ... of the sixteen (SLOPES: of both)
    auto store = [&](int t, const f32x4v (&v)[2]) __attribute__((always_inline)) {
      const int token = 16 * t + r;
      const size_t units = (size_t)T * L.d_ff;
      if constexpr (SLOPES) {
#pragma unroll
        for (int m = 0; m < 2; ++m) {
          const int unit = unit_of(i) + 16 * m + 4 * q;
          if (token >= T || unit >= L.d_ff) continue;  // d_ff is a multiple of 8
          const size_t at = (size_t)token * L.d_ff + unit;
          if (part) {
            *reinterpret_cast<f32x4v*>(part + blockIdx.y * units + at) = v[m];
            continue;
          }
          const uint2 gd = *reinterpret_cast<const uint2*>(kept.g + at), ud = *reinterpret_cast<const uint2*>(kept.u + at);
          const uint2 ld = *reinterpret_cast<const uint2*>(kept.low + at);
          const uint32_t g[2] = {gd.x, gd.y}, u[2] = {ud.x, ud.y}, low[2] = {ld.x, ld.y};
          float dgv[4], duv[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int shift = e % 2 * 16;
            const uint32_t l = low[e / 2] >> shift;
            const float gv = __uint_as_float((g[e / 2] >> shift) << 16 | (l & 0xFFu) << 8);
            const float uv = __uint_as_float((u[e / 2] >> shift) << 16 | (l & 0xFF00u));
            float slope;
            const float a = activation_of(L.act, gv, &slope);
            dgv[e] = v[m][e] * uv * slope;
            duv[e] = v[m][e] * a;
          }
          *reinterpret_cast<uint2*>(dg + at) = pack4(dgv);
          *reinterpret_cast<uint2*>(du + at) = pack4(duv);
        }
      } else {
        const int unit = unit_of(i) + 4 * q;
        if (token >= T || unit >= L.d_ff) return;
        const size_t at = (size_t)token * L.d_ff + unit;
        const f32x4v g = v[0], u = v[1];
        if (part) {
          float* sums = part + 2 * blockIdx.y * units + at;
          *reinterpret_cast<f32x4v*>(sums) = g;
          *reinterpret_cast<f32x4v*>(sums + units) = u;
          return;
        }
        float h[4], slope;
#pragma unroll
        for (int e = 0; e < 4; ++e) h[e] = activation_of(L.act, g[e], &slope) * u[e];
        *reinterpret_cast<uint2*>(kept.h + at) = pack4(h);
        if constexpr (NT == 1) {
#pragma unroll
          for (int e = 0; e < 4; ++e) h[e] = bf16_rest(h[e]);
          *reinterpret_cast<uint2*>(kept.rest + at) = pack4(h);
        }
        if (kept.g) {
          *reinterpret_cast<uint2*>(kept.g + at) = make_uint2(upper_pair(g[0], g[1]), upper_pair(g[2], g[3]));
          *reinterpret_cast<uint2*>(kept.u + at) = make_uint2(upper_pair(u[0], u[1]), upper_pair(u[2], u[3]));
          *reinterpret_cast<uint2*>(kept.low + at) =
              make_uint2(lower_pair(g[0], u[0], g[1], u[1]), lower_pair(g[2], u[2], g[3], u[3]));
        }
      }
    };
    if constexpr (SPAN == 1) {
#pragma unroll
      for (int t = 0; t < NT; ++t) store(t, {acc[0][t], acc[1][t]});
    } else {
      if (i > 0) lds_barrier();  // the sums before are read
#pragma unroll
      for (int m = 0; m < 2; ++m)
#pragma unroll
        for (int t = 0; t < NT; ++t) join[((wave * 2 + m) * NT + t) * 64 + lane] = acc[m][t];
      lds_barrier();
      for (int t = in_span; t < NT; t += SPAN) {
        const f32x4v* first = join + ((wave - in_span) * 2 * NT + t) * 64 + lane;
        f32x4v v[2] = {first[0], first[NT * 64]};
#pragma unroll
        for (int w = 1; w < SPAN; ++w) v[0] += first[w * 2 * NT * 64], v[1] += first[(w * 2 + 1) * NT * 64];
        store(t, v);
      }
    }
  }
}

struct FirstLayer {
  GatedLayer L;
  const uint16_t* x;
  int T;
  GatedKept kept;
  uint16_t *dg, *du;  // SLOPES
  float* part;
};
template <bool SLOPES, int NT, int SPAN>
hipError_t launch_span(const FirstLayer& f, int parts, int part_cols, hipStream_t s) {
  constexpr int kUnits = (SLOPES ? 32 : 16) * (kStreamWaves / SPAN);
  const int batches = (f.L.d_ff + kUnits - 1) / kUnits, each = 256 / parts;
  const hipError_t e = launch(&k_gated_stream<SLOPES, NT, SPAN>, dim3((unsigned)(batches < each ? batches : each), (unsigned)parts),
                              dim3(64 * kStreamWaves), 0, s, f.L, f.x, f.T, part_cols, f.kept, f.dg, f.du,
                              parts > 1 ? f.part : nullptr);
  if (e != hipSuccess || parts == 1) return e;
  const long long units = (long long)f.T * f.L.d_ff;
  const dim3 grid(join_blocks(units / 8)), block(256);
  return with_activation(f.L.act, [&](auto act) {
    constexpr int ACT = decltype(act)::value;
    if constexpr (SLOPES) return launch(&k_join_slopes<ACT>, grid, block, 0, s, f.part, parts, units, f.kept, f.dg, f.du);
    else return launch(&k_join_gated<ACT>, grid, block, 0, s, f.part, parts, units, f.kept);
  });
}
template <bool SLOPES, int NT>
hipError_t launch_tiles(const FirstLayer& f, hipStream_t s) {
  const int d = f.L.d, parts = gated_stream_parts(d), part_cols = (d / 8 + parts - 1) / parts * 8;
  if (part_cols <= kStreamCols) return launch_span<SLOPES, NT, 1>(f, parts, part_cols, s);
  if (part_cols <= 2 * kStreamCols) return launch_span<SLOPES, NT, 2>(f, parts, part_cols, s);
  return launch_span<SLOPES, NT, 4>(f, parts, part_cols, s);
}
template <bool SLOPES>
hipError_t launch_first_layer(const FirstLayer& f, hipStream_t s) {
  switch ((f.T + 15) / 16) {
    case 1: return launch_tiles<SLOPES, 1>(f, s);
    case 2: return launch_tiles<SLOPES, 2>(f, s);
    case 3: return launch_tiles<SLOPES, 3>(f, s);
    default: return launch_tiles<SLOPES, 4>(f, s);
  }
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
  constexpr bool REST = NT == 1;  // two terms of the tokens' values
  static_assert(kGatedRestTokens == 16, "one sixteen");
  constexpr int kTerms = REST ? 2 : 1, kPlaces = NT * kTerms <= 2 ? 4 : 3, kPlace = kDownMatrix + NT * kTerms * 1024;
  constexpr int kBlocks = kDownCols / 16;
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
      const size_t at = (size_t)min(16 * t + token, T - 1) * d_ff + k0 + 8 * chunk;
      const bool there = k0 + 8 * chunk < d_ff;
      gemm_load_at(there ? (const void*)(from.h[pair] + at) : (const void*)kGemmZeros, lds + kDownMatrix + t * 1024);
      if constexpr (REST)
        gemm_load_at(there ? (const void*)(from.rest[pair] + at) : (const void*)kGemmZeros, lds + kDownMatrix + (NT + t) * 1024);
    }
  };
  constexpr int kLoads = kDownLoads + NT * kTerms;
  for (int i = 0; i < kPlaces - 1 && i < n; ++i) request(i);
  f32x4v acc[NT * kTerms][kBlocks] = {};
  for (int i = 0; i < n; ++i) {
    if (i + kPlaces - 2 < n)
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"((kPlaces - 2) * kLoads) : "memory");
    else if (kPlaces == 4 && i + 1 < n)
      asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(kLoads) : "memory");
    else
      asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)" ::: "memory");
    if (i + kPlaces - 1 < n) request(i + kPlaces - 1);  // where the block before was
    const char* place = smem + (wave * kPlaces + i % kPlaces) * kPlace;
    bf16x8v hf[NT * kTerms];
#pragma unroll
    for (int t = 0; t < NT * kTerms; ++t)
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
      for (int t = 0; t < NT * kTerms; ++t) acc[t][c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(col, hf[t], acc[t][c], 0, 0, 0);
    }
  }
  if constexpr (REST) {
    // the first terms' sum stays as it is where it is not finite (gated.h, first_term)
#pragma unroll
    for (int c = 0; c < kBlocks; ++c)
#pragma unroll
      for (int e = 0; e < 4; ++e) acc[0][c][e] += fabsf(acc[0][c][e]) <= kLargestFloat ? acc[1][c][e] : 0.0f;
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
  return launch_first_layer<false>(FirstLayer{L, x, T, kept, nullptr, nullptr, part}, s);
}
hipError_t launch_gated_stream_slopes(const GatedLayer& L, const uint16_t* dy, int T, const GatedKept& kept, uint16_t* dg, uint16_t* du,
                                      float* part, hipStream_t s) {
  return launch_first_layer<true>(FirstLayer{L, dy, T, kept, dg, du, part}, s);
}

}  // namespace hire
