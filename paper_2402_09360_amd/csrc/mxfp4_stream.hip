// Product of many packed rows with a few tokens: bound by reading the rows once.
//   A wave keeps what it needs of the tokens in registers for as long as it lives, 512 or 1024 columns of them, and works on sixteen rows
// of these columns after the other.  The codes come to LDS by asynchronous loads of whole runs of 256 or 512 bytes, seven or three sixteens ahead
// (26 KB on their way for each of the four waves of a compute unit), without a barrier: every wave has its own places.  SPAN waves
// share rows of up to COLS SPAN columns and add their sums; longer rows are split into parts.  Against tokens that come from the L2
// or LDS and codes that come to registers one step ahead, in pieces of 64 bytes: 60000 rows of 8192 columns, two bf16 tokens 74 ->
// 55 us (4.8 TB/s), sixteen 88 -> 61, sixteen packed ones 78 -> 60.
#include "mxfp4.h"

#include "dense_epilogue.h"

namespace hire {
namespace {

constexpr int kStreamWaves = 4;

// COLS: of a wave, 1024 or 512.
template <int COLS>
struct StreamPlace {
  static constexpr int kSteps = COLS / 128, kChunks = COLS / 32, kCodes = 16 * COLS / 2, kScales = 16 * COLS / kMxBlock;
  static constexpr int kBytes = kCodes + kScales, kLoads = kCodes / 1024 + 1, kPlaces = 4096 / COLS;
};

template <bool PACKED, int NT, int COLS, int SPAN>
__global__ __launch_bounds__(64 * kStreamWaves) __attribute__((amdgpu_waves_per_eu(1, 1))) void k_mx_stream(
    const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales, const void* __restrict__ x,
    const uint8_t* __restrict__ x_scales, int T, int rows, int cols, int part_cols, void* __restrict__ y, int y_bf16,
    float* __restrict__ part) {
  using P = StreamPlace<COLS>;
  constexpr int kGroups = kStreamWaves / SPAN;  // sixteens of rows at a time
  __shared__ __align__(1024) char smem[kStreamWaves * P::kPlaces * P::kBytes];
  __shared__ f32x4v join[SPAN > 1 ? kStreamWaves * NT * 64 : 1];
  const int wave = __builtin_amdgcn_readfirstlane(wave_id()), lane = lane_id(), r = lane & 15, q = lane >> 4;
  const int in_span = wave % SPAN, blocks = cols / kMxBlock;
  const int col_end = min(((int)blockIdx.y + 1) * part_cols, cols), col0 = (int)blockIdx.y * part_cols + in_span * COLS;
  const int there = max(col_end - col0, 0) / kMxBlock;  // blocks of this wave, a multiple of sixteen

  // the tokens
  uint4 xv[NT][P::kSteps][PACKED ? 1 : 4];
  uint32_t xs[NT][PACKED ? P::kSteps : 1];
#pragma unroll
  for (int t = 0; t < NT; ++t) {
    const size_t token = (size_t)min(16 * t + r, T - 1);
#pragma unroll
    for (int s = 0; s < P::kSteps; ++s) {
      const uint4 zeros = make_uint4(0u, 0u, 0u, 0u);
      if constexpr (PACKED) {
        const bool in = 4 * s + q < there;
        const size_t block = token * blocks + (in ? col0 / kMxBlock + 4 * s + q : 0);
        const uint4 v = reinterpret_cast<const uint4*>(x)[block];
        xv[t][s][0] = in ? v : zeros;
        xs[t][s] = in ? x_scales[block] : 127u;
      } else {
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const bool in = 4 * s + j < there;
          const uint4 v = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(x) + token * cols +
                                                         (in ? col0 + (4 * s + j) * kMxBlock : 0))[q];
          xv[t][s][j] = in ? v : zeros;
        }
      }
    }
  }

  const int groups = (rows + 15) / 16, batches = (groups + kGroups - 1) / kGroups;
  const int n = (batches - (int)blockIdx.x + (int)gridDim.x - 1) / (int)gridDim.x;  // at least one
  auto row_of = [&](int i) { return (((int)blockIdx.x + i * (int)gridDim.x) * kGroups + wave / SPAN) * 16; };
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(gemm_lds_offset(smem)) + (uint32_t)wave * P::kPlaces * P::kBytes;
  const uint32_t ld = (uint32_t)cols / 2;
  // The sixteen bytes c of row r lie at c ^ r.  Blocks behind the last one are read as zeros.
  auto request = [&](int i) __attribute__((always_inline)) {
    const int row0 = min(row_of(i), rows - 1), last = rows - 1 - row0;
    const uint32_t lds = lds0 + (uint32_t)(i % P::kPlaces) * P::kBytes;
    const char* base = reinterpret_cast<const char*>(codes) + (size_t)row0 * ld + col0 / 2;
#pragma unroll
    for (int p = 0; p < P::kCodes / 1024; ++p) {
      const int row = 64 / P::kChunks * p + lane / P::kChunks, chunk = (lane % P::kChunks) ^ row;
      const uint32_t off = (uint32_t)min(row, last) * ld + (uint32_t)chunk * 16;
      if (there >= P::kChunks)
        gemm_load(base, off, lds + p * 1024);
      else
        gemm_load_at(chunk < there ? (const void*)(base + off) : (const void*)kGemmZeros, lds + p * 1024);
    }
    if (lane < P::kScales / 16) {  // sixteen bytes for 512 columns of a row
      constexpr int kEach = COLS / 512;
      const int row = min(lane / kEach, last), in = lane % kEach;
      const uint8_t* from = scales + (size_t)(row0 + row) * blocks + col0 / kMxBlock + 16 * in;
      gemm_load_at(16 * in < there ? (const void*)from : (const void*)kGemmZeros, lds + P::kCodes);
    }
  };
  auto wait = [&](auto younger) __attribute__((always_inline)) {
    asm volatile("s_waitcnt vmcnt(%0) lgkmcnt(0)" ::"n"(decltype(younger)::value * P::kLoads) : "memory");
  };
  for (int i = 0; i < P::kPlaces - 1 && i < n; ++i) request(i);
  for (int i = 0; i < n; ++i) {
    if (i + P::kPlaces - 2 < n)
      wait(std::integral_constant<int, P::kPlaces - 2>{});
    else if (P::kPlaces > 4 && i + 4 < n)
      wait(std::integral_constant<int, 4>{});
    else if (P::kPlaces > 4 && i + 2 < n)
      wait(std::integral_constant<int, 2>{});
    else if (i + 1 < n)
      wait(std::integral_constant<int, 1>{});
    else
      wait(std::integral_constant<int, 0>{});
    if (i + P::kPlaces - 1 < n) request(i + P::kPlaces - 1);  // where the sixteen before had theirs
    const char* place = smem + (wave * P::kPlaces + i % P::kPlaces) * P::kBytes;
    uint32_t sc[P::kSteps];
#pragma unroll
    for (int w = 0; w < P::kSteps; w += 4)
      *reinterpret_cast<uint4*>(&sc[w]) = *reinterpret_cast<const uint4*>(place + P::kCodes + (r * P::kSteps + w) * 4);
    f32x4v acc[NT] = {};
#pragma unroll
    for (int s = 0; s < P::kSteps; ++s) {
      uint4 c[1] = {*reinterpret_cast<const uint4*>(place + r * (COLS / 2) + (((4 * s + q) ^ r) << 4))};
      if constexpr (PACKED) {
        const i32x8v cv = {(int)c[0].x, (int)c[0].y, (int)c[0].z, (int)c[0].w, 0, 0, 0, 0};
#pragma unroll
        for (int t = 0; t < NT; ++t) {
          const i32x8v tv = {(int)xv[t][s][0].x, (int)xv[t][s][0].y, (int)xv[t][s][0].z, (int)xv[t][s][0].w, 0, 0, 0, 0};
          acc[t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(cv, tv, acc[t], 4, 4, 0, (int)(sc[s] >> (8 * q)), 0,
                                                                    (int)xs[t][s]);
        }
      } else {
        exchange_blocks<1>(c);
        auto block = [&](auto which, uint32_t word) {
          constexpr int J = decltype(which)::value;
          const uint4 w4 = mx_to_bf16(word, mx_scale_of<J>(sc[s]));
          bf16x8v wv;
          __builtin_memcpy(&wv, &w4, 16);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            bf16x8v xf;
            __builtin_memcpy(&xf, &xv[t][s][J], 16);
            acc[t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv, xf, acc[t], 0, 0, 0);
          }
        };
        block(std::integral_constant<int, 0>{}, c[0].x);
        block(std::integral_constant<int, 1>{}, c[0].y);
        block(std::integral_constant<int, 2>{}, c[0].z);
        block(std::integral_constant<int, 3>{}, c[0].w);
      }
    }
    // Every lane takes part in the instructions above, also those that store nothing below: without this the compiler moves the
    // scaled ones and the reads in front of them behind that condition.
#pragma unroll
    for (int t = 0; t < NT; ++t) asm volatile("" : "+v"(acc[t]));
    // acc[t]: token 16 t + lane % 16, rows 4 q ... of the sixteen
    auto store = [&](int t, int from, const f32x4v& v) __attribute__((always_inline)) {
      store_rows(gridDim.y > 1 ? part + (size_t)blockIdx.y * T * rows : y, gridDim.y > 1 ? 0 : y_bf16, T, rows,
                 16 * t + (from & 15), row_of(i) + 4 * (from >> 4), v);
    };
    if constexpr (SPAN == 1) {
#pragma unroll
      for (int t = 0; t < NT; ++t) store(t, lane, acc[t]);
    } else {
      if (i > 0) lds_barrier();  // the sums before are read
#pragma unroll
      for (int t = 0; t < NT; ++t) join[(wave * NT + t) * 64 + lane] = acc[t];
      lds_barrier();
      for (int t = in_span; t < NT; t += SPAN) {
        const f32x4v* first = join + ((wave - in_span) * NT + t) * 64 + lane;
        f32x4v v = first[0];
#pragma unroll
        for (int w = 1; w < SPAN; ++w) v += first[w * NT * 64];
        store(t, lane, v);
      }
    }
  }
}

template <bool PACKED, int NT, int COLS, int SPAN>
hipError_t launch_stream(const MxProduct& p, int parts, int part_cols, hipStream_t s) {
  const int batches = (p.rows + 16 * (kStreamWaves / SPAN) - 1) / (16 * (kStreamWaves / SPAN)), each = 256 / parts;
  float* part = static_cast<float*>(p.workspace);
  const hipError_t e = launch(&k_mx_stream<PACKED, NT, COLS, SPAN>, dim3((unsigned)(batches < each ? batches : each), (unsigned)parts),
                              dim3(64 * kStreamWaves), 0, s, p.codes, p.scales, p.x, p.x_scales, p.T, p.rows, p.cols, part_cols, p.y,
                              p.y_bf16, part);
  if (e != hipSuccess || parts == 1) return e;
  return launch_join_parts(part, p.y, p.y_bf16 != 0, parts, (long long)p.T * p.rows, s);
}
template <bool PACKED, int NT, int COLS>
hipError_t launch_by_columns(const MxProduct& p, hipStream_t s) {
  const int parts = mx_stream_shape(PACKED, p.T, p.rows, p.cols).parts, part_cols = (p.cols / 512 + parts - 1) / parts * 512;
  if (part_cols <= COLS) return launch_stream<PACKED, NT, COLS, 1>(p, parts, part_cols, s);
  if (part_cols <= 2 * COLS) return launch_stream<PACKED, NT, COLS, 2>(p, parts, part_cols, s);
  return launch_stream<PACKED, NT, COLS, 4>(p, parts, part_cols, s);
}
template <bool PACKED, int NT>
hipError_t launch_by_shape(const MxProduct& p, hipStream_t s) {
  if constexpr (PACKED || NT <= 2)
    if (mx_stream_shape(PACKED, p.T, p.rows, p.cols).cols == 1024) return launch_by_columns<PACKED, NT, 1024>(p, s);
  return launch_by_columns<PACKED, NT, 512>(p, s);
}

}  // namespace

// Columns of a wave.  More than 32 bf16 tokens: 512, all that the registers hold.  Else 512 take less of a start (the tokens come to
// registers first) and 1024 have longer runs and fewer parts.  us with 1024 / 512: 8192 rows of 2048 columns, 16 bf16 tokens 7.3 /
// 6.4, 20 packed 6.4 / 5.6, 64 packed 11.4 / 8.5; 16384 of 2048, two bf16 8.1 / 8.8, one packed 7.0 / 7.7, 64 packed 13.6 / 11.9;
// 256000 of 2048, 16 bf16 57 / 67, 48 packed 69 / 72; 2048 of 4096, one packed 4.4 / 6.0.  20 bf16 tokens: 8192 of 8192 20.7 /
// 19.8, 60000 of 8192 72 / 77, 16384 of 2048 13.2 / 10.9, 30000 of 2048 18.5 / 17.1.
MxStreamShape mx_stream_shape(bool packed, int T, int rows, int cols) {
  const long long values = (long long)rows * cols;
  bool narrow;
  if (packed)
    narrow = cols <= 2048 && values < (T <= 32 ? 1 << 25 : 1 << 26);
  else if (T <= 16)
    narrow = cols <= 2048 && values < 1 << 25;
  else
    narrow = T > 32 || (cols < 4096 ? values < 1 << 28 : rows < 16384);
  const int wave = narrow ? 512 : 1024, parts = (cols + 4 * wave - 1) / (4 * wave);
  const int part_cols = (cols / 512 + parts - 1) / parts * 512;
  const int waves = part_cols <= wave ? 1 : (part_cols <= 2 * wave ? 2 : 4);
  return MxStreamShape{wave, parts, 8ll * cols >= 7ll * parts * waves * wave};
}

hipError_t launch_mx_stream(const MxProduct& p, hipStream_t s) {
  const int tiles = (p.T + 15) / 16;
  if (p.x_scales) {
    if (tiles == 1) return launch_by_shape<true, 1>(p, s);
    if (tiles == 2) return launch_by_shape<true, 2>(p, s);
    if (tiles == 3) return launch_by_shape<true, 3>(p, s);
    return launch_by_shape<true, 4>(p, s);
  }
  if (tiles == 1) return launch_by_shape<false, 1>(p, s);
  if (tiles == 2) return launch_by_shape<false, 2>(p, s);
  if (tiles == 3) return launch_by_shape<false, 3>(p, s);
  return launch_by_shape<false, 4>(p, s);
}

}  // namespace hire
