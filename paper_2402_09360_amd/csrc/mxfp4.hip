// Microscaled 4-bit floating point: packing, reading back, and the product of packed rows with tokens in bf16 or packed
// themselves.  Layout: codes [rows, cols / 2], the lower column in the low nibble; scale bytes [rows, cols / 32].
#include "mxfp4.h"

#include "dense_epilogue.h"

namespace hire {
namespace {

// ---- packing ----------------------------------------------------------------
// A block is eight values in each of four lanes.  Its power of two is that of its largest magnitude, less two (6 = 1.5 2^2 is
// the largest code), so only magnitudes in (6, 8) 2^e saturate; e is at least -127.  The quotients are exact, and the
// conversion rounds half steps to the even code.
__global__ __launch_bounds__(256) void k_pack_mxfp4(const uint4* __restrict__ w, long long eights, uint32_t* __restrict__ codes,
                                                    uint8_t* __restrict__ scales) {
  typedef unsigned short u16x2 __attribute__((ext_vector_type(2)));
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < eights; i += (long long)gridDim.x * 256) {
    const uint4 v = w[i];
    const uint32_t d[4] = {v.x, v.y, v.z, v.w};
    u16x2 m = {0, 0};
#pragma unroll
    for (int q = 0; q < 4; ++q) {
      u16x2 a;
      const uint32_t magnitude = d[q] & 0x7FFF7FFFu;
      __builtin_memcpy(&a, &magnitude, 4);
      m = __builtin_elementwise_max(m, a);
    }
    uint32_t top = m[0] > m[1] ? m[0] : m[1];
    top = max(top, dpp_move<0xB1, 0xF>(0u, top));  // lanes 1 0 3 2 of every four
    top = max(top, dpp_move<0x4E, 0xF>(0u, top));  // lanes 2 3 0 1
    const uint32_t exponent = top >> 7;
    uint32_t byte = exponent > 2u ? exponent - 2u : 0u;
    if (top == 0u) byte = 127u;
    const bool finite = top < 0x7F80u;
    const float scale = mx_scale(byte);
    uint32_t c = 0u;
    bf16x2v pair[4];
    __builtin_memcpy(pair, d, 16);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, pair[0], scale, 0);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, pair[1], scale, 1);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, pair[2], scale, 2);
    c = __builtin_amdgcn_cvt_scalef32_pk_fp4_bf16(c, pair[3], scale, 3);
    codes[i] = finite ? c : 0u;
    if ((i & 3) == 0) scales[i >> 2] = finite ? (uint8_t)byte : (uint8_t)255;
  }
}

__global__ __launch_bounds__(256) void k_unpack_mxfp4(const uint32_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                      long long eights, uint4* __restrict__ w) {
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < eights; i += (long long)gridDim.x * 256)
    w[i] = mx_to_bf16(codes[i], mx_scale(scales[i >> 2]));
}

// ---- few tokens -----------------------------------------------------------------
// A wave multiplies RU times sixteen rows with NT times sixteen tokens in steps of 128 columns, four blocks; the WAVES waves of a
// workgroup take the steps in turn, and their sums are added in LDS in a fixed order.  A lane gets one block (sixteen bytes) of
// one row: block q = lane / 16 of row lane % 16.
//   Packed tokens: the same of a token, and one scaled instruction for the four blocks.
//   bf16 tokens: one instruction per block, whose lane holds columns 8 q ... of the block; so the four lanes of a row first
// exchange words, after which word q of block j is word j of lane q.  Then sixteen bytes of a token are 64 in a row of four
// lanes; of a lane's own block they would be 16 bytes every 64.
// The four scale bytes of blocks 4 s ... of a row; behind the last one: 127 (the codes there are zeros).
__device__ __forceinline__ uint32_t scale_word(const uint8_t* row, int s, int blocks, bool words) {
  if (words) return reinterpret_cast<const uint32_t*>(row)[s];
  uint32_t v = 0u;
#pragma unroll
  for (int e = 0; e < 4; ++e) v |= (4 * s + e < blocks ? (uint32_t)row[min(4 * s + e, blocks - 1)] : 127u) << (8 * e);
  return v;
}

// The words of TURN neighbouring steps, s0 a multiple of TURN: one load, in which neighbouring lanes of a row take neighbouring
// words, so that a line of scale bytes is asked for once for all of them and not for every step again.
template <int TURN>
__device__ __forceinline__ uint32_t scale_words(const uint8_t* row, int s0, int blocks, bool words) {
  const int s = s0 + ((lane_id() >> 4) & (TURN - 1));
  return scale_word(row, min(s, (blocks - 1) / 4), blocks, words);
}
template <int TURN>
__device__ __forceinline__ void spread_words(uint32_t mine, uint32_t (&word)[TURN]) {
  static_assert(TURN == 1 || TURN == 2 || TURN == 4, "lanes of a row");
  if constexpr (TURN == 1) {
    word[0] = mine;
  } else if constexpr (TURN == 2) {
    const auto w = __builtin_amdgcn_permlane16_swap(mine, mine, false, false);
    word[0] = w[0], word[1] = w[1];
  } else {
    const auto h = __builtin_amdgcn_permlane32_swap(mine, mine, false, false);
    const auto lo = __builtin_amdgcn_permlane16_swap(h[0], h[0], false, false);
    const auto hi = __builtin_amdgcn_permlane16_swap(h[1], h[1], false, false);
    word[0] = lo[0], word[1] = lo[1], word[2] = hi[0], word[3] = hi[1];
  }
}

template <bool PACKED_TOKENS, int NT, int RU, int WAVES, int TURN>
__global__ __launch_bounds__(64 * WAVES) void k_mx_few(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                       const void* __restrict__ x, const uint8_t* __restrict__ x_scales, int T,
                                                       int rows, int cols, int words, void* __restrict__ y, int y_bf16,
                                                       float* __restrict__ part) {
  __shared__ float sums[WAVES][RU * NT * 256];
  const int lane = lane_id(), wave = wave_id(), q = lane >> 4, blocks = cols / kMxBlock;
  const int row0 = blockIdx.x * 16 * RU;
  const uint8_t *row[RU], *row_scale[RU];
#pragma unroll
  for (int r = 0; r < RU; ++r) {
    const int at = min(row0 + 16 * r + (lane & 15), rows - 1);
    row[r] = codes + (size_t)at * (cols / 2);
    row_scale[r] = scales + (size_t)at * blocks;
  }
  size_t token[NT];
#pragma unroll
  for (int t = 0; t < NT; ++t) token[t] = (size_t)min(16 * t + (lane & 15), T - 1);

  f32x4v acc[RU][NT] = {};
  const int turns = (blocks + 4 * TURN - 1) / (4 * TURN), steps = (blocks + 3) / 4;
  const int first = (int)((long long)turns * blockIdx.y / gridDim.y), last = (int)((long long)turns * (blockIdx.y + 1) / gridDim.y);
  const uint4 zeros = make_uint4(0u, 0u, 0u, 0u);
  auto step = [&](int s, const uint32_t (&sc)[RU]) __attribute__((always_inline)) {
    const bool there = 4 * s + q < blocks;
    const int b = there ? 4 * s + q : blocks - 1;
    uint4 c[RU];
#pragma unroll
    for (int r = 0; r < RU; ++r) c[r] = reinterpret_cast<const uint4*>(row[r])[b];
    if constexpr (PACKED_TOKENS) {
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        uint4 xc = reinterpret_cast<const uint4*>(static_cast<const uint8_t*>(x) + token[t] * (cols / 2))[b];
        const uint32_t xs = there ? x_scales[token[t] * blocks + b] : 127u;
        if (!there) xc = zeros;
        const i32x8v xv = {(int)xc.x, (int)xc.y, (int)xc.z, (int)xc.w, 0, 0, 0, 0};
#pragma unroll
        for (int r = 0; r < RU; ++r) {
          const i32x8v cv = {(int)c[r].x, (int)c[r].y, (int)c[r].z, (int)c[r].w, 0, 0, 0, 0};
          acc[r][t] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(cv, xv, acc[r][t], 4, 4, 0, (int)(sc[r] >> (8 * q)), 0,
                                                                       (int)xs);
        }
      }
    } else {
      uint4 xv[NT][4];
#pragma unroll
      for (int t = 0; t < NT; ++t) {
        const uint4* p = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(x) + token[t] * cols) + q;
#pragma unroll
        for (int j = 0; j < 4; ++j) xv[t][j] = p[4 * min(4 * s + j, blocks - 1)];
      }
      if (4 * s + 4 > blocks) {  // uniform: the last blocks are not there
#pragma unroll
        for (int r = 0; r < RU; ++r)
          if (!there) c[r] = zeros;
#pragma unroll
        for (int j = 0; j < 4; ++j)
          if (4 * s + j >= blocks) {
#pragma unroll
            for (int t = 0; t < NT; ++t) xv[t][j] = zeros;
          }
      }
      exchange_blocks<RU>(c);
#pragma unroll
      for (int r = 0; r < RU; ++r) {
        auto block = [&](auto which, uint32_t code) {
          constexpr int J = decltype(which)::value;
          const uint4 w4 = mx_to_bf16(code, mx_scale_of<J>(sc[r]));
          bf16x8v wv;
          __builtin_memcpy(&wv, &w4, 16);
#pragma unroll
          for (int t = 0; t < NT; ++t) {
            bf16x8v xf;
            __builtin_memcpy(&xf, &xv[t][J], 16);
            acc[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv, xf, acc[r][t], 0, 0, 0);
          }
        };
        block(std::integral_constant<int, 0>{}, c[r].x);
        block(std::integral_constant<int, 1>{}, c[r].y);
        block(std::integral_constant<int, 2>{}, c[r].z);
        block(std::integral_constant<int, 3>{}, c[r].w);
      }
    }
  };
  for (int turn = first + wave; turn < last; turn += WAVES) {
    uint32_t word[RU][TURN];
#pragma unroll
    for (int r = 0; r < RU; ++r) spread_words<TURN>(scale_words<TURN>(row_scale[r], turn * TURN, blocks, words), word[r]);
#pragma unroll
    for (int u = 0; u < TURN; ++u) {
      if (TURN > 1 && turn * TURN + u >= steps) break;
      uint32_t sc[RU];
#pragma unroll
      for (int r = 0; r < RU; ++r) sc[r] = word[r][u];
      step(turn * TURN + u, sc);
    }
  }
  // acc[r][t]: token 16 t + lane % 16, rows 16 r + 4 (lane / 16) ... of this wave's columns
#pragma unroll
  for (int r = 0; r < RU; ++r)
#pragma unroll
    for (int t = 0; t < NT; ++t)
      *reinterpret_cast<f32x4v*>(&sums[wave][((r * NT + t) * 64 + lane) * 4]) = acc[r][t];
  __syncthreads();
  const bool parts = gridDim.y > 1;
  float* out = parts ? part + (size_t)blockIdx.y * T * rows : static_cast<float*>(y);
  for (int i = threadIdx.x; i < RU * NT * 256; i += 64 * WAVES) {
    // neighbouring threads: neighbouring rows of one token
    const int n = i % (16 * RU), tok = i / (16 * RU), at = ((n / 16 * NT + tok / 16) * 64 + (n % 16 / 4) * 16 + tok % 16) * 4 + n % 4;
    float v = sums[0][at];
#pragma unroll
    for (int w = 1; w < WAVES; ++w) v += sums[w][at];
    if (tok < T && row0 + n < rows) {
      const size_t o = (size_t)tok * rows + row0 + n;
      if (y_bf16 && !parts)
        static_cast<__bf16*>(y)[o] = (__bf16)v;
      else
        out[o] = v;
    }
  }
}

// ---- one bf16 token ---------------------------------------------------------------------
// Whole rows by vector instructions: LPR lanes of a wave share a row, a lane has one block of it and the token's 32 values that go
// with it, in registers for as long as the wave lives; so a wave's loads are whole rows without gaps, which the matrix
// instructions' layout (64 bytes of sixteen rows) does not give.  SPAN waves share rows of more than 2048 columns.  A wave has the
// kOneRows groups of rows that it works on and the next ones in flight.  256000 rows of 2048 columns: 50 us (5.6 TB/s; by matrix
// instructions 66), 16384 rows 6.5 (7.3).  Two tokens this way take as long as by matrix instructions, 68 us: the additions.
constexpr int kOneRows = 4;

template <int LPR, int SPAN>
__global__ __launch_bounds__(64 * SPAN) void k_mx_one(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                      const uint16_t* __restrict__ x, int rows, int cols, void* __restrict__ y,
                                                      int y_bf16) {
  constexpr int kRows = kWave / LPR, kBatch = kRows * kOneRows;
  __shared__ float join[SPAN > 1 ? 2 * SPAN * kBatch : 1];
  const int lane = lane_id(), wave = SPAN > 1 ? wave_id() : 0, blocks = cols / kMxBlock;
  const int block = wave * LPR + lane % LPR, at = min(block, blocks - 1);
  const bool there = block < blocks;
  float xv[32];
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    uint4 v = reinterpret_cast<const uint4*>(x + (size_t)at * 32)[p];
    if (!there) v = make_uint4(0u, 0u, 0u, 0u);
    const uint32_t d[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) xv[8 * p + 2 * e] = bf16_lo(d[e]), xv[8 * p + 2 * e + 1] = bf16_hi(d[e]);
  }
  const int stride = gridDim.x * kBatch;
  uint4 next[kOneRows];
  uint32_t next_scale[kOneRows];
  auto request = [&](int row0) __attribute__((always_inline)) {
#pragma unroll
    for (int u = 0; u < kOneRows; ++u) {
      const size_t row = (size_t)min(row0 + u * kRows + lane / LPR, rows - 1);
      next[u] = load_streaming(reinterpret_cast<const uint4*>(codes + row * (cols / 2)) + at);
      next_scale[u] = scales[row * blocks + at];
    }
  };
  int turn = 0;
  request(blockIdx.x * kBatch);
  for (int row0 = blockIdx.x * kBatch; row0 < rows; row0 += stride, turn ^= 1) {
    uint4 code[kOneRows];
    uint32_t sc[kOneRows];
#pragma unroll
    for (int u = 0; u < kOneRows; ++u) code[u] = next[u], sc[u] = next_scale[u];
    request(min(row0 + stride, rows - 1));  // not used behind the last row
    float mine = 0.0f;  // lane u kRows + r of the first kBatch: that row's sum
#pragma unroll
    for (int u = 0; u < kOneRows; ++u) {
      const float scale = mx_scale(there ? sc[u] : 127u);
      const uint32_t d[4] = {code[u].x, code[u].y, code[u].z, code[u].w};
      float s = 0.0f;
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const uint32_t word = there ? d[p] : 0u;
        float w[8];
        auto pair = [&](auto which) {
          constexpr int P = decltype(which)::value;
          const auto v = __builtin_amdgcn_cvt_scalef32_pk_f32_fp4(word, scale, P);
          w[2 * P] = v[0], w[2 * P + 1] = v[1];
        };
        pair(std::integral_constant<int, 0>{});
        pair(std::integral_constant<int, 1>{});
        pair(std::integral_constant<int, 2>{});
        pair(std::integral_constant<int, 3>{});
#pragma unroll
        for (int e = 0; e < 8; ++e) s = fmaf(w[e], xv[8 * p + e], s);
      }
      // the sum of the row's lanes, in its last one
      s += dpp_move<0x111, 0xF>(0.0f, s);
      s += dpp_move<0x112, 0xF>(0.0f, s);
      s += dpp_move<0x114, 0xF>(0.0f, s);
      if constexpr (LPR >= 16) s += dpp_move<0x118, 0xF>(0.0f, s);
      if constexpr (LPR >= 32) s += dpp_move<0x142, 0xA>(0.0f, s);
      if constexpr (LPR >= 64) s += dpp_move<0x143, 0xC>(0.0f, s);
#pragma unroll
      for (int r = 0; r < kRows; ++r) {
        const float sum = read_lane(s, r * LPR + LPR - 1);
        if (lane == u * kRows + r) mine = sum;
      }
    }
    if constexpr (SPAN > 1) {
      float* place = join + turn * SPAN * kBatch;
      if (lane < kBatch) place[wave * kBatch + lane] = mine;
      lds_barrier();
      if (wave == 0 && lane < kBatch)
        for (int w = 1; w < SPAN; ++w) mine += place[w * kBatch + lane];
    }
    if (wave == 0 && lane < kBatch && row0 + lane < rows) {
      if (y_bf16)
        static_cast<__bf16*>(y)[row0 + lane] = (__bf16)mine;
      else
        static_cast<float*>(y)[row0 + lane] = mine;
    }
  }
}

// ---- few bf16 tokens, the tokens shared in LDS -----------------------------------------
// RW waves of a workgroup have RU times sixteen rows each, all of them the same columns, and KW such groups of waves share the
// four-block steps of a chunk of 256 columns; the tokens' chunk is in LDS, so what comes from the L2 for the tokens is shared by 16 RU RW
// rows.  The next chunk's tokens and the wave's own codes of it are on their way while one is multiplied.
// x in LDS: [16 NT tokens][512 bytes], 16-byte piece c of token t at c ^ (t % 16).
constexpr int kSharedChunk = 256;
constexpr int kSharedSteps = kSharedChunk / 128;

template <int NT, int RU, int RW, int KW>
__global__ __launch_bounds__(64 * RW * KW) void k_mx_shared(const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                            const uint16_t* __restrict__ x, int T, int rows, int cols, int words,
                                                            void* __restrict__ y, int y_bf16) {
  constexpr int kWaves = RW * KW, kSteps = kSharedSteps / KW, kPlace = 16 * NT * kSharedChunk * 2, kLoads = kPlace / 1024 / kWaves;
  static_assert(KW <= 2 && kLoads * kWaves * 1024 == kPlace, "whole loads");
  constexpr int kJoin = KW > 1 ? RW * RU * NT * 1024 : 0;
  __shared__ __align__(1024) char smem[2 * kPlace > kJoin ? 2 * kPlace : kJoin];
  const int lane = lane_id(), wave = __builtin_amdgcn_readfirstlane(wave_id()), q = lane >> 4, blocks = cols / kMxBlock;
  const int kw = wave % KW, row0 = (blockIdx.x * RW + wave / KW) * 16 * RU;
  const uint8_t *row[RU], *row_scale[RU];
#pragma unroll
  for (int r = 0; r < RU; ++r) {
    const int at = min(row0 + 16 * r + (lane & 15), rows - 1);
    row[r] = codes + (size_t)at * (cols / 2);
    row_scale[r] = scales + (size_t)at * blocks;
  }
  const int chunks = (cols + kSharedChunk - 1) / kSharedChunk;
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(gemm_lds_offset(smem));
  auto request_tokens = [&](int c) {
#pragma unroll
    for (int i = 0; i < kLoads; ++i) {
      constexpr int kLanes = kSharedChunk / 8;  // of a token
      const int piece = i * kWaves + wave, t = (piece * 64 + lane) / kLanes;
      const int at = c * kSharedChunk + ((lane & (kLanes - 1)) ^ (t & 15)) * 8;
      const void* from = x + (size_t)min(t, T - 1) * cols + at;
      gemm_load_at(at < cols ? from : (const void*)kGemmZeros, lds0 + (uint32_t)(c & 1) * kPlace + piece * 1024);
    }
  };
  uint4 next[kSteps][RU];
  uint32_t next_scale[RU];  // of all steps of the chunk, as scale_words has them
  auto request_codes = [&](int c) {
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      const int s = kSharedSteps * c + kw * kSteps + u, b = min(4 * s + q, blocks - 1);
#pragma unroll
      for (int r = 0; r < RU; ++r) {
        next[u][r] = reinterpret_cast<const uint4*>(row[r])[b];
      }
    }
#pragma unroll
    for (int r = 0; r < RU; ++r) next_scale[r] = scale_words<kSteps>(row_scale[r], kSharedSteps * c + kw * kSteps, blocks, words);
  };
  f32x4v acc[RU][NT] = {};
  request_codes(0);
  request_tokens(0);
  for (int c = 0; c < chunks; ++c) {
    asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
    uint4 code[kSteps][RU];
    uint32_t sc[RU][kSteps];
#pragma unroll
    for (int u = 0; u < kSteps; ++u)
#pragma unroll
      for (int r = 0; r < RU; ++r) {
        // in registers before the next requests go out: behind them the compiler would wait for those too
        asm volatile("" : "+v"(next[u][r].x), "+v"(next[u][r].y), "+v"(next[u][r].z), "+v"(next[u][r].w), "+v"(next_scale[r]));
        code[u][r] = next[u][r];
        if ((kSharedSteps * c + kw * kSteps + u) * 4 + q >= blocks) code[u][r] = make_uint4(0u, 0u, 0u, 0u);
      }
#pragma unroll
    for (int r = 0; r < RU; ++r) spread_words<kSteps>(next_scale[r], sc[r]);
    if (c + 1 < chunks) {
      request_codes(c + 1);
      request_tokens(c + 1);
    }
    const char* place = smem + (c & 1) * kPlace;
#pragma unroll
    for (int u = 0; u < kSteps; ++u) {
      exchange_blocks<RU>(code[u]);
      const int step = kw * kSteps + u;
      auto block = [&](auto which) {
        constexpr int J = decltype(which)::value;
        bf16x8v xf[NT];
#pragma unroll
        for (int t = 0; t < NT; ++t)
          xf[t] = *reinterpret_cast<const bf16x8v*>(place + (16 * t + (lane & 15)) * (2 * kSharedChunk) +
                                                    ((((4 * step + J) * 4 + q) ^ (lane & 15)) << 4));
#pragma unroll
        for (int r = 0; r < RU; ++r) {
          const uint32_t word = J == 0 ? code[u][r].x : (J == 1 ? code[u][r].y : (J == 2 ? code[u][r].z : code[u][r].w));
          const uint4 w4 = mx_to_bf16(word, mx_scale_of<J>(sc[r][u]));
          bf16x8v wv;
          __builtin_memcpy(&wv, &w4, 16);
#pragma unroll
          for (int t = 0; t < NT; ++t) acc[r][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wv, xf[t], acc[r][t], 0, 0, 0);
        }
      };
      block(std::integral_constant<int, 0>{});
      block(std::integral_constant<int, 1>{});
      block(std::integral_constant<int, 2>{});
      block(std::integral_constant<int, 3>{});
    }
  }
  if constexpr (KW > 1) {
    __syncthreads();
    f32x4v* join = reinterpret_cast<f32x4v*>(smem) + (size_t)(wave / KW) * RU * NT * 64 + lane;
    if (kw == 1) {
#pragma unroll
      for (int r = 0; r < RU; ++r)
#pragma unroll
        for (int t = 0; t < NT; ++t) join[(r * NT + t) * 64] = acc[r][t];
    }
    __syncthreads();
    if (kw == 1) return;
#pragma unroll
    for (int r = 0; r < RU; ++r)
#pragma unroll
      for (int t = 0; t < NT; ++t) acc[r][t] += join[(r * NT + t) * 64];
  }
  // acc[r][t]: token 16 t + lane % 16, rows 16 r + 4 (lane / 16) ...
#pragma unroll
  for (int r = 0; r < RU; ++r)
#pragma unroll
    for (int t = 0; t < NT; ++t) {
      const int token = 16 * t + (lane & 15), n = row0 + 16 * r + 4 * q;
      store_rows(y, y_bf16, T, rows, token, n, acc[r][t]);
    }
}

// ---- packed tokens in tiles ----------------------------------------------------------
// y's rows out of the sums: whole vectors where the row length admits them.  Parts of the columns follow one another, in fp32.
struct StoreProduct {
  void* y;
  int bf16;
  template <int MB, int NB>
  __device__ __forceinline__ void store(const f32x16v (&acc)[MB][NB], char* smem, int m0, int n0, int M, int N, int, int split) const {
    for_rows<false>(acc, smem, m0, n0, M, N, NoFetch{}, [&](int m, int n, const float (&v)[1][8], int) {
      const size_t at = ((size_t)split * M + m) * N + n;
      if (N % 8 != 0) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (n + e < N) {
            if (bf16)
              static_cast<__bf16*>(y)[at + e] = (__bf16)v[0][e];
            else
              static_cast<float*>(y)[at + e] = v[0][e];
          }
      } else if (bf16) {
        *reinterpret_cast<uint4*>(static_cast<uint16_t*>(y) + at) = pack8(v[0]);
      } else {
        float4* to = reinterpret_cast<float4*>(static_cast<float*>(y) + at);
        to[0] = make_float4(v[0][0], v[0][1], v[0][2], v[0][3]);
        to[1] = make_float4(v[0][4], v[0][5], v[0][6], v[0][7]);
      }
    });
  }
};

// Scale bytes in rows of whole sixteens, 127 behind the last block: what the product reads where the columns are no multiple of
// 512 (or the caller's bytes start elsewhere).
__global__ __launch_bounds__(256) void k_pad_scales(const uint8_t* __restrict__ scales, long long rows, int blocks, int words,
                                                    uint32_t* __restrict__ out) {
  for (long long i = (long long)blockIdx.x * 256 + threadIdx.x; i < rows * words; i += (long long)gridDim.x * 256) {
    const long long row = i / words;
    const int b = (int)(i - row * words) * 4;
    uint32_t v = 0u;
#pragma unroll
    for (int e = 0; e < 4; ++e) v |= (b + e < blocks ? (uint32_t)scales[row * blocks + b + e] : 127u) << (8 * e);
    out[i] = v;
  }
}

bool whole_words(const MxProduct& p) { return p.cols % 128 == 0 && reinterpret_cast<uintptr_t>(p.scales) % 4 == 0; }

// How the rows are divided: `groups` sixteens of them for a workgroup, whose waves take the columns in turns of `turn` steps.  More
// rows share what is read of the tokens (16 kB per step of 64 tokens, against 1 kB of sixteen rows), but 256 workgroups should be
// left; where they are fewer the columns are split and the parts joined.  us with 4 groups, 8 waves / 2, 8 / 1, 16 (and 4, 4 in
// turns of four): 64 tokens, 1000 rows of 4096 14.4 / 11.3 / 12.9, 2500 15.4 / 13.3 / 19.0, 5000 18.2 / 22.0 / 36.6, of 1024 11.9
// / 8.7 / 12.8, 9000 of 4096 28.0 / 42.5 / 54.2, 16384 29.8 / 43.6 / 73.3 (29.0), of 2048 18.6 / - / - (17.1); 20 tokens, 9000 of
// 1024 7.0 / 7.4 / 9.3, 2500 6.7 / 6.1 / 6.1.
//   Up to sixteen tokens a wave has to have three turns for the join to pay: 100 rows, two tokens / sixteen, us without / with
// parts: of 8192 columns 8.0 / 12.8, 5.9 / 7.5, of 32768 25.2 / 44.0, 8.6 / 11.0; 1000 rows of 4096 (two turns) 5.7 / 8.1, 6.1 / 7.4.
struct FewShape {
  int groups, waves, turn;
};
FewShape few_shape(int T, int rows) {
  const int sixteens = (rows + 15) / 16;
  if (sixteens >= 4 * 256) return FewShape{4, 4, 4};
  if (T > 16) return sixteens >= 2 * 256 ? FewShape{4, 8, 1} : FewShape{2, 8, 1};
  return sixteens >= 2 * 256 ? FewShape{2, 8, 1} : FewShape{1, 16, 1};
}
int few_splits(int T, int rows, int cols) {
  const FewShape f = few_shape(T, rows);
  const int workgroups = (rows + 16 * f.groups - 1) / (16 * f.groups), turns = (cols + 128 * f.turn - 1) / (128 * f.turn);
  const int fill = 256 / workgroups, most = turns / f.waves;  // a turn for every wave
  if (T <= 16 && most < 3) return 1;
  const int splits = fill < most ? fill : most;
  return splits < 1 ? 1 : splits;
}

template <bool PACKED, int NT, int RU, int WAVES, int TURN>
hipError_t launch_few(const MxProduct& p, hipStream_t s) {
  const int splits = few_splits(p.T, p.rows, p.cols);
  float* part = static_cast<float*>(p.workspace);
  const hipError_t e = launch(&k_mx_few<PACKED, NT, RU, WAVES, TURN>,
                              dim3((unsigned)((p.rows + 16 * RU - 1) / (16 * RU)), (unsigned)splits), dim3(64 * WAVES), 0, s, p.codes,
                              p.scales, p.x, p.x_scales, p.T, p.rows, p.cols, whole_words(p) ? 1 : 0, p.y, p.y_bf16, part);
  if (e != hipSuccess || splits == 1) return e;
  return launch_join_parts(part, p.y, p.y_bf16 != 0, splits, (long long)p.T * p.rows, s);
}

template <int LPR, int SPAN>
hipError_t launch_one(const MxProduct& p, hipStream_t s) {
  const int batch = kWave / LPR * kOneRows, batches = (p.rows + batch - 1) / batch, most = 4096 / SPAN;
  return launch(&k_mx_one<LPR, SPAN>, dim3((unsigned)(batches < most ? batches : most)), dim3(64 * SPAN), 0, s, p.codes, p.scales,
                static_cast<const uint16_t*>(p.x), p.rows, p.cols, p.y, p.y_bf16);
}
constexpr int kOneMaxCols = 16 * 2048;
hipError_t launch_one_token(const MxProduct& p, hipStream_t s) {
  const int blocks = p.cols / kMxBlock;
  if (blocks <= 8) return launch_one<8, 1>(p, s);
  if (blocks <= 16) return launch_one<16, 1>(p, s);
  if (blocks <= 32) return launch_one<32, 1>(p, s);
  if (blocks <= 64) return launch_one<64, 1>(p, s);
  if (blocks <= 128) return launch_one<64, 2>(p, s);
  if (blocks <= 256) return launch_one<64, 4>(p, s);
  return launch_one<64, 16>(p, s);
}

template <int NT, int RU, int RW, int KW>
hipError_t launch_shared(const MxProduct& p, hipStream_t s) {
  return launch(&k_mx_shared<NT, RU, RW, KW>, dim3((unsigned)((p.rows + 16 * RU * RW - 1) / (16 * RU * RW))), dim3(64 * RW * KW), 0, s,
                p.codes, p.scales, static_cast<const uint16_t*>(p.x), p.T, p.rows, p.cols, whole_words(p) ? 1 : 0, p.y, p.y_bf16);
}

// Tokens shared in LDS where the rows still fill the chip in workgroups of 128 or 256.  2048 columns, us through the L2 / shared:
// 256000 rows, four tokens 69 / 71, sixteen 80 / 72, 33 127 / 86, 64 247 / 103; 32768 rows of 4096, sixteen 23.3 / 22.9, 33 35.2 /
// 27.4, 64 53.9 / 31.5; 16384 rows, 33 12.5 / 15.5, 64 17.1 / 16.9.
template <bool PACKED, int NT>  // NT: sixteens of tokens
hipError_t launch_few_by_rows(const MxProduct& p, hipStream_t s) {
  if constexpr (!PACKED) {
    if (p.rows >= 256 * 256 && p.T > 4) return launch_shared<NT, 2, 8, 1>(p, s);
    if constexpr (NT > 1)
      if (p.rows >= 128 * 256) return launch_shared<NT, 2, 4, 2>(p, s);
  }
  const FewShape f = few_shape(p.T, p.rows);
  if (f.turn == 4) return launch_few<PACKED, NT, 4, 4, 4>(p, s);
  if constexpr (NT > 1) return f.groups == 4 ? launch_few<PACKED, NT, 4, 8, 1>(p, s) : launch_few<PACKED, NT, 2, 8, 1>(p, s);
  return f.groups == 2 ? launch_few<PACKED, NT, 2, 8, 1>(p, s) : launch_few<PACKED, NT, 1, 16, 1>(p, s);
}
template <bool PACKED>
hipError_t launch_few_tokens(const MxProduct& p, hipStream_t s) {
  if constexpr (!PACKED)
    if (p.T == 1 && p.cols <= kOneMaxCols) return launch_one_token(p, s);
  switch ((p.T + 15) / 16) {
    case 1: return launch_few_by_rows<PACKED, 1>(p, s);
    case 2: return launch_few_by_rows<PACKED, 2>(p, s);
    case 3: return launch_few_by_rows<PACKED, 3>(p, s);
    default: return launch_few_by_rows<PACKED, 4>(p, s);
  }
}

}  // namespace

hipError_t launch_pack_mxfp4(const uint16_t* w, int rows, int cols, uint8_t* codes, uint8_t* scales, hipStream_t s) {
  const long long eights = (long long)rows * cols / 8, groups = (eights + 255) / 256;
  return launch(&k_pack_mxfp4, dim3((unsigned)(groups < 16384 ? groups : 16384)), dim3(256), 0, s, reinterpret_cast<const uint4*>(w),
                eights, reinterpret_cast<uint32_t*>(codes), scales);
}

hipError_t launch_unpack_mxfp4(const uint8_t* codes, const uint8_t* scales, int rows, int cols, uint16_t* w, hipStream_t s) {
  const long long eights = (long long)rows * cols / 8, groups = (eights + 255) / 256;
  return launch(&k_unpack_mxfp4, dim3((unsigned)(groups < 16384 ? groups : 16384)), dim3(256), 0, s,
                reinterpret_cast<const uint32_t*>(codes), scales, eights, reinterpret_cast<uint4*>(w));
}

namespace {
bool mx_pads_scales(const MxProduct& p) {
  return p.cols % 512 != 0 || reinterpret_cast<uintptr_t>(p.x_scales) % 16 != 0 || reinterpret_cast<uintptr_t>(p.scales) % 16 != 0;
}
// Packed tokens as tiles of a dense product: always from 65 on, and where the rows are many enough for tiles of 128 of them; a few
// tokens' tiles are mostly empty, but the tokens then come to LDS once for 128 rows.  us with the few tokens' kernel / as tiles,
// 2048 columns: 256000 rows, 17 tokens 77 / 71, 64 128 / 79; 16384, 17 8.7 / 9.7, 33 10.2 / 9.9, 64 13.0 / 10.5; 1000 of 8192, 64
// 11.1 / 27.4.
bool mx_tiles(int T, int rows) {
  return T > kMxFewTokens || (T > 32 && rows >= 16384) || (T > 8 && rows >= 65536);
}
size_t mx_padded_bytes(int T, int rows, int cols) {
  return (((size_t)T + rows) * ((cols / kMxBlock + 15) / 16) * 16 + 255) / 256 * 256;
}
// Tiles that leave compute units idle in parts of the columns, whose sums are joined.  us without / with: 100 tokens on 1000 rows
// of 8192 columns 28.2 / 12.7, on 8192 rows 30.5 / 19.9; 1000 on 1024 of 8192 28.2 / 23.3; 128 on 2048 of 4096 16.5 / 11.7.  Every
// other tile and number of parts was timed for 16 such sizes: at most 9 % better.
ProductShape mx_shape(int T, int rows, int cols) { return product_shape(T, rows, (cols + 127) / 128, 1, 32); }
// Rows streamed past the tokens (mxfp4_stream.hip): matrices that keep every compute unit at it for a while.  us without / with it:
//   bf16, two / sixteen tokens: 4096 rows of 4096 columns 6.1, 5.6 / 8.4, 7.6, of 1024 3.7, 5.0 / 4.4, 5.1 (no), 8192 of 2048 5.4,
// 5.9 / 6.9, 6.5, 256000 of 2048 69.5, 58.2 / 76.6, 64.3, 12000 of 8192 23.6, 19.0 / 32.6, 21.4; parts pay later: 4096 of 8192 9.8,
// 10.1 / 14.1, 12.6.  20 / 48: 1000 of 2048 7.1, 5.9 / 9.5, 8.8, 20000 of 8192 50.1, 34.6 / 72.0, 42.2, 60000 of 8192 93.9, 77.3 /
// 105, 97; 4096 of 1024 5.7, 6.1 / 7.8, 9.1 (no), 65536 of 2048 24.5, 25.9 / 26.5, 31.2 (no), 2048 of 4096, 48 11.1, 11.4 (no).
//   packed, one / sixteen: 1000 of 2048 3.5, 3.2 / 4.3, 3.6, 8192 of 1024 4.0, 3.9 / 4.6, 4.1, 256000 of 2048 65.1, 56.1 / 67.5, 61.0,
// 16384 of 16384 48.8, 33.4 / 52.4, 34.8; 20 / 64: 1000 of 2048 6.6, 4.0 / 9.2, 6.5, 8192 of 2048 9.0, 5.7 / 14.5, 8.6, 20000 of 8192
// 42.5, 26.3 / 35.9, 33.3, but 64 on 65536 of 2048 22.9, 26.6 (no: tiles).
//   Over 140 drawn sizes 0.93 of the time without it as a geometric mean, 0.49 to 1.1.
bool mx_streams(int T, int rows, int cols, bool packed) {
  if (cols % 512 != 0 || cols < 1024 || T > kMxFewTokens || (T == 1 && !packed)) return false;
  const long long values = (long long)rows * cols;
  const MxStreamShape shape = mx_stream_shape(packed, T, rows, cols);
  if (!shape.full || shape.parts > 64 || values < 3 << 19) return false;
  const bool long_rows = cols >= 4096;
  if (T <= 16) {
    if (shape.parts > 1 && T <= 8 && values <= 1 << 26) return false;
    return packed || values >= 1 << 24 || (T > 8 && cols >= 2048);
  }
  if (packed) return T <= 32 || rows < 16384 || long_rows;
  return (rows < 32768 || long_rows) && (cols >= 2048 || values >= 1 << 23) && (T <= 32 || shape.parts == 1 || values >= 1 << 24);
}
size_t mx_parts_bytes(int splits, int T, int rows) { return splits > 1 ? (size_t)splits * T * rows * sizeof(float) : 0; }
}  // namespace

// Room for the parts of the sums and, with tiles, for padded scale bytes in front of them, whichever a call of this size needs.
size_t mx_workspace_bytes(int T, int rows, int cols) {
  const size_t tiles =
      mx_tiles(T, rows) ? mx_padded_bytes(T, rows, cols) + mx_parts_bytes(mx_shape(T, rows, cols).splits, T, rows) : 0;
  if (T > kMxFewTokens) return tiles;
  // a call's alignment and tokens may allow the rows to be streamed or not
  int splits = few_splits(T, rows, cols);
  for (const bool packed : {false, true})
    if (mx_streams(T, rows, cols, packed)) {
      const int streams = mx_stream_shape(packed, T, rows, cols).parts;
      if (streams > splits) splits = streams;
    }
  const size_t parts = mx_parts_bytes(splits, T, rows);
  return parts > tiles ? parts : tiles;
}

hipError_t launch_mx_product(const MxProduct& p, hipStream_t s) {
  if (mx_streams(p.T, p.rows, p.cols, p.x_scales != nullptr) && reinterpret_cast<uintptr_t>(p.scales) % 16 == 0)
    return launch_mx_stream(p, s);
  if (!p.x_scales) return launch_few_tokens<false>(p, s);
  if (!mx_tiles(p.T, p.rows)) return launch_few_tokens<true>(p, s);
  const int blocks = p.cols / kMxBlock, words = (blocks + 15) / 16 * 4;
  GemmArgs g{};
  g.a[0] = p.x, g.b[0] = p.codes;
  g.M = p.T, g.N = p.rows, g.K = p.cols / 4, g.lda = g.ldb = (uint32_t)p.cols / 2;
  const ProductShape shape = mx_shape(p.T, p.rows, p.cols);
  g.segments = g.products = 1, g.splits = shape.splits;
  g.a_scales = p.x_scales, g.b_scales = p.scales, g.scale_ld = 4u * words;
  if (mx_pads_scales(p)) {
    uint32_t* padded = static_cast<uint32_t*>(p.workspace);
    auto pad = [&](const uint8_t* from, int rows, uint32_t* to) {
      const long long groups = ((long long)rows * words + 255) / 256;
      return launch(&k_pad_scales, dim3((unsigned)(groups < 4096 ? groups : 4096)), dim3(256), 0, s, from, (long long)rows, blocks,
                    words, to);
    };
    hipError_t e = pad(p.x_scales, p.T, padded);
    if (e == hipSuccess) e = pad(p.scales, p.rows, padded + (size_t)p.T * words);
    if (e != hipSuccess) return e;
    g.a_scales = reinterpret_cast<const uint8_t*>(padded);
    g.b_scales = reinterpret_cast<const uint8_t*>(padded + (size_t)p.T * words);
  }
  if (g.splits == 1) return launch_product<true, true, false, true>(g, shape.tile, StoreProduct{p.y, p.y_bf16}, s);
  float* part = reinterpret_cast<float*>(static_cast<char*>(p.workspace) + mx_padded_bytes(p.T, p.rows, p.cols));
  const hipError_t e = launch_product<true, true, false, true>(g, shape.tile, StoreProduct{part, 0}, s);
  return e != hipSuccess ? e : launch_join_parts(part, p.y, p.y_bf16 != 0, g.splits, (long long)p.T * p.rows, s);
}

}  // namespace hire
