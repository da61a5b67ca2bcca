// The dense gated FFN for up to 64 tokens, forward and backward: bound by reading the three matrices once (6 d d_ff bytes), and by
// writing their gradients.  Tokens are the small side of 16 x 16 x 32 matrix instructions, whose other operand comes straight from
// memory into registers; large layers are streamed through LDS instead (gated_stream.hip).
#include "gated.h"

namespace hire {
namespace {

// ---- the first layer's products ------------------------------------------------------
// g and u of RU times sixteen units for NT times sixteen tokens: one wave's part of k, in steps of 64 that the SLICES waves of a
// workgroup take in turn.  A lane holds 32 bytes of one row of each matrix per step (k 64 s + 16 q ... of row lane % 16, q =
// lane / 16) and of one token of each tile: which k meet in an instruction is the same for both, so any order of them will do.
// Every workgroup starts at another step: rows are a power of two apart more often than not, and where all start with their first
// columns the requests crowd on a few of the memory's channels (one token, d = 2048, 16384 units: 31.6 -> 24.7 us).
// MATRICES: 2, or 1 (the backward pass's product with the second layer's rows).
template <int MATRICES, int NT, int RU, int SLICES>
__device__ __forceinline__ void up_products(const uint16_t* __restrict__ x, int T, int d, int d_ff,
                                            const uint16_t* const (&w)[MATRICES], int unit0, int slice,
                                            f32x4v (&sums)[RU][MATRICES][NT]) {
  const int lane = lane_id(), q = lane >> 4, chunks = d / 8, steps = (chunks + 7) / 8;
  const int turn = (int)((blockIdx.x * 5u) % (unsigned)steps);
  const uint4 *pw[RU][MATRICES], *px[NT];
#pragma unroll
  for (int r = 0; r < RU; ++r)
#pragma unroll
    for (int m = 0; m < MATRICES; ++m)
      pw[r][m] = reinterpret_cast<const uint4*>(w[m] + (size_t)min(unit0 + 16 * r + (lane & 15), d_ff - 1) * d);
#pragma unroll
  for (int t = 0; t < NT; ++t) px[t] = reinterpret_cast<const uint4*>(x + (size_t)min(16 * t + (lane & 15), T - 1) * d);
  auto chunk_of = [&](int s) { return 8 * (s + turn < steps ? s + turn : s + turn - steps) + 2 * q; };
  auto load = [&](int s, uint4 (&wv)[RU][MATRICES][2], uint4 (&xv)[NT][2]) __attribute__((always_inline)) {
    const int c = chunk_of(s), a = min(c, chunks - 1), b = min(c + 1, chunks - 1);
#pragma unroll
    for (int r = 0; r < RU; ++r)
#pragma unroll
      for (int m = 0; m < MATRICES; ++m) wv[r][m][0] = pw[r][m][a], wv[r][m][1] = pw[r][m][b];
#pragma unroll
    for (int t = 0; t < NT; ++t) xv[t][0] = px[t][a], xv[t][1] = px[t][b];
  };
  auto multiply = [&](int s, const uint4 (&wv)[RU][MATRICES][2], const uint4 (&xv)[NT][2]) __attribute__((always_inline)) {
    const int c = chunk_of(s);
#pragma unroll
    for (int e = 0; e < 2; ++e) {
      const uint32_t keep = c + e < chunks ? 0xFFFFFFFFu : 0u;  // behind the end of k both are zeros
      auto masked = [&](const uint4& v) {
        const uint4 m = make_uint4(v.x & keep, v.y & keep, v.z & keep, v.w & keep);
        bf16x8v b;
        __builtin_memcpy(&b, &m, 16);
        return b;
      };
      bf16x8v xf[NT];
#pragma unroll
      for (int t = 0; t < NT; ++t) xf[t] = masked(xv[t][e]);
#pragma unroll
      for (int r = 0; r < RU; ++r) {
        bf16x8v wf[MATRICES];
#pragma unroll
        for (int m = 0; m < MATRICES; ++m) wf[m] = masked(wv[r][m][e]);
#pragma unroll
        for (int t = 0; t < NT; ++t)
#pragma unroll
          for (int m = 0; m < MATRICES; ++m)
            sums[r][m][t] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(wf[m], xf[t], sums[r][m][t], 0, 0, 0);
      }
    }
  };
  uint4 wa[RU][MATRICES][2], xa[NT][2];
  if constexpr (RU > 1) {  // the sums leave room for one step; the waves of a SIMD overlap theirs
    for (int s = slice; s < steps; s += SLICES) {
      load(s, wa, xa);
      multiply(s, wa, xa);
    }
  } else {
    uint4 wb[RU][MATRICES][2], xb[NT][2];
    int s = slice;
    if (s >= steps) return;
    load(s, wa, xa);
    for (; s + SLICES < steps; s += 2 * SLICES) {
      load(s + SLICES, wb, xb);
      multiply(s, wa, xa);
      load(min(s + 2 * SLICES, steps - 1), wa, xa);  // not used where it repeats the last step
      multiply(s + SLICES, wb, xb);
    }
    if (s < steps) multiply(s, wa, xa);
  }
}

// Adds the slices' sums in their order; red: LDS, [SLICES][MATRICES NT 256] of sixteen units.  f(unit, token, sums) for value i.
template <int MATRICES, int NT, int SLICES, typename F>
__device__ __forceinline__ void join_slices(const float* red, int i, F f) {
  const int unit = i & 15, token = i >> 4, at = (token >> 4) * 256 + ((unit >> 2) * 16 + (token & 15)) * 4 + (unit & 3);
  float v[MATRICES];
#pragma unroll
  for (int m = 0; m < MATRICES; ++m) v[m] = red[m * NT * 256 + at];
#pragma unroll
  for (int s = 1; s < SLICES; ++s)
#pragma unroll
    for (int m = 0; m < MATRICES; ++m) v[m] += red[(s * MATRICES + m) * NT * 256 + at];
  f(unit, token, v);
}
template <int MATRICES, int NT>
__device__ __forceinline__ void leave_slice(float* red, const f32x4v (&sums)[MATRICES][NT]) {
#pragma unroll
  for (int m = 0; m < MATRICES; ++m)
#pragma unroll
    for (int t = 0; t < NT; ++t) *reinterpret_cast<f32x4v*>(red + ((m * NT + t) * 64 + lane_id()) * 4) = sums[m][t];
}
__device__ __forceinline__ void put_bf16(uint16_t* to, float v) {
  const __bf16 b = (__bf16)v;
  __builtin_memcpy(to, &b, 2);
}
__device__ __forceinline__ void keep_gated(const GatedKept& kept, size_t at, float g, float u) {
  kept.g[at] = (uint16_t)(__float_as_uint(g) >> 16);
  kept.u[at] = (uint16_t)(__float_as_uint(u) >> 16);
  kept.low[at] = (uint16_t)((__float_as_uint(g) >> 8 & 0xFFu) | (__float_as_uint(u) & 0xFF00u));
}

struct KeptValue {
  uint16_t h, g, u, low;
  __device__ __forceinline__ void load(const GatedKept& kept, size_t at) {
    h = kept.h[at], g = kept.g[at], u = kept.u[at], low = kept.low[at];
  }
  __device__ __forceinline__ float gate() const { return __uint_as_float((uint32_t)g << 16 | (low & 0xFFu) << 8); }
  __device__ __forceinline__ float up() const { return __uint_as_float((uint32_t)u << 16 | (low & 0xFF00u)); }
};

constexpr int kUpWaves = 4;

template <int NT, int RU>
__global__ __launch_bounds__(64 * kUpWaves) void k_gated_up(GatedLayer L, const uint16_t* __restrict__ x, int T, GatedKept kept) {
  __shared__ float red[kUpWaves * 2 * NT * 256];
  const int unit0 = blockIdx.x * 16 * RU;
  f32x4v sums[RU][2][NT] = {};
  up_products<2, NT, RU, kUpWaves>(x, T, L.d, L.d_ff, {L.wg, L.wu}, unit0, wave_id(), sums);
#pragma unroll
  for (int r = 0; r < RU; ++r) {
    if (r > 0) __syncthreads();
    leave_slice<2, NT>(red + wave_id() * 2 * NT * 256, sums[r]);
    __syncthreads();
    for (int i = threadIdx.x; i < NT * 256; i += 64 * kUpWaves)
      join_slices<2, NT, kUpWaves>(red, i, [&](int unit, int token, const float (&v)[2]) {
        const int f = unit0 + 16 * r + unit;
        if (token >= T || f >= L.d_ff) return;
        const size_t at = (size_t)token * L.d_ff + f;
        float slope;
        const float h = activation_of(L.act, v[0], &slope) * v[1];
        put_bf16(kept.h + at, h);
        if (kept.rest) put_bf16(kept.rest + at, bf16_rest(h));
        if (kept.g) keep_gated(kept, at, v[0], v[1]);
      });
  }
}

// The backward pass's first product: dh of the units, and from it and what was kept dg and du.
template <int NT, int RU>
__global__ __launch_bounds__(64 * kUpWaves) void k_gated_slopes(GatedLayer L, const uint16_t* __restrict__ dy, int T, GatedKept kept,
                                                                GatedSlopes to) {
  __shared__ float red[kUpWaves * NT * 256];
  const int unit0 = blockIdx.x * 16 * RU;
  // up to sixteen tokens, a value for each thread: asked for in front of the products
  constexpr bool kAhead = NT == 1;
  KeptValue ahead[RU];
  if constexpr (kAhead) {
#pragma unroll
    for (int r = 0; r < RU; ++r) {
      const int f = min(unit0 + 16 * r + ((int)threadIdx.x & 15), L.d_ff - 1), token = min((int)threadIdx.x >> 4, T - 1);
      ahead[r].load(kept, (size_t)token * L.d_ff + f);
    }
  }
  f32x4v sums[RU][1][NT] = {};
  up_products<1, NT, RU, kUpWaves>(dy, T, L.d, L.d_ff, {L.w2u}, unit0, wave_id(), sums);
#pragma unroll
  for (int r = 0; r < RU; ++r) {
    if (r > 0) __syncthreads();
    leave_slice<1, NT>(red + wave_id() * NT * 256, sums[r]);
    __syncthreads();
    for (int i = threadIdx.x; i < NT * 256; i += 64 * kUpWaves)
      join_slices<1, NT, kUpWaves>(red, i, [&](int unit, int token, const float (&dh)[1]) {
        const int f = unit0 + 16 * r + unit;
        if (token >= T || f >= L.d_ff) return;
        const size_t at = (size_t)token * L.d_ff + f;
        KeptValue k;
        if constexpr (kAhead)
          k = ahead[r];
        else
          k.load(kept, at);
        float slope;
        const float a = activation_of(L.act, k.gate(), &slope);
        const float dg = dh[0] * k.up() * slope, du = dh[0] * a;
        put_bf16(to.dg + at, dg);
        put_bf16(to.du + at, du);
        if (to.dg_rest) {
          put_bf16(to.dg_rest + at, bf16_rest(dg));
          put_bf16(to.du_rest + at, bf16_rest(du));
          put_bf16(to.h_rest + at, rest_of(a * k.up(), bf16_lo(k.h)));
        }
      });
  }
}

// What the rounding left of the kept h, where no other kernel of the backward pass reads g and u.
__global__ __launch_bounds__(256) void k_gated_rest(int act, int values, GatedKept kept, uint16_t* __restrict__ rest) {
  for (int i = blockIdx.x * 256 + threadIdx.x; i < values; i += gridDim.x * 256) {
    KeptValue k;
    k.load(kept, i);
    float slope;
    put_bf16(rest + i, rest_of(activation_of(act, k.gate(), &slope) * k.up(), bf16_lo(k.h)));
  }
}

// ---- the second layer ---------------------------------------------------------------------
// 32 rows by 128 columns of the matrix by NT tiles of tokens: lane l has eight columns (8 (l % 16) ...) of eight rows (8 (l / 16)
// ...).  Column c of the eight, taken from all lanes, is one instruction's operand: its k are the rows, its columns 8 n + c.
__device__ __forceinline__ bf16x8v column_of(const uint4 (&rows)[8], int c) {
  uint32_t d[4];
#pragma unroll
  for (int p = 0; p < 4; ++p) {
    const uint32_t lo[4] = {rows[2 * p].x, rows[2 * p].y, rows[2 * p].z, rows[2 * p].w};
    const uint32_t hi[4] = {rows[2 * p + 1].x, rows[2 * p + 1].y, rows[2 * p + 1].z, rows[2 * p + 1].w};
    d[p] = __builtin_amdgcn_perm(hi[c / 2], lo[c / 2], c % 2 ? 0x07060302u : 0x05040100u);
  }
  bf16x8v v;
  __builtin_memcpy(&v, d, 16);
  return v;
}
// Rows row0 + 8 (l / 16) ... of eight, as far as they lie in front of `end` (others: zeros, nothing of them is used).
__device__ __forceinline__ void load_rows(const uint16_t* __restrict__ w, int d, int chunk, int row0, int end, uint4 (&rows)[8]) {
  const int first = row0 + 8 * (lane_id() >> 4);
#pragma unroll
  for (int r = 0; r < 8; ++r)
    rows[r] = load_streaming(reinterpret_cast<const uint4*>(w + (size_t)min(first + r, end - 1) * d) + chunk);
}
__device__ __forceinline__ void mask_rows(int row0, int end, uint4 (&rows)[8]) {
  const int first = row0 + 8 * (lane_id() >> 4);
#pragma unroll
  for (int r = 0; r < 8; ++r)
    if (first + r >= end) rows[r] = make_uint4(0u, 0u, 0u, 0u);
}

constexpr int kMostStreamParts = 8;

// Parts of the rows: a workgroup for every compute unit, which has its LDS, with two blocks of 32 rows for each of its four
// waves.  us of both layers, 17 / 48 tokens, with one, two, four blocks: d = 512, 8192 units 19.1, 17.1, 17.1 / 23.2, 21.1, 20.8;
// 800, 2504 14.0, 13.4, 15.2 / 16.9, 15.9, 17.6.
int down_parts(int d, int rows) {
  const int columns = (d + 127) / 128, most = rows / (32 * 4 * 2), parts = 256 / columns;
  const int fewer = parts < most ? parts : most;
  return fewer < 1 ? 1 : fewer;
}

// ---- both layers in one kernel: the fewest tokens ---------------------------------------------
// A workgroup takes 16 GROUPS units through both layers: their g and u, h through LDS, and the contribution of their
// rows of the second matrix to y, whose loads go out before the waves join their sums.  The workgroups' parts of y, T d values
// each, are added by k_join_units.
template <int ACT, int GROUPS, int kOneWaves>
__global__ __launch_bounds__(64 * kOneWaves) void k_gated_one(GatedLayer L, const uint16_t* __restrict__ x, int T, GatedKept kept,
                                                              float* __restrict__ part) {
  constexpr int kSlices = kOneWaves / GROUPS, kUnits = 16 * GROUPS, kBlocks = (kUnits + 31) / 32;
  __shared__ float red[kOneWaves * 512];
  __shared__ __align__(16) __bf16 hidden[2][16 * kBlocks * 32];  // and what the rounding left
  const int lane = lane_id(), wave = wave_id(), unit0 = blockIdx.x * kUnits, end = min(unit0 + kUnits, L.d_ff);
  const int group = wave % GROUPS, columns = (L.d + 127) / 128;
  f32x4v products[1][2][1] = {};
  up_products<2, 1, 1, kSlices>(x, T, L.d, L.d_ff, {L.wg, L.wu}, unit0 + 16 * group, wave / GROUPS, products);
  auto chunk_of = [&](int block) { return min(16 * block + (lane & 15), L.d / 8 - 1); };
  uint4 rows[kBlocks][8];
#pragma unroll
  for (int b = 0; b < kBlocks; ++b) load_rows(L.w2u, L.d, chunk_of(min(wave, columns - 1)), unit0 + 32 * b, end, rows[b]);
  leave_slice<2, 1>(red + (group * kSlices + wave / GROUPS) * 512, products[0]);
  for (int i = threadIdx.x; i < 16 * kBlocks * 32; i += 64 * kOneWaves) hidden[0][i] = hidden[1][i] = (__bf16)0.0f;
  __syncthreads();
  for (int i = threadIdx.x; i < GROUPS * 256; i += 64 * kOneWaves)
    join_slices<2, 1, kSlices>(red + i / 256 * kSlices * 512, i % 256, [&](int unit, int token, const float (&v)[2]) {
      const int in = i / 256 * 16 + unit;
      if (token >= T || unit0 + in >= L.d_ff) return;
      float slope;
      const float h = activation<ACT>(v[0], &slope) * v[1];
      hidden[0][token * kBlocks * 32 + in] = (__bf16)h;
      hidden[1][token * kBlocks * 32 + in] = (__bf16)bf16_rest(h);
      const size_t at = (size_t)token * L.d_ff + unit0 + in;
      put_bf16(kept.h + at, h);  // also for k_join_units
      if (kept.g) keep_gated(kept, at, v[0], v[1]);
    });
  __syncthreads();
  for (int block = wave; block < columns; block += kOneWaves) {
    f32x4v acc[8] = {};
#pragma unroll
    for (int b = 0; b < kBlocks; ++b) {
      if (unit0 + 32 * b + 32 > end) mask_rows(unit0 + 32 * b, end, rows[b]);
#pragma unroll
      for (int t = 0; t < 2; ++t) {
        const bf16x8v hf = *reinterpret_cast<const bf16x8v*>(hidden[t] + ((lane & 15) * kBlocks + b) * 32 + 8 * (lane >> 4));
#pragma unroll
        for (int c = 0; c < 8; ++c) acc[c] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(hf, column_of(rows[b], c), acc[c], 0, 0, 0);
      }
      if (block + kOneWaves < columns) load_rows(L.w2u, L.d, chunk_of(block + kOneWaves), unit0 + 32 * b, end, rows[b]);
    }
    const int col = 128 * block + 8 * (lane & 15);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int token = 4 * (lane >> 4) + i;
      if (token < T && col < L.d) {
        float4* to = reinterpret_cast<float4*>(part + ((size_t)blockIdx.x * T + token) * L.d + col);
        to[0] = make_float4(acc[0][i], acc[1][i], acc[2][i], acc[3][i]);
        to[1] = make_float4(acc[4][i], acc[5][i], acc[6][i], acc[7][i]);
      }
    }
  }
}

// Sum of many parts of few values: sixteen threads share four values, each adds every sixteenth part.  A sum that is not finite is that
// of the first terms alone (first_term), which the same threads then form from h and the rows.  In k_gated_one, which would have to
// keep both terms' sums apart, or the rows, this took its registers beyond the 128 of the small layers: 7.3 -> 9.1 us.
__global__ __launch_bounds__(256) void k_join_units(GatedLayer L, const float* __restrict__ part, const uint16_t* __restrict__ h,
                                                    uint16_t* __restrict__ y, int parts, int quads) {
  __shared__ float4 sums[256];
  const int quad = blockIdx.x * 16 + (int)threadIdx.x % 16, at = min(quad, quads - 1);
  float4 s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 8
  for (int r = (int)threadIdx.x / 16; r < parts; r += 16) {
    const float4 v = reinterpret_cast<const float4*>(part)[(size_t)r * quads + at];
    s.x += v.x, s.y += v.y, s.z += v.z, s.w += v.w;
  }
  auto join = [&](const float4& mine, float (&joined)[4]) {
    sums[threadIdx.x] = mine;
    __syncthreads();
    if (threadIdx.x >= 16) return;
    const float4* all = sums + threadIdx.x;
    joined[0] = mine.x, joined[1] = mine.y, joined[2] = mine.z, joined[3] = mine.w;
    for (int r = 1; r < 16; ++r) {
      const float4 v = all[16 * r];
      joined[0] += v.x, joined[1] += v.y, joined[2] += v.z, joined[3] += v.w;
    }
  };
  float f[4];
  join(s, f);
  const bool mine = threadIdx.x < 16 && quad < quads;
  const uint64_t others = __ballot(mine && !all_finite(f));  // the first wave's
  __shared__ int again;
  if (threadIdx.x == 0) again = others != 0ull;
  __syncthreads();
  if (again) {
    const int token = 4 * at / L.d, col = 4 * at % L.d;
    s = make_float4(0.0f, 0.0f, 0.0f, 0.0f);
#pragma unroll 4
    for (int unit = (int)threadIdx.x / 16; unit < L.d_ff; unit += 16) {
      const float hv = bf16_lo(h[(size_t)token * L.d_ff + unit]);
      const uint2 row = *reinterpret_cast<const uint2*>(L.w2u + (size_t)unit * L.d + col);
      s.x = fmaf(hv, bf16_lo(row.x), s.x), s.y = fmaf(hv, bf16_hi(row.x), s.y);
      s.z = fmaf(hv, bf16_lo(row.y), s.z), s.w = fmaf(hv, bf16_hi(row.y), s.w);
    }
    float first[4];
    join(s, first);
#pragma unroll
    for (int e = 0; e < 4; ++e) f[e] = first_term(f[e], first[e]);
  }
  if (mine) reinterpret_cast<uint2*>(y)[quad] = pack4(f);
}

// Sixteens of units of a workgroup: a workgroup for every compute unit, but no more than are resident at once.  d = 2048, one
// token, us with 1 / 2 / 4 of them: 5000 units 26.5 / 18.7 / -, 9000 - / 33.3 / 31.0, 16384 - / 41.7 / 38.3.
int one_groups(int d_ff) {
  const int groups = (d_ff + 15) / 16;
  return groups > 512 ? 4 : (groups > 256 ? 2 : 1);
}
int one_parts(int d_ff) { return (d_ff + 16 * one_groups(d_ff) - 1) / (16 * one_groups(d_ff)); }
// One kernel and the join of its parts saves about 4 us against two and a join.  It loses what its parts take on their way through
// memory (6.5 TB/s there and back) and, where its workgroups come short of the compute units, a part of the matrices' time (at 5.6
// TB/s; three quarters of the units are enough for all of it).  us, one kernel / two: d = 2048, 16384 units, one token 39.3 / 43.5,
// four 40.6 / 43.9, eight 43.3 / 44.2; 2560, 10240 (160 workgroups), one 43.3 / 37.4; 2048, 20000 (313), one 62.0 / 50.1; 4096,
// 8192, two 43.6 / 45.4, four 46.6 / 46.2; 1024, 4096, four 13.3 / 15.1, sixteen 18.4 / 15.7; 512, 2048, sixteen 11.2 / 13.0;
// 256, 1024, one 7.6 / 8.8.  Over 25 such layers and up to sixteen tokens it is at most 14 % off.
bool one_kernel(int T, int d, int d_ff) {
  if (T > 16) return false;
  const int parts = one_parts(d_ff), rounds = (parts + 255) / 256;
  const double filled = 1.35 * parts / (256.0 * rounds), matrices = 6.0 * d * d_ff / 5.6e6;
  const double lost = (double)parts * T * d * 8.0 / 6.5e6 + (filled < 1.0 ? matrices * (1.0 / filled - 1.0) : 0.0);
  return lost <= 4.0;
}

template <int GROUPS, int kOneWaves>
hipError_t launch_one(const GatedLayer& L, const uint16_t* x, int T, uint16_t* y, const GatedKept& kept, float* part, hipStream_t s) {
  const int parts = one_parts(L.d_ff), quads = T * L.d / 4;
  const hipError_t e = with_activation(L.act, [&](auto act) {
    return launch(&k_gated_one<decltype(act)::value, GROUPS, kOneWaves>, dim3((unsigned)parts), dim3(64 * kOneWaves), 0, s, L, x, T, kept, part);
  });
  return e != hipSuccess ? e
                         : launch(&k_join_units, dim3((unsigned)((quads + 15) / 16)), dim3(256), 0, s, L, part, kept.h, y, parts,
                                  quads);
}

// out = the sum over the pairs' rows, in parts where they are many.
hipError_t launch_down(const GatedDown& from, int T, int d, int d_ff, uint16_t* out, float* part, hipStream_t s) {
  const int parts = down_parts(d, from.pairs * d_ff);
  const hipError_t e = launch_gated_down_stream(from, T, d, d_ff, parts, out, part, s);
  if (e != hipSuccess || parts == 1) return e;
  return launch_join_parts(part, out, true, parts, (long long)T * d, s);
}

// The first layer's rows streamed past the tokens (gated_stream.hip): where they keep every compute unit at it for a while.  us of
// both layers without / with it, 17 / 48 tokens: d = 2048, 16384 units 49.7, 48.6 / 58.9, 53.7; 2560, 10240 57.9, 41.3 / 71.5,
// 47.9; 8192, 8192 98, 88 / 121, 93; 1024, 8192 24.1, 23.3 / 28.9, 27.3; not 1024, 4096 16.7, 17.4 / 20.7, 22.5 or 512, 8192 17.4,
// 18.8 / 21.5, 23.8.
bool few_streams(int d, int d_ff) { return d >= 1024 && (long long)d * d_ff >= 1 << 23 && gated_stream_parts(d) <= kMostStreamParts; }

template <int NT, int RU>
hipError_t launch_few(const GatedLayer& L, const uint16_t* x, int T, uint16_t* y, const GatedKept& kept, float* part, hipStream_t s) {
  const hipError_t e = few_streams(L.d, L.d_ff) ? launch_gated_stream(L, x, T, kept, part, s)
                                               : launch(&k_gated_up<NT, RU>, dim3((unsigned)((L.d_ff + 16 * RU - 1) / (16 * RU))),
                                                        dim3(64 * kUpWaves), 0, s, L, x, T, kept);
  if (e != hipSuccess) return e;
  return launch_down(GatedDown{{L.w2u, nullptr}, {kept.h, nullptr}, {kept.rest, nullptr}, 1}, T, L.d, L.d_ff, y, part, s);
}

template <int NT>
hipError_t launch_slopes(const GatedLayer& L, const uint16_t* dy, int T, const GatedKept& kept, const GatedSlopes& slopes,
                         hipStream_t s) {
  const int groups = (L.d_ff + 15) / 16;
  if (groups >= 2 * 256)
    return launch(&k_gated_slopes<NT, 2>, dim3((unsigned)((groups + 1) / 2)), dim3(64 * kUpWaves), 0, s, L, dy, T, kept, slopes);
  return launch(&k_gated_slopes<NT, 1>, dim3((unsigned)groups), dim3(64 * kUpWaves), 0, s, L, dy, T, kept, slopes);
}

// ---- the weights' gradients -------------------------------------------------------------------
// out[f, c] = sum over the tokens of a[token, f] b[token, c], bound by writing it.  A workgroup has both operands of its 128 x 128
// tile in LDS as a whole (32 tokens STEPS times), so little of it that four share a compute unit and fill each other's waits.  d =
// 2048, 16384 units, one token, us of the three: 75 as tiles of the many tokens' kernel, 60 this way, 36 with streaming stores.
//   REST, up to sixteen tokens: a's second terms are k 16 ... of the one stage, with the same tokens of b.
template <int STEPS, bool REST>
__global__ __launch_bounds__(256) void k_gated_outer(GemmArgs g, GatedRests rest, StoreBf16<true> out) {
  static_assert(!REST || (STEPS == 1 && kGatedRestTokens == 16), "two terms of sixteen tokens in a stage");
  using Tile = GemmTile<128, 4, false, false>;
  constexpr int kTiles = 2 * STEPS * Tile::kBytes, kRows = 4 * 32 * kRowFloats * 4;
  __shared__ __align__(1024) char smem[kTiles > kRows ? kTiles : kRows];
  const int tiles_m = (g.M + 127) / 128, tiles_n = (g.N + 127) / 128, tiles = tiles_m * tiles_n;
  const int w = gemm_place((int)blockIdx.x, (int)gridDim.x), product = w / tiles, t = w % tiles;
  const int m0 = t / tiles_n * 128, n0 = t % tiles_n * 128, wave = __builtin_amdgcn_readfirstlane(wave_id());
  Tile ta, tb;
  ta.init(m0, g.M, g.lda);
  tb.init(n0, g.N, g.ldb);
  const uint32_t lds0 = __builtin_amdgcn_readfirstlane(gemm_lds_offset(smem));
  const char* a = static_cast<const char*>(g.a[product]) + 2 * (size_t)m0;
  const char* b = static_cast<const char*>(g.b[product]) + 2 * (size_t)n0;
  if constexpr (REST) {
    const char* r = reinterpret_cast<const char*>(rest.of[product]) + 2 * (size_t)m0;
#pragma unroll
    for (int i = 0; i < Tile::kLoads; ++i) {
      const int piece = i * 4 + wave, k = Tile::k_of_lane(piece);
      const bool there = (k & 15) < g.K;
      const char* from_a = (k < 16 ? a : r) + (ta.off[i] - (uint32_t)(k & 16) * g.lda);
      const char* from_b = b + (tb.off[i] - (uint32_t)(k & 16) * g.ldb);
      gemm_load_at(there ? (const void*)from_a : (const void*)kGemmZeros, lds0 + piece * 1024);
      gemm_load_at(there ? (const void*)from_b : (const void*)kGemmZeros, lds0 + Tile::kBytes + piece * 1024);
    }
  }
#pragma unroll
  for (int s = 0; s < (REST ? 0 : STEPS); ++s) {
    const int k = s * kGemmStep;
    ta.request(a + (size_t)k * g.lda, nullptr, g.K - k, lds0 + 2 * s * Tile::kBytes, wave);
    tb.request(b + (size_t)k * g.ldb, nullptr, g.K - k, lds0 + (2 * s + 1) * Tile::kBytes, wave);
  }
  asm volatile("s_waitcnt vmcnt(0)\n\ts_barrier" ::: "memory");
  const int wm = wave / 2 * 64, wn = wave % 2 * 64;
  f32x16v acc[2][2] = {};
#pragma unroll
  for (int s = 0; s < STEPS; ++s)
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      bf16x8v fa[2], fb[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
        fa[i] = Tile::fragment(smem + 2 * s * Tile::kBytes, wm + 32 * i, ks);
        fb[i] = Tile::fragment(smem + (2 * s + 1) * Tile::kBytes, wn + 32 * i, ks);
      }
#pragma unroll
      for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) acc[i][j] = __builtin_amdgcn_mfma_f32_32x32x16_bf16(fb[j], fa[i], acc[i][j], 0, 0, 0);
    }
  lds_barrier();  // LDS is the epilogue's
  if constexpr (REST) {
    for_rows<false>(acc, smem, m0 + wm, n0 + wn, g.M, g.N, NoFetch{}, [&](int m, int n, const float (&sums)[1][8], int) {
      uint16_t* to = out.c[product] + (size_t)m * g.N + n;
      store_streaming(to, pack8(sums[0]));
      if (all_finite(sums[0])) return;
      uint32_t other = 0u;  // columns that are the first terms' (a loop, for little code)
#pragma unroll
      for (int e = 0; e < 8; ++e) other |= (fabsf(sums[0][e]) <= kLargestFloat ? 0u : 1u) << e;
#pragma unroll 1
      for (int e = 0; e < 8; ++e) {
        if ((other >> e & 1u) == 0u) continue;
        const uint16_t* of_a = static_cast<const uint16_t*>(g.a[product]) + m;
        const uint16_t* of_b = static_cast<const uint16_t*>(g.b[product]) + n + e;
        float first = 0.0f;
#pragma unroll 1
        for (int k = 0; k < g.K; ++k)
          first = fmaf(bf16_lo(of_a[(size_t)k * (g.lda / 2)]), bf16_lo(of_b[(size_t)k * (g.ldb / 2)]), first);
        put_bf16(to + e, first);
      }
    });
  } else {
    out.store(acc, smem, m0 + wm, n0 + wn, g.M, g.N, product, 0);
  }
}

// f with the number of tiles of sixteen tokens as a type.
template <typename F>
hipError_t with_tiles(int T, F f) {
  switch ((T + 15) / 16) {
    case 1: return f(std::integral_constant<int, 1>{});
    case 2: return f(std::integral_constant<int, 2>{});
    case 3: return f(std::integral_constant<int, 3>{});
    default: return f(std::integral_constant<int, 4>{});
  }
}

// Units of a workgroup of the first layer, in sixteens.  More of them share what is read of the tokens, which comes from the L2
// for every workgroup; but 256 workgroups should be left.
template <int NT, int WIDEST>
hipError_t launch_few_by_width(const GatedLayer& L, const uint16_t* x, int T, uint16_t* y, const GatedKept& kept, float* part,
                               hipStream_t s) {
  const int groups = (L.d_ff + 15) / 16;
  if constexpr (WIDEST >= 4)
    if (groups >= 4 * 256) return launch_few<NT, 4>(L, x, T, y, kept, part, s);
  if (groups >= 2 * 256) return launch_few<NT, 2>(L, x, T, y, kept, part, s);
  return launch_few<NT, 1>(L, x, T, y, kept, part, s);
}

}  // namespace

size_t gated_few_part_bytes(int T, int d, int d_ff, int pairs) {
  if (pairs == 1 && one_kernel(T, d, d_ff)) return (size_t)one_parts(d_ff) * T * d * sizeof(float);
  const int parts = down_parts(d, pairs * d_ff), streams = few_streams(d, d_ff) ? gated_stream_parts(d) : 1;
  const size_t down = parts > 1 ? (size_t)parts * T * d * sizeof(float) : 0;
  const size_t up = streams > 1 ? (pairs == 1 ? 2 : 1) * (size_t)streams * T * d_ff * sizeof(float) : 0;  // g and u, or dh
  return down > up ? down : up;
}

hipError_t launch_gated_few(const GatedLayer& L, const uint16_t* x, int T, uint16_t* y, const GatedKept& kept, float* part,
                            hipStream_t s) {
  if (one_kernel(T, L.d, L.d_ff)) {
    const int groups = one_groups(L.d_ff);
    if (groups == 4) return launch_one<4, 8>(L, x, T, y, kept, part, s);
    return groups == 2 ? launch_one<2, 8>(L, x, T, y, kept, part, s) : launch_one<1, 16>(L, x, T, y, kept, part, s);
  }
  return with_tiles(T, [&](auto tiles) {
    constexpr int NT = decltype(tiles)::value;
    return launch_few_by_width<NT, NT <= 2 ? 2 : 4>(L, x, T, y, kept, part, s);
  });
}

hipError_t launch_gated_few_slopes(const GatedLayer& L, const uint16_t* dy, int T, const GatedKept& kept, const GatedSlopes& slopes,
                                   float* part, hipStream_t s) {
  // streamed or not, us of this and dx: 17 / 64 tokens, d = 2560, 10240 units 45.7 / 57.8, 51.0 / 72.0, 8192, 2048 32.4 / 40.9, 38.3 /
  // 64.6, 2048, 16384 50.3 / 64.2, 52.6 / 69.9; sixteen 48.6, 47.6; of 1024, 8192 23.9 / 35.5, 22.2 / 30.7
  if (T > 16 && few_streams(L.d, L.d_ff) && (long long)L.d * L.d_ff >= 1 << 24)
    return launch_gated_stream_slopes(L, dy, T, kept, slopes.dg, slopes.du, part, s);
  return with_tiles(T, [&](auto tiles) { return launch_slopes<decltype(tiles)::value>(L, dy, T, kept, slopes, s); });
}

hipError_t launch_gated_few_weights(const GemmArgs& g, const GatedRests& rest, const StoreBf16<true>& out, hipStream_t s) {
  const long long tiles = (long long)((g.M + 127) / 128) * ((g.N + 127) / 128) * g.products;
  const auto kernel = rest.of[0] ? &k_gated_outer<1, true> : (g.K <= kGemmStep ? &k_gated_outer<1, false> : &k_gated_outer<2, false>);
  return launch(kernel, dim3((unsigned)tiles), dim3(256), 0, s, g, rest, out);
}

hipError_t launch_gated_rest(const GatedLayer& L, int T, const GatedKept& kept, uint16_t* rest, hipStream_t s) {
  const int values = T * L.d_ff;
  return launch(&k_gated_rest, dim3(join_blocks(values)), dim3(256), 0, s, L.act, values, kept, rest);
}

hipError_t launch_gated_few_dx(const GatedLayer& L, int T, const GatedSlopes& slopes, uint16_t* dx, float* part, hipStream_t s) {
  return launch_down(GatedDown{{L.wg, L.wu}, {slopes.dg, slopes.du}, {slopes.dg_rest, slopes.du_rest}, 2}, T, L.d, L.d_ff, dx, part,
                     s);
}

}  // namespace hire
