// Verification of drafted tokens: which of them the target's probabilities accept under given random numbers, and the token
// that follows, drawn from what the draft leaves of the target's distribution.
//   token i is accepted iff u_i q_i(d_i) < p_i(d_i); behind a accepted ones the next token is the first v with
//   sum_{w <= v} r(w) > s sum_w r(w),  r = max(p_a - q_a, 0) where token a was refused, p_a where none was left
// Probabilities are fp32 and everything computed from them is fp64: products are exact, differences all but (one rounding of 2^-53), and
// a running sum has at most some 130 additions behind one another (dense: 70 to the sum of a slice, 16 over the slices, 44 in the
// slice), so that it is off by less than 2^-45 of the whole.  A token's even share of the largest vocabulary is 2^-22 of it.  A
// mark s times the whole that lies within 2^-45 of the border between two tokens may thus fall to either.
#include "kernels.h"
#include "select.h"

#include <type_traits>

namespace hire {
namespace {

constexpr int kVerifyThreads = 256;  // one workgroup for a sequence; or that sums a part of a dense row
constexpr int kVerifyWaves = kVerifyThreads / kWave;
constexpr int kPartSlices = kVerifyWaves;  // of a part, one per wave

// Places of the first entries of two lists that name a token, -1: none (k = 0: no list); whole wave, every lane gets them.
__device__ __forceinline__ void find_in_lists(const int32_t* a, int ka, const int32_t* b, int kb, int token, int* at_a, int* at_b) {
  constexpr int kAhead = 8;  // loads of each list under way
  *at_a = *at_b = -1;
  for (int j0 = 0; j0 < ka || j0 < kb; j0 += kWave * kAhead) {
    int32_t of_a[kAhead], of_b[kAhead];
    const bool more_a = j0 < ka && *at_a < 0, more_b = j0 < kb && *at_b < 0;  // uniform
    if (!more_a && !more_b) return;
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int j = j0 + u * kWave + lane_id();
      if (more_a) of_a[u] = a[min(j, ka - 1)];
      if (more_b) of_b[u] = b[min(j, kb - 1)];
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      const int j = j0 + u * kWave + lane_id();
      const uint64_t hit_a = __ballot(more_a && j < ka && of_a[u] == token), hit_b = __ballot(more_b && j < kb && of_b[u] == token);
      if (*at_a < 0 && hit_a != 0ull) *at_a = j0 + u * kWave + (int)__builtin_ctzll(hit_a);
      if (*at_b < 0 && hit_b != 0ull) *at_b = j0 + u * kWave + (int)__builtin_ctzll(hit_b);
    }
  }
}

__device__ __forceinline__ const float* target_row(const DraftArgs& a, int b, int i) {
  return a.target + ((size_t)b * (a.n + 1) + i) * (a.target_idx ? a.target_k : a.vocab);
}
__device__ __forceinline__ const int32_t* target_list(const DraftArgs& a, int b, int i) {
  return a.target_idx + ((size_t)b * (a.n + 1) + i) * a.target_k;
}
__device__ __forceinline__ const float* draft_row(const DraftArgs& a, int b, int i) {
  return a.draft + ((size_t)b * a.n + i) * (a.draft_idx ? a.draft_k : a.vocab);
}
__device__ __forceinline__ const int32_t* draft_list(const DraftArgs& a, int b, int i) {
  return a.draft_idx + ((size_t)b * a.n + i) * a.draft_k;
}
__device__ __forceinline__ int draft_length(const DraftArgs& a, int b) {
  return a.lengths ? min(max(a.lengths[b], 0), a.n) : a.n;
}

// Number of accepted tokens of sequence b, for the whole workgroup; ok: LDS, kMaxDraft words.
__device__ __forceinline__ int accepted_tokens(const DraftArgs& a, int b, int length, int* ok) {
  auto drafted = [&](int i) { return a.tokens[(size_t)b * a.n + i]; };
  auto decide = [&](int i, float p, float q) { return (double)a.accept_u[(size_t)b * a.n + i] * (double)q < (double)p ? 1 : 0; };
  if (!a.target_idx && !a.draft_idx) {  // a lane for each token
    const int i = (int)threadIdx.x;
    if (i < kMaxDraft && i < length) {
      const int d = drafted(i);
      ok[i] = (unsigned)d < (unsigned)a.vocab ? decide(i, target_row(a, b, i)[d], a.draft ? draft_row(a, b, i)[d] : 1.0f) : 0;
    }
  } else {  // a wave for each
    for (int i = wave_id(); i < length; i += (int)(blockDim.x / kWave)) {
      const int d = drafted(i);
      int yes = 0;
      if ((unsigned)d < (unsigned)a.vocab) {
        int in_p, in_q;
        find_in_lists(a.target_idx ? target_list(a, b, i) : nullptr, a.target_idx ? a.target_k : 0,
                      a.draft_idx ? draft_list(a, b, i) : nullptr, a.draft_idx ? a.draft_k : 0, d, &in_p, &in_q);
        if (!a.target_idx) in_p = d;
        if (!a.draft_idx) in_q = d;
        const float p = in_p >= 0 ? target_row(a, b, i)[in_p] : 0.0f;
        const float q = !a.draft ? 1.0f : (in_q >= 0 ? draft_row(a, b, i)[in_q] : 0.0f);
        yes = decide(i, p, q);
      }
      if (lane_id() == 0) ok[i] = yes;
    }
  }
  __syncthreads();
  const bool refused = lane_id() < length && ok[min(lane_id(), kMaxDraft - 1)] == 0;
  const uint64_t mask = __ballot(refused);
  return mask == 0ull ? length : __builtin_ctzll(mask);
}

// Two sums over the workgroup's threads, in front of each thread and of all of them, in a fixed order.
struct Running {
  double before[2], total[2];
};
template <int WAVES>
__device__ __forceinline__ Running running_sums(double x, double y, double (&waves)[2][WAVES]) {
  auto add = [](double p, double q) { return p + q; };
  const double ix = wave_prefix(x, 0.0, add), iy = wave_prefix(y, 0.0, add);
  if (lane_id() == kWave - 1) waves[0][wave_id()] = ix, waves[1][wave_id()] = iy;
  __syncthreads();
  Running r{{0.0, 0.0}, {0.0, 0.0}};
#pragma unroll
  for (int w = 0; w < WAVES; ++w) {
    if (w == wave_id()) r.before[0] = r.total[0], r.before[1] = r.total[1];
    r.total[0] += waves[0][w];
    r.total[1] += waves[1][w];
  }
  // a starting point only, which may be off in its last place: the search takes the first value that goes beyond the mark
  r.before[0] += ix - x;
  r.before[1] += iy - y;
  return r;
}

// Thread t has the values w[0 ... EACH - 1] of places EACH t ...; the first place whose running sum is beyond the mark, else the
// last one with a positive value, else -1.  *start: the running sum in front of it.
struct Found {
  int hit, last;
  double before_hit, before_last;
};
template <int EACH, int WAVES>
__device__ __forceinline__ int find_place(const double (&w)[EACH], double before, double mark, Found (&waves)[WAVES],
                                          double* start) {
  Found f{-1, -1, 0.0, 0.0};
  double sum = before;
#pragma unroll
  for (int e = 0; e < EACH; ++e)
    if (w[e] > 0.0) {
      f.last = (int)threadIdx.x * EACH + e;
      f.before_last = sum;
      sum += w[e];
      if (f.hit < 0 && sum > mark) f.hit = f.last, f.before_hit = f.before_last;
    }
  const uint64_t hits = __ballot(f.hit >= 0), any = __ballot(f.last >= 0);
  const int h = hits ? (int)__builtin_ctzll(hits) : 0, l = any ? 63 - (int)__builtin_clzll(any) : 0;
  f = Found{read_lane(f.hit, h), read_lane(f.last, l), read_lane(f.before_hit, h), read_lane(f.before_last, l)};
  if (lane_id() == 0) waves[wave_id()] = f;
  __syncthreads();
  Found r{-1, -1, 0.0, 0.0};
#pragma unroll
  for (int v = WAVES - 1; v >= 0; --v) {
    const Found o = waves[v];
    if (o.hit >= 0) r.hit = o.hit, r.before_hit = o.before_hit;
    if (r.last < 0 && o.last >= 0) r.last = o.last, r.before_last = o.before_last;
  }
  *start = r.hit >= 0 ? r.before_hit : r.before_last;
  return r.hit >= 0 ? r.hit : r.last;
}

__device__ __forceinline__ void write_tokens(const DraftArgs& a, int b, int accepted, int next) {
  for (int i = threadIdx.x; i <= a.n; i += blockDim.x)
    a.out_tokens[(size_t)b * (a.n + 1) + i] = i < accepted ? a.tokens[(size_t)b * a.n + i] : (i == accepted ? next : -1);
  if (threadIdx.x == 0) a.accepted[b] = accepted;
}

// ---- target as lists: a workgroup per sequence ------------------------------------
// Bound by the chain of its steps, not by bytes.  Four drafted tokens, 64 sequences, lists of 1024 of 32000 tokens: 16.9 us (21.3
// with four waves, four entries in a thread).
// A table in LDS tells for a token the first place of a list that names it: open addressing, at most half full.
struct PlaceTable {
  int32_t* key;
  int32_t* place;
  int mask;
  __device__ __forceinline__ void clear() const {
    for (int i = threadIdx.x; i <= mask; i += (int)blockDim.x) key[i] = -1, place[i] = 0x7FFFFFFF;
    __syncthreads();
  }
  __device__ __forceinline__ int slot(int token) const { return (int)((uint32_t)token * 2654435761u >> 16) & mask; }
  __device__ __forceinline__ void insert(int token, int at) const {
    for (int s = slot(token);; s = (s + 1) & mask) {
      const int was = atomicCAS(&key[s], -1, token);
      if (was == -1 || was == token) {
        atomicMin(&place[s], at);
        return;
      }
    }
  }
  __device__ __forceinline__ int find(int token) const {  // 0x7FFFFFFF: not there
    for (int s = slot(token);; s = (s + 1) & mask) {
      if (key[s] == token) return place[s];
      if (key[s] == -1) return 0x7FFFFFFF;
    }
  }
};

template <int THREADS, int EACH>  // places of a thread
__global__ __launch_bounds__(THREADS) void k_verify_lists(DraftArgs a) {
  constexpr int kSlots = 2 * EACH * THREADS;
  __shared__ int ok[kMaxDraft];
  __shared__ double waves[2][THREADS / kWave];
  __shared__ Found found[THREADS / kWave];
  __shared__ int32_t keys[kSlots], places[kSlots];
  const int b = blockIdx.x, length = draft_length(a, b);
  const double sample = (double)a.sample_u[b];
  const PlaceTable table{keys, places, kSlots - 1};
  table.clear();
  const int accepted = accepted_tokens(a, b, length, ok);
  const float* p = target_row(a, b, accepted);
  const int32_t* tokens = target_list(a, b, accepted);
  const bool refused = accepted < length, by_list = refused && a.draft_idx;
  const int first = (int)threadIdx.x * EACH;

  int token[EACH], other[EACH];
  double whole[EACH], rest[EACH];
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    const int at = min(first + i, a.target_k - 1);
    token[i] = tokens[at];
    whole[i] = (double)p[at];
    if (by_list) other[i] = draft_list(a, b, accepted)[min((int)threadIdx.x + i * THREADS, a.draft_k - 1)];
  }
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    if (first + i >= a.target_k || (unsigned)token[i] >= (unsigned)a.vocab) token[i] = -1;
    if (token[i] >= 0) table.insert(token[i], first + i);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < EACH; ++i)
    if (token[i] < 0 || table.find(token[i]) != first + i || !(whole[i] > 0.0)) whole[i] = 0.0, token[i] = -1;
  if (by_list) {
    __syncthreads();
    table.clear();
#pragma unroll
    for (int i = 0; i < EACH; ++i) {
      const int j = (int)threadIdx.x + i * THREADS;
      if (j < a.draft_k && (unsigned)other[i] < (unsigned)a.vocab) table.insert(other[i], j);
    }
    __syncthreads();
  }
  double sums[2] = {0.0, 0.0};
#pragma unroll
  for (int i = 0; i < EACH; ++i) {
    double q = 0.0;
    if (refused && token[i] >= 0) {
      if (a.draft_idx) {
        const int at = table.find(token[i]);
        if (at != 0x7FFFFFFF) q = (double)draft_row(a, b, accepted)[at];
      } else if (a.draft) {
        q = (double)draft_row(a, b, accepted)[token[i]];
      } else {
        q = token[i] == a.tokens[(size_t)b * a.n + accepted] ? 1.0 : 0.0;
      }
    }
    rest[i] = fmax(whole[i] - q, 0.0);
    sums[0] += rest[i];
    sums[1] += whole[i];
  }
  const Running r = running_sums(sums[0], sums[1], waves);
  const bool nothing = !(r.total[0] > 0.0);  // the draft's covers the target's everywhere: the target's itself
#pragma unroll
  for (int i = 0; i < EACH; ++i) rest[i] = nothing ? whole[i] : rest[i];
  double start;
  const int at = find_place(rest, nothing ? r.before[1] : r.before[0], sample * (nothing ? r.total[1] : r.total[0]), found,
                                  &start);
  write_tokens(a, b, accepted, at >= 0 ? tokens[at] : -1);
}

// Short lists (or a draft that was certain): a wave for every position takes its lists into registers before it is known which
// positions are reached, so that everything is asked for at once; the wave of the position behind the accepted tokens then does
// the rest alone.  Eight sequences of four drafted tokens with lists of 64: 5.9 us (12.6 by a workgroup
// that takes one step after the other, as k_verify_lists does).
constexpr int kShortEach = 4;                       // entries of a lane
constexpr int kShortList = kShortEach * kWave;      // longest list
constexpr int kShortWaves = 16;                     // most positions
template <int EACH>
struct ShortList {
  int token[EACH];
  float prob[EACH];
  __device__ __forceinline__ void load(const float* p, const int32_t* idx, int k, bool there) {
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const int j = e * kWave + lane_id(), at = there && j < k ? j : 0;
      token[e] = idx[at];
      prob[e] = p[at];
      if (!there || j >= k) token[e] = -1, prob[e] = 0.0f;
    }
  }
  // Probability of `wanted` by the first entry that names it.
  __device__ __forceinline__ float find(int wanted) const {
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      const uint64_t hit = __ballot(token[e] == wanted);
      if (hit != 0ull) return read_lane(prob[e], (int)__builtin_ctzll(hit));
    }
    return 0.0f;
  }
};

template <int EACH>
__global__ __launch_bounds__(kWave* kShortWaves) void k_verify_short(DraftArgs a) {
  __shared__ int ok[kShortWaves];
  __shared__ int32_t keys[2 * kShortList], places[2 * kShortList];
  const int b = blockIdx.x, i = __builtin_amdgcn_readfirstlane(wave_id()), lane = lane_id();
  const bool drafted = i < a.n;
  const size_t at = (size_t)b * a.n + (drafted ? i : 0);
  ShortList<EACH> p, q;
  p.load(target_row(a, b, i), target_list(a, b, i), a.target_k, true);
  if (a.draft) q.load(draft_row(a, b, drafted ? i : 0), draft_list(a, b, drafted ? i : 0), a.draft_k, drafted);
  const int length = draft_length(a, b), token = drafted ? a.tokens[at] : -1;
  const float u = drafted ? a.accept_u[at] : 0.0f, mark_at = a.sample_u[b];
  int yes = 0;
  if (i < length && (unsigned)token < (unsigned)a.vocab)
    yes = (double)u * (a.draft ? (double)q.find(token) : 1.0) < (double)p.find(token) ? 1 : 0;
  if (lane == 0) ok[i] = yes;
  __syncthreads();
  const uint64_t refusals = __ballot(lane < length && ok[min(lane, kShortWaves - 1)] == 0);
  const int accepted = refusals == 0ull ? length : (int)__builtin_ctzll(refusals);
  int32_t* out = a.out_tokens + (size_t)b * (a.n + 1);
  if (i != accepted) {
    if (lane == 0) out[i] = i < accepted ? token : -1;
    return;
  }
  // this wave alone from here on: LDS in the order of the program
  const bool refused = accepted < length;
  PlaceTable table{keys, places, 2 * kWave * EACH - 1};
  auto clear = [&]() {
    for (int j = lane; j <= table.mask; j += kWave) keys[j] = -1, places[j] = 0x7FFFFFFF;
    __builtin_amdgcn_wave_barrier();
  };
  clear();
  double whole[EACH], rest[EACH];
#pragma unroll
  for (int e = 0; e < EACH; ++e)
    if ((unsigned)p.token[e] < (unsigned)a.vocab) table.insert(p.token[e], e * kWave + lane);
  __builtin_amdgcn_wave_barrier();
#pragma unroll
  for (int e = 0; e < EACH; ++e) {
    const bool first = (unsigned)p.token[e] < (unsigned)a.vocab && table.find(p.token[e]) == e * kWave + lane;
    whole[e] = first && p.prob[e] > 0.0f ? (double)p.prob[e] : 0.0;
    rest[e] = whole[e];
  }
  if (refused && !a.draft) {
#pragma unroll
    for (int e = 0; e < EACH; ++e)
      if (p.token[e] == token) rest[e] = fmax(whole[e] - 1.0, 0.0);
  } else if (refused) {
    __builtin_amdgcn_wave_barrier();
    clear();
#pragma unroll
    for (int e = 0; e < EACH; ++e)
      if ((unsigned)q.token[e] < (unsigned)a.vocab) table.insert(q.token[e], e * kWave + lane);
    __builtin_amdgcn_wave_barrier();
    // Probabilities by place, in the keys' words once the places are found: as bits of the same type, for a store through another
    // one may be moved in front of the reads of the keys, and the barriers here are the wave's only
    int found[EACH];
#pragma unroll
    for (int e = 0; e < EACH; ++e) found[e] = whole[e] > 0.0 ? table.find(p.token[e]) : 0x7FFFFFFF;
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int e = 0; e < EACH; ++e) keys[e * kWave + lane] = __float_as_int(q.prob[e]);
    __builtin_amdgcn_wave_barrier();
#pragma unroll
    for (int e = 0; e < EACH; ++e)
      if (found[e] != 0x7FFFFFFF) rest[e] = fmax(whole[e] - (double)__int_as_float(keys[found[e]]), 0.0);
  }
  // running sums in the order of the places: blocks of 64 one after the other
  auto pick = [&](const double (&w)[EACH], int* next) {
    double sums[EACH], total = 0.0;
#pragma unroll
    for (int e = 0; e < EACH; ++e) {
      sums[e] = total + wave_prefix(w[e], 0.0, [](double x, double y) { return x + y; });
      total = read_lane63(sums[e]);
    }
    if (!(total > 0.0)) return false;
    const double mark = (double)mark_at * total;
    int last = -1;
#pragma unroll
    for (int e = EACH - 1; e >= 0; --e) {
      const uint64_t beyond = __ballot(w[e] > 0.0 && sums[e] > mark), any = __ballot(w[e] > 0.0);
      if (beyond != 0ull) *next = read_lane(p.token[e], (int)__builtin_ctzll(beyond)), last = -2;
      if (last == -1 && any != 0ull) last = e;
      if (last == e) *next = read_lane(p.token[e], 63 - (int)__builtin_clzll(any));
    }
    return true;
  };
  int next = -1;
  if (!pick(rest, &next)) pick(whole, &next);
  if (lane == 0) {
    out[i] = next;
    a.accepted[b] = accepted;
  }
}

// ---- target dense: parts of the row in workgroups of their own, then one per sequence --------
// The draft's probabilities of a part's tokens, q(v) for v of [v0, v0 + size): from the row, from the list's entries that fall
// into the part (their places are left in LDS), or of the one token.
enum { kDraftCertain, kDraftDense, kDraftList };
template <int KIND>
struct PartDraft {
  const float* row;
  int32_t* places;
  int v0, token;
  bool refused;  // nothing is taken off where all tokens were accepted
  __device__ __forceinline__ double at(int v) const {
    if (!refused) return 0.0;
    if constexpr (KIND == kDraftDense) return (double)row[v];
    if constexpr (KIND == kDraftList) {
      const int j = places[v - v0];
      return j != 0x7FFFFFFF ? (double)row[j] : 0.0;
    }
    return v == token ? 1.0 : 0.0;
  }
};
template <int KIND>
__device__ __forceinline__ PartDraft<KIND> part_draft(const DraftArgs& a, int b, int accepted, bool refused, int v0, int size,
                                                int32_t* places) {
  PartDraft<KIND> d{nullptr, places, v0, -1, refused};
  if (!refused) return d;
  if constexpr (KIND == kDraftCertain) {
    d.token = a.tokens[(size_t)b * a.n + accepted];
    return d;
  }
  d.row = draft_row(a, b, accepted);
  if constexpr (KIND == kDraftList) {
    const int4 none = make_int4(0x7FFFFFFF, 0x7FFFFFFF, 0x7FFFFFFF, 0x7FFFFFFF);
    for (int i = threadIdx.x; i < size / 4; i += blockDim.x) reinterpret_cast<int4*>(places)[i] = none;
    __syncthreads();
    const int32_t* list = draft_list(a, b, accepted);
    for (int j = threadIdx.x; j < a.draft_k; j += blockDim.x) {
      const int v = list[j] - v0;
      if ((unsigned)v < (unsigned)size && list[j] < a.vocab) atomicMin(&places[v], j);
    }
    __syncthreads();
  }
  return d;
}

// A wave sums a quarter of the workgroup's part, so that the one behind has less to look through; the first workgroup of a
// sequence leaves how many tokens were accepted.  VEC: rows start at multiples of 16 bytes.
// PART: the most tokens of a part.
template <int KIND, bool VEC, int PART>
__global__ __launch_bounds__(kVerifyThreads) void k_verify_sums(DraftArgs a) {
  __shared__ int ok[kMaxDraft];
  __shared__ __align__(16) int32_t places[KIND == kDraftList ? PART : 4];
  const int b = blockIdx.y, length = draft_length(a, b);
  const int accepted = accepted_tokens(a, b, length, ok);
  if (blockIdx.x == 0 && threadIdx.x == 0) a.accepted[b] = accepted;
  const int v0 = blockIdx.x * a.part_size;
  const float* p = target_row(a, b, accepted);
  const PartDraft<KIND> q = part_draft<KIND>(a, b, accepted, accepted < length, v0, a.part_size, places);
  const int slice = a.part_size / kPartSlices, w0 = v0 + wave_id() * slice, w1 = min(w0 + slice, a.vocab), lane = lane_id();
  double rest = 0.0, whole = 0.0;
  auto add = [&](float pv, double qv) {
    const double w = fmax((double)pv, 0.0);
    whole += w;
    rest += fmax(w - qv, 0.0);
  };
  if constexpr (VEC) {
    constexpr int kAhead = 4;
    for (int v = w0 + 4 * lane; v < w1; v += 256 * kAhead) {  // w1 is a multiple of 4
      float4 pv[kAhead], qv[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int at = min(v + 256 * u, w1 - 4);
        pv[u] = *reinterpret_cast<const float4*>(p + at);
        if constexpr (KIND == kDraftDense) qv[u] = *reinterpret_cast<const float4*>((q.refused ? q.row : p) + at);
      }
#pragma unroll
      for (int u = 0; u < kAhead; ++u) {
        const int at = v + 256 * u;
        if (at >= w1) break;
        const float pe[4] = {pv[u].x, pv[u].y, pv[u].z, pv[u].w};
        if constexpr (KIND == kDraftDense) {
          const float qe[4] = {qv[u].x, qv[u].y, qv[u].z, qv[u].w};
#pragma unroll
          for (int e = 0; e < 4; ++e) add(pe[e], q.refused ? (double)qe[e] : 0.0);
        } else if constexpr (KIND == kDraftList) {
          int4 in = make_int4(0x7FFFFFFF, 0x7FFFFFFF, 0x7FFFFFFF, 0x7FFFFFFF);
          if (q.refused) in = *reinterpret_cast<const int4*>(places + (at - v0));
          const int j[4] = {in.x, in.y, in.z, in.w};
#pragma unroll
          for (int e = 0; e < 4; ++e) add(pe[e], j[e] != 0x7FFFFFFF ? (double)q.row[j[e]] : 0.0);
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) add(pe[e], q.at(at + e));
        }
      }
    }
  } else {
#pragma unroll 8
    for (int v = w0 + lane; v < w1; v += kWave) add(p[v], q.at(v));
  }
  rest = wave_sum(rest);
  whole = wave_sum(whole);
  if (lane == 0) {
    double* out = a.part + 2 * (((size_t)b * a.parts + blockIdx.x) * kPartSlices + wave_id());
    out[0] = rest;
    out[1] = whole;
  }
}

// A workgroup per sequence: the slice of the row in which the running sum passes the mark, then the place in it, whose values stay in
// registers between the sum and the search.
constexpr int kMostSlices = 4 * kVerifyThreads;

// EACH: values of a slice in a thread.
template <int KIND, int EACH>
__global__ __launch_bounds__(kVerifyThreads) void k_verify_pick(DraftArgs a) {
  constexpr int kSlices = kMostSlices / kVerifyThreads, kEach = EACH;
  __shared__ double waves[2][2][kVerifyWaves];
  __shared__ Found found[2][kVerifyWaves];
  __shared__ __align__(16) int32_t places[KIND == kDraftList ? EACH * kVerifyThreads : 4];
  const int b = blockIdx.x, slices = a.parts * kPartSlices, slice = a.part_size / kPartSlices;
  const double2* part = reinterpret_cast<const double2*>(a.part) + (size_t)b * slices;
  double w[kSlices], whole[kSlices], sums[2] = {0.0, 0.0};
#pragma unroll
  for (int e = 0; e < kSlices; ++e) {
    const int at = (int)threadIdx.x * kSlices + e;
    const double2 v = part[min(at, slices - 1)];
    w[e] = at < slices ? v.x : 0.0;
    whole[e] = at < slices ? v.y : 0.0;
  }
  const int length = draft_length(a, b), accepted = a.accepted[b];
  const double sample = (double)a.sample_u[b];
#pragma unroll
  for (int e = 0; e < kSlices; ++e) sums[0] += w[e], sums[1] += whole[e];
  const Running r = running_sums(sums[0], sums[1], waves[0]);
  const bool nothing = !(r.total[0] > 0.0);
#pragma unroll
  for (int e = 0; e < kSlices; ++e) w[e] = nothing ? whole[e] : w[e];
  const double mark = sample * (nothing ? r.total[1] : r.total[0]);
  double start, unused;
  const int at_slice = find_place(w, nothing ? r.before[1] : r.before[0], mark, found[0], &start);
  int next = -1;
  if (at_slice >= 0) {
    const int v0 = at_slice * slice, size = min(slice, a.vocab - v0), first = (int)threadIdx.x * kEach;
    const float* p = target_row(a, b, accepted) + v0;
    const PartDraft<KIND> q = part_draft<KIND>(a, b, accepted, accepted < length && !nothing, v0, slice, places);
    double x[kEach], sum = 0.0;
    // neighbouring threads load neighbouring values; in the order of the places they go through LDS
    __shared__ float staged[EACH * kVerifyThreads];
    float pv[kEach];
#pragma unroll
    for (int i = 0; i < kEach; ++i) pv[i] = p[min((int)threadIdx.x + i * kVerifyThreads, size - 1)];
#pragma unroll
    for (int i = 0; i < kEach; ++i) {
      const int at = (int)threadIdx.x + i * kVerifyThreads;
      if (at < slice) staged[at] = at < size ? (float)pv[i] : 0.0f;
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < kEach; ++i)
      x[i] = first + i < size ? fmax(fmax((double)staged[first + i], 0.0) - q.at(v0 + first + i), 0.0) : 0.0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) sum += x[i];
    const Running in = running_sums(sum, 0.0, waves[1]);
    next = find_place(x, start + in.before[0], mark, found[1], &unused);
    if (next >= 0) next += v0;
  }
  write_tokens(a, b, accepted, next);
}

// Parts of a dense row: about a thousand workgroups over the batch, of at least 1024 tokens; the slices of all of them are
// what the workgroup that picks holds.  With a draft's list a part's places lie in LDS, and parts of up to 4096 tokens leave room
// for eight workgroups on a compute unit: 64 sequences of 2 tokens, 256000 in the vocabulary, 32.4 -> 26.6 us.
constexpr int kListPart = 4096;
bool small_parts(const DraftArgs& a) { return a.draft_idx && a.vocab <= kListPart * (kMostSlices / kPartSlices); }
DraftParts draft_parts(const DraftArgs& a) {
  int parts = 1024 / a.B;
  parts = parts < 16 ? 16 : (parts > kMostSlices / kPartSlices ? kMostSlices / kPartSlices : parts);
  int size = ((a.vocab + parts - 1) / parts + 1023) / 1024 * 1024;
  const int most = small_parts(a) ? kListPart : kMaxDraftPart;
  if (size > most) size = most;
  return DraftParts{(a.vocab + size - 1) / size, size};
}

}  // namespace

size_t draft_part_bytes(const DraftArgs& a) { return (size_t)a.B * draft_parts(a).count * kPartSlices * 2 * sizeof(double); }

hipError_t launch_verify(DraftArgs a, hipStream_t s) {
  if (a.target_idx) {
    const int longest = a.draft_idx && a.draft_k > a.target_k ? a.draft_k : a.target_k;
    if (longest <= kShortList && a.n < kShortWaves && (!a.draft || a.draft_idx)) {
      const dim3 grid((unsigned)a.B), block((unsigned)(kWave * (a.n + 1)));
      return longest <= kWave ? launch(&k_verify_short<1>, grid, block, 0, s, a) : launch(&k_verify_short<kShortEach>, grid, block, 0, s, a);
    }
    const dim3 grid((unsigned)a.B);
    if (longest <= 512) return launch(&k_verify_lists<512, 1>, grid, dim3(512), 0, s, a);
    if (longest <= 1024) return launch(&k_verify_lists<1024, 1>, grid, dim3(1024), 0, s, a);
    return launch(&k_verify_lists<1024, kMaxDraftList / 1024>, grid, dim3(1024), 0, s, a);
  }
  const DraftParts parts = draft_parts(a);
  a.parts = parts.count;
  a.part_size = parts.size;
  const bool vec = a.vocab % 4 == 0 && reinterpret_cast<uintptr_t>(a.target) % 16 == 0 &&
                   (!a.draft || a.draft_idx || reinterpret_cast<uintptr_t>(a.draft) % 16 == 0);
  auto both = [&](auto kind) {
    constexpr int KIND = decltype(kind)::value;
    auto sums = [&](auto part) {
      constexpr int PART = decltype(part)::value;
      const dim3 grid((unsigned)a.parts, (unsigned)a.B);
      return vec ? launch(&k_verify_sums<KIND, true, PART>, grid, dim3(kVerifyThreads), 0, s, a)
                 : launch(&k_verify_sums<KIND, false, PART>, grid, dim3(kVerifyThreads), 0, s, a);
    };
    hipError_t e;
    if constexpr (KIND == kDraftList)
      e = small_parts(a) ? sums(std::integral_constant<int, kListPart>{}) : sums(std::integral_constant<int, kMaxDraftPart>{});
    else
      e = sums(std::integral_constant<int, 0>{});
    if (e != hipSuccess) return e;
    const dim3 grid((unsigned)a.B), block(kVerifyThreads);
    const int each = a.part_size / kPartSlices / kVerifyThreads;  // at least one: a part is whole thousands
    if (each <= 1) return launch(&k_verify_pick<KIND, 1>, grid, block, 0, s, a);
    if (each <= 4) return launch(&k_verify_pick<KIND, 4>, grid, block, 0, s, a);
    return launch(&k_verify_pick<KIND, kMaxDraftPart / kPartSlices / kVerifyThreads>, grid, block, 0, s, a);
  };
  if (!a.draft) return both(std::integral_constant<int, kDraftCertain>{});
  if (!a.draft_idx) return both(std::integral_constant<int, kDraftDense>{});
  return both(std::integral_constant<int, kDraftList>{});
}

}  // namespace hire
