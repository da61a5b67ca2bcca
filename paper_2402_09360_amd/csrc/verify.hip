// Verification of drafted tokens: which of them the target's probabilities accept under given random numbers, and the token
// that follows, drawn from what the draft leaves of the target's distribution.
//   token i is accepted iff u_i q_i(d_i) < p_i(d_i); behind a accepted ones the next token is the first v with
//   sum_{w <= v} r(w) > s sum_w r(w),  r = max(p_a - q_a, 0) where token a was refused, p_a where none was left
// Probabilities are fp32 and everything computed from them is fp64: products and differences are exact (or all but), and sums
// over a whole vocabulary keep about 45 bits more than a probability's share of one needs.
#include "kernels.h"
#include "select.h"

namespace hire {
namespace {

constexpr int kVerifyThreads = 1024;  // one workgroup for a sequence
constexpr int kPartThreads = 256;     // workgroups that sum a part of a dense row

// Probability of a token by the first entry of a list that names it; whole wave, every lane gets it.
__device__ __forceinline__ float list_at(const float* prob, const int32_t* idx, int k, int token) {
  for (int j0 = 0; j0 < k; j0 += kWave) {
    const int j = j0 + lane_id();
    const uint64_t hit = __ballot(j < k && idx[min(j, k - 1)] == token);
    if (hit != 0ull) return prob[j0 + __builtin_ctzll(hit)];
  }
  return 0.0f;
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
  auto decide = [&](int i, auto p_of, auto q_of) {
    const int d = a.tokens[(size_t)b * a.n + i];
    if ((unsigned)d >= (unsigned)a.vocab) return 0;
    const double p = p_of(i, d), q = q_of(i, d);
    return (double)a.accept_u[(size_t)b * a.n + i] * q < p ? 1 : 0;
  };
  if (!a.target_idx && !a.draft_idx) {  // a lane for each token
    if (threadIdx.x < kMaxDraft && (int)threadIdx.x < length)
      ok[threadIdx.x] = decide((int)threadIdx.x, [&](int i, int d) { return target_row(a, b, i)[d]; },
                               [&](int i, int d) { return a.draft ? draft_row(a, b, i)[d] : 1.0f; });
  } else {  // a wave for each
    for (int i = wave_id(); i < length; i += (int)(blockDim.x / kWave)) {
      const int yes = decide(
          i,
          [&](int t, int d) {
            return a.target_idx ? list_at(target_row(a, b, t), target_list(a, b, t), a.target_k, d) : target_row(a, b, t)[d];
          },
          [&](int t, int d) {
            return a.draft_idx ? list_at(draft_row(a, b, t), draft_list(a, b, t), a.draft_k, d)
                               : (a.draft ? draft_row(a, b, t)[d] : 1.0f);
          });
      if (lane_id() == 0) ok[i] = yes;
    }
  }
  __syncthreads();
  const bool refused = lane_id() < length && ok[min(lane_id(), kMaxDraft - 1)] == 0;
  const uint64_t mask = __ballot(refused);
  return mask == 0ull ? length : __builtin_ctzll(mask);
}

// Sum over the workgroup's threads in front of this one, and of all of them; in a fixed order.  waves: LDS, a value per wave.
__device__ __forceinline__ double block_prefix(double v, double* waves, double* total) {
  const double incl = wave_prefix(v, 0.0, [](double x, double y) { return x + y; });
  if (lane_id() == kWave - 1) waves[wave_id()] = incl;
  __syncthreads();
  double before = 0.0, all = 0.0;
  for (int w = 0; w < (int)(blockDim.x / kWave); ++w) {
    if (w == wave_id()) before = all;
    all += waves[w];
  }
  __syncthreads();
  *total = all;
  const double excl = incl - v;  // only a starting point: the picking below takes the first place beyond the mark
  return before + excl;
}

// The first of this workgroup's places whose running sum is beyond `mark`, else the last place that counts at all.  A thread has
// the places first + 0 ... count - 1, in order; weight(i) is that of place i.  found: two LDS words.
template <typename Weight>
__device__ __forceinline__ int pick_place(double before, double mark, int first, int count, Weight weight, int* found) {
  if (threadIdx.x == 0) found[0] = 0x7FFFFFFF, found[1] = -1;
  __syncthreads();
  double sum = before;
  int last = -1, hit = 0x7FFFFFFF;
  for (int i = 0; i < count; ++i) {
    const double w = weight(first + i);
    if (!(w > 0.0)) continue;
    sum += w;
    last = first + i;
    if (sum > mark) {
      hit = last;
      break;
    }
  }
  if (hit != 0x7FFFFFFF) atomicMin(&found[0], hit);
  if (last >= 0) atomicMax(&found[1], last);
  __syncthreads();
  return found[0] != 0x7FFFFFFF ? found[0] : found[1];
}

__device__ __forceinline__ void write_tokens(const DraftArgs& a, int b, int accepted, int next) {
  for (int i = threadIdx.x; i <= a.n; i += blockDim.x)
    a.out_tokens[(size_t)b * (a.n + 1) + i] = i < accepted ? a.tokens[(size_t)b * a.n + i] : (i == accepted ? next : -1);
  if (threadIdx.x == 0) a.accepted[b] = accepted;
}

// ---- target as lists: a workgroup per sequence ------------------------------------
// A table in LDS tells for a token the first place of a list that names it: open addressing, at most half full.
struct PlaceTable {
  int32_t* key;
  int32_t* place;
  int mask;
  __device__ __forceinline__ void clear() const {
    for (int i = threadIdx.x; i <= mask; i += kVerifyThreads) key[i] = -1, place[i] = 0x7FFFFFFF;
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

constexpr int kListEach = kMaxDraftList / kVerifyThreads;

__global__ __launch_bounds__(kVerifyThreads) void k_verify_lists(DraftArgs a) {
  __shared__ int ok[kMaxDraft], found[2];
  __shared__ double waves[kVerifyThreads / kWave];
  __shared__ int32_t keys[2 * kMaxDraftList], places[2 * kMaxDraftList];
  const int b = blockIdx.x, length = draft_length(a, b);
  const int accepted = accepted_tokens(a, b, length, ok);
  const float* p = target_row(a, b, accepted);
  const int32_t* tokens = target_list(a, b, accepted);
  const bool refused = accepted < length;
  const int each = (a.target_k + kVerifyThreads - 1) / kVerifyThreads, first = (int)threadIdx.x * each;
  const int count = min(max(a.target_k - first, 0), each);

  PlaceTable table{keys, places, 63};
  const int longest = max(a.target_k, a.draft_idx ? a.draft_k : 0);
  while (table.mask + 1 < 2 * longest) table.mask = 2 * table.mask + 1;
  table.clear();
  int token[kListEach];
  double whole[kListEach], rest[kListEach];
#pragma unroll
  for (int i = 0; i < kListEach; ++i) {
    const bool there = i < count;
    token[i] = there ? tokens[first + i] : -1;
    whole[i] = there ? (double)p[first + i] : 0.0;
    if ((unsigned)token[i] >= (unsigned)a.vocab) token[i] = -1;
    if (token[i] >= 0) table.insert(token[i], first + i);
  }
  __syncthreads();
#pragma unroll
  for (int i = 0; i < kListEach; ++i)
    if (token[i] < 0 || table.find(token[i]) != first + i || !(whole[i] > 0.0)) whole[i] = 0.0, token[i] = -1;
  __syncthreads();
  if (refused && a.draft_idx) {
    table.clear();
    const int32_t* list = draft_list(a, b, accepted);
    for (int j = threadIdx.x; j < a.draft_k; j += kVerifyThreads)
      if ((unsigned)list[j] < (unsigned)a.vocab) table.insert(list[j], j);
    __syncthreads();
  }
  double sums[2] = {0.0, 0.0};
#pragma unroll
  for (int i = 0; i < kListEach; ++i) {
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
  double total, total_whole;
  double before = block_prefix(sums[0], waves, &total);
  const double before_whole = block_prefix(sums[1], waves, &total_whole);
  const bool nothing = !(total > 0.0);  // the draft's covers the target's everywhere: the target's itself
  if (nothing) before = before_whole, total = total_whole;
  const double mark = (double)a.sample_u[b] * total;
  auto weight = [&](int at) {
    double w = 0.0;
#pragma unroll
    for (int i = 0; i < kListEach; ++i)
      if (at == first + i) w = nothing ? whole[i] : rest[i];
    return w;
  };
  const int at = pick_place(before, mark, first, count, weight, found);
  write_tokens(a, b, accepted, at >= 0 ? tokens[at] : -1);
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
    for (int i = threadIdx.x; i < size; i += blockDim.x) places[i] = 0x7FFFFFFF;
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

template <int KIND>
__global__ __launch_bounds__(kPartThreads) void k_verify_sums(DraftArgs a) {
  __shared__ int ok[kMaxDraft];
  __shared__ double waves[2][kPartThreads / kWave];
  __shared__ int32_t places[KIND == kDraftList ? kMaxDraftPart : 1];
  const int b = blockIdx.y, length = draft_length(a, b);
  const int accepted = accepted_tokens(a, b, length, ok);
  const int v0 = blockIdx.x * a.part_size, v1 = min(v0 + a.part_size, a.vocab);
  const float* p = target_row(a, b, accepted);
  const PartDraft<KIND> q = part_draft<KIND>(a, b, accepted, accepted < length, v0, a.part_size, places);
  double rest = 0.0, whole = 0.0;
#pragma unroll 8
  for (int v = v0 + (int)threadIdx.x; v < v1; v += kPartThreads) {
    const double w = fmax((double)p[v], 0.0);
    whole += w;
    rest += fmax(w - q.at(v), 0.0);
  }
  rest = wave_sum(rest);
  whole = wave_sum(whole);
  if (lane_id() == 0) waves[0][wave_id()] = rest, waves[1][wave_id()] = whole;
  __syncthreads();
  if (threadIdx.x == 0) {
    for (int w = 1; w < kPartThreads / kWave; ++w) rest += waves[0][w], whole += waves[1][w];
    double* out = a.part + 2 * ((size_t)b * a.parts + blockIdx.x);
    out[0] = rest;
    out[1] = whole;
  }
}

template <int KIND>
__global__ __launch_bounds__(kVerifyThreads) void k_verify_pick(DraftArgs a) {
  __shared__ int ok[kMaxDraft], found[2];
  __shared__ double waves[kVerifyThreads / kWave], start;
  __shared__ int32_t places[KIND == kDraftList ? kMaxDraftPart : 1];
  const int b = blockIdx.x, length = draft_length(a, b);
  const int accepted = accepted_tokens(a, b, length, ok);
  const bool mine = (int)threadIdx.x < a.parts;
  const double* part = a.part + 2 * ((size_t)b * a.parts + (mine ? threadIdx.x : 0));
  double rest = mine ? part[0] : 0.0;
  const double whole = mine ? part[1] : 0.0;
  double total, total_whole;
  double before = block_prefix(rest, waves, &total);
  const double before_whole = block_prefix(whole, waves, &total_whole);
  const bool nothing = !(total > 0.0);
  if (nothing) before = before_whole, total = total_whole, rest = whole;
  const double mark = (double)a.sample_u[b] * total;
  // the part, then the place in it
  const int at_part = pick_place(before, mark, (int)threadIdx.x, mine ? 1 : 0, [&](int) { return rest; }, found);
  if ((int)threadIdx.x == at_part) start = before;
  __syncthreads();
  int next = -1;
  if (at_part >= 0) {
    const int v0 = at_part * a.part_size, size = min(a.part_size, a.vocab - v0);
    const float* p = target_row(a, b, accepted);
    const PartDraft<KIND> q = part_draft<KIND>(a, b, accepted, accepted < length && !nothing, v0, a.part_size, places);
    const int each = (size + kVerifyThreads - 1) / kVerifyThreads, first = v0 + (int)threadIdx.x * each;
    const int count = min(max(v0 + size - first, 0), each);
    auto weight = [&](int v) { return fmax(fmax((double)p[v], 0.0) - q.at(v), 0.0); };
    double sum = 0.0, all;
    for (int i = 0; i < count; ++i) sum += weight(first + i);
    const double inside = block_prefix(sum, waves, &all);
    next = pick_place(start + inside, mark, first, count, weight, found);
  }
  write_tokens(a, b, accepted, next);
}

}  // namespace

// Parts of a dense row: about a thousand workgroups over the batch, none with fewer than 1024 tokens.
DraftParts draft_parts(int B, int vocab) {
  int parts = 1024 / B;
  parts = parts < 16 ? 16 : (parts > 256 ? 256 : parts);
  int size = ((vocab + parts - 1) / parts + 1023) / 1024 * 1024;
  if (size > kMaxDraftPart) size = kMaxDraftPart;
  return DraftParts{(vocab + size - 1) / size, size};
}

hipError_t launch_verify(DraftArgs a, hipStream_t s) {
  if (a.target_idx) return launch(&k_verify_lists, dim3((unsigned)a.B), dim3(kVerifyThreads), 0, s, a);
  const DraftParts parts = draft_parts(a.B, a.vocab);
  a.parts = parts.count;
  a.part_size = parts.size;
  auto both = [&](void (*sums)(DraftArgs), void (*pick)(DraftArgs)) {
    const hipError_t e = launch(sums, dim3((unsigned)a.parts, (unsigned)a.B), dim3(kPartThreads), 0, s, a);
    return e != hipSuccess ? e : launch(pick, dim3((unsigned)a.B), dim3(kVerifyThreads), 0, s, a);
  };
  if (!a.draft) return both(&k_verify_sums<kDraftCertain>, &k_verify_pick<kDraftCertain>);
  if (!a.draft_idx) return both(&k_verify_sums<kDraftDense>, &k_verify_pick<kDraftDense>);
  return both(&k_verify_sums<kDraftList>, &k_verify_pick<kDraftList>);
}

}  // namespace hire
