// The largest logits of a row from its logits and its groups' maxima, and what a beam search makes of them.
#pragma once
#include "logit_tiles.h"

namespace flce {

constexpr int TOPK_MAX = 256;             // most logits kept of a row
constexpr int SELECT_THREADS = 256;
constexpr int SELECT_SORT = 512;          // candidates that are ranked against each other
constexpr int SELECT_KEYS = 8192;         // group maxima held in LDS

// Order of a logit as an unsigned number: NaN above everything, -0 equal to +0.
__device__ __forceinline__ uint32_t order_key(float x) {
  if (x != x) return 0xFFFFFFFFu;
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
// That of a group: by its maximum, which does not see NaN; its sum does.
__device__ __forceinline__ uint32_t group_key(float2 s) { return s.y != s.y ? 0xFFFFFFFFu : order_key(s.x); }

struct Threshold {
  uint32_t key;       // at least `need` keys are >= key, fewer than that are > key
  int above, equal;   // how many are > key, == key
};

// The need-th largest of n keys (1 <= need <= n) by radix selection, 8 bits at a time from the top: every pass counts the keys
// that agree with the digits found so far by their next digit.  All threads of a block of SELECT_THREADS call it.
template <typename GET>
__device__ __forceinline__ Threshold find_threshold(GET get, int n, int need, int* hist, int* word) {
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  uint32_t prefix = 0;
  int above = 0, equal = 0;
#pragma unroll
  for (int shift = 24; shift >= 0; shift -= 8) {
    hist[t] = 0;
    __syncthreads();
    for (int i = t; i < n; i += SELECT_THREADS) {
      const uint32_t k = get(i);
      if (shift == 24 || (k ^ prefix) >> (shift + 8) == 0) atomicAdd(&hist[k >> shift & 255], 1);
    }
    __syncthreads();
    // thread t has digit 255 - t: counts of the digits above it by a prefix sum
    const int c = hist[255 - t];
    int sum = c;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(sum, o, 64);
      if (lane >= o) sum += x;
    }
    if (lane == 63) word[4 + wave] = sum;
    __syncthreads();
#pragma unroll
    for (int w = 0; w < 3; ++w) if (w < wave) sum += word[4 + w];
    if (above + sum >= need && above + sum - c < need) { word[0] = 255 - t; word[1] = above + sum - c; word[2] = c; }
    __syncthreads();
    prefix |= (uint32_t)word[0] << shift;
    above = word[1];
    equal = word[2];
  }
  return Threshold{prefix, above, equal};
}

// The places of the need largest of n keys: those above the threshold and of those equal to it the first ones, into out[].
// (The order of out is not fixed.)
template <typename GET>
__device__ __forceinline__ void collect(GET get, int n, int need, const Threshold& th, int* out, int* word) {
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const bool all = th.above + th.equal == need;
  if (t == 0) word[3] = 0;
  __syncthreads();
  for (int i = t; i < n; i += SELECT_THREADS) {
    const uint32_t k = get(i);
    if (all ? k >= th.key : k > th.key) out[atomicAdd(&word[3], 1)] = i;
  }
  if (!all) {
    int taken = th.above;           // equal ones in order of their place: 256 at a time, wavefront after wavefront
    for (int i0 = 0; i0 < n && taken < need; i0 += SELECT_THREADS) {
      const int i = i0 + t;
      const bool eq = i < n && get(i) == th.key;
      const uint64_t m = __ballot(eq);
      __syncthreads();
      if (lane == 0) word[4 + wave] = __popcll(m);
      __syncthreads();
      int at = taken + __popcll(m & ((1ull << lane) - 1));
#pragma unroll
      for (int w = 0; w < SELECT_THREADS / 64; ++w) {
        if (w < wave) at += word[4 + w];
        taken += word[4 + w];
      }
      if (eq && at < need) out[at] = i;
    }
  }
  __syncthreads();
}

// One block per row: the row's K largest logits in order (equal ones by id), their ids, and its log-sum-exp.
//   1. K groups hold them: the first K by (maximum, position), since an element of another group has K better ones in these.
//   2. The K-th of those maxima is a lower bound of the K-th logit: of the K groups' elements only the ones that reach it are
//      candidates, some more than K as a rule.  Where there are more than fit (many equal logits, a band of large ones in
//      consecutive positions) the K among them are selected first.
//   3. A candidate's rank is the number of larger (logit, lower id) pairs.
// Reads the groups' maxima and K groups of logits; a chain of latencies and barriers, a few us, many rows at a time.
template <int G>      // positions per group
__global__ __launch_bounds__(SELECT_THREADS) void select_kernel(const float* __restrict__ z, int64_t ldz, const float2* __restrict__ stats,
                                                                int64_t ld_stats, int n_groups, int V, int K, float* __restrict__ logits_out,
                                                                int64_t* __restrict__ ids_out, float* __restrict__ lse_out) {
  __shared__ uint32_t keys[SELECT_KEYS];
  __shared__ int hist[SELECT_THREADS], word[8], groups[TOPK_MAX];
  __shared__ unsigned long long cand[SELECT_SORT];
  __shared__ float red[2 * SELECT_THREADS / 64];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int64_t row = blockIdx.x;
  z += row * ldz;
  stats += row * ld_stats;
  const bool in_lds = n_groups <= SELECT_KEYS;

  float m = NEG_INF;
  for (int g = t; g < n_groups; g += SELECT_THREADS) {
    const float2 s = stats[g];
    m = fmaxf(m, s.x);
    if (in_lds) keys[g] = group_key(s);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
  if (lane == 0) red[wave] = m;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < SELECT_THREADS / 64; ++w) m = fmaxf(m, red[w]);
  float sum = 0.f;
  for (int g = t; g < n_groups; g += SELECT_THREADS) {
    const float2 s = stats[g];
    // a group without a finite maximum is relative to 0 (and adds nothing, or +inf)
    if (s.y != 0.f) sum += s.y * fast_exp2((finite_or_zero(s.x) - finite_or_zero(m)) * LOG2E);
  }
  sum = wave_sum(sum);
  if (lane == 0) red[SELECT_THREADS / 64 + wave] = sum;
  __syncthreads();
  if (t == 0) {
    float a = 0.f;
#pragma unroll
    for (int w = 0; w < SELECT_THREADS / 64; ++w) a += red[SELECT_THREADS / 64 + w];
    lse_out[row] = finite_or_zero(m) + logf(a);
  }

  auto key_of_group = [&](int g) { return in_lds ? keys[g] : group_key(stats[g]); };
  const int kg = min(K, n_groups);
  Threshold th{0u, 0, n_groups};
  if (kg < n_groups) th = find_threshold(key_of_group, n_groups, kg, hist, word);
  collect(key_of_group, n_groups, kg, th, groups, word);

  const int n = kg * G;
  auto place = [&](int i) { return groups[i / G] * G + i % G; };
  // a position past the vocabulary's end lies below everything, -inf included (whose key is not 0)
  auto key_of = [&](int i) { const int v = place(i); return v < V ? order_key(z[v]) : 0u; };
  if (t == 0) word[3] = 0;
  __syncthreads();
  const uint32_t low = kg == K ? max(th.key, 1u) : 1u;     // fewer groups than K: every element is a candidate
  for (int i = t; i < n; i += SELECT_THREADS) {
    const uint32_t k = key_of(i);
    if (k >= low) {
      const int at = atomicAdd(&word[3], 1);
      if (at < SELECT_SORT) cand[at] = (unsigned long long)k << 32 | (uint32_t)~place(i);
    }
  }
  __syncthreads();
  int count = word[3];
  __syncthreads();
  if (count > SELECT_SORT) {
    // in order of their ids, so that the first of equal ones are the lowest
    int rank = 0, mine = t < kg ? groups[t] : 0;
    for (int g = 0; g < kg; ++g) rank += groups[g] < mine;
    __syncthreads();
    if (t < kg) groups[rank] = mine;
    __syncthreads();
    const Threshold te = find_threshold(key_of, n, K, hist, word);
    int* chosen = reinterpret_cast<int*>(cand);            // K <= 256 places, then their pairs in the same memory
    collect(key_of, n, K, te, chosen, word);
    const int i = t < K ? chosen[t] : 0;
    __syncthreads();
    if (t < K) cand[t] = (unsigned long long)key_of(i) << 32 | (uint32_t)~place(i);
    __syncthreads();
    count = K;
  }
  for (int i = t; i < count; i += SELECT_THREADS) {
    const unsigned long long c = cand[i];
    int rank = 0;
    for (int o = 0; o < count; ++o) rank += cand[o] > c;
    if (rank < K) {
      const int v = (int)~(uint32_t)c;
      logits_out[row * K + rank] = z[v];
      ids_out[row * K + rank] = v;
    }
  }
}

// A beam's candidates in order: the rows' largest logits as scores; a finished beam's is the one that it is.
// One block per batch element.  A candidate's rank is its place in its own beam's list plus the number of candidates of the
// other beams that come before it (a binary search in each list, which is in order): larger score first, equal ones by beam.
__global__ __launch_bounds__(SELECT_THREADS) void beam_select_kernel(const float* __restrict__ logits, const int64_t* __restrict__ ids,
                                                                     const float* __restrict__ lse, const float* __restrict__ scores,
                                                                     const uint8_t* __restrict__ finished, int beams, int K, int n_out,
                                                                     int64_t eos_id, int64_t pad_id, float* __restrict__ scores_out,
                                                                     int64_t* __restrict__ tokens_out, int64_t* __restrict__ parents_out,
                                                                     uint8_t* __restrict__ finished_out) {
  extern __shared__ __align__(16) char dyn[];
  uint32_t* key = reinterpret_cast<uint32_t*>(dyn);        // [beams][K]
  int* len = reinterpret_cast<int*>(key + beams * K);      // [beams]
  const int b = blockIdx.x;
  const int64_t row0 = (int64_t)b * beams;
  auto score = [&](int j, int k) {
    const float s = scores[row0 + j];
    // (NaN and +inf stay what they are, so that a beam's scores are in order whatever its logits)
    return (finished && finished[row0 + j]) || !(s < __builtin_inff()) ? s : s + (logits[(row0 + j) * K + k] - lse[row0 + j]);
  };
  for (int i = threadIdx.x; i < beams * K; i += SELECT_THREADS) key[i] = order_key(score(i / K, i % K));
  for (int j = threadIdx.x; j < beams; j += SELECT_THREADS) len[j] = finished && finished[row0 + j] ? 1 : K;
  __syncthreads();
  int total = 0;
  for (int j = 0; j < beams; ++j) total += len[j];
  for (int i = threadIdx.x; i < beams * K; i += SELECT_THREADS) {
    const int j = i / K, k = i % K;
    if (k >= len[j]) continue;
    const uint32_t mine = key[i];
    int rank = k;
    for (int o = 0; o < beams && rank < n_out; ++o) {
      if (o == j) continue;
      int lo = 0, hi = len[o];         // how many of beam o come first: larger ones, of a lower beam equal ones too
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        const uint32_t x = key[o * K + mid];
        if (x > mine || (x == mine && o < j)) lo = mid + 1; else hi = mid;
      }
      rank += lo;
    }
    if (rank >= n_out) continue;
    const bool done = finished && finished[row0 + j];
    const int64_t token = done ? pad_id : ids[(row0 + j) * K + k];
    const int64_t at = (int64_t)b * n_out + rank;
    scores_out[at] = score(j, k);
    tokens_out[at] = token;
    parents_out[at] = j;
    finished_out[at] = done || token == eos_id;
  }
  // fewer candidates than places: dead results
  for (int r = total + threadIdx.x; r < n_out; r += SELECT_THREADS) {
    const int64_t at = (int64_t)b * n_out + r;
    scores_out[at] = NEG_INF;
    tokens_out[at] = pad_id;
    parents_out[at] = 0;
    finished_out[at] = 1;
  }
}

// States of beams reordered: row (o, b, j) of dst = row (o, b, parents[b][j]) of src, row_bytes of it.
// A thread has one vector of NB rows (one run of them per blockIdx.z) of an (o, b): it loads what every destination row takes before
// it stores any, so that src and dst may be the same memory where there is one run (rows that keep their place are then left
// alone), and has up to NB loads in flight.
// A parent outside [0, beams_in) leaves its row as it was and sets *status.  One read and one write of memory per byte.
template <typename Vec, int NB>
__global__ __launch_bounds__(256) void beam_reorder_kernel(const char* src, char* dst, const int64_t* __restrict__ parents, int batch,
                                                           int beams_in, int beams_out, int64_t n_vec, int64_t src_row, int64_t src_outer,
                                                           int64_t dst_row, int64_t dst_outer, int32_t* __restrict__ status) {
  const int b = blockIdx.y % batch, o = blockIdx.y / batch;
  src += o * src_outer + (int64_t)b * beams_in * src_row;
  const int j0 = blockIdx.z * NB;
  dst += o * dst_outer + ((int64_t)b * beams_out + j0) * dst_row;
  __shared__ int from[NB];            // -1: nothing to copy
  if (threadIdx.x < NB) {
    const int j = j0 + threadIdx.x;
    int f = -1;
    if (j < beams_out) {
      const int64_t p = parents[(int64_t)b * beams_out + j];
      if (p >= 0 && p < beams_in) f = (int)p;
      else if (status) *status = FLCE_ERR_TARGET_RANGE;
    }
    from[threadIdx.x] = src == dst && f == j ? -1 : f;
  }
  __syncthreads();
  for (int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x; i < n_vec; i += (int64_t)gridDim.x * 256) {
    Vec v[NB];
#pragma unroll
    for (int j = 0; j < NB; ++j) {
      const int f = __builtin_amdgcn_readfirstlane(from[j]);
      if (f >= 0) v[j] = reinterpret_cast<const Vec*>(src + f * src_row)[i];
    }
#pragma unroll
    for (int j = 0; j < NB; ++j)
      if (__builtin_amdgcn_readfirstlane(from[j]) >= 0) reinterpret_cast<Vec*>(dst + j * dst_row)[i] = v[j];
  }
}

}  // namespace flce
