// The largest logits of a row from its logits and its groups' maxima, and what a beam search makes of them.
#pragma once
#include "logit_tiles.h"

namespace flce {

constexpr int TOPK_MAX = 256;             // most logits kept of a row
constexpr int SELECT_THREADS = 256;
constexpr int SELECT_SORT = 512;          // candidates that are ranked against each other
constexpr int SELECT_GROUPS = 320;        // groups that are looked into: K and a quarter or 16 more
constexpr int SELECT_HELD = 16;           // group pairs that a thread keeps in registers

// Order of a logit as an unsigned number: NaN above everything, -0 equal to +0.
__device__ __forceinline__ uint32_t order_key(float x) {
  if (x != x) return 0xFFFFFFFFu;
  const uint32_t b = __float_as_uint(x + 0.f);
  return b & 0x80000000u ? ~b : b | 0x80000000u;
}
// That of a group: by its maximum, which does not see NaN; its sum does.
__device__ __forceinline__ uint32_t group_key(float2 s) { return s.y != s.y ? 0xFFFFFFFFu : order_key(s.x); }

__device__ __forceinline__ float value_of(uint32_t key) {
  return key == 0xFFFFFFFFu ? __builtin_nanf("") : __uint_as_float(key & 0x80000000u ? key ^ 0x80000000u : ~key);
}

// A lower bound of the need-th largest of a set of keys: `above` keys lie above the interval of keys that starts at `low`, `equal` in it,
// above < need <= above + equal.  The interval is one key where no wider one has above + equal <= limit.
struct Bound { uint32_t low; int above, equal; };

// By radix selection between the smallest and the largest key, 8 bits at a time from the top: each pass counts the keys of the present
// interval by their next digit, and ends the search once few enough keys lie above its lower end.  each(f) calls f(key) for every
// key of the calling thread.  hist: four histograms, zero and a barrier behind them.  Every wavefront reads the histogram for itself, four
// digits per lane: one barrier per pass.
template <typename EACH>
__device__ __forceinline__ Bound find_bound(EACH each, uint32_t kmin, uint32_t kmax, int need, int limit, int (*hist)[256]) {
  const int lane = threadIdx.x & 63;
  uint32_t low = kmin;
  int bits = 32 - __builtin_clz(kmax - kmin | 1u), above = 0, equal = 0;      // digits that are left
  for (int pass = 0;; ++pass) {
    const int shift = max(0, bits - 8);
    const uint32_t span = (bits == 32 ? 0u : 1u << bits) - 1u;                // of the present interval
    each([&](uint32_t k) {
      if (k - low <= span && k >= low) atomicAdd(&hist[pass][(k - low) >> shift], 1);
    });
    __syncthreads();
    // lane l has the digits 255 - 4 l .. 252 - 4 l
    const int4 c = *reinterpret_cast<const int4*>(&hist[pass][252 - 4 * lane]);
    const int mine = c.x + c.y + c.z + c.w;
    int sum = mine;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(sum, o, 64);
      if (lane >= o) sum += x;
    }
    const int at = __builtin_ctzll(__ballot(above + sum >= need));            // (the last lane's sum reaches it)
    int before = above + sum - mine, digit = 255 - 4 * lane, count = c.w;
    if (before + count < need) { before += count; --digit; count = c.z; }
    if (before + count < need) { before += count; --digit; count = c.y; }
    if (before + count < need) { before += count; --digit; count = c.x; }
    above = __builtin_amdgcn_readlane(before, at);
    equal = __builtin_amdgcn_readlane(count, at);
    low += (uint32_t)__builtin_amdgcn_readlane(digit, at) << shift;
    bits = shift;
    if (shift == 0 || above + equal <= limit) return Bound{low, above, equal};
  }
}

// The places of the need largest of n keys (get(i), by threads i, i + 256, ...) in order of their place where they are equal: those above
// b.low and the first ones equal to it, into out[].  For sets that have more than `limit` keys from a single key on.
template <typename GET>
__device__ __forceinline__ void collect_first(GET get, int n, int need, const Bound& b, int* out, int* word) {
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  if (t == 0) word[0] = 0;
  __syncthreads();
  int taken = b.above;
  for (int i0 = 0; i0 < n; i0 += SELECT_THREADS) {         // 256 at a time, wavefront after wavefront
    const int i = i0 + t;
    const uint32_t k = i < n ? get(i) : 0u;
    const bool eq = i < n && k == b.low;
    if (i < n && k > b.low) out[atomicAdd(&word[0], 1)] = i;
    const uint64_t m = __ballot(eq);
    if (lane == 0) word[4 + wave] = __popcll(m);
    __syncthreads();
    int at = taken + __popcll(m & ((1ull << lane) - 1));
#pragma unroll
    for (int w = 0; w < SELECT_THREADS / 64; ++w) {
      if (w < wave) at += word[4 + w];
      taken += word[4 + w];
    }
    if (eq && at < need) out[at] = i;
    __syncthreads();
  }
}

// out[] gets what f says of the calling thread's items: each(g) calls g(keep, value) the same number of times in all lanes of a wavefront.
template <typename V, typename EACH>
__device__ __forceinline__ void append(EACH each, V* out, int room, int* count) {
  const int lane = threadIdx.x & 63;
  each([&](bool keep, V value) {
    const uint64_t m = __ballot(keep);
    if (m == 0ull) return;
    int base = 0;
    if (lane == 0) base = atomicAdd(count, __popcll(m));
    base = __builtin_amdgcn_readfirstlane(base) + __popcll(m & ((1ull << lane) - 1));
    if (keep && base < room) out[base] = value;
  });
}

// A beam search's step on top of the selection: the rows of a search hand their candidates over, and the block that does so last ranks
// them all (a launch of its own took 4 to 5 us).
struct BeamStep {
  const float* scores; const uint8_t* finished;
  int64_t row0; int beams, n_out;
  int64_t eos_id, pad_id;
  float* scores_out; int64_t* tokens_out; int64_t* parents_out; uint8_t* finished_out;
  uint32_t* arrived;                // [search], zero
  unsigned long long* cand;         // [row][K]: (key, ~id) in order
  unsigned long long* norm;         // [row]: (M, log sum exp(z - M)), M the largest logit
  __device__ __forceinline__ bool done(int64_t row) const { return finished && finished[row]; }
};

// Scores of a beam's candidates, s + ((z - M) - log sum exp(z - M)), are in order as its logits are: z - (M + log sum) would lose the
// logarithm beside a large M (a beam whose logits are all the mask's value is uniform, -log V).  A finished beam is its own one candidate.  A candidate's rank is its
// place in its own beam's list plus the number of candidates of the other beams that come before it (a binary search in each list):
// larger score first, equal ones by beam.  key: [beams][K], len: [beams] in LDS.
__device__ __forceinline__ void rank_beams(const BeamStep& s, int K, int64_t search, uint32_t* key, int* len) {
  const int64_t row0 = search * s.beams;
  auto pair = [&](int i) {          // (written by other blocks of this launch: read past this XCD's own caches)
    return __hip_atomic_load(s.cand + row0 * K + i, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  };
  for (int i = threadIdx.x; i < s.beams * K; i += SELECT_THREADS) {
    const int j = i / K;
    float x = s.scores[row0 + j];
    // (NaN and +inf stay what they are, so that a beam's scores are in order whatever its logits)
    if (!s.done(row0 + j) && x < __builtin_inff()) {
      const float2 n = __builtin_bit_cast(float2, __hip_atomic_load(s.norm + row0 + j, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT));
      x += (value_of((uint32_t)(pair(i) >> 32)) - n.x) - n.y;
    }
    key[i] = order_key(x);
  }
  for (int j = threadIdx.x; j < s.beams; j += SELECT_THREADS) len[j] = s.done(row0 + j) ? 1 : K;
  __syncthreads();
  int total = 0;
  for (int j = 0; j < s.beams; ++j) total += len[j];
  for (int i = threadIdx.x; i < s.beams * K; i += SELECT_THREADS) {
    const int j = i / K, k = i % K;
    if (k >= len[j]) continue;
    const uint32_t mine = key[i];
    int rank = k;
    for (int o = 0; o < s.beams && rank < s.n_out; ++o) {
      if (o == j) continue;
      int lo = 0, hi = len[o];         // how many of beam o come first: larger ones, of a lower beam equal ones too
      while (lo < hi) {
        const int mid = (lo + hi) >> 1;
        const uint32_t x = key[o * K + mid];
        if (x > mine || (x == mine && o < j)) lo = mid + 1; else hi = mid;
      }
      rank += lo;
    }
    if (rank >= s.n_out) continue;
    const bool done = s.done(row0 + j);
    const int64_t token = done ? s.pad_id : (int64_t)(int)~(uint32_t)pair(i);
    const int64_t at = search * s.n_out + rank;
    s.scores_out[at] = value_of(mine);
    s.tokens_out[at] = token;
    s.parents_out[at] = j;
    s.finished_out[at] = done || token == s.eos_id;
  }
  // fewer candidates than places: dead results
  for (int r = total + threadIdx.x; r < s.n_out; r += SELECT_THREADS) {
    const int64_t at = search * s.n_out + r;
    s.scores_out[at] = NEG_INF;
    s.tokens_out[at] = s.pad_id;
    s.parents_out[at] = 0;
    s.finished_out[at] = 1;
  }
}

// The end of a row's block: what it has stored has reached the point the other XCDs read from before it counts as arrived.
__device__ __forceinline__ void arrive(const BeamStep& s, int K, int64_t row) {
  extern __shared__ __align__(16) char dyn[];
  __shared__ int last;
  const int64_t search = (s.row0 + row) / s.beams;
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  __syncthreads();
  if (threadIdx.x == 0)
    last = __hip_atomic_fetch_add(s.arrived + search, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)s.beams - 1;
  __syncthreads();
  if (last) {
    uint32_t* key = reinterpret_cast<uint32_t*>(dyn);
    rank_beams(s, K, search, key, reinterpret_cast<int*>(key + s.beams * K));
  }
}

// One block per row: the row's K largest logits in order (equal ones by id), their ids, and its log-sum-exp.
//   1. Any set of groups that has the K with the largest maxima (of equal ones the first) holds them: an element of another group has K
//      better ones in these.  A bound of the K-th maximum that leaves a few more than K is found first.
//   2. That bound is a lower bound of the K-th logit too: of those groups' elements only the ones that reach it are candidates, some
//      more than K as a rule.  Where there are more than fit (many equal logits, a band of large ones in consecutive
//      positions) the search is repeated on them.
//   3. A candidate's rank is the number of larger (logit, lower id) pairs.
// Reads the groups' pairs once, where a thread's fit its registers, and some more than K groups of logits; a chain of latencies and seven
// barriers.
// OUT: Largest, or BeamStep with beams (K + 1) words of dynamic LDS.
struct Largest { float* logits; int64_t* ids; float* lse; const float* floor; };    // [row][K], [row][K], [row], [row] or null; the launch's rows
template <int G, typename OUT>      // positions per group
__device__ __forceinline__ void select_row(const float* __restrict__ z, int64_t ldz, const float2* __restrict__ stats, int64_t ld_stats,
                                           int n_groups, int V, int K, const OUT& out) {
  constexpr bool BEAM = std::is_same<OUT, BeamStep>::value;
  __shared__ __align__(16) int hist[4][256];
  __shared__ int word[8], groups[SELECT_GROUPS];
  __shared__ __align__(16) unsigned long long cand[SELECT_SORT];
  __shared__ float wm[SELECT_THREADS / 64], ws[SELECT_THREADS / 64];
  __shared__ uint32_t klo[SELECT_THREADS / 64], khi[SELECT_THREADS / 64];
  const int t = threadIdx.x, lane = t & 63, wave = t >> 6;
  const int64_t row = blockIdx.x;
  z += row * ldz;
  stats += row * ld_stats;
  const bool held = n_groups <= SELECT_HELD * SELECT_THREADS;

  // Groups' pairs: log-sum-exp, keys and their range.  (A place past the end has key 0, which no logit has.)
  uint32_t key[SELECT_HELD];
  float m = NEG_INF, sum = 0.f;
  uint32_t lo = 0xFFFFFFFFu, hi = 0u;
  auto take = [&](float2 s) {
    m = fmaxf(m, s.x);
    const uint32_t k = group_key(s);
    lo = min(lo, k); hi = max(hi, k);
    return k;
  };
  // a group without a finite maximum is relative to 0 (and adds nothing, or +inf)
  auto add = [&](float2 s) { if (s.y != 0.f) sum += s.y * fast_exp2((finite_or_zero(s.x) - finite_or_zero(m)) * LOG2E); };
  auto wave_max = [&] {
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      m = fmaxf(m, __shfl_xor(m, o, 64));
      lo = min(lo, (uint32_t)__shfl_xor((int)lo, o, 64));
      hi = max(hi, (uint32_t)__shfl_xor((int)hi, o, 64));
    }
  };
  if (held) {
    float2 s[SELECT_HELD];
#pragma unroll
    for (int u = 0; u < SELECT_HELD; ++u)
      if (u * SELECT_THREADS < n_groups) s[u] = stats[min(t + u * SELECT_THREADS, n_groups - 1)];
#pragma unroll
    for (int u = 0; u < SELECT_HELD; ++u) key[u] = t + u * SELECT_THREADS < n_groups ? take(s[u]) : 0u;
    wave_max();
#pragma unroll
    for (int u = 0; u < SELECT_HELD; ++u)
      if (key[u] != 0u) add(s[u]);
  } else {
    for (int g = t; g < n_groups; g += SELECT_THREADS) take(stats[g]);
    wave_max();
    for (int g = t; g < n_groups; g += SELECT_THREADS) add(stats[g]);
  }
  sum = wave_sum(sum);
#pragma unroll
  for (int p = 0; p < 4; ++p) hist[p][t] = 0;
  if (lane == 0) { wm[wave] = m; ws[wave] = sum; klo[wave] = lo; khi[wave] = hi; }
  if (t < 2) word[t] = 0;
  __syncthreads();
#pragma unroll
  for (int w = 0; w < SELECT_THREADS / 64; ++w) { lo = min(lo, klo[w]); hi = max(hi, khi[w]); }
  if (t == 0) {
    float M = NEG_INF, a = 0.f;
#pragma unroll
    for (int w = 0; w < SELECT_THREADS / 64; ++w) M = fmaxf(M, wm[w]);
#pragma unroll
    for (int w = 0; w < SELECT_THREADS / 64; ++w)
      if (ws[w] != 0.f) a += ws[w] * fast_exp2((finite_or_zero(wm[w]) - finite_or_zero(M)) * LOG2E);
    const float2 norm{finite_or_zero(M), logf(a)};
    if constexpr (BEAM)
      __hip_atomic_store(out.norm + out.row0 + row, __builtin_bit_cast(unsigned long long, norm), __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    else out.lse[row] = norm.x + norm.y;
  }

  auto group_keys = [&](auto f) {
    if (held) {
#pragma unroll
      for (int u = 0; u < SELECT_HELD; ++u)
        if (key[u] != 0u) f(key[u]);
    } else {
      for (int g = t; g < n_groups; g += SELECT_THREADS) f(group_key(stats[g]));
    }
  };
  const int want = min(K, n_groups);
  Bound b{0u, 0, n_groups};
  if (n_groups > want) b = find_bound(group_keys, lo, hi, want, want + max(16, want / 4), hist);
  int n_held = b.above + b.equal;
  // below the row's floor, itself a lower bound of the K-th maximum, nothing was kept
  if constexpr (!BEAM) { if (out.floor) b.low = max(b.low, order_key(out.floor[row])); }
  if (n_held <= SELECT_GROUPS) {
    append<int>([&](auto f) {
      if (held) {
#pragma unroll
        for (int u = 0; u < SELECT_HELD; ++u)
          if (u * SELECT_THREADS < n_groups) f(key[u] >= max(b.low, 1u), t + u * SELECT_THREADS);
      } else {
        for (int g0 = 0; g0 < n_groups; g0 += SELECT_THREADS) f(g0 + t < n_groups && group_key(stats[g0 + t]) >= b.low, g0 + t);
      }
    }, groups, SELECT_GROUPS, &word[0]);
    __syncthreads();
    n_held = word[0];
  } else {
    n_held = want;
    collect_first([&](int g) { return group_key(stats[g]); }, n_groups, want, b, groups, word);
  }

  const int n = n_held * G;
  auto place = [&](int i) { return groups[i / G] * G + i % G; };
  // a position past the vocabulary's end lies below everything, -inf included (whose key is not 0)
  auto key_of = [&](int i) { const int v = place(i); return v < V ? order_key(z[v]) : 0u; };
  const uint32_t low = n_groups >= K ? max(b.low, 1u) : 1u;     // fewer groups than K: every element is a candidate
  append<unsigned long long>([&](auto f) {
    constexpr int U = 4;
    for (int i0 = 0; i0 < n; i0 += U * SELECT_THREADS) {
      uint32_t k[U];
#pragma unroll
      for (int u = 0; u < U; ++u) k[u] = key_of(min(i0 + u * SELECT_THREADS + t, n - 1));
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const int i = i0 + u * SELECT_THREADS + t;
        f(i < n && k[u] >= low, (unsigned long long)k[u] << 32 | (uint32_t)~place(min(i, n - 1)));
      }
    }
  }, cand, SELECT_SORT, &word[1]);
  __syncthreads();
  int count = word[1];
  if (count > SELECT_SORT) {
    // in order of their ids, so that the first of equal ones are the lowest
    __syncthreads();
    int rank[2] = {0, 0}, mine[2];
#pragma unroll
    for (int u = 0; u < 2; ++u) {
      mine[u] = t + u * SELECT_THREADS < n_held ? groups[t + u * SELECT_THREADS] : 0;
      for (int g = 0; g < n_held; ++g) rank[u] += groups[g] < mine[u];
    }
#pragma unroll
    for (int p = 0; p < 4; ++p) hist[p][t] = 0;
    if (t == 0) word[1] = 0;
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 2; ++u)
      if (t + u * SELECT_THREADS < n_held) groups[rank[u]] = mine[u];
    __syncthreads();
    const Bound e = find_bound([&](auto f) { for (int i = t; i < n; i += SELECT_THREADS) f(key_of(i)); }, 0u, 0xFFFFFFFFu, K, SELECT_SORT, hist);
    count = e.above + e.equal;
    if (count <= SELECT_SORT) {
      append<unsigned long long>([&](auto f) {
        for (int i0 = 0; i0 < n; i0 += SELECT_THREADS) {
          const int i = min(i0 + t, n - 1);
          const uint32_t k = key_of(i);
          f(i0 + t < n && k >= e.low, (unsigned long long)k << 32 | (uint32_t)~place(i));
        }
      }, cand, SELECT_SORT, &word[1]);
    } else {
      int* chosen = reinterpret_cast<int*>(cand);          // K <= 256 places, then their pairs in the same memory
      collect_first(key_of, n, K, e, chosen, word);
      const int i = t < K ? chosen[t] : 0;
      __syncthreads();
      if (t < K) cand[t] = (unsigned long long)key_of(i) << 32 | (uint32_t)~place(i);
      count = K;
    }
    __syncthreads();
  }
  for (int i = t; i < count; i += SELECT_THREADS) {
    const unsigned long long c = cand[i];
    int rank = 0;
    for (int o = 0; o < count; ++o) rank += cand[o] > c;
    if (rank < K) {
      if constexpr (BEAM) {
        __hip_atomic_store(out.cand + (out.row0 + row) * K + rank, c, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
      } else {
        out.logits[row * K + rank] = value_of((uint32_t)(c >> 32));
        out.ids[row * K + rank] = (int)~(uint32_t)c;
      }
    }
  }
}

template <int G, typename OUT>
__global__ __launch_bounds__(SELECT_THREADS) void select_kernel(const float* __restrict__ z, int64_t ldz, const float2* __restrict__ stats,
                                                                int64_t ld_stats, int n_groups, int V, int K, OUT out) {
  if constexpr (std::is_same<OUT, BeamStep>::value) {
    if (!out.done(out.row0 + blockIdx.x)) select_row<G>(z, ldz, stats, ld_stats, n_groups, V, K, out);
    arrive(out, K, blockIdx.x);
  } else {
    select_row<G>(z, ldz, stats, ld_stats, n_groups, V, K, out);
  }
}

// A lower bound of every row's K-th logit from its first n_groups groups (n_groups > K), one block per row: what the rest of the
// vocabulary has to reach to be kept.  Finite or -inf: what lies above the largest number is kept whatever the floor.
static __global__ __launch_bounds__(SELECT_THREADS) void floor_kernel(const float2* __restrict__ stats, int64_t ld_stats, int n_groups, int K,
                                                                      float* __restrict__ floor) {
  __shared__ __align__(16) int hist[4][256];
  __shared__ uint32_t klo[SELECT_THREADS / 64], khi[SELECT_THREADS / 64];
  const int t = threadIdx.x;
  stats += (int64_t)blockIdx.x * ld_stats;
  uint32_t lo = 0xFFFFFFFFu, hi = 0u;
  for (int g = t; g < n_groups; g += SELECT_THREADS) {
    const uint32_t k = group_key(stats[g]);
    lo = min(lo, k); hi = max(hi, k);
  }
#pragma unroll
  for (int o = 32; o > 0; o >>= 1) {
    lo = min(lo, (uint32_t)__shfl_xor((int)lo, o, 64));
    hi = max(hi, (uint32_t)__shfl_xor((int)hi, o, 64));
  }
#pragma unroll
  for (int p = 0; p < 4; ++p) hist[p][t] = 0;
  if ((t & 63) == 0) { klo[t >> 6] = lo; khi[t >> 6] = hi; }
  __syncthreads();
#pragma unroll
  for (int w = 0; w < SELECT_THREADS / 64; ++w) { lo = min(lo, klo[w]); hi = max(hi, khi[w]); }
  const Bound b = find_bound([&](auto f) { for (int g = t; g < n_groups; g += SELECT_THREADS) f(group_key(stats[g])); }, lo, hi, K, K + 2, hist);
  if (t == 0) floor[blockIdx.x] = fminf(value_of(b.low), 3.402823466e38f);          // (NaN: the other operand)
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
