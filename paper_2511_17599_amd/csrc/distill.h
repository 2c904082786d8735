// Distillation from a teacher's largest logits: the lists by tile for the forward's tiles, a row's loss, the shares the backward
// subtracts, and their place in G.
//   p_k = softmax over the list of t_k / T;  loss = T^2 sum_k p_k (log p_k - z_{id_k} / T + lse),  lse = log sum_v exp(z_v / T)
//   d loss / d z_v = T (exp(z_v / T - lse) - sum of p_k with id_k = v)
// An entry with a negative id is absent, one whose logit is -inf has no share; a row without a share does not count.
#pragma once
#include "logit_tiles.h"

namespace flce {

constexpr int DISTILL_MAX = 256;          // entries of a list
constexpr int LIST_BUCKETS = 8192;

// Entries of each row tile sorted by vocabulary tile (in no order inside one: each has a place of its own to write to).
// One block per row tile: count, prefix sum, place; a chain of latencies, two reads of the lists.
template <int E>
__global__ __launch_bounds__(1024) void distill_lists_kernel(const int64_t* __restrict__ ids, const float* __restrict__ t, int N, int V, int K,
                                                             int n_vt, int* __restrict__ list_begin, uint32_t* __restrict__ entries,
                                                             float* __restrict__ zt, Header* __restrict__ hdr) {
  __shared__ int cnt[LIST_BUCKETS];
  __shared__ int wsum[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n0 = blockIdx.x * E, total = min(E, N - n0) * K;
  ids += (int64_t)n0 * K; t += (int64_t)n0 * K; zt += (int64_t)n0 * K;
  list_begin += (int64_t)blockIdx.x * (n_vt + 1);
  entries += (int64_t)blockIdx.x * E * K;
  if (blockIdx.x == 0 && tid == 0) hdr->arrived = 0;      // for the loss that follows on the stream
  auto listed = [&](int i, int64_t& id) {
    id = ids[i];
    return id >= 0 && id < V && t[i] != NEG_INF;
  };
  int base = 0;
  for (int q0 = 0; q0 < n_vt; q0 += LIST_BUCKETS) {
    for (int i = tid; i < LIST_BUCKETS; i += 1024) cnt[i] = 0;
    __syncthreads();
    for (int i = tid; i < total; i += 1024) {
      int64_t id;
      const bool in = listed(i, id);
      if (q0 == 0 && !in) zt[i] = 0.f;
      const int q = in ? (int)id / E - q0 : -1;
      if (q >= 0 && q < LIST_BUCKETS) atomicAdd(&cnt[q], 1);
    }
    __syncthreads();
    constexpr int PER = LIST_BUCKETS / 1024;
    int own[PER], sum = 0;
#pragma unroll
    for (int k = 0; k < PER; ++k) { own[k] = cnt[tid * PER + k]; sum += own[k]; }
    int incl = sum;
#pragma unroll
    for (int o = 1; o < 64; o <<= 1) {
      const int x = __shfl_up(incl, o, 64);
      if (lane >= o) incl += x;
    }
    if (lane == 63) wsum[wave] = incl;
    __syncthreads();
    int at = base + incl - sum, all = 0;
#pragma unroll
    for (int w = 0; w < 16; ++w) { if (w < wave) at += wsum[w]; all += wsum[w]; }
#pragma unroll
    for (int k = 0; k < PER; ++k) {
      const int q = tid * PER + k;
      cnt[q] = at;
      if (q0 + q <= n_vt) list_begin[q0 + q] = at;        // (the one behind the last tile: the end)
      at += own[k];
    }
    __syncthreads();
    for (int i = tid; i < total; i += 1024) {
      int64_t id;
      if (!listed(i, id)) continue;
      const int q = (int)id / E - q0;
      if (q >= 0 && q < LIST_BUCKETS) entries[atomicAdd(&cnt[q], 1)] = list_entry(i / K, (int)id % E, i % K);
    }
    base += all;
    __syncthreads();
  }
  if (n_vt % LIST_BUCKETS == 0 && tid == 0) list_begin[n_vt] = base;
}

// One row's list in the lanes of a wavefront: entry lane + 64 u is the lane's u-th.
struct RowList {
  static constexpr int U = DISTILL_MAX / 64;
  int id[U];                // -1: absent or without a share
  float x[U], p[U];         // (t - max) / T, share
  float log_sum;            // log sum exp x
  bool counts, out_of_range;
  __device__ __forceinline__ void load(const int64_t* __restrict__ ids, const float* __restrict__ t, int K, int V, float inv_T) {
    const int lane = threadIdx.x & 63;
    bool oor = false, any = false;
    float tt[U], m = NEG_INF;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = lane + 64 * u;
      const int64_t v = k < K ? ids[k] : -1;
      tt[u] = k < K ? t[k] : NEG_INF;
      oor |= v >= V;
      id[u] = v >= 0 && v < V && tt[u] != NEG_INF ? (int)v : -1;
      any |= id[u] >= 0;
      if (id[u] >= 0) m = fmaxf(m, tt[u]);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    float sum = 0.f;
#pragma unroll
    for (int u = 0; u < U; ++u) {
      x[u] = (tt[u] - m) * inv_T;
      p[u] = id[u] >= 0 ? fast_exp2(x[u] * LOG2E) : 0.f;
      sum += p[u];
    }
    sum = wave_sum(sum);
    log_sum = logf(sum);
    const float inv = 1.f / sum;
#pragma unroll
    for (int u = 0; u < U; ++u) if (id[u] >= 0) p[u] *= inv;
    out_of_range = __ballot(oor) != 0ull;
    counts = __ballot(any) != 0ull && !out_of_range;
  }
};

// The forward's end, a wavefront per row: lse from the groups' (max, sum), the row's loss; per-block sums in fixed order, and
// the call's loss from them by the block that hands its sums in last (merge_rows_kernel's way).  Bound by the read of the groups' pairs.
constexpr int DISTILL_ROWS = 4;
struct DistillRowArgs {
  const int64_t* ids; const float* t; const float* zt;
  int row0, rows, V, K, n_groups;
  const float2* stats; int64_t ld_stats;
  float temperature, inv_T, z_scale;
  float* lse_out; float* loss_rows_out;
  LossOut o; int blk0, n_blk;             // this launch's first block among all of the call's
};
static __global__ __launch_bounds__(64 * DISTILL_ROWS) void distill_rows_kernel(DistillRowArgs a) {
  __shared__ float sl[DISTILL_ROWS];
  __shared__ int sc[DISTILL_ROWS], so[DISTILL_ROWS], last;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r = blockIdx.x * DISTILL_ROWS + wave;
  float loss = 0.f;
  bool counts = false, oor = false;
  if (r < a.rows) {
    const int64_t n = a.row0 + r;
    const float2* __restrict__ s = a.stats + (int64_t)r * a.ld_stats;
    RowList list;
    list.load(a.ids + n * a.K, a.t + n * a.K, a.K, a.V, a.inv_T);
    float z[RowList::U];
#pragma unroll
    for (int u = 0; u < RowList::U; ++u) z[u] = list.id[u] >= 0 ? a.zt[n * a.K + lane + 64 * u] : 0.f;
    float m = NEG_INF;
#pragma unroll 8
    for (int g = lane; g < a.n_groups; g += 64) m = fmaxf(m, s[g].x);
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    m = finite_or_zero(m);
    float sum = 0.f;
#pragma unroll 8
    for (int g = lane; g < a.n_groups; g += 64) {
      const float2 x = s[g];
      if (x.y != 0.f) sum += x.y * fast_exp2((finite_or_zero(x.x) - m) * a.z_scale);
    }
    sum = wave_sum(sum);
    const float lse = fmaf(m, a.inv_T, logf(sum));
    counts = list.counts;
    oor = list.out_of_range;
    float kl = 0.f;
#pragma unroll
    for (int u = 0; u < RowList::U; ++u)
      if (list.id[u] >= 0 && list.p[u] != 0.f) kl += list.p[u] * ((list.x[u] - list.log_sum) + fmaf(-z[u], a.inv_T, lse));
    kl = wave_sum(kl);
    loss = counts ? a.temperature * a.temperature * kl : 0.f;
    if (lane == 0) {
      a.lse_out[n] = lse;
      if (a.loss_rows_out) a.loss_rows_out[n] = loss;
    }
  }
  if (lane == 0) { sl[wave] = loss; sc[wave] = counts; so[wave] = oor; }
  __syncthreads();
  if (threadIdx.x == 0) {
    float l = 0.f;
    int c = 0, bad = 0;
#pragma unroll
    for (int w = 0; w < DISTILL_ROWS; ++w) { l += sl[w]; c += sc[w]; bad |= so[w]; }
    const int b = a.blk0 + blockIdx.x;
    __hip_atomic_store(a.o.blk_loss + b, l, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(a.o.blk_cnt + b, c, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(a.o.blk_oor + b, bad, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // the three stores have reached the point the other XCDs read from
    last = __hip_atomic_fetch_add(&a.o.hdr->arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == (uint32_t)a.n_blk - 1;
  }
  __syncthreads();
  if (last) finalize_loss(a.o, a.n_blk);
}

// The backward's start, a wavefront per row: shares (the whole share of an id at its first place in the row, -1 at the others and
// where there is none), the targets that the row preparation counts rows by (V: counts, matches no column; -1: does not count;
// V + 1: out of range), upstream gradients times T.
struct DistillPrepArgs {
  const int64_t* ids; const float* t; int N, V, K; float inv_T, temperature;
  float* share; int64_t* target;
  const float* grad_loss; const float* grad_rows; float* grad_loss_T; float* grad_rows_T;
};
static __global__ __launch_bounds__(64 * DISTILL_ROWS) void distill_prep_kernel(DistillPrepArgs a) {
  __shared__ int sid[DISTILL_ROWS][DISTILL_MAX];
  __shared__ float sp[DISTILL_ROWS][DISTILL_MAX];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t n = (int64_t)blockIdx.x * DISTILL_ROWS + wave;
  if (n == 0 && lane == 0 && a.grad_loss) *a.grad_loss_T = *a.grad_loss * a.temperature;
  const bool row = n < a.N;
  RowList list;
  if (row) {
    list.load(a.ids + n * a.K, a.t + n * a.K, a.K, a.V, a.inv_T);
#pragma unroll
    for (int u = 0; u < RowList::U; ++u) { sid[wave][lane + 64 * u] = list.id[u]; sp[wave][lane + 64 * u] = list.p[u]; }
  }
  __syncthreads();
  if (!row) return;
  if (lane == 0) {
    a.target[n] = list.out_of_range ? (int64_t)a.V + 1 : list.counts ? a.V : -1;
    if (a.grad_rows) a.grad_rows_T[n] = a.grad_rows[n] * a.temperature;
  }
#pragma unroll
  for (int u = 0; u < RowList::U; ++u) {
    const int k = lane + 64 * u;
    if (64 * u >= a.K) break;
    float sum = 0.f;
    bool first = list.id[u] >= 0;
    for (int o = 0; o < a.K; ++o) {
      const bool same = sid[wave][o] == list.id[u];
      if (same) sum += sp[wave][o];
      first = first && !(same && o < k);
    }
    if (k < a.K) a.share[n * a.K + k] = first ? sum : -1.f;
  }
}

// The listed elements of a staged chunk of G: exp(z / T - lse) - share, from the forward's logit and in one rounding, over what the
// recompute step wrote there (which knows no lists).  A thread per entry of the chunk's rows.
template <typename T, typename L, bool PER_ROW>
__global__ __launch_bounds__(256) void distill_scatter_kernel(RecomputeArgs<T> a, DistillLists x, const int* __restrict__ rowmap) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int rl = (int)(i / x.K), k = (int)(i - (int64_t)rl * x.K);          // row of the chunk, place in its list
  const int c = a.nt0 * L::TILE + rl;
  if (rl >= a.n_nt * L::TILE || c >= a.hdr->n_valid) return;
  const int64_t at = (int64_t)rowmap[c] * x.K + k;
  const float share = x.share[at];
  if (share < 0.f) return;
  const int64_t v = x.ids[at] - (int64_t)a.vt0 * L::TILE;
  if (v < 0 || v >= (int64_t)a.n_vt * L::TILE) return;
  float g = fast_exp2(fmaf(x.zt[at], x.z_scale, -x.lse[rowmap[c]] * LOG2E)) - share;
  if constexpr (PER_ROW) g *= a.gam_c[c];
  if constexpr (L::TUNED)
    *reinterpret_cast<T*>(reinterpret_cast<char*>(a.G) + (int64_t)(rl >> 4) * a.ldG + (v >> 5) * 1024 + (rl & 15) * 64 + (v & 31) * 2) = Pack4<T>::one(g);
  else
    a.G[(int64_t)rl * a.ldG + v] = Pack4<T>::one(g);
  if constexpr (!L::TRANSPOSING) a.GT[v * a.ldGT + rl] = Pack4<T>::one(g);
}

}  // namespace flce
