// Distillation from a teacher's largest logits: the lists by tile, the forward's tiles, a row's loss and the shares that the backward
// subtracts, and their place in G.
//   p_k = softmax over the list of t_k / T;  loss = T^2 sum_k p_k (log p_k - z_{id_k} / T + lse),  lse = log sum_v exp(z_v / T)
//   d loss / d z_v = T (exp(z_v / T - lse) - sum of p_k with id_k = v)
// An entry with a negative id is absent, one whose logit is -inf has no share; a row without a share does not count.
#pragma once
#include "plan.h"
#include "recompute.h"

namespace flce {

constexpr int DISTILL_MAX = 256;          // entries of a list
// A listed logit of a tile: token row in the tile (bits 0-7), vocabulary position in the tile (8-15), place in the row's list (16-23).
constexpr uint32_t NO_ENTRY = 0xFFFFFFFFu;
__host__ __device__ __forceinline__ constexpr uint32_t list_entry(int row, int pos, int k) {
  return (uint32_t)row | (uint32_t)pos << 8 | (uint32_t)k << 16;
}
constexpr int LIST_BUCKETS = 8192;

// Entries of each row tile sorted by vocabulary tile and, inside it, by the wavefront that computes them (2 along the positions, NW along
// the rows; in no order beyond that: each entry has a place of its own to write to).
// One block per row tile: count, prefix sum, place.  A chain of latencies: a thread's first LIST_HELD entries are loaded together and
// stay in registers (256 rows x 32 entries are all of them), further ones are read twice, four at a time.  (2048 rows x 32 entries 18.4 us without that,
// 11.0 with it.)
constexpr int LIST_HELD = 8;
template <int E, int NW>
__global__ __launch_bounds__(1024) void distill_lists_kernel(const int64_t* __restrict__ ids, const float* __restrict__ t, int N, int V, int K,
                                                             int n_vt_all, int* __restrict__ list_begin, uint32_t* __restrict__ entries,
                                                             Header* __restrict__ hdr) {
  constexpr int S = 2 * NW;
  const int n_vt = n_vt_all * S;          // buckets
  __shared__ int cnt[LIST_BUCKETS];
  __shared__ int wsum[16];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int n0 = blockIdx.x * E, total = min(E, N - n0) * K;
  ids += (int64_t)n0 * K; t += (int64_t)n0 * K;
  list_begin += (int64_t)blockIdx.x * (n_vt + 1);
  entries += (int64_t)blockIdx.x * E * K;
  if (blockIdx.x == 0 && tid == 0) hdr->arrived = 0;      // for the loss that follows on the stream
  // id of entry i, -1 where it has no share
  auto share_id = [&](int64_t id, float x) { return id >= 0 && id < V && x != NEG_INF ? (int)id : -1; };
  int held[LIST_HELD];
  {
    int64_t id[LIST_HELD];
    float x[LIST_HELD];
#pragma unroll
    for (int u = 0; u < LIST_HELD; ++u) {
      if (u * 1024 >= total) break;
      const int i = min(tid + u * 1024, total - 1);
      id[u] = ids[i]; x[u] = t[i];
    }
#pragma unroll
    for (int u = 0; u < LIST_HELD; ++u)          // (all ones past the end, without a mask kept for each)
      held[u] = u * 1024 < total ? share_id(id[u], x[u]) | ((total - 1 - tid - u * 1024) >> 31) : -1;
  }
  // f(i, id) for every entry with a share
  auto each = [&](auto f) {
#pragma unroll
    for (int u = 0; u < LIST_HELD; ++u)
      if (held[u] >= 0) f(tid + u * 1024, held[u]);
    for (int i0 = LIST_HELD * 1024; i0 < total; i0 += 4 * 1024) {
      int id[4];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int i = min(i0 + u * 1024 + tid, total - 1);
        id[u] = share_id(ids[i], t[i]);
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (i0 + u * 1024 + tid < total && id[u] >= 0) f(i0 + u * 1024 + tid, id[u]);
    }
  };
  auto bucket = [&](int i, int id) { return id / E * S + id % E / (E / 2) * NW + i / K / (E / NW); };
  int base = 0;
  for (int q0 = 0; q0 < n_vt; q0 += LIST_BUCKETS) {
    const int nq = min(LIST_BUCKETS, n_vt + 1 - q0);        // (with the one behind the last tile: the end)
    for (int i = tid; i < LIST_BUCKETS; i += 1024) cnt[i] = 0;
    __syncthreads();
    each([&](int i, int id) {
      const int q = bucket(i, id) - q0;
      if (q >= 0 && q < LIST_BUCKETS) atomicAdd(&cnt[q], 1);
    });
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
    for (int k = 0; k < PER; ++k) { cnt[tid * PER + k] = at; at += own[k]; }
    __syncthreads();
    for (int i = tid; i < nq; i += 1024) list_begin[q0 + i] = cnt[i];
    __syncthreads();
    each([&](int i, int id) {
      const int q = bucket(i, id) - q0;
      if (q >= 0 && q < LIST_BUCKETS) entries[atomicAdd(&cnt[q], 1)] = list_entry(i / K, id % E, i % K);
    });
    base += all;
    __syncthreads();
  }
  if (n_vt % LIST_BUCKETS == 0 && tid == 0) list_begin[n_vt] = base;
}

// Merge of (m, a) pairs in units of 1 / T in slot order, as merge_fixed does it; NaN and +inf go through.
template <int S>
__device__ __forceinline__ void merge_scaled(const float (&m)[S], const float (&a)[S], float z_scale, float& M, float& A) {
  M = NEG_INF;
#pragma unroll
  for (int k = 0; k < S; ++k) M = fmaxf(M, m[k]);
  A = 0.f;
#pragma unroll
  for (int k = 0; k < S; ++k) if (a[k] != 0.f) A += a[k] * fast_exp2((m[k] - M) * z_scale);
}

// Token columns of a block, and a loop's wavefronts along the rows: the lists are sorted for two times these.
template <typename L>
constexpr int list_columns() { return L::ROWS == 64 ? 16 : 32; }
template <typename L>
constexpr int list_waves() {
  constexpr int waves = L::TILE / (L::WN * list_columns<L>());
  static_assert(L::THREADS == 64 * 2 * waves, "two wavefronts along the positions");
  return waves;
}

// Where the slices are: in the stage that the tuned loop leaves free between tiles, anywhere with the others.
template <typename L>
__host__ __device__ constexpr int list_lds() {
  if constexpr (L::TUNED) return L::FREE_LDS_OFFSET;
  else return 0;
}

template <typename T>
struct DistillTileArgs {
  const T* H; const T* HT; const T* W;
  int N, d, V, n_rb, n_win, n_vt;
  double vt_per_win;
  float z_scale;                        // log2(e) / T
  float* part; int64_t npad;            // [2][n_win][npad]: m, a per (window, row)
  int item_begin;
  // per row tile TILE * K entries, those of bucket b (vocabulary tile, wavefront) from list_begin[b] to list_begin[b + 1]
  const int* list_begin; const uint32_t* entries; int K; float2* saved;  // saved[row][place].y: the logit
};

// The forward's tiles: its walk over a window's vocabulary tiles, its online (m, a) in units of 1 / T, and after each tile the logits
// that the lists name there: a wavefront's entries 64 at a time, one per lane; a column of its blocks that holds some (ballot) goes through
// the wavefront's slice of LDS, from where each entry's lane takes its logit, however many they are.  Bound by the matrix
// instructions; a tile without entries costs a load and a comparison.  The logit handed out is the one in the row's sum bit
// for bit, which exp(z - lse) - share needs where both are near 1 (a dot product of its own would also read N K rows of W, 2.1 GB
// at 8192 x 4096 with 32 entries a row).
template <typename T, typename L, bool HKR>
__global__ __launch_bounds__(L::THREADS, L::MIN_WAVES) void distill_tiles_kernel(DistillTileArgs<T> a) {
  extern __shared__ __align__(16) char lds[];
  constexpr int COLS = list_columns<L>(), NW = list_waves<L>();
  constexpr int POS = L::WM * L::ROWS;                  // positions of a wavefront's column of blocks
  static_assert(list_lds<L>() + L::THREADS / 64 * (COLS * POS * 4) <= L::LDS, "a slice per wavefront");
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int id = a.item_begin + xcd_contiguous_id(blockIdx.x, gridDim.x);
  int rb, win;
  grouped_raster(id, a.n_rb, a.n_win, FLCE_FWD_GROUP, rb, win);
  // (as the cross-entropy's forward places its windows)
  const int vt_begin = __builtin_amdgcn_readfirstlane((int)(win * a.vt_per_win));
  const int vt_end = win + 1 < a.n_win ? __builtin_amdgcn_readfirstlane((int)((win + 1) * a.vt_per_win)) : a.n_vt;
  const int n0 = rb * L::TILE;
  const int64_t ld_bytes = (int64_t)a.d * sizeof(T);
  // The lists run two tiles ahead: a tile's range is loaded while the tile before the last is computed, its first entries while the
  // last is, so that neither load is waited for ahead of a request.  A range is one vector register, its begin in even lanes
  // and its end in odd ones: the loop has no scalar registers for it.
  auto load_range = [&](int vt) { return a.list_begin[(int64_t)rb * (a.n_vt * 2 * NW + 1) + vt * 2 * NW + wave + (lane & 1)]; };
  auto load_entry = [&](int range, int first) {
    const int at = __builtin_amdgcn_readlane(range, 0) + first + lane;
    return at < __builtin_amdgcn_readlane(range, 1) ? a.entries[(int64_t)rb * (L::TILE * a.K) + at] : NO_ENTRY;
  };
  float m[L::WN], s[L::WN];
#pragma unroll
  for (int j = 0; j < L::WN; ++j) { m[j] = NEG_INF; s[j] = 0.f; }
  int range = 0, range_next = 0;
  uint32_t entry = NO_ENTRY;
  typename L::Acc acc;
  typename L::template Stream<HKR> stream;
  if (vt_begin < vt_end) {
    if constexpr (L::TUNED) {
      range = load_range(vt_begin);
      range_next = load_range(min(vt_begin + 1, a.n_vt - 1));
      entry = load_entry(range, 0);
      asm volatile("" : "+v"(entry), "+v"(range_next));
    }
    stream.start(a.W, ld_bytes, vt_begin * L::TILE, a.V, a.H, a.HT, ld_bytes, n0, a.N, a.d, lds);
  }
  for (int vt = vt_begin; vt < vt_end; ++vt) {
    const int v0 = vt * L::TILE;
    uint32_t entry_next = NO_ENTRY;
    int range2 = 0;
    stream.run(lds, acc, [&] {
      if (vt + 1 < vt_end) {
        if constexpr (L::TUNED) {
          entry_next = load_entry(range_next, 0);
          range2 = load_range(min(vt + 2, a.n_vt - 1));
        }
        stream.start(a.W, ld_bytes, v0 + L::TILE, a.V, a.H, a.HT, ld_bytes, n0, a.N, a.d, lds);
      }
    });
#pragma unroll
    for (int j = 0; j < L::WN; ++j) {
#pragma unroll
      for (int i = 0; i < L::WM; ++i) {
        const int blk0 = v0 + __builtin_amdgcn_readfirstlane(L::tile_m(i, 0) & ~(L::ROWS - 1));   // first row of the block
        if (blk0 >= a.V) continue;
        float z[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) z[r] = acc.get(i, j, r);
        if (blk0 + L::ROWS > a.V) {
          const int live = a.V - blk0 - L::lane_row();
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if ((r >> 2) * L::QUAD + (r & 3) >= live) z[r] = NEG_INF;
        }
        float bmax = z[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) bmax = fmaxf(bmax, z[r]);
        const float mn = fmaxf(m[j], bmax);
        const float ms = (mn == NEG_INF) ? 0.f : mn;     // nothing but padding so far: keep exp arguments finite
        // (the difference first: a logit's product with z_scale may be no number where the difference is one)
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += fast_exp2((z[r] - ms) * a.z_scale);
        s[j] = s[j] * fast_exp2((m[j] - ms) * a.z_scale) + sum;
        m[j] = mn;
        __builtin_amdgcn_sched_barrier(0);     // one block at a time in VGPRs
      }
    }
    if constexpr (!L::TUNED) {              // nothing is requested ahead, and no registers to spare across that main loop
      range = load_range(vt);
      entry = load_entry(range, 0);
    }
    const int count = __builtin_amdgcn_readlane(range, 1) - __builtin_amdgcn_readlane(range, 0);
    // [column][position], the 16-byte chunk number XOR-ed with the column: what a store or a read touches lies in different banks
    float* slice = reinterpret_cast<float*>(lds + list_lds<L>() + wave * (COLS * POS * 4));
    auto slot = [](int col, int chunk) { return col * POS + ((chunk ^ (col & (POS / 4 < 16 ? POS / 4 - 1 : 15))) << 2); };
    for (int c = 0; c < count; c += 64) {
      const uint32_t e = c == 0 ? entry : load_entry(range, c);
      const int row = e & (L::WN * COLS - 1), pos = e >> 8 & (POS - 1);       // in the wavefront's part of the tile
      const int ej = e != NO_ENTRY ? row / COLS : -1;
#pragma unroll
      for (int j = 0; j < L::WN; ++j) {
        if (__ballot(ej == j) == 0ull) continue;
        int ln = lane;
        asm volatile("" : "+v"(ln));          // (nothing derived from it is kept across the main loop)
        const int col = ln & (COLS - 1);
#pragma unroll
        for (int i = 0; i < L::WM; ++i) {
#pragma unroll
          for (int rq = 0; rq < 4; ++rq)
            *reinterpret_cast<f32x4*>(slice + slot(col, (i * L::ROWS + rq * L::QUAD) / 4 + ln / COLS)) =
                f32x4{acc.get(i, j, rq * 4), acc.get(i, j, rq * 4 + 1), acc.get(i, j, rq * 4 + 2), acc.get(i, j, rq * 4 + 3)};
          __builtin_amdgcn_sched_barrier(0);
        }
        // (a wavefront's LDS operations complete in order)
        if (ej == j) a.saved[(int64_t)(n0 + (int)(e & 255)) * a.K + (e >> 16)].y = slice[slot(row & (COLS - 1), pos / 4) + (pos & 3)];
      }
    }
    if constexpr (!L::TUNED) __syncthreads();       // the next tile's operands go where the slices are
    if constexpr (L::TUNED) {
      asm volatile("" : "+v"(entry_next), "+v"(range2));
      entry = entry_next; range = range_next; range_next = range2;
    }
  }

  // SLOTS lanes hold partial state of each token: merged in fixed slot order through LDS (free after the main loop's last barrier)
  constexpr int S = L::SLOTS;
  float* sm = reinterpret_cast<float*>(lds);
  float* sa = sm + S * L::TILE;
  const int slot = L::slot();
#pragma unroll
  for (int j = 0; j < L::WN; ++j) {
    sm[slot * L::TILE + L::tile_n(j)] = m[j];
    sa[slot * L::TILE + L::tile_n(j)] = s[j];
  }
  __syncthreads();
  if (threadIdx.x < L::TILE) {
    float pm[S], pa[S];
#pragma unroll
    for (int k = 0; k < S; ++k) { pm[k] = sm[k * L::TILE + threadIdx.x]; pa[k] = sa[k * L::TILE + threadIdx.x]; }
    float M, A;
    merge_scaled<S>(pm, pa, a.z_scale, M, A);
    const int64_t o = (int64_t)win * a.npad + n0 + threadIdx.x;
    a.part[o] = M;
    a.part[(int64_t)a.n_win * a.npad + o] = A;
  }
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

// The forward's end, a wavefront per row: lse from the windows' (m, a), the row's loss, and what the backward needs: shares (the
// whole share of an id at its first place in the row, -1 at the others and where there is none) and the target that the row preparation
// counts rows by (V: counts, matches no column; -1: does not count; V + 1: out of range).  Per-block sums in fixed order, and the
// call's loss from them by the block that hands its sums in last (merge_rows_kernel's way).  A chain of latencies; R rows per block:
// 16, since the blocks count in one word, one after the other (7911 rows 15 us, in blocks of 4 31), but 4 where that leaves few blocks for a
// list's comparisons (190 rows x 105 entries 10 us, in blocks of 16 16).
constexpr int DISTILL_ROWS = 16, DISTILL_FEW_ROWS = 4, DISTILL_FEW = 1024;
inline int distill_rows_per_block(int64_t N) { return N <= DISTILL_FEW ? DISTILL_FEW_ROWS : DISTILL_ROWS; }
struct DistillRowArgs {
  const int64_t* ids; const float* t; float2* saved; int64_t* target;
  int N, V, K, n_win;
  const float* part; int64_t npad;
  float temperature, inv_T, z_scale;
  float* lse_out; float* loss_rows_out;
  LossOut o;
};
template <int R>
__global__ __launch_bounds__(64 * R) void distill_rows_kernel(DistillRowArgs a) {
  __shared__ int2 entry[R][DISTILL_MAX];        // (id, share's bits)
  __shared__ float sl[R];
  __shared__ int sc[R], so[R], last;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int64_t n = (int64_t)blockIdx.x * R + wave;
  float loss = 0.f;
  bool counts = false, oor = false;
  if (n < a.N) {
    const float* __restrict__ pm = a.part + n;
    const float* __restrict__ pa = pm + (int64_t)a.n_win * a.npad;
    float m = NEG_INF, sum = 0.f;
    RowList list;
    float2* __restrict__ saved = a.saved + n * a.K;
    float z[RowList::U];
#pragma unroll
    for (int u = 0; u < RowList::U; ++u) z[u] = lane + 64 * u < a.K ? saved[lane + 64 * u].y : 0.f;      // (undefined without a share)
    list.load(a.ids + n * a.K, a.t + n * a.K, a.K, a.V, a.inv_T);
#pragma unroll
    for (int u = 0; u < RowList::U; ++u) entry[wave][lane + 64 * u] = int2{list.id[u], __float_as_int(list.p[u])};
    for (int w0 = 0; w0 < a.n_win; w0 += 4 * 64) {          // four windows per lane at a time, all their loads in flight together
      float mw[5], aw[5];
#pragma unroll
      for (int u = 0; u < 4; ++u) {
        const int w = w0 + u * 64 + lane;
        const int64_t at = (int64_t)min(w, a.n_win - 1) * a.npad;
        mw[u] = pm[at]; aw[u] = pa[at];
      }
#pragma unroll
      for (int u = 0; u < 4; ++u)
        if (w0 + u * 64 + lane >= a.n_win) { mw[u] = NEG_INF; aw[u] = 0.f; }
      mw[4] = m; aw[4] = sum;
      merge_scaled<5>(mw, aw, a.z_scale, m, sum);
    }
#pragma unroll
    for (int o = 32; o > 0; o >>= 1) {
      const float mw[2] = {m, __shfl_xor(m, o, 64)}, aw[2] = {sum, __shfl_xor(sum, o, 64)};
      merge_scaled<2>(mw, aw, a.z_scale, m, sum);
    }
    // (m / T and log sum are kept apart in the loss: where the largest logit is far from 0 their sum has lost the logarithm)
    const float log_a = logf(sum), lse = fmaf(m, a.inv_T, log_a);
    counts = list.counts;
    oor = list.out_of_range;
    float kl = 0.f;
#pragma unroll
    for (int u = 0; u < RowList::U; ++u)
      if (list.id[u] >= 0 && list.p[u] != 0.f) kl += list.p[u] * ((list.x[u] - list.log_sum) + fmaf(m - z[u], a.inv_T, log_a));
    kl = wave_sum(kl);
    loss = counts ? a.temperature * a.temperature * kl : 0.f;
    // every entry against all of the row's, eight at a time (a wavefront reads what it wrote: LDS operations of one are in order)
    float share[RowList::U];
    int earlier[RowList::U];
#pragma unroll
    for (int u = 0; u < RowList::U; ++u) { share[u] = 0.f; earlier[u] = 0; }
    for (int o0 = 0; o0 < a.K; o0 += 8) {          // (past K there are entries without an id)
      int2 e[8];
#pragma unroll
      for (int o = 0; o < 8; ++o) e[o] = entry[wave][o0 + o];
#pragma unroll
      for (int u = 0; u < RowList::U; ++u) {
        if (64 * u >= a.K) break;
#pragma unroll
        for (int o = 0; o < 8; ++o) {
          const int same = e[o].x == list.id[u] ? -1 : 0;
          share[u] += __int_as_float(e[o].y & same);
          earlier[u] |= same & (o0 + o - (lane + 64 * u));        // (negative: an entry with the id stands before this one)
        }
      }
    }
#pragma unroll
    for (int u = 0; u < RowList::U; ++u) {
      const int k = lane + 64 * u;
      if (k < a.K) saved[k] = float2{list.id[u] >= 0 && earlier[u] >= 0 ? share[u] : -1.f, list.id[u] >= 0 ? z[u] : 0.f};
    }
    if (lane == 0) {
      a.lse_out[n] = lse;
      a.target[n] = oor ? (int64_t)a.V + 1 : counts ? a.V : -1;
      if (a.loss_rows_out) a.loss_rows_out[n] = loss;
    }
  }
  if (lane == 0) { sl[wave] = loss; sc[wave] = counts; so[wave] = oor; }
  __syncthreads();
  if (threadIdx.x == 0) {
    float l = 0.f;
    int c = 0, bad = 0;
#pragma unroll
    for (int w = 0; w < R; ++w) { l += sl[w]; c += sc[w]; bad |= so[w]; }
    const int b = blockIdx.x;
    __hip_atomic_store(a.o.blk_loss + b, l, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(a.o.blk_cnt + b, c, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    __hip_atomic_store(a.o.blk_oor + b, bad, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");      // the three stores have reached the point the other XCDs read from
    last = __hip_atomic_fetch_add(&a.o.hdr->arrived, 1u, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) == gridDim.x - 1;
  }
  __syncthreads();
  if (last) finalize_loss(a.o, gridDim.x);
}

// The listed elements of a staged chunk of G: exp(z / T - lse) - share, from the forward's logit and in one rounding, over what the
// recompute step wrote there (which knows no lists).  A thread per entry of the chunk's rows.
// Rounded to T as all of G is, whose matrix instructions take no wider one: dH and dW in bf16 are 2.3e-3 of their norm away from 64 bits,
// where the rounding of the results alone makes 1.65e-3 (2048 x 1024 x 32000 and 8192 x 4096 x 128256).
template <typename T, typename L, bool PER_ROW>
__global__ __launch_bounds__(256) void distill_scatter_kernel(RecomputeArgs<T> a, DistillLists x, const int* __restrict__ rowmap) {
  const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
  const int rl = (int)(i / x.K), k = (int)(i - (int64_t)rl * x.K);          // row of the chunk, place in its list
  const int c = a.nt0 * L::TILE + rl;
  if (rl >= a.n_nt * L::TILE || c >= a.hdr->n_valid) return;
  const int64_t at = (int64_t)rowmap[c] * x.K + k;
  const float2 saved = x.saved[at];
  if (saved.x < 0.f) return;
  const int64_t v = x.ids[at] - (int64_t)a.vt0 * L::TILE;
  if (v < 0 || v >= (int64_t)a.n_vt * L::TILE) return;
  float g = fast_exp2(fmaf(saved.y, x.z_scale, -x.lse[rowmap[c]] * LOG2E)) - saved.x;
  if constexpr (PER_ROW) g *= a.gam_c[c] * x.temperature;
  if constexpr (L::TUNED)
    *reinterpret_cast<T*>(reinterpret_cast<char*>(a.G) + (int64_t)(rl >> 4) * a.ldG + (v >> 5) * 1024 + (rl & 15) * 64 + (v & 31) * 2) = Pack4<T>::one(g);
  else
    a.G[(int64_t)rl * a.ldG + v] = Pack4<T>::one(g);
  if constexpr (!L::TRANSPOSING) a.GT[v * a.ldGT + rl] = Pack4<T>::one(g);
}

}  // namespace flce
