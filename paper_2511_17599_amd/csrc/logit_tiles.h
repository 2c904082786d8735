// Logit tiles for calls that keep a few logits of each row: what a row's softmax needs, by groups of consecutive vocabulary
// positions, and either every logit (a chunk of rows, for the selection that follows) or the logits that a list names.
#pragma once
#include "plan.h"
#include "recompute.h"

namespace flce {

// A listed logit of a tile: token row in the tile (bits 0-7), vocabulary position in the tile (8-15), place in the row's list (16-23).
constexpr uint32_t NO_ENTRY = 0xFFFFFFFFu;
__host__ __device__ __forceinline__ constexpr uint32_t list_entry(int row, int pos, int k) {
  return (uint32_t)row | (uint32_t)pos << 8 | (uint32_t)k << 16;
}

template <typename T>
struct LogitArgs {
  const T* H; const T* HT; const T* W;
  int N, d, V, nt0, n_nt, n_vt;         // row tiles nt0 .. nt0 + n_nt - 1 by all vocabulary tiles
  float z_scale;                        // log2(e) / temperature
  float2* stats; int64_t ld_stats;      // [row - first row][group]: (max z, sum exp((z - max) / temperature))
  float* z; int64_t ldz;                // KEEP: [row - first row][position], up to whole tiles
  // otherwise: per row tile TILE * K entries, those of vocabulary tile q from list_begin[q] to list_begin[q + 1]
  const int* list_begin; const uint32_t* entries; int K; float* zt;      // zt[row][place]
};

// The lanes of a wavefront that share a token column: their maximum, their sum, in a fixed order.
template <int COLS>
__device__ __forceinline__ float columns_max(float v) {
  if constexpr (COLS == 16) v = fmaxf(v, __shfl_xor(v, 16, 64));
  return fmaxf(v, __shfl_xor(v, 32, 64));
}
template <int COLS>
__device__ __forceinline__ float columns_sum(float v) {
  if constexpr (COLS == 16) v += __shfl_xor(v, 16, 64);
  return v + __shfl_xor(v, 32, 64);
}
// The value a group's exponentials are taken relative to: its maximum, but 0 where there is none (all -inf) and where it is
// +inf: the sum is then 0 or +inf, and NaN only where a logit is NaN.
__device__ __forceinline__ float finite_or_zero(float m) { return fabsf(m) == __builtin_inff() ? 0.f : m; }

// Workgroups walk the tiles as the recompute step's do (same raster, the next tile's first K stages requested before the current
// one is post-processed).  A group is a block of L::ROWS consecutive positions, all of one wavefront: two or four lanes share a token.
// Bound by the matrix instructions; per logit the post-processing adds an exponential and (KEEP) 4 bytes stored, 64 consecutive
// ones of a row per store instruction.
template <typename T, typename L, bool HKR, bool KEEP>
__global__ __launch_bounds__(L::THREADS, L::MIN_WAVES) void logit_tiles_kernel(LogitArgs<T> a) {
  extern __shared__ __align__(16) char lds[];
  constexpr int COLS = L::ROWS == 64 ? 16 : 32;         // token columns of a block
  const int lane = threadIdx.x & 63;
  const int total = a.n_nt * a.n_vt;
  int t = blockIdx.x;
  if (t >= total) return;
  auto place = [&](int tile, int& p, int& q) {
    // (opaque per tile: the divisions' constants would be kept in scalar registers)
    const int n_nt = fast::scalar(a.n_nt), n_vt = fast::scalar(a.n_vt);
    grouped_raster(xcd_contiguous_id(tile, n_nt * n_vt), n_nt, n_vt, 8, p, q);
  };
  typename L::template Stream<HKR> stream;
  auto start = [&](int p, int q) {
    const int64_t ld_bytes = (int64_t)a.d * sizeof(T);
    stream.start(a.W, ld_bytes, q * L::TILE, a.V, a.H, a.HT, ld_bytes, (a.nt0 + p) * L::TILE, a.N, a.d, lds);
  };
  // The lists run two tiles ahead with the tuned loop: a tile's range is loaded while the tile before the last is computed, its first
  // entries while the last is, so that neither load is waited for ahead of a request.  A range is one vector register, its begin
  // in even lanes and its end in odd ones: the loop has no scalar registers for it.
  auto load_range = [&](int tile) {
    int p, q;
    place(tile, p, q);
    return a.list_begin[(int64_t)(a.nt0 + p) * (a.n_vt + 1) + q + (lane & 1)];
  };
  auto load_entry = [&](int p, int range, int first) {
    const int at = __builtin_amdgcn_readlane(range, 0) + first + lane;
    return at < __builtin_amdgcn_readlane(range, 1) ? a.entries[(int64_t)(a.nt0 + p) * (L::TILE * a.K) + at] : NO_ENTRY;
  };
  int p, q, range = 0, range_next = 0;
  uint32_t entry = NO_ENTRY;
  place(t, p, q);
  if constexpr (!KEEP) {
    range = load_range(t);
    if (t + (int)gridDim.x < total) range_next = load_range(t + gridDim.x);
    entry = load_entry(p, range, 0);
    asm volatile("" : "+v"(entry), "+v"(range_next));
  }
  start(p, q);
  typename L::Acc acc;
  for (;;) {
    const int t_next = t + gridDim.x;
    const bool more = L::TUNED && t_next < total;      // (a loop with nothing to request ahead gets one tile per workgroup)
    uint32_t entry_next = NO_ENTRY;
    int range2 = 0;
    stream.run(lds, acc, [&] {
      if (more) {
        int p_next, q_next;
        place(t_next, p_next, q_next);
        if constexpr (!KEEP) {
          entry_next = load_entry(p_next, range_next, 0);
          if (t_next + (int)gridDim.x < total) range2 = load_range(t_next + gridDim.x);
        }
        start(p_next, q_next);
      }
    });

    place(t, p, q);         // (again: no scalar registers to keep it across the main loop)
    const int v0 = q * L::TILE, n0 = p * L::TILE;      // n0: relative to the launch's first row
    float2* __restrict__ stats = a.stats + (int64_t)n0 * a.ld_stats + v0 / L::ROWS;
#pragma unroll
    for (int j = 0; j < L::WN; ++j) {
      const int n = L::tile_n(j);
      float* __restrict__ zrow = nullptr;
      if constexpr (KEEP) zrow = a.z + (int64_t)(n0 + n) * a.ldz + v0 + L::lane_row();
#pragma unroll
      for (int i = 0; i < L::WM; ++i) {
        const int blk = __builtin_amdgcn_readfirstlane(L::tile_m(i, 0) & ~(L::ROWS - 1));   // first row of the block in the tile
        float z[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) z[r] = acc.get(i, j, r);
        if constexpr (KEEP) {
#pragma unroll
          for (int rq = 0; rq < 4; ++rq)
            *reinterpret_cast<f32x4*>(zrow + blk + rq * L::QUAD) = f32x4{z[rq * 4], z[rq * 4 + 1], z[rq * 4 + 2], z[rq * 4 + 3]};
        }
        if (v0 + blk + L::ROWS > a.V) {
          const int live = a.V - v0 - blk - L::lane_row();
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if ((r >> 2) * L::QUAD + (r & 3) >= live) z[r] = NEG_INF;
        }
        float m = z[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) m = fmaxf(m, z[r]);
        m = columns_max<COLS>(m);
        const float ms = -finite_or_zero(m) * a.z_scale;
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += fast_exp2(fmaf(z[r], a.z_scale, ms));
        sum = columns_sum<COLS>(sum);
        if (lane < COLS) stats[(int64_t)n * a.ld_stats + blk / L::ROWS] = float2{m, sum};
        __builtin_amdgcn_sched_barrier(0);     // one block at a time in VGPRs
      }
    }
    if constexpr (!KEEP) {
      // Listed logits of this tile, 64 entries at a time, one per lane; a block that holds one (ballot) is read again.
      const int count = __builtin_amdgcn_readlane(range, 1) - __builtin_amdgcn_readlane(range, 0);
      for (int c = 0; c < count; c += 64) {
        const uint32_t e = c == 0 ? entry : load_entry(p, range, c);
        // the wavefront's block that holds the lane's entry, if one does (blocks are aligned to their size)
        const int bj = ((int)(e & 255) - (L::tile_n(0) & ~(COLS - 1))) / COLS, bi = ((int)(e >> 8 & 255) - (L::tile_m(0, 0) & ~(L::ROWS - 1))) / L::ROWS;
        const bool mine = e != NO_ENTRY && (int)(e & 255) >= (L::tile_n(0) & ~(COLS - 1)) && bj < L::WN &&
                          (int)(e >> 8 & 255) >= (L::tile_m(0, 0) & ~(L::ROWS - 1)) && bi < L::WM;
        const int block = mine ? bj * L::WM + bi : -1;
#pragma unroll
        for (int j = 0; j < L::WN; ++j) {
#pragma unroll
          for (int i = 0; i < L::WM; ++i) {
            uint64_t hits = __ballot(block == j * L::WM + i);
            if (hits != 0ull) {
              float z[16];
#pragma unroll
              for (int r = 0; r < 16; ++r) z[r] = acc.get(i, j, r);
              do {
                const int from = __builtin_ctzll(hits);
                hits &= hits - 1;
                const uint32_t h = __builtin_amdgcn_readlane(e, from);
                // row rel of a block is register 4 (rel / QUAD) + rel % 4 of the lanes of quarter (or half) rel % QUAD / 4
                const int rel = h >> 8 & (L::ROWS - 1), in = rel % L::QUAD, r = rel / L::QUAD * 4 + (in & 3);
                float v = z[0];
#pragma unroll
                for (int k = 1; k < 16; ++k) v = r == k ? z[k] : v;
                if (lane == in / 4 * COLS + (int)(h & (COLS - 1)))
                  a.zt[(int64_t)((a.nt0 + p) * L::TILE + (int)(h & 255)) * a.K + (h >> 16)] = v;
              } while (hits != 0ull);
            }
            __builtin_amdgcn_sched_barrier(0);
          }
        }
      }
    }
    if (!more) break;
    t = t_next;
    if constexpr (!KEEP) {
      asm volatile("" : "+v"(entry_next), "+v"(range2));
      entry = entry_next; range = range_next; range_next = range2;
    }
  }
}

template <typename T, typename L, bool KEEP>
hipError_t logit_tiles_allowance() {
  static OncePerDevice once;
  return once([] {
    if constexpr (L::TUNED) {
      const hipError_t e = allow_big_lds(logit_tiles_kernel<T, L, true, KEEP>, L::LDS);
      if (e != hipSuccess) return e;
    }
    return allow_big_lds(logit_tiles_kernel<T, L, false, KEEP>, L::LDS);
  });
}

// One launch; at most one round of workgroups with the tuned loop.
template <typename T, typename L, bool KEEP>
void launch_logit_tiles(const LogitArgs<T>& a, hipStream_t st) {
  int grid = a.n_nt * a.n_vt;
  if constexpr (L::TUNED) {
    if (grid > NUM_CU * L::PER_CU) grid = NUM_CU * L::PER_CU;
    if (a.HT) { logit_tiles_kernel<T, L, true, KEEP><<<grid, L::THREADS, L::LDS, st>>>(a); return; }
  }
  logit_tiles_kernel<T, L, false, KEEP><<<grid, L::THREADS, L::LDS, st>>>(a);
}

}  // namespace flce
