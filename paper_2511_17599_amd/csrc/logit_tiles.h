// Logit tiles for the selection of a row's largest logits: every logit of a chunk of rows, and by groups of consecutive vocabulary
// positions the maximum and the sum of exponentials.
#pragma once
#include "plan.h"
#include "recompute.h"

namespace flce {

// Words that a later kernel on the stream counts in.
struct ZeroWords {
  uint32_t* word; int n;
  __device__ __forceinline__ void by_first_block() const {
    if (blockIdx.x == 0)
      for (int i = threadIdx.x; i < n; i += blockDim.x) word[i] = 0u;
  }
};

template <typename T>
struct LogitArgs {
  const T* H; const T* HT; const T* W;
  int N, d, V, nt0, n_nt, n_vt;         // row tiles nt0 .. nt0 + n_nt - 1 by vocabulary tiles vt0 .. vt0 + n_vt - 1
  float2* stats; int64_t ld_stats;      // [row - first row][group]: (max z, sum exp(z - max))
  float* z; int64_t ldz;                // [row - first row][position], up to whole tiles; groups whose maximum is below the row's floor are not kept
  const float* floor;                   // [row - first row], or null
  int vt0;                              // first vocabulary tile
  ZeroWords zero;
};

// The lanes of a wavefront that share a token column (every sixteenth or every thirty-second): their maximum, their sum, in a fixed
// order.  By exchanges of register halves: a lone wavefront per SIMD would wait for the LDS that a general shuffle goes through.
template <int COLS, typename F>
__device__ __forceinline__ float over_columns(float v, F f) {
  if constexpr (COLS == 16) {
    const auto x = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
    v = f(__uint_as_float(x[0]), __uint_as_float(x[1]));
  }
  const auto x = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return f(__uint_as_float(x[0]), __uint_as_float(x[1]));
}
// The value a group's exponentials are taken relative to: its maximum, but 0 where there is none (all -inf) and where it is
// +inf: the sum is then 0 or +inf, and NaN only where a logit is NaN.  Subtracted before the factor log2(e): the product of a logit
// beyond 2.36e38 with it (a vocabulary masked with the type's lowest value) is no number, the difference has none such.
__device__ __forceinline__ float finite_or_zero(float m) { return fabsf(m) == __builtin_inff() ? 0.f : m; }

// Workgroups walk the tiles as the recompute step's do (same raster, the next tile's first K stages requested before the current
// one is post-processed).  A group is a block of L::ROWS consecutive positions, all of one wavefront: two or four lanes share a token.
// Bound by the matrix instructions; per logit the post-processing adds an exponential and 4 bytes stored, 64 consecutive
// ones of a row per store instruction.
template <typename T, typename L, bool HKR, bool FLOOR>
__global__ __launch_bounds__(L::THREADS, L::MIN_WAVES) void logit_tiles_kernel(LogitArgs<T> a) {
  extern __shared__ __align__(16) char lds[];
  constexpr int COLS = L::ROWS == 64 ? 16 : 32;         // token columns of a block
  const int lane = threadIdx.x & 63;
  a.zero.by_first_block();
  const int total = a.n_nt * a.n_vt;
  const int64_t ld_bytes = (int64_t)a.d * sizeof(T);
  int t = blockIdx.x;
  if (t >= total) return;
  auto place = [&](int tile, int& p, int& q) {
    grouped_raster(xcd_contiguous_id(tile, total), a.n_nt, a.n_vt, 8, p, q);
  };
  typename L::template Stream<HKR> stream;
  auto start = [&](int p, int q) {
    stream.start(a.W, ld_bytes, (a.vt0 + q) * L::TILE, a.V, a.H, a.HT, ld_bytes, (a.nt0 + p) * L::TILE, a.N, a.d, lds);
  };
  // The rows' floors come with a tile's first requests (as the recompute step's inputs do), -inf without any.  A row past the end has
  // +inf: nothing of it is kept.
  float fl[L::WN], fl_next[L::WN];
  const int rows = a.N - a.nt0 * L::TILE;
  auto load_floor = [&](int p, float (&f)[L::WN]) {
#pragma unroll
    for (int j = 0; j < L::WN; ++j) {
      const int n = p * L::TILE + L::tile_n(j);
      f[j] = n >= rows ? __builtin_inff() : FLOOR ? a.floor[n] : NEG_INF;
    }
  };
  int p, q;
  place(t, p, q);
  if constexpr (L::TUNED) load_floor(p, fl);
  start(p, q);
  typename L::Acc acc;
  for (;;) {
    const int t_next = t + gridDim.x;
    const bool more = L::TUNED && t_next < total;      // (a loop with nothing to request ahead gets one tile per workgroup)
    int p_next = 0, q_next = 0;
    stream.run(lds, acc, [&] {
      if constexpr (!L::TUNED) load_floor(p, fl);          // no registers to spare across that main loop
#pragma unroll
      for (int j = 0; j < L::WN; ++j) asm volatile("" : "+v"(fl[j]));
      if (more) {
        place(t_next, p_next, q_next);
        load_floor(p_next, fl_next);
        start(p_next, q_next);
      }
    });

    const int v0 = (a.vt0 + q) * L::TILE, n0 = p * L::TILE;      // n0: relative to the launch's first row
    float2* __restrict__ stats = a.stats + (int64_t)n0 * a.ld_stats + v0 / L::ROWS;
#pragma unroll
    for (int j = 0; j < L::WN; ++j) {
      const int n = L::tile_n(j);
      float* __restrict__ zrow = a.z + (int64_t)(n0 + n) * a.ldz + v0 + L::lane_row();
#pragma unroll
      for (int i = 0; i < L::WM; ++i) {
        const int blk = __builtin_amdgcn_readfirstlane(L::tile_m(i, 0) & ~(L::ROWS - 1));   // first row of the block in the tile
        float z[16];
#pragma unroll
        for (int r = 0; r < 16; ++r) z[r] = acc.get(i, j, r);
        if (v0 + blk + L::ROWS > a.V) {
          const int live = a.V - v0 - blk - L::lane_row();
#pragma unroll
          for (int r = 0; r < 16; ++r)
            if ((r >> 2) * L::QUAD + (r & 3) >= live) z[r] = NEG_INF;
        }
        float m = z[0];
#pragma unroll
        for (int r = 1; r < 16; ++r) m = fmaxf(m, z[r]);
        m = over_columns<COLS>(m, [](float x, float y) { return fmaxf(x, y); });
        const float ref = finite_or_zero(m);
        float sum = 0.f;
#pragma unroll
        for (int r = 0; r < 16; ++r) sum += fast_exp2((z[r] - ref) * LOG2E);
        sum = over_columns<COLS>(sum, [](float x, float y) { return x + y; });
        if (lane < COLS) stats[(int64_t)n * a.ld_stats + blk / L::ROWS] = float2{m, sum};
        if (!(m < fl[j]) || (sum != sum && fl[j] < __builtin_inff())) {
#pragma unroll
          for (int rq = 0; rq < 4; ++rq)
            *reinterpret_cast<f32x4*>(zrow + blk + rq * L::QUAD) = f32x4{z[rq * 4], z[rq * 4 + 1], z[rq * 4 + 2], z[rq * 4 + 3]};
        }
        __builtin_amdgcn_sched_barrier(0);     // one block at a time in VGPRs
      }
    }
    if (!more) break;
    t = t_next; p = p_next; q = q_next;
#pragma unroll
    for (int j = 0; j < L::WN; ++j) { asm volatile("" : "+v"(fl_next[j])); fl[j] = fl_next[j]; }
  }
}

// Whether a loop's kernel has a form with floors: large calls alone need one, with the copy of H; the ragged hidden sizes' has no
// scalar registers left for it.
template <typename L>
constexpr bool has_floors() {
  if constexpr (L::TUNED) return std::is_same<L, typename L::Even>::value;
  else return false;
}

template <typename T, typename L>
hipError_t logit_tiles_allowance() {
  static OncePerDevice once;
  return once([] {
    if constexpr (L::TUNED) {
      hipError_t e = allow_big_lds(logit_tiles_kernel<T, L, true, false>, L::LDS);
      if constexpr (has_floors<L>()) { if (e == hipSuccess) e = allow_big_lds(logit_tiles_kernel<T, L, true, true>, L::LDS); }
      if (e != hipSuccess) return e;
    }
    return allow_big_lds(logit_tiles_kernel<T, L, false, false>, L::LDS);
  });
}

// One launch; at most one round of workgroups with the tuned loop.
template <typename T, typename L>
void launch_logit_tiles(const LogitArgs<T>& a, hipStream_t st) {
  int grid = a.n_nt * a.n_vt;
  if constexpr (L::TUNED) {
    if (grid > NUM_CU * L::PER_CU) grid = NUM_CU * L::PER_CU;
    if constexpr (has_floors<L>()) {
      if (a.HT && a.floor) { logit_tiles_kernel<T, L, true, true><<<grid, L::THREADS, L::LDS, st>>>(a); return; }
    }
    if (a.HT) { logit_tiles_kernel<T, L, true, false><<<grid, L::THREADS, L::LDS, st>>>(a); return; }
  }
  logit_tiles_kernel<T, L, false, false><<<grid, L::THREADS, L::LDS, st>>>(a);
}

}  // namespace flce
