// Logits of a few rows (single new tokens, the beams of a few sentences): one read of W.
#pragma once
#include "logit_tiles.h"

namespace flce {

constexpr int FEW_ROWS = 64;          // rows up to which this kernel is used
constexpr int FEW_WAVES = 4;

// 64 bytes of K of 16 rows per step and fragment: lane l holds 16 bytes of row l % 16, from byte 16 (l / 16) on.
template <typename T> struct FewMma;
template <> struct FewMma<bf16_t> {
  static __device__ __forceinline__ void run(const u32x4& a, const u32x4& b, f32x4& c) {
    c = __builtin_amdgcn_mfma_f32_16x16x32_bf16(__builtin_bit_cast(bf16x8, a), __builtin_bit_cast(bf16x8, b), c, 0, 0, 0);
  }
};
template <> struct FewMma<float> {    // element e of every lane together: K indices 4 (l / 16) + e
  static __device__ __forceinline__ void run(const u32x4& a, const u32x4& b, f32x4& c) {
#pragma unroll
    for (int e = 0; e < 4; ++e)
      c = __builtin_amdgcn_mfma_f32_16x16x4f32(__uint_as_float(a[e]), __uint_as_float(b[e]), c, 0, 0, 0);
  }
};

// One workgroup: 16 MB vocabulary rows (a group) by 16 NT token rows.  Its four wavefronts take every fourth K step each, so
// that together they read 256 consecutive bytes of a row of W, and their sums are added in wavefront order through LDS.
// W goes from memory to the matrix instruction's registers without a stop in LDS: no element of it is used twice by a wavefront.
// Bound by the read of W; H (N d elements, from the L2) is read once per workgroup.
template <typename T, int MB, int NT>
__global__ __launch_bounds__(64 * FEW_WAVES) void few_rows_kernel(const T* __restrict__ H, const T* __restrict__ W, int N, int d, int V,
                                                                  float* __restrict__ z, int64_t ldz, float2* __restrict__ stats,
                                                                  int64_t ld_stats) {
  constexpr int VEC = 16 / (int)sizeof(T), STEP = 4 * VEC, U = MB * NT >= 8 ? 2 : 4, GROUP = 16 * MB, LD = GROUP + 4;
  constexpr int TURN = MB * NT >= 16 ? NT / 2 : NT;       // blocks of tokens that go through LDS at a time (35 KiB at most)
  __shared__ __align__(16) float part[FEW_WAVES][16 * TURN][LD];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = lane & 15, k0 = (lane >> 4) * VEC;
  const int v0 = blockIdx.x * GROUP;
  const T* wp[MB];
  const T* hp[NT];
#pragma unroll
  for (int i = 0; i < MB; ++i) wp[i] = W + (int64_t)min(v0 + i * 16 + row, V - 1) * d + k0;
#pragma unroll
  for (int j = 0; j < NT; ++j) hp[j] = H + (int64_t)min(j * 16 + row, N - 1) * d + k0;
  f32x4 acc[MB][NT];
#pragma unroll
  for (int i = 0; i < MB; ++i)
#pragma unroll
    for (int j = 0; j < NT; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int steps = (d + STEP - 1) / STEP, whole = d / STEP;
  int s = wave;
  for (; s + (U - 1) * FEW_WAVES < whole; s += U * FEW_WAVES) {
    u32x4 a[U][MB], b[U][NT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int k = (s + u * FEW_WAVES) * STEP;
#pragma unroll
      for (int i = 0; i < MB; ++i) a[u][i] = *reinterpret_cast<const u32x4*>(wp[i] + k);
#pragma unroll
      for (int j = 0; j < NT; ++j) b[u][j] = *reinterpret_cast<const u32x4*>(hp[j] + k);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) FewMma<T>::run(a[u][i], b[u][j], acc[i][j]);
  }
  for (; s < steps; s += FEW_WAVES) {
    const int k = s * STEP;
    const bool in = k + k0 < d;         // d is a multiple of 8: 16 bytes are inside or outside
    u32x4 a[MB], b[NT];
#pragma unroll
    for (int i = 0; i < MB; ++i) a[i] = in ? *reinterpret_cast<const u32x4*>(wp[i] + k) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
    for (int j = 0; j < NT; ++j) b[j] = in ? *reinterpret_cast<const u32x4*>(hp[j] + k) : u32x4{0u, 0u, 0u, 0u};
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j) FewMma<T>::run(a[i], b[j], acc[i][j]);
  }
  // GROUP lanes per token
  constexpr int PER_WAVE = 64 / GROUP;
  const int pos = lane % GROUP, v = v0 + pos;
#pragma unroll
  for (int j0 = 0; j0 < NT; j0 += TURN) {
    if (j0 > 0) __syncthreads();
    // block (i, j): element r of a lane is vocabulary row 4 (l / 16) + r, token l % 16
#pragma unroll
    for (int i = 0; i < MB; ++i)
#pragma unroll
      for (int j = 0; j < TURN; ++j)
        *reinterpret_cast<f32x4*>(&part[wave][j * 16 + row][i * 16 + (lane >> 4) * 4]) = acc[i][j0 + j];
    __syncthreads();
#pragma unroll 4
    for (int nl = wave * PER_WAVE; nl < 16 * TURN; nl += FEW_WAVES * PER_WAVE) {
      if (j0 * 16 + nl >= N) break;
      const int n = j0 * 16 + nl + lane / GROUP;
      float x = 0.f;
#pragma unroll
      for (int w = 0; w < FEW_WAVES; ++w) x += part[w][nl + lane / GROUP][pos];
      if (v >= V) x = NEG_INF;
      float m = x;
#pragma unroll
      for (int o = GROUP / 2; o > 0; o >>= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
      float e = fast_exp2((x - finite_or_zero(m)) * LOG2E);
#pragma unroll
      for (int o = GROUP / 2; o > 0; o >>= 1) e += __shfl_xor(e, o, 64);
      if (n < N) {
        z[(int64_t)n * ldz + v] = x;
        if (pos == 0) stats[(int64_t)n * ld_stats + blockIdx.x] = float2{m, e};
      }
    }
  }
}

// Vocabulary rows per workgroup (16, 32 or 64): as many as leave 512 workgroups, two per CU.
inline int few_rows_group(int64_t V) { return V >= 64 * 512 ? 64 : V >= 32 * 512 ? 32 : 16; }

template <typename T>
void launch_few_rows(const T* H, const T* W, int N, int d, int V, float* z, int64_t ldz, float2* stats, int64_t ld_stats, hipStream_t st) {
  const int group = few_rows_group(V), grid = (V + group - 1) / group;
  auto go = [&](auto kernel) { kernel<<<grid, 64 * FEW_WAVES, 0, st>>>(H, W, N, d, V, z, ldz, stats, ld_stats); };
  auto by_group = [&](auto nt) {
    constexpr int NT = decltype(nt)::value;
    if (group == 64) go(few_rows_kernel<T, 4, NT>);
    else if (group == 32) go(few_rows_kernel<T, 2, NT>);
    else go(few_rows_kernel<T, 1, NT>);
  };
  if (N <= 16) by_group(std::integral_constant<int, 1>{});
  else if (N <= 32) by_group(std::integral_constant<int, 2>{});
  else by_group(std::integral_constant<int, 4>{});
}

}  // namespace flce
