// Logits of a few rows (single new tokens, the beams of a few sentences): one read of W.
#pragma once
#include "logit_tiles.h"

namespace flce {

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

// f(e, p[e]) for n consecutive floats of LDS, by as wide reads as there are.
template <int n, typename F>
__device__ __forceinline__ void for_each_value(const float* p, F f) {
  if constexpr (n >= 4) {
#pragma unroll
    for (int q = 0; q < n; q += 4) {
      const f32x4 x = *reinterpret_cast<const f32x4*>(p + q);
#pragma unroll
      for (int e = 0; e < 4; ++e) f(q + e, x[e]);
    }
  } else {
#pragma unroll
    for (int e = 0; e < n; ++e) f(e, p[e]);
  }
}

// One workgroup: 16 MB vocabulary rows by 16 NT token rows.  Its four wavefronts take U consecutive K steps (64 U bytes of a row of W) in
// turn, and their sums are added in wavefront order through LDS.
// W goes from memory to the matrix instruction's registers without a stop in LDS: no element of it is used twice by a wavefront.
// Bound by the read of W (128256 x 4096 in bf16: this kernel alone with 1 row 195 us or 5.4 TB/s, with 32 rows 227); H (N d elements, from the
// L2) is read once per workgroup.  Tried and no faster: a wavefront per group with H shared through LDS or the L1 (32 rows 251 to
// 283), the next run's loads issued ahead of the products (registers for them cost more wavefronts than they gain), loads of W
// that pass the caches (291).
template <typename T, int MB, int NT, int U>
__global__ __launch_bounds__(64 * FEW_WAVES) void few_rows_kernel(const T* __restrict__ H, const T* __restrict__ W, int N, int d, int V,
                                                                  float* __restrict__ z, int64_t ldz, float2* __restrict__ stats,
                                                                  int64_t ld_stats, ZeroWords zero) {
  constexpr int VEC = 16 / (int)sizeof(T), STEP = 4 * VEC, GB = MB < 4 ? MB : 4, GROUP = 16 * GB, LD = GROUP + 4;
  __shared__ __align__(16) float part[FEW_WAVES][16 * NT][LD];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int row = lane & 15, k0 = (lane >> 4) * VEC;
  const int v0 = blockIdx.x * (16 * MB);
  zero.by_first_block();
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

  int k = wave * U * STEP;
  for (; k + U * STEP <= d; k += FEW_WAVES * U * STEP) {
    u32x4 a[U][MB], b[U][NT];
#pragma unroll
    for (int u = 0; u < U; ++u) {
#pragma unroll
      for (int i = 0; i < MB; ++i) a[u][i] = *reinterpret_cast<const u32x4*>(wp[i] + k + u * STEP);
#pragma unroll
      for (int j = 0; j < NT; ++j) b[u][j] = *reinterpret_cast<const u32x4*>(hp[j] + k + u * STEP);
    }
#pragma unroll
    for (int u = 0; u < U; ++u)
#pragma unroll
      for (int i = 0; i < MB; ++i)
#pragma unroll
        for (int j = 0; j < NT; ++j) FewMma<T>::run(a[u][i], b[u][j], acc[i][j]);
  }
  for (const int end = min(d, k + U * STEP); k < end; k += STEP) {     // the wavefront that has the last, shorter run
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

  // One group of the workgroup's at a time: TPT neighbouring lanes have a token, VPT positions each.
  constexpr int TPT = 64 * FEW_WAVES / (16 * NT), VPT = GROUP / TPT;
  static_assert(VPT >= 1 && (VPT & (VPT - 1)) == 0, "lanes and positions of a token");
  const int n = threadIdx.x / TPT, pos = threadIdx.x % TPT * VPT;
#pragma unroll
  for (int i0 = 0; i0 < MB; i0 += GB) {
    const int g0 = v0 + i0 * 16;
    if (g0 >= V) break;
    if (i0 > 0) __syncthreads();
    // block (i, j): element r of a lane is vocabulary row 4 (l / 16) + r, token l % 16
#pragma unroll
    for (int i = 0; i < GB; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j)
        *reinterpret_cast<f32x4*>(&part[wave][j * 16 + row][i * 16 + (lane >> 4) * 4]) = acc[i0 + i][j];
    __syncthreads();
    float x[VPT];
    for_each_value<VPT>(&part[0][n][pos], [&](int e, float y) { x[e] = y; });
#pragma unroll
    for (int w = 1; w < FEW_WAVES; ++w) for_each_value<VPT>(&part[w][n][pos], [&](int e, float y) { x[e] += y; });
    float m = NEG_INF;
#pragma unroll
    for (int e = 0; e < VPT; ++e) {
      if (g0 + pos + e >= V) x[e] = NEG_INF;
      m = fmaxf(m, x[e]);
    }
#pragma unroll
    for (int o = 1; o < TPT; o <<= 1) m = fmaxf(m, __shfl_xor(m, o, 64));
    const float ref = finite_or_zero(m);
    float sum = 0.f;
#pragma unroll
    for (int e = 0; e < VPT; ++e) sum += fast_exp2((x[e] - ref) * LOG2E);
#pragma unroll
    for (int o = 1; o < TPT; o <<= 1) sum += __shfl_xor(sum, o, 64);
    if (n < N) {
      float* __restrict__ zn = z + (int64_t)n * ldz + g0 + pos;
#pragma unroll
      for (int e = 0; e < VPT; e += VPT < 4 ? VPT : 4) {
        if constexpr (VPT >= 4) *reinterpret_cast<f32x4*>(zn + e) = f32x4{x[e], x[e + 1], x[e + 2], x[e + 3]};
        else if constexpr (VPT == 2) *reinterpret_cast<float2*>(zn) = float2{x[0], x[1]};
        else zn[0] = x[0];
      }
      if (pos == 0) stats[(int64_t)n * ld_stats + g0 / GROUP] = float2{m, sum};
    }
  }
}

// Consecutive positions per group (16, 32 or 64): as many as leave 512 workgroups, two per CU.
inline int few_rows_group(int64_t V) { return V >= 64 * 512 ? 64 : V >= 32 * 512 ? 32 : 16; }
// Whether this kernel takes a call (otherwise the tiles of the forward's loop do, whose logits take 256 rows of the workspace however few are
// asked for: 131 MB at 128256 positions, this kernel's one row 0.5).  Whole calls of the selection, this kernel / tiles, us: bf16 50257 x 768
// 1 row 27.6 / 31.0, 4 rows 25.5 / 28.6, 32 rows 33.2 / 30.9; 16000 x 1024 1 row 13.6 / 16.4, 32 rows 20.5 / 17.2, 64 rows 28.4 / 18.1; 8192 x 4096
// 64 rows 46.8 / 52.4; 32000 x 1024 32 rows 26.4 / 24.2, 64 rows 36.3 / 25.2; 128256 x 4096 1 row 203 / 192, 32 rows 236 / 208, 64 rows 277 / 226;
// fp32 50257 x 768 4 rows 42 / 82, 32 rows 60 / 84, 64 rows 90 / 83; 128256 x 4096 1 row 391 / 724, 32 rows 508 / 776.
inline bool few_rows_ok(int64_t N, int64_t V) { return N <= 32 || (N <= 64 && few_rows_group(V) == 16); }

// 17 to 32 rows over a long vocabulary take two groups per workgroup and longer runs, which pays with whole rounds of workgroups (whole calls:
// 32 rows of 128256 x 4096 236 us, one group 253; fp32 508, one group 523) and loses just past one (516 workgroups: 32 rows of 66000 x 4096 189,
// one group 154).  Up to 16 rows the registers that it takes cost more than it gives (1 row 203, two groups 234).
template <typename T>
void launch_few_rows(const T* H, const T* W, int N, int d, int V, float* z, int64_t ldz, float2* stats, int64_t ld_stats, ZeroWords zero,
                     hipStream_t st) {
  const int group = few_rows_group(V);
  auto by = [&](auto mb, auto nt, auto u) {
    constexpr int MB = decltype(mb)::value, NT = decltype(nt)::value, U = decltype(u)::value;
    few_rows_kernel<T, MB, NT, U><<<(V + 16 * MB - 1) / (16 * MB), 64 * FEW_WAVES, 0, st>>>(H, W, N, d, V, z, ldz, stats, ld_stats, zero);
  };
  using std::integral_constant;
  const integral_constant<int, 1> one{};
  const integral_constant<int, 2> two{};
  const integral_constant<int, 4> four{};
  auto by_group = [&](auto nt) {
    if (group == 64) by(four, nt, two);
    else if (group == 32) by(two, nt, two);
    else by(one, nt, two);
  };
  if (N <= 16) by_group(one);
  else if (N > 32) by(one, four, two);
  else if (V >= 128 * 512) by(integral_constant<int, 8>{}, two, four);
  else by_group(two);
}

}  // namespace flce
