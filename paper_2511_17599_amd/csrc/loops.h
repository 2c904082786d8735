// The main-loop policies (bf16 tuned, bf16 generic, fp32) as the kernels use them, and what several kernels share: the layout
// of pre-tiled copies, the workspace header, packing, the target test, sums in fixed order.
#pragma once
#include <type_traits>

#include "mainloop_f32.h"
#include "mainloop_fast.h"
#include "tile_mma.h"

namespace flce {

// Byte offset of row block rb in a pre-tiled copy of a matrix with d columns: the block's ceil(d / 32) images of 16 KiB
// plus a skew, so that the blocks do not start a power of two apart (the workgroups resident at one time stream
// several dozen blocks side by side, and blocks exactly 2^k bytes apart land on the same DRAM banks).
#ifndef FLCE_PACK_SKEW
#define FLCE_PACK_SKEW 17408
#endif
__host__ __device__ __forceinline__ int64_t packed_block_offset(int rb, int d) {
  return (int64_t)rb * ((int64_t)((d + 31) / 32 * 32) * (TILE * 2) + FLCE_PACK_SKEW);
}
// The same for the transposed pre-tiled copy of a matrix with `rows` rows (a multiple of 256): byte offset of the
// block of column tile q (256 columns), which holds rows / 32 images.
__host__ __device__ __forceinline__ int64_t packed_cols_offset(int q, int rows) {
  return (int64_t)q * ((int64_t)rows * (TILE * 2) + FLCE_PACK_SKEW);
}

// Main-loop policies.  A kernel is written once against this interface:
//   THREADS, MIN_WAVES (launch bounds), TILE (output tile edge), LDS (dynamic LDS bytes), WM x WN (accumulator blocks per wavefront, 16 values of a
//   lane in one N column of ROWS rows each), Acc: a finished tile's accumulators, get(i, j, r) element r of block (i, j)
//   (i, j, r constants after unrolling), tile_m(i, r) / tile_n(j): its position inside the tile; inside its block it is row
//   (r / 4) QUAD + lane_row() + r % 4,
//   slot(): which of the SLOTS lanes that share an N column this lane is,
//   TRANSPOSING: can take an operand whose K index runs over memory rows (otherwise K-contiguous copies are made),
//   TUNED: the bf16 loop with its persistent launches, pre-tiled copies and blocked G.
template <int WM, int WN>
struct VectorAcc {        // of the loops that leave the accumulators to the compiler
  f32x16 v[WM][WN];
  __device__ __forceinline__ float get(int i, int j, int r) const { return v[i][j][r]; }
};
struct GenericLoop {      // bf16 where the tuned loop does not reach (address windows); 8 wavefronts 2 x 4
  static constexpr int TILE = flce::TILE, THREADS = flce::THREADS, WM = flce::WM, WN = flce::WN, LDS = LDS_BYTES;
  static constexpr bool TRANSPOSING = false, TUNED = false;
  static constexpr int MIN_WAVES = 1;
  static constexpr int ROWS = 32, QUAD = 8, SLOTS = 4;
  using Acc = VectorAcc<WM, WN>;
  static __device__ __forceinline__ int lane_row() { return (threadIdx.x & 32) >> 3; }
  static __device__ __forceinline__ int tile_m(int i, int r) { return flce::tile_m(i, r); }
  static __device__ __forceinline__ int tile_n(int j) { return flce::tile_n(j); }
  static __device__ __forceinline__ int slot() {
    return ((threadIdx.x >> 6) >> 2) * 2 + ((threadIdx.x & 63) >> 5);
  }
  // A sequence of tiles A[a_row0 ..][:] x B[b_row0 ..][:] over K = k_elems; start() names the next tile, run() computes
  // it and calls `released` when the next start() may come.  This loop has nothing to request ahead: start() only records the operands.
  template <bool BT>
  struct Stream {
    TileSrc As, Bs;
    int k_bytes;
    __device__ __forceinline__ void start(const bf16_t* A, int64_t lda_bytes, int a_row0, int a_rows, const bf16_t* B,
                                          const bf16_t*, int64_t ldb_bytes, int b_row0, int b_rows, int k_elems, char*) {
      As = TileSrc{reinterpret_cast<const char*>(A), lda_bytes, a_row0, a_rows};
      Bs = TileSrc{reinterpret_cast<const char*>(B), ldb_bytes, b_row0, b_rows};
      k_bytes = k_elems * (int)sizeof(bf16_t);
    }
    template <typename F>
    __device__ __forceinline__ void run(char* lds, Acc& acc, F released) {
      tile_mainloop(As, Bs, k_bytes, lds, acc.v);
      released();
    }
  };
  static __device__ __forceinline__ void run(const void* A, int64_t lda_bytes, int a_row0, int a_rows, const void* B,
                                             int64_t ldb_bytes, int b_row0, int b_rows, int k_bytes, char* lds,
                                             Acc& acc) {
    const TileSrc As{static_cast<const char*>(A), lda_bytes, a_row0, a_rows};
    const TileSrc Bs{static_cast<const char*>(B), ldb_bytes, b_row0, b_rows};
    tile_mainloop(As, Bs, k_bytes, lds, acc.v);
  }
};

template <int T>
struct F32Loop {          // fp32; T x T tiles, 4 wavefronts 2 x 2, two workgroups per CU
  static constexpr int TILE = T, THREADS = f32::THREADS, WM = T / 64, WN = T / 64, LDS = f32::lds_bytes<T>();
  static constexpr bool TRANSPOSING = true, TUNED = false;
  // wavefronts per SIMD that the compiler has to leave registers for: two workgroups of 128-row tiles need it told (64-row ones have
  // room anyway, and are 1 % faster with their sums in the accumulation registers)
  static constexpr int MIN_WAVES = T == 128 ? 2 : 1;
  static constexpr int ROWS = 32, QUAD = 8, SLOTS = 4;
  using Acc = VectorAcc<WM, WN>;
  static __device__ __forceinline__ int lane_row() { return (threadIdx.x & 32) >> 3; }
  static __device__ __forceinline__ int tile_m(int i, int r) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    return (wave >> 1) * (T / 2) + i * 32 + (r >> 2) * 8 + (lane >> 5) * 4 + (r & 3);
  }
  static __device__ __forceinline__ int tile_n(int j) {
    const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
    return (wave & 1) * (T / 2) + j * 32 + (lane & 31);
  }
  static __device__ __forceinline__ int slot() { return fast::slot_of_lane(); }
  template <bool BT>
  struct Stream {         // as GenericLoop::Stream: the other resident workgroup covers a tile's first requests
    f32::Operand As, Bs;
    int k_elems;
    __device__ __forceinline__ void start(const float* A, int64_t lda_bytes, int a_row0, int a_rows, const float* B,
                                          const float*, int64_t ldb_bytes, int b_row0, int b_rows, int k, char*) {
      As = f32::Operand{reinterpret_cast<const char*>(A), lda_bytes, a_row0, a_rows, 0};
      Bs = f32::Operand{reinterpret_cast<const char*>(B), ldb_bytes, b_row0, b_rows, 0};
      k_elems = k;
    }
    template <typename F>
    __device__ __forceinline__ void run(char* lds, Acc& acc, F released) {
      f32::mainloop<T, f32::KC, f32::KC>(As, Bs, k_elems, lds, acc.v);
      released();
    }
  };
};

// The tuned bf16 loop; 4 wavefronts 2 x 2 of 32 B rows x 32 B columns, global -> LDS DMA.
// RAGGED: the hidden size is a multiple of 8 but not of 32 (the K extent of the forward and the recompute; the
// contractions' K extents are whole tiles, they always run with the plain form).
template <bool RAGGED, int B>
struct TunedLoop {
  static constexpr int TILE = 64 * B, THREADS = fast::THREADS, WM = B / 2, WN = 2 * B;
  static constexpr bool TRANSPOSING = true, TUNED = true;
  static constexpr int MIN_WAVES = 1;
  static constexpr int ROWS = 64, QUAD = 16, SLOTS = 8;
  using Acc = fast::Acc<2 * B, 2 * B>;
  // 256-row tiles: one workgroup per CU, 4 stages of 32 KiB; 128-row tiles: two, 5 stages of 16 KiB each
  static constexpr int PER_CU = B == 4 ? 1 : 2, STAGES = B == 4 ? fast::NS : 5, STAGE = B * 8192, LDS = STAGES * STAGE;
  template <int LA, int LB, bool RG = false> using Pipe = fast::Pipe<LA, LB, true, B, STAGES, RG, B>;
  // LDS that post-processing may use while the next tile's first K stages are being filled: the last stage
  static constexpr int FREE_LDS_OFFSET = (STAGES - 1) * STAGE;
  static __device__ __forceinline__ int lane_row() { return (threadIdx.x & 48) >> 2; }
  static __device__ __forceinline__ int tile_m(int i, int r) {
    const int wave = threadIdx.x >> 6;
    return (wave >> 1) * (B * 32) + i * ROWS + (r >> 2) * QUAD + lane_row() + (r & 3);
  }
  static __device__ __forceinline__ int tile_n(int j) {
    const int wave = threadIdx.x >> 6;
    return (wave & 1) * (B * 32) + j * 16 + (threadIdx.x & 15);
  }
  static __device__ __forceinline__ int slot() { return (threadIdx.x >> 7) * 4 + ((threadIdx.x & 63) >> 4); }
  // A sequence of tiles with the same B operand: start() requests the first K stages of a tile (all LDS stages must
  // be free: every wavefront is past the previous run()), run() computes it.  BP: B is also given pre-tiled (Bp:
  // per 256-row block and K step the 16 KiB image of its LDS tile, see pack_rows_kernel), and that copy is read.
  template <bool BP>
  struct Stream {
    Pipe<fast::KC, BP ? fast::PK : fast::KC, RAGGED> pipe;
    __device__ __forceinline__ void start(const bf16_t* A, int64_t lda_bytes, int a_row0, int a_rows, const bf16_t* Bm,
                                          const bf16_t* Bp, int64_t ldb_bytes, int b_row0, int b_rows, int k_elems,
                                          char* lds) {
      const fast::Operand As{reinterpret_cast<const char*>(A), lda_bytes, a_row0, a_rows, 0};
      if constexpr (BP) {
        // the block's images follow each other, one per K step, 64 bytes per row
        const fast::Operand Bs{reinterpret_cast<const char*>(Bp) + packed_block_offset(b_row0 / flce::TILE, k_elems) +
                                   b_row0 % flce::TILE * 64, 0, 0, 0, 0};
        pipe.start(As, Bs, k_elems, lds);
      } else {
        const fast::Operand Bs{reinterpret_cast<const char*>(Bm), ldb_bytes, b_row0, b_rows, 0};
        pipe.start(As, Bs, k_elems, lds);
      }
    }
    template <typename F>
    __device__ __forceinline__ void run(char* lds, Acc& acc, F released) { pipe.run(lds, released); }
  };
  // A wavefront's pieces of 16 rows x (32 B) columns of bf16 on their way through its slice of the free stage, rows of
  // ROW_BYTES in 16-byte chunks whose number is XOR-ed with mix(row), so that the 16 rows (x 2 neighbouring 8-byte halves)
  // one write cycle touches lie in different banks, and likewise the four rows x four neighbouring chunks of a read
  // cycle (blocks of G; output rows are read in the order of the places, and the store takes the chunks as they come).  Counted
  // bank conflicts, of the LDS's busy cycles: recompute 3 % at 8192 x 4096 x 128256, 12 % at 4096 x 768 x 50257, dW up to 2.5 %.
  // piece_slot: where a lane writes its 4 columns of quad rq of block i in row r; piece_chunk: where chunk c of row r is read.
  static constexpr int ROW_BYTES = 64 * B, CHUNKS = ROW_BYTES / 16, ROWS_PER_STORE = 64 / CHUNKS;
  static __device__ __forceinline__ int mix(int r) {
    return B == 4 ? ((r & 3) << 2 | r >> 2) : ((r >> 1 & 1) << 2 | r >> 2);
  }
  static __device__ __forceinline__ int piece_slot(int r, int i, int rq) {      // chunk i * 8 + rq * 2 + (lane / 32), half (lane / 16) % 2
    const int quarter = (threadIdx.x & 63) >> 4;
    return r * ROW_BYTES + (((i * 8 + rq * 2 + (quarter >> 1)) ^ mix(r)) << 4) + ((quarter & 1) << 3);
  }
  static __device__ __forceinline__ int piece_chunk(int r, int c) { return r * ROW_BYTES + ((c ^ mix(r)) << 4); }
};
template <bool RAGGED> struct FastLoop : TunedLoop<RAGGED, 4> { using Even = FastLoop<false>; };
template <bool RAGGED> struct SmallLoop : TunedLoop<RAGGED, 2> { using Even = SmallLoop<false>; };

#ifndef FLCE_FWD_GROUP
#define FLCE_FWD_GROUP 8     // row blocks per raster patch of the forward (x 32 / this many windows per XCD)
#endif
constexpr float LOG2E = 1.4426950408889634f;
constexpr float NEG_INF = -__builtin_inff();

// First 256 bytes of every workspace.
struct Header {
  int32_t status;      // 0 or FLCE_ERR_TARGET_RANGE
  int32_t pad0;
  int64_t n_valid;     // number of counted rows
  float loss_sum;      // un-normalised sum of per-row losses (forward only)
  uint32_t arrived;    // blocks of the window merge that have handed in their sums (forward only)
};

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Four consecutive elements of the storage type <-> four floats.
template <typename T> struct Pack4;
template <> struct Pack4<float> {
  static __device__ __forceinline__ void store(float* p, float a, float b, float c, float d) {
    *reinterpret_cast<f32x4*>(p) = f32x4{a, b, c, d};
  }
  static __device__ __forceinline__ void load(const float* p, float (&v)[4]) {
    const f32x4 x = *reinterpret_cast<const f32x4*>(p);
    v[0] = x[0]; v[1] = x[1]; v[2] = x[2]; v[3] = x[3];
  }
  static __device__ __forceinline__ float one(float v) { return v; }
};
template <> struct Pack4<bf16_t> {
  static __device__ __forceinline__ void store(bf16_t* p, float a, float b, float c, float d) {
    uint2 v;
    v.x = f32x2_to_bf16x2_bits(a, b);
    v.y = f32x2_to_bf16x2_bits(c, d);
    *reinterpret_cast<uint2*>(p) = v;
  }
  static __device__ __forceinline__ void load(const bf16_t* p, float (&v)[4]) {
    const uint2 x = *reinterpret_cast<const uint2*>(p);
    v[0] = __uint_as_float(x.x << 16); v[1] = __uint_as_float(x.x & 0xFFFF0000u);
    v[2] = __uint_as_float(x.y << 16); v[3] = __uint_as_float(x.y & 0xFFFF0000u);
  }
  static __device__ __forceinline__ bf16_t one(float v) { return bf16_t{f32_to_bf16_bits(v)}; }
};


// Whether a row counts towards the loss: its target is not the ignore index and lies in
// [0, V_total); a target outside that range that is not the ignore index is reported through `oor`.
__device__ __forceinline__ bool target_counts(int64_t y, int64_t ignore_index, int64_t V_total, bool& oor) {
  oor = false;
  if (y == ignore_index) return false;
  if (y < 0 || y >= V_total) { oor = true; return false; }
  return true;
}

// A counted target as a column of the vocabulary slice [v_begin, v_begin + Vs) that a call works
// on: its column inside the slice, or `outside` when it lies in another slice; -1 for rows that do
// not count.  The whole vocabulary as the slice is v_begin = 0, Vs = V_total.
__device__ __forceinline__ int classify_target_in_slice(int64_t y, int64_t ignore_index, int64_t V_total,
                                                        int64_t v_begin, int Vs, int outside, bool& oor) {
  if (!target_counts(y, ignore_index, V_total, oor)) return -1;
  const int64_t c = y - v_begin;
  return (c >= 0 && c < (int64_t)Vs) ? (int)c : outside;
}

// Merge of safe-softmax partials (m_k, a_k) in slot order; slots with a == 0 are
// the identity.  Returns (M, A) with A relative to M.
template <int S>
__device__ __forceinline__ void merge_fixed(const float (&m)[S], const float (&a)[S], float& M, float& A) {
  M = NEG_INF;
#pragma unroll
  for (int s = 0; s < S; ++s) if (a[s] > 0.f) M = fmaxf(M, m[s]);
  A = 0.f;
#pragma unroll
  for (int s = 0; s < S; ++s) if (a[s] > 0.f) A += a[s] * fast_exp2((m[s] - M) * LOG2E);
}

// Sum over the 64 lanes of a wavefront in a fixed tree (every lane gets it).
template <typename V>
__device__ __forceinline__ V wave_sum(V v) {
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) v += __shfl_xor(v, s, 64);
  return v;
}

// Upstream gradient of the scalar loss: a device word times a host factor if there is one, the host value otherwise.
struct GradLoss {
  float value; const float* word;
  __device__ __forceinline__ float get() const { return word ? *word * value : value; }
};

// Where the reduced loss of a call goes.
struct LossOut {
  float* blk_loss; int* blk_cnt; int* blk_oor;      // one entry per block of the merge
  Header* hdr; float* loss; int mean;
  int32_t* status; int64_t* n_valid;                // the caller's own words, or null
};

// The call's loss, by one thread: normalisation, header.
__device__ __forceinline__ void write_loss(const LossOut& o, double total, int64_t nv, int any) {
  double loss = total;
  if (o.mean) loss = nv > 0 ? total / (double)nv : 0.0;
  o.hdr->status = any ? 4 : 0;
  o.hdr->pad0 = 0;
  o.hdr->n_valid = nv;
  o.hdr->loss_sum = (float)total;
  *o.loss = (float)loss;
  if (o.status) *o.status = any ? 4 : 0;
  if (o.n_valid) *o.n_valid = nv;
}

// The second half of the reduction, by one block: fixed-order fp64 sum of the per-block partials.
__device__ __forceinline__ void finalize_loss(const LossOut& o, int n_blk) {
  __shared__ double sl[16];
  __shared__ long long sc[16];
  __shared__ int so[16];
  double l = 0.0; long long c = 0; int bad = 0;
  for (int b = threadIdx.x; b < n_blk; b += blockDim.x) {
    // (written by other blocks of this launch when the merge calls this: read past this XCD's own caches)
    l += (double)__hip_atomic_load(o.blk_loss + b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    c += __hip_atomic_load(o.blk_cnt + b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
    bad |= __hip_atomic_load(o.blk_oor + b, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT);
  }
  l = wave_sum(l); c = wave_sum(c); bad = __ballot(bad != 0) != 0ull;
  const int wave = threadIdx.x >> 6, n_waves = blockDim.x >> 6;
  if ((threadIdx.x & 63) == 0) { sl[wave] = l; sc[wave] = c; so[wave] = bad; }
  __syncthreads();
  if (threadIdx.x == 0) {
    double total = 0.0; long long nv = 0; int any = 0;
    for (int w = 0; w < n_waves; ++w) { total += sl[w]; nv += sc[w]; any |= so[w]; }
    write_loss(o, total, nv, any);
  }
}

// 16 bytes of the storage type as floats.
template <typename T>
struct Vec16 {
  static constexpr int N = 16 / (int)sizeof(T);
  static __device__ __forceinline__ void load(const T* p, float (&v)[N]) {
    const u32x4 x = *reinterpret_cast<const u32x4*>(p);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      if constexpr (sizeof(T) == 2) { v[2 * e] = __uint_as_float(x[e] << 16); v[2 * e + 1] = __uint_as_float(x[e] & 0xFFFF0000u); }
      else v[e] = __uint_as_float(x[e]);
    }
  }
};

}  // namespace flce
