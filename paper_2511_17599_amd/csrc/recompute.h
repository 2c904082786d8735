// The backward's recompute step: logit tiles again, G staged.
#pragma once
#include "loops.h"

namespace flce {

// ------------------------------------------------------------------------------------
// Backward, step 1 (on the compacted rows): logit tile recomputed exactly as in the
// forward (the same products added up in the same order; fp32 on the same tile edge, see plan_base), then
//   g = exp(z - lse_row) - [v == y_row]            (unscaled; Gamma comes later)
// rounded to T and written to the staging tile
//   G [row - chunk_n0][vocab - chunk_v0]   (ldG  elements per row; with the tuned loop in blocks of 16 rows x 32
//                                           positions of 1 KiB, ldG = BYTES from one group of 16 rows to the next)
// and, for main loops that need K-contiguous operands, also transposed:
//   GT[vocab - chunk_v0][row - chunk_n0]   (ldGT elements per row)
// Padded vocabulary columns and the padding rows behind the last counted row are 0.
// Tiles that lie entirely behind the last counted row return at once; the
// contractions never read them.
// ------------------------------------------------------------------------------------
template <typename T>
struct RecomputeArgs {
  const T* Hc; const T* HcT; const T* W; const int* tgt_c; const float* lse_c; const Header* hdr;
  int npad, d, V, nt0, n_nt, vt0, n_vt;
  T* G; int64_t ldG; T* GT; int64_t ldGT;
  // per-row variant only: upstream gradient of each compact row, label-smoothing constants
  const float* gam_c; float onehot_weight; float uniform_part;   // 1 - eps, eps / V
};

// TEMP: the softmax of z / temperature; lse_c belongs to that.
template <typename T>
struct RecomputeTempArgs : RecomputeArgs<T> {
  float z_scale;        // log2(e) / temperature
  float temperature;    // PER_ROW: G = temperature * Gamma_row * (p - ...)
};

// Per-row inputs of a recompute tile, one set per token column a lane owns.
template <typename L>
struct RowMeta {
  int tgt[L::WN];       // target column inside the slice, -1 for a padding row
  float lse[L::WN];
  float gam[L::WN];     // per-row variant only
};

// The recompute step.  With the tuned loop the launch has at most one round of workgroups (NUM_CU * L::PER_CU: 256 with
// 256-row tiles, 512 with 128-row ones) and workgroup b takes tiles b, b + gridDim.x, ... of the chunk; with the other loops
// it has one per tile.  With the tuned loop the first K stages of a workgroup's next tile (and that tile's per-row inputs) are
// requested before the current tile's G is formed and stored, so the latency of a tile's first operands hides behind
// the previous tile's post-processing: it matters when the K loop is short (small d).
// PER_ROW: g = Gamma_row * (p - (1 - eps) [v == y_row] - eps / V), the upstream gradient applied here because
// it differs from row to row (Alg. 2 with a per-position Gamma); otherwise g = p - [v == y_row] and the
// scalar Gamma is applied when the contractions write out.
// TEMP: p = exp(z / temperature - lse).
template <typename T, typename L, bool HKR, bool PER_ROW = false, bool TEMP = false>
__global__ __launch_bounds__(L::THREADS, L::MIN_WAVES) void recompute_kernel(
    std::conditional_t<TEMP, RecomputeTempArgs<T>, RecomputeArgs<T>> a) {
  float z_scale = LOG2E;
  if constexpr (TEMP) z_scale = a.z_scale;
  extern __shared__ __align__(16) char lds[];
  const T* __restrict__ Hc = a.Hc; const T* __restrict__ HcT = a.HcT; const T* __restrict__ W = a.W;
  const int npad = a.npad, d = a.d, V = a.V;
  T* __restrict__ G = a.G; T* __restrict__ GT = a.GT; const int64_t ldG = a.ldG, ldGT = a.ldGT;
  // Only the row tiles that hold counted rows are rastered (their number is known on the device
  // alone), so the XCDs share the work evenly however many rows are ignored; workgroups beyond the
  // useful tiles of a launch sized for N rows leave at once.
  const int n_nt = max(0, min(a.n_nt, ((int)a.hdr->n_valid - a.nt0 * L::TILE + L::TILE - 1) / L::TILE));
  const int useful = n_nt * a.n_vt;
  int t = blockIdx.x;
  if (t >= useful) return;
  const int64_t ld_bytes = (int64_t)d * sizeof(T);
  auto place = [&](int tile, int& p, int& q) {     // row tile, vocabulary tile inside the chunk
    grouped_raster(xcd_contiguous_id(tile, useful), n_nt, a.n_vt, 8, p, q);
  };
  auto load_meta = [&](int n0, RowMeta<L>& m) {
#pragma unroll
    for (int j = 0; j < L::WN; ++j) {
      const int n = n0 + L::tile_n(j);
      m.tgt[j] = a.tgt_c[n];
      m.lse[j] = a.lse_c[n];
      if constexpr (PER_ROW) m.gam[j] = a.gam_c[n];
    }
  };
  // Marks the point where a tile's per-row inputs must have arrived: the compiler's wait for them lands here (it
  // cannot see the main loop's own requests, so a wait placed later would also wait for the next tile's operands).
  auto need_meta = [&](RowMeta<L>& m) {
#pragma unroll
    for (int j = 0; j < L::WN; ++j) {
      asm volatile("" : "+v"(m.tgt[j]), "+v"(m.lse[j]));
      if constexpr (PER_ROW) asm volatile("" : "+v"(m.gam[j]));
    }
  };
  typename L::template Stream<HKR> stream;
  int p, q;
  place(t, p, q);
  RowMeta<L> meta;
  if constexpr (L::TUNED) load_meta((a.nt0 + p) * L::TILE, meta);
  stream.start(W, ld_bytes, (a.vt0 + q) * L::TILE, V, Hc, HcT, ld_bytes, (a.nt0 + p) * L::TILE, npad, d, lds);
  typename L::Acc acc;
  for (;;) {
    const int t_next = t + gridDim.x;
    // (a main loop with nothing to request ahead gets one tile per workgroup)
    const bool more = L::TUNED && t_next < useful;
    int p_next = 0, q_next = 0;
    RowMeta<L> meta_next;
    stream.run(lds, acc, [&] {
      if constexpr (!L::TUNED) load_meta((a.nt0 + p) * L::TILE, meta);   // no registers to spare across that main loop
      need_meta(meta);
      if (more) {
        place(t_next, p_next, q_next);
        load_meta((a.nt0 + p_next) * L::TILE, meta_next);
        stream.start(W, ld_bytes, (a.vt0 + q_next) * L::TILE, V, Hc, HcT, ld_bytes, (a.nt0 + p_next) * L::TILE, npad, d, lds);
      }
    });

    const int v0 = (a.vt0 + q) * L::TILE;
    if constexpr (L::TUNED) {
      // Tuned loop.  A lane holds, of 16 token rows x (32 B) vocabulary positions per j, scattered 8-byte pieces of one
      // row; stored as they lie, every store instruction would touch 16 different memory rows in 32-byte pieces.  Each wavefront
      // therefore passes its piece (4 KiB of bf16 with 256-row tiles) through its own slice of the free LDS stage and
      // writes whole blocks of G, 1 KiB of consecutive bytes per instruction.
      static_assert(sizeof(T) == 2, "the tuned epilogue is laid out for bf16");
      constexpr int POS = L::WM * L::ROWS;                        // vocabulary positions of a piece
      const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
      char* stage = lds + L::FREE_LDS_OFFSET + wave * (16 * L::ROW_BYTES);
      const int wrow = lane & 15;                                 // writer: token row of the piece
      const int rrow = lane >> 2, rchunk = lane & 3;              // reader: row and 16-byte chunk inside a block
      const int vbase = v0 + (wave >> 1) * POS;                   // first vocabulary position of the piece
#pragma unroll
      for (int j = 0; j < L::WN; ++j) {
        const int tgt = meta.tgt[j];
        // exp(z - lse) = 2^(z * log2e - lse * log2e); a padding row (tgt < 0) gets lse = +inf here, so its p is
        // exactly 0, and no column equals its target: its row of G is 0 without a mask
        const float ll = tgt >= 0 ? -meta.lse[j] * LOG2E : NEG_INF;
        float gam = 1.f;
        if constexpr (PER_ROW) gam = tgt >= 0 ? meta.gam[j] : 0.f;
        if constexpr (PER_ROW && TEMP) gam *= a.temperature;
        const float unif = tgt >= 0 ? a.uniform_part : 0.f;
        // A whole column of blocks without a target of the wavefront and inside the vocabulary (almost all are: POS of V
        // positions) needs no tests (step of 4326 x 232 x 74697 1044 -> 1008 us, 1144 x 576 x 191782 1306 -> 1264,
        // 4096 x 768 x 50257 1198 -> 1178).
        if (vbase + POS <= V && __ballot((unsigned)(tgt - vbase) < (unsigned)POS) == 0ull) {
#pragma unroll
          for (int i = 0; i < L::WM; ++i) {
#pragma unroll
            for (int rq = 0; rq < 4; ++rq) {
              float g[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) {
                g[e] = fast_exp2(fmaf(acc.get(i, j, rq * 4 + e), z_scale, ll));
                if constexpr (PER_ROW) g[e] = gam * (g[e] - unif);
              }
              uint2 packed;
              packed.x = f32x2_to_bf16x2_bits(g[0], g[1]);
              packed.y = f32x2_to_bf16x2_bits(g[2], g[3]);
              *reinterpret_cast<uint2*>(stage + L::piece_slot(wrow, i, rq)) = packed;
            }
            __builtin_amdgcn_sched_barrier(0);   // one accumulator block at a time in VGPRs
          }
        } else {
#pragma unroll
          for (int i = 0; i < L::WM; ++i) {
            const int blk0 = vbase + i * L::ROWS;                   // wave-uniform
            const bool whole = blk0 + L::ROWS <= V;
            // Does any token column of this wavefront have its target among the block's vocabulary positions?
            // Almost never, and then the one-hot term costs nothing: a wave-uniform branch.
            const bool hit = __ballot((unsigned)(tgt - blk0) < (unsigned)L::ROWS) != 0ull;
#pragma unroll
            for (int rq = 0; rq < 4; ++rq) {
              const int vpos = blk0 + rq * L::QUAD + L::lane_row();   // first of this lane's 4 consecutive positions
              float g[4];
#pragma unroll
              for (int e = 0; e < 4; ++e) g[e] = fast_exp2(fmaf(acc.get(i, j, rq * 4 + e), z_scale, ll));
              if (hit) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  if (vpos + e == tgt) g[e] -= PER_ROW ? a.onehot_weight : 1.f;
              }
              if constexpr (PER_ROW) {
#pragma unroll
                for (int e = 0; e < 4; ++e) g[e] = gam * (g[e] - unif);
              }
              if (!whole) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                  if (vpos + e >= V) g[e] = 0.f;
              }
              uint2 packed;
              packed.x = f32x2_to_bf16x2_bits(g[0], g[1]);
              packed.y = f32x2_to_bf16x2_bits(g[2], g[3]);
              *reinterpret_cast<uint2*>(stage + L::piece_slot(wrow, i, rq)) = packed;
            }
            __builtin_amdgcn_sched_barrier(0);   // one accumulator block at a time in VGPRs
          }
        }
        // the piece is complete in LDS (a wavefront's LDS operations complete in order): write it out, a block at a
        // time.  G is stored in blocks of 16 rows x 32 positions (1 KiB; the blocks of a row
        // group along the vocabulary, row groups ldG BYTES apart), so that both contractions fetch whole blocks.
        const int row0 = p * L::TILE + (wave & 1) * (L::WN * 16) + j * 16;          // a row group
        char* __restrict__ gdst = reinterpret_cast<char*>(G) + (int64_t)(row0 >> 4) * ldG +
                                  (int64_t)(q * (L::TILE / 32) + (wave >> 1) * (POS / 32)) * 1024 + lane * 16;
#pragma unroll
        for (int k = 0; k < POS / 32; ++k)
          *reinterpret_cast<u32x4*>(gdst + k * 1024) = *reinterpret_cast<const u32x4*>(stage + L::piece_chunk(rrow, k * 4 + rchunk));
      }
    } else {
    // Blocks in (i, j) order, i outermost: what depends on the vocabulary position only (the padding masks of a
    // block that straddles the vocabulary's end) is then shared by the four j of one i and dies with it.
#pragma unroll
    for (int i = 0; i < L::WM; ++i) {
      // All 32 vocabulary positions of a block belong to one wavefront: "behind the vocabulary's end" and
      // "straddles the end" are wave-uniform tests, and only a straddling block masks single elements.
      const int blk0 = v0 + __builtin_amdgcn_readfirstlane(L::tile_m(i, 0) & ~31);
      const bool whole = blk0 + 32 <= V;
#pragma unroll
      for (int j = 0; j < L::WN; ++j) {
        const int nl = p * L::TILE + L::tile_n(j);       // row inside the staging tile
        // this lane's first position in the row; block (i, rq) lies a constant 32 i + 8 rq further on
        T* __restrict__ grow = G + (int64_t)nl * ldG + q * L::TILE + L::tile_m(0, 0);
        const int tgt = meta.tgt[j];
        // exp(z - lse) = 2^(z * log2e - lse * log2e); a padding row (tgt < 0) gets lse = +inf here, so its p is
        // exactly 0, and no column equals its target: its row of G is 0 without a mask
        const float ll = tgt >= 0 ? -meta.lse[j] * LOG2E : NEG_INF;
        float gam = 1.f;
        if constexpr (PER_ROW) gam = tgt >= 0 ? meta.gam[j] : 0.f;
        if constexpr (PER_ROW && TEMP) gam *= a.temperature;
        const float unif = tgt >= 0 ? a.uniform_part : 0.f;
        // Does any token column of this wavefront have its target among the block's 32 vocabulary positions?
        // Almost never (32 of V positions), and then the one-hot term costs nothing: a wave-uniform branch.
        const bool hit = __ballot((unsigned)(tgt - blk0) < 32u) != 0ull;
#pragma unroll
        for (int rq = 0; rq < 4; ++rq) {
          const int mloc = L::tile_m(i, rq * 4);    // first of 4 consecutive vocabulary positions
          float g[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) g[e] = fast_exp2(fmaf(acc.get(i, j, rq * 4 + e), z_scale, ll));
          if (hit) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (v0 + mloc + e == tgt) g[e] -= PER_ROW ? a.onehot_weight : 1.f;
          }
          if constexpr (PER_ROW) {
#pragma unroll
            for (int e = 0; e < 4; ++e) g[e] = gam * (g[e] - unif);
          }
          if (!whole) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (v0 + mloc + e >= V) g[e] = 0.f;
          }
          const int vl = q * L::TILE + mloc;
          Pack4<T>::store(grow + (i * 32 + rq * 8), g[0], g[1], g[2], g[3]);
          if constexpr (!L::TRANSPOSING) {
#pragma unroll
            for (int e = 0; e < 4; ++e) GT[(int64_t)(vl + e) * ldGT + nl] = Pack4<T>::one(g[e]);
          }
        }
        __builtin_amdgcn_sched_barrier(0);   // one 32x32 block at a time in VGPRs
      }
    }
    }
    if (!more) break;
    need_meta(meta_next);
    t = t_next; p = p_next; q = q_next;
    meta = meta_next;
  }
}

}  // namespace flce
