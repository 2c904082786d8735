// The launch plan of a shape and what else the library's sources share on the host.
#pragma once
#include "../../include/flce.h"

#include <hip/hip_runtime.h>

#include <mutex>

#include "recompute.h"

namespace flce {

constexpr int64_t ALIGN = 256;
constexpr int NUM_CU = 256;   // MI355X; the plan must not depend on a device query
// Most bytes that a plan spends on the forward's copy of H at a ragged hidden size, and on the fp32 tiles of the K slices of
// one contraction launch (60000 random shapes up to 140000 x 8192 x 262144: five would take more, 617 MB at most).
constexpr int64_t BYTES_CAP = (int64_t)512 << 20;


inline int64_t align_up(int64_t x, int64_t a) { return (x + a - 1) / a * a; }
inline int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }

inline bool aligned16(const void* p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

struct Plan {
  int64_t N, d, V;
  int esize;
  int n_rb, n_vt;          // 256-row tiles of tokens / vocabulary
  int tile, fwd_tile;      // output tile edge of the main loop, backward and forward (bf16: 256 or 128, fp32: 128 or 64)
  int64_t npad;
  // forward
  int n_win;
  int64_t off_part, off_blk_loss, off_blk_cnt, off_blk_oor, off_wpart, off_wsum, off_zbar, off_fHT, fwd_bytes;
  // backward
  int n_vch, n_nch;        // chunks along vocabulary / tokens
  int vc_tiles, nc_tiles;  // largest chunk, in tiles
  int64_t ld_v, ld_n;      // elements per row of the buffers whose rows run over a vocabulary / row chunk: the
                           // chunk's extent plus 64, so that rows never lie a power of two apart
  bool fast;               // tuned bf16 loop: W, Hc and G read in place by the contractions
  bool ragged;             // its form for hidden sizes that are no multiple of a K step's 32 elements
  bool hkr;                // forward / recompute read a pre-tiled copy of H (tuned loop, unless the caller rules the copy out)
  bool fwd_copy;           // the forward makes that copy (long enough for it to pay)
  int split_dh, split_dw;  // K slices of the dH / dW contraction launches (1 = unsplit)
  bool pair;               // dW and dH of the only chunk go out as one launch
  int64_t off_Hc, off_rowmap, off_tgt, off_lsec, off_gamc, off_HT, off_WT, off_G, off_GT, off_dHacc, off_dWacc, off_partial, off_partial_dh, bwd_bytes;
};

enum : int { PLAN_FORWARD = 1, PLAN_BACKWARD = 2, PLAN_BOTH = 3 };   // 0: the shape's check only
// allow_h_copy: the caller has a workspace for the pre-tiled copy of H.
bool make_plan(int parts, int64_t N, int64_t d, int64_t V, flce_dtype dt, Plan& p, bool allow_h_copy = true, bool wide = true);

// One launch class of flce_profile_*, while recording is on.
struct ProfScope {
  hipStream_t st;
  hipEvent_t b = nullptr;
  ProfScope(int cls, hipStream_t s);
  ~ProfScope();
};

template <typename K>
hipError_t allow_big_lds(K kernel, int bytes) {
  return hipFuncSetAttribute(reinterpret_cast<const void*>(kernel), hipFuncAttributeMaxDynamicSharedMemorySize, bytes);
}

constexpr int MAX_DEVICES = 64;

// W holds the p.V vocabulary rows [slice.v_begin, slice.v_begin + p.V) of slice.V_total.  With m_out set the
// call stops after the window merge and hands out the slice's (m, a, z_target) per row.
struct Slice { int64_t V_total, v_begin; };
// Per-row variant: the forward writes one loss per row (label-smoothed by eps), the backward takes one
// upstream gradient per row (device arrays of N floats).
struct PerRow { float* loss_rows_out; const float* grad_rows; float eps; };
// Device words of the caller that receive the range flag and the number of counted rows (either may be null).
struct StatusOut { int32_t* status; int64_t* n_valid; };

// The forward's pre-tiled copy of H (p.npad rows, zero behind the last one).
void pack_rows(const Plan& p, const void* H, void* HT, hipStream_t st);

// What a distillation's backward has beside the cross-entropy's: lists of K entries per row, shares and the logits at them.
struct DistillLists {
  const int64_t* ids;     // [N][K]
  const float2* saved;    // [N][K]: the teacher's share of the id at its first place in a row, negative elsewhere; the student's logit
  const float* lse;       // [N], of the logits / temperature
  int K;
  float temperature, z_scale;          // log2(e) / temperature
};
// The recompute step of one chunk with those: G = softmax(z / temperature) - share (times the row's gradient if per_row).
template <typename T, typename L>
hipError_t distill_recompute(const RecomputeArgs<T>& a, int grid, const DistillLists& lists, const int* rowmap, bool per_row,
                             hipStream_t st);

// The checks and launches of every backward; `lists` makes it a distillation's.
flce_status backward_impl(const void* H, const void* W, const int64_t* targets, const float* lse, int64_t N, int64_t d, int64_t V,
                          int64_t ignore_index, flce_reduction reduction, flce_dtype dt, GradLoss grad_loss, void* dH_out,
                          void* dW_out, void* workspace, size_t workspace_bytes, void* hip_stream, Slice slice,
                          PerRow rows = PerRow{nullptr, nullptr, 0.f}, const DistillLists* lists = nullptr);

// f(loop) with the main loop that a plan's forward runs on: a tag with its types.
template <typename ST, typename LOOP> struct LoopTag { using T = ST; using L = LOOP; };
template <typename F>
flce_status with_forward_loop(const Plan& p, F f) {
  if (p.esize == 4) return p.fwd_tile == 64 ? f(LoopTag<float, F32Loop<64>>{}) : f(LoopTag<float, F32Loop<128>>{});
  if (!p.fast) return f(LoopTag<bf16_t, GenericLoop>{});
  if (p.fwd_tile == 128) return p.ragged ? f(LoopTag<bf16_t, SmallLoop<true>>{}) : f(LoopTag<bf16_t, SmallLoop<false>>{});
  return p.ragged ? f(LoopTag<bf16_t, FastLoop<true>>{}) : f(LoopTag<bf16_t, FastLoop<false>>{});
}

// set() once per device, for what is a property of the loaded code there; one OncePerDevice for each kind of it.
struct OncePerDevice {
  std::mutex mu;
  bool done[MAX_DEVICES] = {};
  template <typename F>
  hipError_t operator()(F set) {
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    if (dev < 0 || dev >= MAX_DEVICES) return hipErrorInvalidDevice;
    std::lock_guard<std::mutex> lk(mu);
    if (done[dev]) return hipSuccess;
    if ((e = set()) != hipSuccess) return e;
    done[dev] = true;
    return hipSuccess;
  }
};

}  // namespace flce
