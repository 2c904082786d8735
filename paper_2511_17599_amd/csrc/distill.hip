// C-ABI entry points of the distillation from a teacher's largest logits (see include/flce.h).  Host code: checks, workspaces,
// launches; the backward is the cross-entropy's with another recompute step.
#include <algorithm>
#include <cmath>

#include "distill.h"

namespace flce {

template <typename T, typename L>
hipError_t distill_recompute(const RecomputeArgs<T>& a, int grid, const DistillLists& lists, const int* rowmap, bool per_row,
                             hipStream_t st) {
  static OncePerDevice once;
  const hipError_t e = once([] {
    const hipError_t e = allow_big_lds(recompute_kernel<T, L, L::TUNED, false, true>, L::LDS);
    return e != hipSuccess ? e : allow_big_lds(recompute_kernel<T, L, L::TUNED, true, true>, L::LDS);
  });
  if (e != hipSuccess) return e;
  RecomputeTempArgs<T> x;
  static_cast<RecomputeArgs<T>&>(x) = a;
  x.z_scale = lists.z_scale;
  x.temperature = lists.temperature;
  const unsigned blocks = (unsigned)ceil_div((int64_t)a.n_nt * L::TILE * lists.K, 256);
  if (per_row) {
    recompute_kernel<T, L, L::TUNED, true, true><<<grid, L::THREADS, L::LDS, st>>>(x);
    distill_scatter_kernel<T, L, true><<<blocks, 256, 0, st>>>(a, lists, rowmap);
  } else {
    recompute_kernel<T, L, L::TUNED, false, true><<<grid, L::THREADS, L::LDS, st>>>(x);
    distill_scatter_kernel<T, L, false><<<blocks, 256, 0, st>>>(a, lists, rowmap);
  }
  return hipSuccess;
}
#define FLCE_DISTILL(T, ...) \
  template hipError_t distill_recompute<T, __VA_ARGS__>(const RecomputeArgs<T>&, int, const DistillLists&, const int*, bool, hipStream_t);
FLCE_DISTILL(bf16_t, SmallLoop<true>)
FLCE_DISTILL(bf16_t, SmallLoop<false>)
FLCE_DISTILL(bf16_t, FastLoop<true>)
FLCE_DISTILL(bf16_t, FastLoop<false>)
FLCE_DISTILL(bf16_t, GenericLoop)
FLCE_DISTILL(float, F32Loop<64>)
FLCE_DISTILL(float, F32Loop<128>)
#undef FLCE_DISTILL

namespace {

struct DistillPlan {
  Plan p;
  int n_blk, n_win;
  int64_t off_blk_loss, off_blk_cnt, off_blk_oor, off_part, off_begin, off_entries, off_HT, fwd_bytes;
};

bool make_distill_plan(int parts, int64_t N, int64_t d, int64_t V, int64_t K, flce_dtype dt, DistillPlan& x) {
  if (!make_plan(parts, N, d, V, dt, x.p) || K < 1 || K > DISTILL_MAX) return false;
  const Plan& p = x.p;
  if (parts & PLAN_FORWARD) {
    int64_t tile = 0, buckets = 0;          // of the loop: edge, and wavefronts that the lists of a tile are sorted for
    with_forward_loop(p, [&](auto tag) -> flce_status {
      using L = typename decltype(tag)::L;
      tile = L::TILE;
      buckets = 2 * list_waves<L>();
      return FLCE_OK;
    });
    x.n_blk = (int)ceil_div(N, distill_rows_per_block(N));
    // The cross-entropy's windows, but in fp32 where they leave CUs idle as many as give every CU two workgroups, down to a tile each
    // (its 64-row tiles are planned by 256 positions: 256 x 256 x 4096, 256 tiles, 37 us as four each of 64 workgroups, 11 as one each).
    const int64_t n_rt = ceil_div(N, tile), n_vt = ceil_div(V, tile);
    x.n_win = p.n_win;
    if (p.esize == 4 && n_rt * x.n_win < 2 * NUM_CU) x.n_win = (int)std::min(n_vt, std::max<int64_t>(x.n_win, ceil_div(2 * NUM_CU, n_rt)));
    int64_t o = ALIGN;
    x.off_blk_loss = o; o = align_up(o + (int64_t)x.n_blk * 4, ALIGN);
    x.off_blk_cnt = o;  o = align_up(o + (int64_t)x.n_blk * 4, ALIGN);
    x.off_blk_oor = o;  o = align_up(o + (int64_t)x.n_blk * 4, ALIGN);
    x.off_part = o;     o = align_up(o + 2ll * x.n_win * p.npad * 4, ALIGN);
    x.off_begin = o;    o = align_up(o + n_rt * (n_vt * buckets + 1) * 4, ALIGN);
    x.off_entries = o;  o = align_up(o + n_rt * tile * K * 4, ALIGN);
    x.off_HT = o;       if (p.fwd_copy) o = align_up(o + packed_block_offset(p.n_rb, (int)d), ALIGN);
    x.fwd_bytes = o;
  }
  return true;
}

// What the forward leaves for the backward: targets, then (share, logit) per list entry.
int64_t saved_bytes(int64_t N, int64_t K) { return align_up(N * 8, ALIGN) + N * K * 8; }
int64_t* saved_targets(void* saved) { return static_cast<int64_t*>(saved); }
float2* saved_entries(void* saved, int64_t N) { return reinterpret_cast<float2*>(static_cast<char*>(saved) + align_up(N * 8, ALIGN)); }

template <typename T, typename L>
hipError_t distill_tiles_allowance() {
  static OncePerDevice once;
  return once([] {
    if constexpr (L::TUNED) {
      const hipError_t e = allow_big_lds(distill_tiles_kernel<T, L, true>, L::LDS);
      if (e != hipSuccess) return e;
    }
    return allow_big_lds(distill_tiles_kernel<T, L, false>, L::LDS);
  });
}

bool temperature_ok(float T) { return T > 0.f && std::isfinite(T) && std::isfinite(LOG2E / T) && std::isfinite(T * T) && T * T > 0.f; }
bool bad_workspace(const void* ws, size_t bytes, int64_t need) {
  return !ws || (reinterpret_cast<uintptr_t>(ws) & 255u) || bytes < (size_t)need;
}

}  // namespace
}  // namespace flce

extern "C" {

size_t flce_distill_workspace_bytes(int64_t N, int64_t d, int64_t V, int64_t K, flce_dtype dt, int for_backward) {
  flce::DistillPlan x;
  if (!flce::make_distill_plan(for_backward ? flce::PLAN_BACKWARD : flce::PLAN_FORWARD, N, d, V, K, dt, x)) return 0;
  return (size_t)(for_backward ? x.p.bwd_bytes : x.fwd_bytes);
}

size_t flce_distill_saved_bytes(int64_t N, int64_t K) {
  if (N < 1 || N > 0x7FFFFF00ll || K < 1 || K > flce::DISTILL_MAX) return 0;
  return (size_t)flce::saved_bytes(N, K);
}

flce_status flce_distill_forward(const void* H, const void* W, const int64_t* teacher_ids, const float* teacher_logits, int64_t N, int64_t d,
                                 int64_t V, int64_t K, float temperature, flce_reduction reduction, flce_dtype dt, float* loss_out,
                                 float* loss_rows_out, float* lse_out, void* saved_out, void* workspace, size_t workspace_bytes,
                                 void* hip_stream) {
  using namespace flce;
  if (!H || !W || !teacher_ids || !teacher_logits || (!loss_out && !loss_rows_out) || !lse_out || !saved_out) return FLCE_ERR_BAD_ARG;
  if (reduction != FLCE_REDUCE_MEAN && reduction != FLCE_REDUCE_SUM) return FLCE_ERR_BAD_ARG;
  if (dt != FLCE_DTYPE_BF16 && dt != FLCE_DTYPE_F32) return FLCE_ERR_BAD_ARG;
  if (!temperature_ok(temperature)) return FLCE_ERR_BAD_ARG;
  DistillPlan x;
  if (!make_distill_plan(PLAN_FORWARD, N, d, V, K, dt, x)) return FLCE_ERR_BAD_SHAPE;
  if (!aligned16(H) || !aligned16(W) || !aligned16(saved_out)) return FLCE_ERR_BAD_ARG;
  if (bad_workspace(workspace, workspace_bytes, x.fwd_bytes)) return FLCE_ERR_WORKSPACE;
  int64_t* target = saved_targets(saved_out);
  float2* saved = saved_entries(saved_out, N);
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  char* ws = static_cast<char*>(workspace);
  const Plan& p = x.p;
  Header* hdr = reinterpret_cast<Header*>(ws);
  float* part = reinterpret_cast<float*>(ws + x.off_part);
  int* begin = reinterpret_cast<int*>(ws + x.off_begin);
  uint32_t* entries = reinterpret_cast<uint32_t*>(ws + x.off_entries);
  void* HT = p.fwd_copy ? ws + x.off_HT : nullptr;
  if (HT) pack_rows(p, H, HT, st);
  return with_forward_loop(p, [&](auto tag) -> flce_status {
    using T = typename decltype(tag)::T;
    using L = typename decltype(tag)::L;
    if (distill_tiles_allowance<T, L>() != hipSuccess) return FLCE_ERR_HIP;
    const int n_rb = (int)ceil_div(N, L::TILE), n_vt = (int)ceil_div(V, L::TILE), items = n_rb * x.n_win;
    {
      ProfScope ps(FLCE_PROF_FWD_EPILOGUE, st);
      distill_lists_kernel<L::TILE, list_waves<L>()><<<(unsigned)n_rb, 1024, 0, st>>>(teacher_ids, teacher_logits, (int)N, (int)V, (int)K, n_vt,
                                                                                      begin, entries, hdr);
    }
    {
      // one workgroup per (row block, window), with the tuned loop a round of them per launch, as the cross-entropy's forward
      ProfScope ps(FLCE_PROF_FWD_TILES, st);
      int per_launch = items;
      if constexpr (L::TUNED) per_launch = NUM_CU * L::PER_CU;
      for (int item0 = 0; item0 < items; item0 += per_launch) {
        const DistillTileArgs<T> a{static_cast<const T*>(H), static_cast<const T*>(HT), static_cast<const T*>(W), (int)N, (int)d, (int)V, n_rb,
                                   x.n_win, n_vt, (double)n_vt / x.n_win, LOG2E / temperature, part, p.npad, item0, begin, entries, (int)K,
                                   saved};
        const int grid = std::min(per_launch, items - item0);
        if constexpr (L::TUNED) {
          if (HT) { distill_tiles_kernel<T, L, true><<<grid, L::THREADS, L::LDS, st>>>(a); continue; }
        }
        distill_tiles_kernel<T, L, false><<<grid, L::THREADS, L::LDS, st>>>(a);
      }
    }
    ProfScope ps(FLCE_PROF_FWD_EPILOGUE, st);
    // a call for rows alone has no scalar loss to hand out: the sum goes to a spare word of the header block
    float* scalar = loss_out ? loss_out : reinterpret_cast<float*>(ws + 64);
    const DistillRowArgs rows{
        teacher_ids, teacher_logits, saved, target, (int)N, (int)V, (int)K, x.n_win, part, p.npad, temperature, 1.f / temperature,
        LOG2E / temperature, lse_out, loss_rows_out,
        LossOut{reinterpret_cast<float*>(ws + x.off_blk_loss), reinterpret_cast<int*>(ws + x.off_blk_cnt),
                reinterpret_cast<int*>(ws + x.off_blk_oor), hdr, scalar, reduction == FLCE_REDUCE_MEAN, nullptr, nullptr}};
    if (N <= DISTILL_FEW) distill_rows_kernel<DISTILL_FEW_ROWS><<<x.n_blk, 64 * DISTILL_FEW_ROWS, 0, st>>>(rows);
    else distill_rows_kernel<DISTILL_ROWS><<<x.n_blk, 64 * DISTILL_ROWS, 0, st>>>(rows);
    return hipGetLastError() == hipSuccess ? FLCE_OK : FLCE_ERR_HIP;
  });
}

flce_status flce_distill_backward(const void* H, const void* W, const int64_t* teacher_ids, const float* lse, const void* saved, int64_t N,
                                  int64_t d, int64_t V, int64_t K, float temperature, flce_reduction reduction, flce_dtype dt,
                                  const float* grad_loss, const float* grad_rows, void* dH_out, void* dW_out, void* workspace,
                                  size_t workspace_bytes, void* hip_stream) {
  using namespace flce;
  if (!teacher_ids || !saved || !aligned16(saved) || !grad_loss == !grad_rows || !temperature_ok(temperature)) return FLCE_ERR_BAD_ARG;
  if (!flce_distill_saved_bytes(N, K)) return FLCE_ERR_BAD_SHAPE;
  void* s = const_cast<void*>(saved);       // (read only)
  const DistillLists lists{teacher_ids, saved_entries(s, N), lse, (int)K, temperature, LOG2E / temperature};
  // one vocabulary position more than W has: the targets of rows that count lie there
  return backward_impl(H, W, saved_targets(s), lse, N, d, V, -1, grad_rows ? FLCE_REDUCE_SUM : reduction, dt,
                       grad_rows ? GradLoss{1.f, nullptr} : GradLoss{temperature, grad_loss}, dH_out, dW_out, workspace, workspace_bytes,
                       hip_stream, Slice{V + 1, 0}, PerRow{nullptr, grad_rows, 0.f}, &lists);
}

}  // extern "C"
