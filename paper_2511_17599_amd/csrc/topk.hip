// C-ABI entry points around a row's largest logits (see include/flce.h): the selection itself, a beam search's step on top of
// it and the reordering of the beams' states.  Host code: checks, workspaces, launches.
#include <algorithm>
#include <cmath>

#include "few_rows.h"
#include "select.h"

namespace flce {
namespace {

constexpr int64_t TOPK_MAX_V = (int64_t)1 << 22;
// Logits of a chunk of rows wait in memory for their selection; more rows at a time fill the launch's rounds better.
constexpr int64_t TOPK_STAGE_BYTES = (int64_t)1 << 30;

struct TopkPlan {
  Plan p;
  bool few;
  int group, n_groups;            // consecutive positions per group
  int64_t ldz, ld_stats, rows;    // rows of a chunk
  int first_vt;                   // vocabulary tiles of the first launch of a chunk where the others have a floor, 0: no such thing
  int64_t off_z, off_stats, off_floor, off_HT, bytes;
};

// A store of a tile's logits is drained before the next tile's K loop can wait for its operands (one counter for both): at 5 TB/s 13 us of a
// 256-row tile that takes 95.  The K-th largest of the first positions' group maxima is a floor that most of the others' groups do not
// reach, and those are not stored.  First part f of the vocabulary: the rest passes K / (f groups) of its groups, least in all at f = sqrt(K /
// groups); whole rounds of workgroups, and only where both parts are several.  Without and with floors, us: 4096 x 4096 x 128256 K = 64 3348 /
// 3112, K = 10 3294 / 3037; 4096 x 1024 x 50257 K = 20 510 / 437; 8192 x 768 x 50257 K = 100 1026 / 952; 8192 x 256 x 60000 K = 10 684 / 475.
int first_tiles(int tile, const TopkPlan& t, int64_t K) {
  const int64_t round = tile == TILE ? NUM_CU : 2 * NUM_CU;
  const int64_t n_nt = ceil_div(std::min(t.rows, t.p.N), tile), n_vt = ceil_div(t.p.V, tile), per_round = std::max<int64_t>(1, round / n_nt);
  const double f = std::max(1.0 / 16.0, std::sqrt((double)K / t.n_groups));
  const int64_t first = align_up((int64_t)std::ceil(f * (double)n_vt), per_round);
  const bool pays = f < 0.4 && n_nt * first >= 2 * round && n_nt * (n_vt - first) >= 4 * round && first * (tile / t.group) > 2 * K;
  return pays ? (int)first : 0;
}

bool make_topk_plan(int64_t N, int64_t d, int64_t V, int64_t K, flce_dtype dt, TopkPlan& t, bool floors = true) {
  if (!make_plan(PLAN_FORWARD, N, d, V, dt, t.p)) return false;
  if (K < 1 || K > TOPK_MAX || K > V || V > TOPK_MAX_V) return false;
  const Plan& p = t.p;
  t.few = few_rows_ok(N, V);
  int64_t o = 0;
  t.first_vt = 0;
  if (t.few) {
    t.group = few_rows_group(V);
    t.n_groups = (int)ceil_div(V, t.group);
    t.ldz = (int64_t)t.n_groups * t.group;
    t.ld_stats = t.n_groups;
    t.rows = N;
  } else {
    t.group = p.fast ? 64 : 32;
    t.n_groups = (int)ceil_div(V, t.group);
    const int64_t vpad = align_up(V, TILE);
    t.ldz = vpad + 64;            // rows do not lie a power of two apart
    t.ld_stats = vpad / t.group;
    const int64_t most = std::max<int64_t>(TILE, TOPK_STAGE_BYTES / (t.ldz * 4) / TILE * TILE);
    t.rows = align_up(ceil_div(p.npad, ceil_div(p.npad, most)), TILE);
    if (floors && p.fwd_copy && !p.ragged) t.first_vt = first_tiles(p.fwd_tile, t, K);
  }
  t.off_z = o;     o = align_up(o + t.rows * t.ldz * 4, ALIGN);
  t.off_stats = o; o = align_up(o + t.rows * t.ld_stats * 8, ALIGN);
  t.off_floor = o; o = align_up(o + t.rows * 4, ALIGN);
  t.off_HT = o;    if (!t.few && p.fwd_copy) o = align_up(o + packed_block_offset(p.n_rb, (int)d), ALIGN);
  t.bytes = o;
  return true;
}

// `out` says where the rows' selections go: out(row0) for a launch of rows from row0 on; `lds` is its dynamic LDS.
template <typename OUT>
void launch_select(const TopkPlan& t, int64_t rows, int K, char* ws, const OUT& out, size_t lds, hipStream_t st) {
  const float* z = reinterpret_cast<const float*>(ws + t.off_z);
  const float2* stats = reinterpret_cast<const float2*>(ws + t.off_stats);
  auto go = [&](auto kernel) { kernel<<<(unsigned)rows, SELECT_THREADS, lds, st>>>(z, t.ldz, stats, t.ld_stats, t.n_groups, (int)t.p.V, K, out); };
  if (t.group == 64) go(select_kernel<64, OUT>);
  else if (t.group == 32) go(select_kernel<32, OUT>);
  else go(select_kernel<16, OUT>);
}

template <typename F>
flce_status run_topk(const TopkPlan& t, const void* H, const void* W, int K, char* ws, F out, size_t lds, ZeroWords zero, hipStream_t st) {
  const Plan& p = t.p;
  const int N = (int)p.N, d = (int)p.d, V = (int)p.V;
  float* z = reinterpret_cast<float*>(ws + t.off_z);
  float2* stats = reinterpret_cast<float2*>(ws + t.off_stats);
  if (t.few) {
    {
      ProfScope ps(FLCE_PROF_FWD_TILES, st);
      if (p.esize == 2)
        launch_few_rows(static_cast<const bf16_t*>(H), static_cast<const bf16_t*>(W), N, d, V, z, t.ldz, stats, t.ld_stats, zero, st);
      else
        launch_few_rows(static_cast<const float*>(H), static_cast<const float*>(W), N, d, V, z, t.ldz, stats, t.ld_stats, zero, st);
    }
    ProfScope ps(FLCE_PROF_FWD_EPILOGUE, st);
    launch_select(t, N, K, ws, out(0), lds, st);
    return hipGetLastError() == hipSuccess ? FLCE_OK : FLCE_ERR_HIP;
  }
  void* HT = p.fwd_copy ? ws + t.off_HT : nullptr;
  if (HT) pack_rows(p, H, HT, st);
  return with_forward_loop(p, [&](auto tag) -> flce_status {
    using T = typename decltype(tag)::T;
    using L = typename decltype(tag)::L;
    if (logit_tiles_allowance<T, L>() != hipSuccess) return FLCE_ERR_HIP;
    for (int64_t row0 = 0; row0 < N; row0 += t.rows) {
      const int64_t rows = std::min<int64_t>(t.rows, N - row0);
      LogitArgs<T> a{};
      a.H = static_cast<const T*>(H); a.HT = static_cast<const T*>(HT); a.W = static_cast<const T*>(W);
      a.N = N; a.d = d; a.V = V;
      a.nt0 = (int)(row0 / L::TILE); a.n_nt = (int)ceil_div(rows, L::TILE); a.n_vt = (int)ceil_div(V, L::TILE);
      a.stats = stats; a.ld_stats = t.ld_stats;
      a.z = z; a.ldz = t.ldz;
      if (row0 == 0) a.zero = zero;
      if (t.first_vt) {
        float* floor = reinterpret_cast<float*>(ws + t.off_floor);
        const int all = a.n_vt;
        a.n_vt = t.first_vt;
        {
          ProfScope ps(FLCE_PROF_FWD_TILES, st);
          launch_logit_tiles<T, L>(a, st);
        }
        {
          ProfScope ps(FLCE_PROF_FWD_EPILOGUE, st);
          floor_kernel<<<(unsigned)rows, SELECT_THREADS, 0, st>>>(stats, t.ld_stats, t.first_vt * (L::TILE / t.group), K, floor);
        }
        a.vt0 = t.first_vt; a.n_vt = all - t.first_vt;
        a.floor = floor;
        a.zero.n = 0;
      }
      {
        ProfScope ps(FLCE_PROF_FWD_TILES, st);
        launch_logit_tiles<T, L>(a, st);
      }
      ProfScope ps(FLCE_PROF_FWD_EPILOGUE, st);
      launch_select(t, rows, K, ws, out(row0), lds, st);
    }
    return hipGetLastError() == hipSuccess ? FLCE_OK : FLCE_ERR_HIP;
  });
}

bool bad_workspace(const void* ws, size_t bytes, int64_t need) {
  return !ws || (reinterpret_cast<uintptr_t>(ws) & 255u) || bytes < (size_t)need;
}

// A beam step's workspace: the selection's, then its results for every beam.
constexpr int BEAMS_MAX = 64;
constexpr int REORDER_ROWS = 16;      // rows whose vectors a thread of the reordering holds at a time
struct BeamPlan {
  TopkPlan t;
  int K;
  int64_t off_cand, off_norm, off_arrived, bytes;
};
bool make_beam_plan(int64_t batch, int64_t beams, int64_t d, int64_t V, int64_t n_out, flce_dtype dt, BeamPlan& b) {
  if (batch < 1 || beams < 1 || beams > BEAMS_MAX || n_out < 1 || n_out > BEAMS_MAX || batch > 0x7FFFFF00ll / beams || V < 1) return false;
  b.K = (int)std::min(n_out, V);
  if (!make_topk_plan(batch * beams, d, V, b.K, dt, b.t, /*floors=*/false)) return false;
  const int64_t rows = batch * beams;
  int64_t o = b.t.bytes;
  b.off_cand = o;    o = align_up(o + rows * b.K * 8, ALIGN);
  b.off_norm = o;    o = align_up(o + rows * 8, ALIGN);
  b.off_arrived = o; o = align_up(o + batch * 4, ALIGN);
  b.bytes = o;
  return true;
}

bool overlap(const void* a, int64_t na, const void* b, int64_t nb) {
  const uintptr_t x = reinterpret_cast<uintptr_t>(a), y = reinterpret_cast<uintptr_t>(b);
  return x < y + (uintptr_t)nb && y < x + (uintptr_t)na;
}

}  // namespace
}  // namespace flce

extern "C" {

size_t flce_topk_workspace_bytes(int64_t N, int64_t d, int64_t V, int64_t K, flce_dtype dt) {
  flce::TopkPlan t;
  return flce::make_topk_plan(N, d, V, K, dt, t) ? (size_t)t.bytes : 0;
}

flce_status flce_topk(const void* H, const void* W, int64_t N, int64_t d, int64_t V, int64_t K, flce_dtype dt, float* logits_out,
                      int64_t* ids_out, float* lse_out, void* workspace, size_t workspace_bytes, void* hip_stream) {
  if (!H || !W || !logits_out || !ids_out || !lse_out) return FLCE_ERR_BAD_ARG;
  if (dt != FLCE_DTYPE_BF16 && dt != FLCE_DTYPE_F32) return FLCE_ERR_BAD_ARG;
  flce::TopkPlan t;
  if (!flce::make_topk_plan(N, d, V, K, dt, t)) return FLCE_ERR_BAD_SHAPE;
  if (!flce::aligned16(H) || !flce::aligned16(W)) return FLCE_ERR_BAD_ARG;
  if (flce::bad_workspace(workspace, workspace_bytes, t.bytes)) return FLCE_ERR_WORKSPACE;
  const float* floor = t.first_vt ? reinterpret_cast<const float*>(static_cast<char*>(workspace) + t.off_floor) : nullptr;
  return flce::run_topk(
      t, H, W, (int)K, static_cast<char*>(workspace),
      [&](int64_t row0) { return flce::Largest{logits_out + row0 * K, ids_out + row0 * K, lse_out + row0, floor}; }, 0, flce::ZeroWords{nullptr, 0},
      static_cast<hipStream_t>(hip_stream));
}

size_t flce_beam_workspace_bytes(int64_t batch, int64_t beams, int64_t d, int64_t V, int64_t n_out, flce_dtype dt) {
  flce::BeamPlan b;
  return flce::make_beam_plan(batch, beams, d, V, n_out, dt, b) ? (size_t)b.bytes : 0;
}

flce_status flce_beam_step(const void* H, const void* W, const float* scores, const uint8_t* finished, int64_t batch, int64_t beams,
                           int64_t d, int64_t V, int64_t n_out, int64_t eos_id, int64_t pad_id, flce_dtype dt, float* scores_out,
                           int64_t* tokens_out, int64_t* parents_out, uint8_t* finished_out, void* workspace, size_t workspace_bytes,
                           void* hip_stream) {
  if (!H || !W || !scores || !scores_out || !tokens_out || !parents_out || !finished_out) return FLCE_ERR_BAD_ARG;
  if (dt != FLCE_DTYPE_BF16 && dt != FLCE_DTYPE_F32) return FLCE_ERR_BAD_ARG;
  flce::BeamPlan b;
  if (!flce::make_beam_plan(batch, beams, d, V, n_out, dt, b)) return FLCE_ERR_BAD_SHAPE;
  if (!flce::aligned16(H) || !flce::aligned16(W)) return FLCE_ERR_BAD_ARG;
  const int64_t rows = batch * beams, results = batch * n_out;
  // a batch element's results are written while its scores and flags are still read
  if (flce::overlap(scores, rows * 4, scores_out, results * 4) || (finished && flce::overlap(finished, rows, finished_out, results)))
    return FLCE_ERR_BAD_ARG;
  if (flce::bad_workspace(workspace, workspace_bytes, b.bytes)) return FLCE_ERR_WORKSPACE;
  char* ws = static_cast<char*>(workspace);
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  uint32_t* arrived = reinterpret_cast<uint32_t*>(ws + b.off_arrived);
  const flce::BeamStep out{scores, finished, 0, (int)beams, (int)n_out, eos_id, pad_id, scores_out, tokens_out, parents_out, finished_out,
                           arrived, reinterpret_cast<unsigned long long*>(ws + b.off_cand), reinterpret_cast<unsigned long long*>(ws + b.off_norm)};
  return flce::run_topk(
      b.t, H, W, b.K, ws,
      [&](int64_t row0) {
        flce::BeamStep o = out;
        o.row0 = row0;
        return o;
      },
      (size_t)beams * (b.K + 1) * 4, flce::ZeroWords{arrived, (int)batch}, st);
}

flce_status flce_beam_reorder(const void* src, void* dst, const int64_t* parents, int64_t outer, int64_t batch, int64_t beams_in,
                              int64_t beams_out, int64_t row_bytes, int64_t src_row_stride, int64_t src_outer_stride,
                              int64_t dst_row_stride, int64_t dst_outer_stride, int32_t* status_out, void* hip_stream) {
  if (!src || !dst || !parents) return FLCE_ERR_BAD_ARG;
  if (outer < 1 || batch < 1 || beams_in < 1 || beams_in > flce::BEAMS_MAX || beams_out < 1 || beams_out > flce::BEAMS_MAX ||
      row_bytes < 1 || batch > 0x7FFFFF00ll / flce::BEAMS_MAX || outer > 0x7FFFFF00ll || row_bytes > (int64_t)1 << 40)
    return FLCE_ERR_BAD_SHAPE;
  // rows side by side inside an outer slab, slabs side by side
  const int64_t cap = (int64_t)1 << 47;
  if (src_row_stride < row_bytes || dst_row_stride < row_bytes || src_row_stride > cap / (batch * beams_in) ||
      dst_row_stride > cap / (batch * beams_out))
    return FLCE_ERR_BAD_SHAPE;
  if (outer > 1 && (src_outer_stride < batch * beams_in * src_row_stride || dst_outer_stride < batch * beams_out * dst_row_stride ||
                    src_outer_stride > cap / outer || dst_outer_stride > cap / outer))
    return FLCE_ERR_BAD_SHAPE;
  // the same memory, laid out alike, or memory of its own
  const int64_t src_span = (outer - 1) * src_outer_stride + (batch * beams_in - 1) * src_row_stride + row_bytes;
  const int64_t dst_span = (outer - 1) * dst_outer_stride + (batch * beams_out - 1) * dst_row_stride + row_bytes;
  const bool same = src == dst && beams_in == beams_out && src_row_stride == dst_row_stride && (outer == 1 || src_outer_stride == dst_outer_stride);
  if (!same && flce::overlap(src, src_span, dst, dst_span)) return FLCE_ERR_BAD_ARG;
  if (same && beams_out > flce::REORDER_ROWS) return FLCE_ERR_BAD_SHAPE;
  if (outer == 1) src_outer_stride = dst_outer_stride = 0;

  const uint64_t bits = reinterpret_cast<uintptr_t>(src) | reinterpret_cast<uintptr_t>(dst) | (uint64_t)row_bytes | (uint64_t)src_row_stride |
                        (uint64_t)dst_row_stride | (uint64_t)src_outer_stride | (uint64_t)dst_outer_stride;
  hipStream_t st = static_cast<hipStream_t>(hip_stream);
  const char* s = static_cast<const char*>(src);
  char* t = static_cast<char*>(dst);
  // one slab per 65535 (o, b) pairs: the grid's second extent
  const int64_t per = std::max<int64_t>(1, 65535 / batch);
  for (int64_t o = 0; o < outer; o += per) {
    const int64_t n = std::min(per, outer - o);
    for (int64_t b0 = 0; b0 < batch; b0 += 65535) {
      const int64_t nb = std::min<int64_t>(65535, batch - b0);
      auto go = [&](auto kernel, int vec, int rows_of_run) {
        const int64_t n_vec = row_bytes / vec;
        const unsigned gz = (unsigned)flce::ceil_div(beams_out, rows_of_run);
        const unsigned gx = (unsigned)std::min<int64_t>(flce::ceil_div(n_vec, 256), std::max<int64_t>(1, 16384 / (n * nb * gz)));
        kernel<<<dim3(gx, (unsigned)(n * nb), gz), 256, 0, st>>>(
            s + o * src_outer_stride + b0 * beams_in * src_row_stride, t + o * dst_outer_stride + b0 * beams_out * dst_row_stride,
            parents + b0 * beams_out, (int)nb, (int)beams_in, (int)beams_out, n_vec, src_row_stride, src_outer_stride, dst_row_stride,
            dst_outer_stride, status_out);
      };
      auto by_width = [&](auto rows) {
        constexpr int NB = decltype(rows)::value;
        if (bits % 16 == 0) go(flce::beam_reorder_kernel<flce::u32x4, NB>, 16, NB);
        else if (bits % 4 == 0) go(flce::beam_reorder_kernel<uint32_t, NB>, 4, NB);
        else go(flce::beam_reorder_kernel<uint8_t, NB>, 1, NB);
      };
      if (beams_out <= 4) by_width(std::integral_constant<int, 4>{});
      else if (beams_out <= 8) by_width(std::integral_constant<int, 8>{});
      else by_width(std::integral_constant<int, flce::REORDER_ROWS>{});
    }
  }
  return hipGetLastError() == hipSuccess ? FLCE_OK : FLCE_ERR_HIP;
}

}  // extern "C"
