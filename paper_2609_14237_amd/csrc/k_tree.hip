// Drafted rows (several tokens of a sequence in one step): RoPE and append to
// the paged cache, and attention of each row over the cached tokens and the
// drafted ones its mask names (tree_attention.hpp).
#include "draft.hpp"
#include "kernels.hpp"
#include "tree_attention.hpp"
#include "turn.hpp"

namespace ods {

namespace {

// RoPE of the q and k heads of one drafted row and/or append of its k and v to
// its cache slot. One block per (sequence, drafted row); bound by memory (64
// sequences of 64 rows, 40 heads turned, 8 of keys and of values appended: 23 us,
// two bytes a load 28; heads normalised first (NORM) 29).
template <bool NORM>
__global__ __launch_bounds__(256) void draft_rope_append_kernel(DraftArgs a, int do_rope, int do_append) {
  __shared__ __align__(16) float cs[128], sn[128], exchange[NORM ? 2048 : 4];
  const int b = blockIdx.x, j = blockIdx.y, D = a.D;
  const DraftSeq q = draft_seq(a.row_off, a.ctx_lens, b, a.rows, a.max_rows, a.cols, a.ring);
  if (j >= q.n || q.ctx < 0) return;
  uint16_t *row = a.qkv + (int64_t)(q.r0 + j) * (a.n_q + 2 * a.n_kv) * D;
  if (do_rope) {
    const int rdim = a.freqs ? a.rdim : D, heads = a.n_q + a.n_kv;
    auto turns = [&]() {
      const int p = q.ctx + clamp_depth(a.depth[q.r0 + j], a.max_rows);
      row_turns(rdim / 2, a.freqs ? a.amp : 1.f, cs, sn, [&](int i, float &c, float &s) {
        if (a.freqs)
          turn_by((double)p * a.freqs[i], c, s);
        else
          rope_angle(p, i, D, a.theta, c, s);
      });
    };
    const bool wide = turns_wide(rdim, a.interleaved);
    if constexpr (NORM) {
      const HeadTurn p{heads, a.n_q, D, rdim, a.freqs ? a.interleaved : 0, a.gain_q, a.gain_k, a.eps};
      auto here = [&](int) { return row; };
      auto go = [](int) { return true; };
      const HeadKind kind = head_kind(rdim, p.interleaved);
      if (kind == kHalves) turn_heads<kHalves, 2>(p, 1, 256, here, here, go, cs, sn, exchange, turns);
      if (kind == kPairs) turn_heads<kPairs, 2>(p, 1, 256, here, here, go, cs, sn, exchange, turns);
      if (kind == kAny) turn_heads<kAny, 2>(p, 1, 256, here, here, go, cs, sn, exchange, turns);
    } else if (wide && a.interleaved) {
      turn_row<true>(row, row, heads, D, rdim, cs, sn, turns);
    } else if (wide) {
      turn_row<false>(row, row, heads, D, rdim, cs, sn, turns);
    } else {
      turns();
      turn_row_by_values(row, row, heads, D, rdim, a.interleaved, cs, sn);
    }
    __syncthreads();
  }
  if (!do_append) return;
  const int t = q.ctx + j, slot = t % kPage;
  if (t >= q.cap) return;
  const int page = page_of(a.table, b, t, a.cols, a.ring, a.pool_pages);
  if (page < 0) return;
  const int64_t blk = (int64_t)kPage * D;
  uint16_t *kb = a.pool + (int64_t)page * 2 * a.n_kv * blk, *vb = kb + a.n_kv * blk;
  const uint16_t *k = row + a.n_q * D, *v = k + a.n_kv * D;
  const int log_d = D == 128 ? 7 : 6;
  for (int e = threadIdx.x * 8; e < a.n_kv * D; e += 256 * 8)
    *(u32x4 *)(kb + (e >> log_d) * blk + slot * D + (e & (D - 1))) = *(const u32x4 *)(k + e);
  for (int e = threadIdx.x; e < a.n_kv * D; e += 256)  // dim-major: two bytes a store
    vb[(e >> log_d) * blk + (e & (D - 1)) * kPage + slot] = v[e];
}

// Sequences per launch: what LDS has room for beside the tiles. Larger batches take several launches, one after the other
// on the same records.
constexpr int kTreeBatch = 2048;

template <int D, int NQ, int QW, bool STREAM>
hipError_t go_tree(DraftArgs a, const TreePlan &plan, void *ws, hipStream_t s) {
  using Shape = TreeShape<D, NQ, QW>;
  static std::atomic<uint64_t> lds_set{0};  // devices whose LDS limit is raised
  auto lds = [](int B) { return ((3 * (size_t)B + 1) * 4 + 15) / 16 * 16 + (size_t)Shape::kSlots * Shape::kTileBytes; };
  const auto kern = tree_attention_kernel<D, NQ, QW, STREAM>;
  if (hipError_t e = ensure_lds_limit((const void *)kern, lds(kTreeBatch), lds_set); e != hipSuccess) return e;
  static_assert(sizeof(TreeDesc) <= kTreeDescBytes, "descriptor size");
  TreeDesc *desc = (TreeDesc *)ws;
  float2 *ml = (float2 *)((uint8_t *)ws + (size_t)kTreeDescBytes * plan.grid);
  float *acc = (float *)(ml + (size_t)2 * plan.grid * plan.qt);
  TreeOut out{};
  out.rec_acc = acc;
  out.rec_ml = ml;
  out.desc = desc;
  const float scale = (float)(1.4426950408889634 / sqrt((double)D));
  const int B = a.B;
  for (int b0 = 0; b0 < B; b0 += kTreeBatch) {
    a.B = B - b0 < kTreeBatch ? B - b0 : kTreeBatch;
    const int64_t tasks = (int64_t)a.B * a.n_kv * plan.max_qt;
    const int by_task = tasks <= plan.grid, blocks = by_task ? (int)tasks : plan.grid;
    hipLaunchKernelGGL(kern, dim3(plan.grid), dim3(64 * QW), lds(a.B), s, a, plan.min_tiles, plan.max_qt, by_task, (int)plan.no_cut, scale,
                       out);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    if (!plan.no_cut) {
      if (plan.split_join)
        hipLaunchKernelGGL((tree_join_kernel<D, true>), dim3(blocks, plan.qt), dim3(256), 0, s, a, plan.qt, plan.max_qt,
                           by_task, acc, ml, desc);
      else
        hipLaunchKernelGGL((tree_join_kernel<D, false>), dim3(blocks, plan.qt / 16), dim3(256), 0, s, a, plan.qt, plan.max_qt,
                           by_task, acc, ml, desc);
      if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    }
    a.row_off += a.B;
    a.ctx_lens += a.B;
    a.table += (int64_t)a.B * a.cols;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_draft_rope_append(const DraftArgs &a, bool do_rope, bool do_append, hipStream_t s) {
  const auto kern = do_rope && a.gain_q ? draft_rope_append_kernel<true> : draft_rope_append_kernel<false>;
  hipLaunchKernelGGL(kern, dim3(a.B, a.max_rows), dim3(256), 0, s, a, (int)do_rope, (int)do_append);
  return hipGetLastError();
}

hipError_t launch_tree_attention(const DraftArgs &a, const TreePlan &plan, void *ws, hipStream_t s) {
  auto of = [&](auto d, auto stream) {
    constexpr int D = decltype(d)::value;
    constexpr bool STREAM = decltype(stream)::value;
    switch (plan.qt) {
      case 16: return go_tree<D, 16, 1, STREAM>(a, plan, ws, s);
      case 32: return go_tree<D, 16, 2, STREAM>(a, plan, ws, s);
      case 64: return go_tree<D, 16, 4, STREAM>(a, plan, ws, s);
      case 128:
        if (plan.equal) return go_tree<D, 32, 4, STREAM>(a, plan, ws, s);
        return go_tree<D, 16, 8, STREAM>(a, plan, ws, s);
      case 256: return go_tree<D, 32, 8, STREAM>(a, plan, ws, s);
    }
    return hipErrorInvalidValue;
  };
  using D64 = std::integral_constant<int, 64>;
  using D128 = std::integral_constant<int, 128>;
  if (plan.stream) return a.D == 128 ? of(D128(), std::true_type()) : of(D64(), std::true_type());
  return a.D == 128 ? of(D128(), std::false_type()) : of(D64(), std::false_type());
}

}  // namespace ods
