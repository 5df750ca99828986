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
// sequences of 64 rows, 40 heads turned, 8 of keys and of values appended: 24 us,
// two bytes a load 28).
__global__ __launch_bounds__(256) void draft_rope_append_kernel(DraftArgs a, int do_rope, int do_append) {
  __shared__ __align__(16) float cs[128], sn[128], exchange[2048];
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
    if (a.gain_q) {
      const HeadTurn p{heads, a.n_q, D, rdim, a.freqs ? a.interleaved : 0, a.gain_q, a.gain_k, a.eps};
      auto here = [&](int) { return row; };
      auto go = [](int) { return true; };
      turns();
      const HeadKind kind = head_kind(rdim, p.interleaved);
      if (kind == kHalves) turn_heads<kHalves>(p, 1, here, here, go, cs, sn, exchange);
      if (kind == kPairs) turn_heads<kPairs>(p, 1, here, here, go, cs, sn, exchange);
      if (kind == kAny) turn_heads<kAny>(p, 1, here, here, go, cs, sn, exchange);
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

}  // namespace

hipError_t launch_draft_rope_append(const DraftArgs &a, bool do_rope, bool do_append, hipStream_t s) {
  hipLaunchKernelGGL(draft_rope_append_kernel, dim3(a.B, a.max_rows), dim3(256), 0, s, a, (int)do_rope, (int)do_append);
  return hipGetLastError();
}

hipError_t launch_tree_attention(const DraftArgs &a, const TreePlan &plan, void *ws, hipStream_t s) {
  return plan.stream ? launch_part<kWhole, true>(a, plan, ws, TreeState{}, s) : launch_part<kWhole, false>(a, plan, ws, TreeState{}, s);
}

}  // namespace ods
