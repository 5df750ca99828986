// Drafted rows (several tokens of a sequence in one step): RoPE and append to
// the paged cache, and attention of each row over the cached tokens and the
// drafted ones its mask names.
#include <math.h>

#include "draft.hpp"
#include "kernels.hpp"

namespace ods {

namespace {

// RoPE of the q and k heads of one drafted row and/or append of its k and v to
// its cache slot. One block per (sequence, drafted row).
__global__ __launch_bounds__(256) void draft_rope_append_kernel(DraftArgs a, int do_rope, int do_append) {
  __shared__ float cs[128], sn[128];
  const int b = blockIdx.x, j = blockIdx.y, D = a.D;
  const DraftSeq q = draft_seq(a.row_off, a.ctx_lens, b, a.rows, a.max_rows, a.cols, a.ring);
  if (j >= q.n || q.ctx < 0) return;
  uint16_t *row = a.qkv + (int64_t)(q.r0 + j) * (a.n_q + 2 * a.n_kv) * D;
  if (do_rope) {
    const int p = q.ctx + clamp_depth(a.depth[q.r0 + j], a.max_rows);
    const int rdim = a.freqs ? a.rdim : D, np = rdim / 2;
    if (threadIdx.x < np) {
      float c, s;
      if (a.freqs)
        turn_by((double)p * a.freqs[threadIdx.x], c, s);
      else
        rope_angle(p, threadIdx.x, D, a.theta, c, s);
      cs[threadIdx.x] = a.freqs ? c * a.amp : c;
      sn[threadIdx.x] = a.freqs ? s * a.amp : s;
    }
    __syncthreads();
    for (int t = threadIdx.x; t < (a.n_q + a.n_kv) * np; t += 256) {
      const int i = t % np, at = t / np * D + (a.interleaved ? 2 * i : i), mate = at + (a.interleaved ? 1 : np);
      const float u = bf2f(row[at]), v = bf2f(row[mate]), c = cs[i], s = sn[i];
      row[at] = f2bf(u * c - v * s);
      row[mate] = f2bf(v * c + u * s);
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
  for (int e = threadIdx.x; e < a.n_kv * D; e += 256) {
    const int g = e / D, i = e % D;
    kb[g * blk + slot * D + i] = row[a.n_q * D + e];
    vb[g * blk + i * kPage + slot] = row[(a.n_q + a.n_kv) * D + e];
  }
}

// One wave per (drafted row, query head): lanes take a token each for the
// scores, a dim each for the values; softmax sums and outputs in fp32. What a
// row may not see is not read into its sums at all.
__global__ __launch_bounds__(64) void tree_attention_kernel(DraftArgs a, float scale) {
  __shared__ float sq[128], sp[64];
  __shared__ int spage[64];
  const int b = blockIdx.x, j = blockIdx.y, h = blockIdx.z, D = a.D, lane = threadIdx.x;
  const DraftSeq s = draft_seq(a.row_off, a.ctx_lens, b, a.rows, a.max_rows, a.cols, a.ring);
  if (j >= s.n) return;
  const int64_t row = s.r0 + j;
  const int g = h / (a.n_q / a.n_kv);
  const uint16_t *q = a.qkv + row * (a.n_q + 2 * a.n_kv) * D + h * D;
  for (int i = lane; i < D; i += 64) sq[i] = bf2f(q[i]);
  const int depth = clamp_depth(a.depth[row], a.max_rows);
  const int lo = a.window > 0 ? max(0, s.ctx + depth - a.window + 1) : 0;
  const int words = (a.max_rows + 63) / 64;
  const int64_t blk = (int64_t)kPage * D;
  __syncthreads();
  float m = -INFINITY, l = 0.f, o0 = 0.f, o1 = 0.f;
  const int first = a.window > 0 ? max(0, s.ctx - a.window + 1) / 64 * 64 : 0;
  for (int t0 = first; t0 < s.end; t0 += 64) {
    const int t = t0 + lane;
    bool see = t < s.end && (t < s.ctx ? t >= lo : (a.mask[row * words + (t - s.ctx) / 64] >> ((t - s.ctx) % 64)) & 1);
    if (see && t >= s.ctx && a.window > 0)
      see = clamp_depth(a.depth[s.r0 + t - s.ctx], a.max_rows) > depth - a.window;
    const int page = see ? page_of(a.table, b, t, a.cols, a.ring, a.pool_pages) : -1;
    see = page >= 0;
    float sc = -INFINITY;
    if (see) {
      const uint16_t *k = a.pool + (int64_t)page * 2 * a.n_kv * blk + g * blk + (t % kPage) * D;
      float dot = 0.f;
      for (int i = 0; i < D; ++i) dot += sq[i] * bf2f(k[i]);
      sc = dot * scale;
    }
    const float m_new = fmaxf(m, wave_max(sc));
    if (__ballot(see) == 0) continue;
    const float base = m_new == -INFINITY ? 0.f : m_new;
    const float p = see ? expf(sc - base) : 0.f;
    const float alpha = expf(m - base);
    l = l * alpha + wave_sum(p);
    m = m_new;
    sp[lane] = p;
    spage[lane] = page;
    __syncthreads();
    o0 *= alpha;
    o1 *= alpha;
    for (int i = 0; i < 64; ++i) {
      if (spage[i] < 0) continue;
      const uint16_t *v = a.pool + (int64_t)spage[i] * 2 * a.n_kv * blk + (a.n_kv + g) * blk + (t0 + i) % kPage;
      o0 += sp[i] * bf2f(v[lane * kPage]);
      if (D > 64) o1 += sp[i] * bf2f(v[(lane + 64) * kPage]);
    }
    __syncthreads();
  }
  const float inv = l == 0.f ? 0.f : 1.f / l;
  uint16_t *o = a.o + row * a.n_q * D + h * D;
  o[lane] = f2bf(o0 * inv);
  if (D > 64) o[lane + 64] = f2bf(o1 * inv);
}

}  // namespace

hipError_t launch_draft_rope_append(const DraftArgs &a, bool do_rope, bool do_append, hipStream_t s) {
  hipLaunchKernelGGL(draft_rope_append_kernel, dim3(a.B, a.max_rows), dim3(256), 0, s, a, (int)do_rope, (int)do_append);
  return hipGetLastError();
}

hipError_t launch_tree_attention(const DraftArgs &a, hipStream_t s) {
  hipLaunchKernelGGL(tree_attention_kernel, dim3(a.B, a.max_rows, a.n_q), dim3(64), 0, s, a,
                     (float)(1.0 / sqrt((double)a.D)));
  return hipGetLastError();
}

}  // namespace ods
