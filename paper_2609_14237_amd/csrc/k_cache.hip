// Page operators of the KV cache: copies of whole pages, and the slots of an
// accepted path moved to the front of a sequence's drafted ones.
#include <algorithm>

#include "draft.hpp"
#include "kernels.hpp"

namespace ods {

namespace {

// One block per (16 KB of a page, pair, layer), four 16-byte loads of each thread in flight. Bound by memory:
// 4001 pages of 64 KB in two layers (1.05 GB moved) 210 us, 5.0 TB/s, what a large copy reaches.
constexpr int kCopyLoads = 4;
__global__ __launch_bounds__(256) void copy_pages_kernel(PoolSet pools, const int2 *__restrict__ pairs) {
  const PoolRef r = pools.p[blockIdx.z];
  const int2 pr = pairs[blockIdx.x];  // source, destination
  if (pr.x == pr.y || pr.x < 0 || pr.y < 0 || pr.x >= r.pages || pr.y >= r.pages) return;
  const u32x4 *a = (const u32x4 *)(r.pool + (int64_t)pr.x * r.page_elems);
  u32x4 *b = (u32x4 *)(r.pool + (int64_t)pr.y * r.page_elems);
  const int64_t n = r.page_elems / 8, e0 = (int64_t)blockIdx.y * 256 * kCopyLoads + threadIdx.x;
  u32x4 x[kCopyLoads];
#pragma unroll
  for (int u = 0; u < kCopyLoads; ++u)
    if (e0 + u * 256 < n) x[u] = a[e0 + u * 256];
#pragma unroll
  for (int u = 0; u < kCopyLoads; ++u)
    if (e0 + u * 256 < n) b[e0 + u * 256] = x[u];
}

// Entries of a sequence's path that count: ascending, below its rows, at most path_cols. Whole wave.
__device__ __forceinline__ int path_length(const int32_t *__restrict__ path, int len, int cols, int rows) {
  const int lane = threadIdx.x & 63;
  int n = 0;
  len = min(max(len, 0), cols);
  for (int k0 = 0; k0 < cols; k0 += 64) {
    const int k = min(k0 + lane, cols - 1);  // read whatever the length: the two loads go together
    const int v = path[k], before = k > 0 ? path[k - 1] : -1;
    const uint64_t bad = __ballot(k0 + lane >= len || v <= before || v >= rows);
    if (bad) return k0 + __ffsll((unsigned long long)bad) - 1;
    n = k0 + 64;
  }
  return min(len, n);
}

// The entries of path[0, n) move to slots ctx, ctx + 1, ... in the pages of one KV head; one wave's work, a destination
// page at a time. Everything a page takes is read before it is written, and what later pages read lies behind it: path[k]
// >= k, strictly ascending.
template <int D>
__device__ __forceinline__ void move_slots(const PoolRef &r, const DraftSeq &s, int b, int g,
                                           const int32_t *__restrict__ path, int n) {
  constexpr int N = D / 32;      // 16-byte pieces of a lane: of sixteen K rows, or of a V block's 2 D half rows
  constexpr int LPR = D / 8;     // lanes of a K row
  const int lane = threadIdx.x & 63;
  const int64_t blk = (int64_t)kPage * D;
  uint16_t *const kb = r.pool + g * blk, *const vb = kb + r.n_kv * blk;
  for (int k0 = 0, count; k0 < n; k0 += count) {
    const int to = s.ctx + k0, slot0 = to % kPage;
    count = min(kPage - slot0, n - k0);
    if (to >= s.cap) return;
    // lane k: where entry k0 + k comes from (page -1: nowhere, or it stays)
    int page = -1, slot = 0;
    if (lane < count) {
      const int at = s.ctx + path[k0 + lane];
      if (at != to + lane && at < s.cap) page = page_of(r.table, b, at, r.cols, r.ring, r.pages);
      slot = at % kPage;
    }
    const int to_page = page_of(r.table, b, to, r.cols, r.ring, r.pages);
    const uint64_t moves = __ballot(page >= 0);
    if (to_page < 0 || !moves) continue;
    auto moved = [&](int half, int k) { return (moves << slot0 >> (half * 8 + k) & 1) != 0; };
    auto half_moves = [&](int half) { return (moves << slot0 >> (half * 8) & 0xff) != 0; };
    u32x4 key[N], val[N];
    uint16_t in[N][8];
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = i * (kWave / LPR) + lane / LPR, from = __shfl(page, e, kWave), at = __shfl(slot, e, kWave);
      if (from >= 0) key[i] = *(const u32x4 *)(kb + (int64_t)from * r.page_elems + at * D + lane % LPR * 8);
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int half = i * kWave / D, d = i * kWave % D + lane;
      if (!half_moves(half)) continue;
      val[i] = *(const u32x4 *)(vb + (int64_t)to_page * r.page_elems + d * kPage + half * 8);
#pragma unroll
      for (int k = 0; k < 8; ++k) {
        if (!moved(half, k)) continue;
        const int e = half * 8 + k - slot0;
        const int from = __builtin_amdgcn_readlane(page, e), at = __builtin_amdgcn_readlane(slot, e);
        in[i][k] = vb[(int64_t)from * r.page_elems + d * kPage + at];
      }
    }
    asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const int e = i * (kWave / LPR) + lane / LPR;
      if (__shfl(page, e, kWave) >= 0)
        *(u32x4 *)(kb + (int64_t)to_page * r.page_elems + (slot0 + e) * D + lane % LPR * 8) = key[i];
      const int half = i * kWave / D, d = i * kWave % D + lane;
      if (!half_moves(half)) continue;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (moved(half, 2 * k)) val[i][k] = (val[i][k] & 0xffff0000u) | in[i][2 * k];
        if (moved(half, 2 * k + 1)) val[i][k] = (val[i][k] & 0xffffu) | (uint32_t)in[i][2 * k + 1] << 16;
      }
      *(u32x4 *)(vb + (int64_t)to_page * r.page_elems + d * kPage + half * 8) = val[i];
    }
  }
}

// One wave per (sequence, KV head, layer): a long chain of small loads (rows, path, page ids, slots) that many waves hide.
// V is dim-major, so a slot's values lie in as many 32-byte rows as there are dims: moved ones are two-byte loads, 64 rows
// of a page each; a row's half is then written in one piece (256 trees of 64, 6 of 12 path entries moved, 4 layers of 8
// heads: 40 us; two bytes a store and a block per head 61).
// ctx_out: NULL, or new contexts, where nothing here reads them.
__global__ __launch_bounds__(256) void accept_kernel(AcceptArgs a, PoolSet pools, int32_t *__restrict__ ctx_out) {
  const int b = blockIdx.x, g = blockIdx.y * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const PoolRef r = pools.p[blockIdx.z];
  if (g >= r.n_kv) return;
  const DraftSeq s = draft_seq(a.row_off, a.ctx_lens, b, a.rows, a.max_rows, r.cols, r.ring);
  const int32_t *path = a.path + (int64_t)b * a.path_cols;
  const int n = path_length(path, a.path_len[b], a.path_cols, s.n);
  if (ctx_out && g == 0 && blockIdx.z == 0 && threadIdx.x == 0) {
    const int c = a.ctx_lens[b];
    ctx_out[b] = c < 0 ? c : c + n;
  }
  if (s.ctx < 0) return;
  if (r.D == 128)
    move_slots<128>(r, s, b, g, path, n);
  else
    move_slots<64>(r, s, b, g, path, n);
}

// New contexts in the place of the old ones, after every move has read those. One wave per sequence.
__global__ __launch_bounds__(64) void accept_ctx_kernel(AcceptArgs a, int32_t *ctx_out) {
  const int b = blockIdx.x;
  const DraftSeq s = draft_seq(a.row_off, a.ctx_lens, b, a.rows, a.max_rows, 1, 0);
  const int n = path_length(a.path + (int64_t)b * a.path_cols, a.path_len[b], a.path_cols, s.n);
  const int c = a.ctx_lens[b];
  if (threadIdx.x == 0) ctx_out[b] = c < 0 ? c : c + n;
}

}  // namespace

hipError_t launch_copy_pages(const PoolSet &pools, int n_pools, const int32_t *pairs, int n, hipStream_t s) {
  int64_t most = 0;  // 16-byte pieces of a page
  for (int i = 0; i < n_pools; ++i) most = std::max(most, pools.p[i].page_elems / 8);
  const int parts = (int)((most + 256 * kCopyLoads - 1) / (256 * kCopyLoads));
  for (int64_t at = 0; at < n; at += kMaxGridX) {
    hipLaunchKernelGGL(copy_pages_kernel, dim3((int)std::min<int64_t>(n - at, kMaxGridX), parts, n_pools), dim3(256), 0, s, pools,
                       (const int2 *)pairs + at);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

hipError_t launch_accept(const AcceptArgs &a, const PoolSet &pools, int n_pools, int max_kv, int32_t *ctx_out, hipStream_t s) {
  hipLaunchKernelGGL(accept_kernel, dim3(a.B, (max_kv + 3) / 4, n_pools), dim3(256), 0, s, a, pools, ctx_out);
  return hipGetLastError();
}

hipError_t launch_accept_ctx(const AcceptArgs &a, int32_t *ctx_out, hipStream_t s) {
  hipLaunchKernelGGL(accept_ctx_kernel, dim3(a.B), dim3(64), 0, s, a, ctx_out);
  return hipGetLastError();
}

}  // namespace ods
