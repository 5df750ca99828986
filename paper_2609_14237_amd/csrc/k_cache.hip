// Page operators of the KV cache: copies of whole pages, and the slots of an
// accepted path moved to the front of a sequence's drafted ones.
#include "draft.hpp"
#include "kernels.hpp"

namespace ods {

namespace {

// One block per (pair, layer): the page's keys and values, 16 bytes a thread.
__global__ __launch_bounds__(256) void copy_pages_kernel(PoolSet pools, const int32_t *__restrict__ pairs, int n) {
  const PoolRef r = pools.p[blockIdx.y];
  const int i = blockIdx.x;
  const int src = pairs[2 * i], dst = pairs[2 * i + 1];
  if (src == dst || src < 0 || dst < 0 || src >= r.pages || dst >= r.pages) return;
  const u32x4 *a = (const u32x4 *)(r.pool + (int64_t)src * r.page_elems);
  u32x4 *b = (u32x4 *)(r.pool + (int64_t)dst * r.page_elems);
  for (int64_t e = threadIdx.x; e < r.page_elems / 8; e += 256) b[e] = a[e];
}

// Entries of a sequence's path that count: ascending, below its rows, at most path_cols. Whole wave.
__device__ __forceinline__ int path_length(const int32_t *__restrict__ path, int len, int cols, int rows) {
  const int lane = threadIdx.x & 63;
  len = min(max(len, 0), cols);
  int n = 0;
  for (int k0 = 0; k0 < len; k0 += 64) {
    const int k = k0 + lane;
    bool ok = true;
    if (k < len) {
      const int v = path[k], before = k > 0 ? path[k - 1] : -1;
      ok = v > before && v < rows;
    }
    const uint64_t bad = __ballot(!ok);
    if (bad) return k0 + __ffsll((unsigned long long)bad) - 1;
    n = min(len, k0 + 64);
  }
  return n;
}

// One block per (sequence, KV head, layer). Sixteen path entries at a time are
// read to registers, then written: path[k] >= k, so what later sixteens read
// lies past what earlier ones wrote.
__global__ __launch_bounds__(256) void accept_kernel(AcceptArgs a, PoolSet pools) {
  const int b = blockIdx.x, g = blockIdx.y;
  const PoolRef r = pools.p[blockIdx.z];
  if (g >= r.n_kv) return;
  const int D = r.D;
  const DraftSeq s = draft_seq(a.row_off, a.ctx_lens, b, a.rows, a.max_rows, r.cols, r.ring);
  if (s.ctx < 0) return;
  const int32_t *path = a.path + (int64_t)b * a.path_cols;
  const int n = path_length(path, a.path_len[b], a.path_cols, s.n);
  const int64_t blk = (int64_t)kPage * D;
  const int i = threadIdx.x % D, per = 256 / D;  // this thread's dim, entries moved at once
  for (int k0 = 0; k0 < n; k0 += kPage) {
    uint16_t kv[2][8];
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int k = k0 + threadIdx.x / D + u * per;
      if (k >= min(n, k0 + kPage)) continue;
      const int at = s.ctx + path[k];
      const int page = at < s.cap ? page_of(r.table, b, at, r.cols, r.ring, r.pages) : -1;
      if (page < 0) continue;
      const uint16_t *src = r.pool + (int64_t)page * r.page_elems + g * blk;
      kv[0][u] = src[(at % kPage) * D + i];
      kv[1][u] = src[r.n_kv * blk + i * kPage + at % kPage];
    }
    __syncthreads();
#pragma unroll
    for (int u = 0; u < 8; ++u) {
      const int k = k0 + threadIdx.x / D + u * per;
      if (k >= min(n, k0 + kPage)) continue;
      const int at = s.ctx + path[k], to = s.ctx + k;
      const int from = at < s.cap ? page_of(r.table, b, at, r.cols, r.ring, r.pages) : -1;
      const int page = to < s.cap ? page_of(r.table, b, to, r.cols, r.ring, r.pages) : -1;
      if (from < 0 || page < 0) continue;
      uint16_t *dst = r.pool + (int64_t)page * r.page_elems + g * blk;
      dst[(to % kPage) * D + i] = kv[0][u];
      dst[r.n_kv * blk + i * kPage + to % kPage] = kv[1][u];
    }
    __syncthreads();
  }
}

// New contexts, after every move has read the old ones. One wave per sequence.
__global__ __launch_bounds__(64) void accept_ctx_kernel(AcceptArgs a, int32_t *ctx_out) {
  const int b = blockIdx.x;
  const DraftSeq s = draft_seq(a.row_off, a.ctx_lens, b, a.rows, a.max_rows, 1, 0);
  const int n = path_length(a.path + (int64_t)b * a.path_cols, a.path_len[b], a.path_cols, s.n);
  const int c = a.ctx_lens[b];
  if (threadIdx.x == 0) ctx_out[b] = c < 0 ? c : c + n;
}

}  // namespace

hipError_t launch_copy_pages(const PoolSet &pools, int n_pools, const int32_t *pairs, int n, hipStream_t s) {
  hipLaunchKernelGGL(copy_pages_kernel, dim3(n, n_pools), dim3(256), 0, s, pools, pairs, n);
  return hipGetLastError();
}

hipError_t launch_accept(const AcceptArgs &a, const PoolSet &pools, int n_pools, int max_kv, hipStream_t s) {
  hipLaunchKernelGGL(accept_kernel, dim3(a.B, max_kv, n_pools), dim3(256), 0, s, a, pools);
  return hipGetLastError();
}

hipError_t launch_accept_ctx(const AcceptArgs &a, int32_t *ctx_out, hipStream_t s) {
  hipLaunchKernelGGL(accept_ctx_kernel, dim3(a.B), dim3(64), 0, s, a, ctx_out);
  return hipGetLastError();
}

}  // namespace ods
