// Device helpers of the drafted-row kernels: a sequence's rows and tokens.
#pragma once
#include "common.hpp"

namespace ods {

// Drafted rows and cache extent of one sequence, whatever the device arrays
// hold: rows [r0, r0 + n) lie inside the buffers, ctx is the cached tokens
// (-1: the sequence is left alone), tokens [0, end) can be attended, and slots
// below cap can be written.
struct DraftSeq {
  int r0, n;
  int ctx, end, cap;
};

// Arrays a kernel only reads, as constant memory: a uniform index becomes a scalar load, which does not queue behind the
// vector loads in flight.
typedef const __attribute__((address_space(4))) int32_t *ConstInts;

template <typename Ints>  // const int32_t * or ConstInts
__device__ __forceinline__ DraftSeq draft_seq(Ints row_off, Ints ctx_lens, int b, int rows, int max_rows, int cols,
                                              int ring) {
  DraftSeq s;
  const int a = row_off[b], e = row_off[b + 1], c = ctx_lens[b];
  s.r0 = a;
  s.n = a < 0 || a >= rows || e <= a ? 0 : min(min(e, rows) - a, max_rows);
  s.cap = ring > 0 ? 0x7fffffff : cols * kPage;
  s.ctx = c < 0 ? -1 : min(c, 0x7fff0000);  // positions and slots past it stay inside 31 bits
  s.end = s.ctx < 0 || s.n == 0 ? 0 : min(s.ctx + s.n, s.cap);
  return s;
}

// Page of token position t of sequence b (-1 if it has none in the pool).
__device__ __forceinline__ int page_of(const int32_t *__restrict__ table, int b, int t, int cols, int ring,
                                       int64_t pool_pages) {
  const int lp = t / kPage;
  if (ring <= 0 && lp >= cols) return -1;
  const int page = table[(int64_t)b * cols + (ring > 0 ? lp % ring : lp)];
  return page >= 0 && page < pool_pages ? page : -1;
}

__device__ __forceinline__ int clamp_depth(int d, int max_rows) { return min(max(d, 0), max_rows - 1); }

}  // namespace ods
