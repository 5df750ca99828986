// Rotary positions of arbitrary rows (ods_rope_rows): y = x turned to each
// row's position, half or interleaved pairs, part of the head, frequencies
// from a table of doubles.
#include <algorithm>

#include "kernels.hpp"
#include "turn.hpp"

namespace ods {

namespace {

// One block per row. Bound by memory: a value is read once and written once. 8192 rows of 40 heads, half of each turned,
// 168 MB: 32 us, 5.2 TB/s, what a copy reaches (two bytes a load: 61 us). WIDE as by turns_wide.
template <bool WIDE, bool INTERLEAVED>
__global__ __launch_bounds__(256) void rope_rows_kernel(const uint16_t *x, int64_t xs, uint16_t *y, int64_t ys, int heads,
                                                        int D, int rdim, const double *__restrict__ freqs, float amp,
                                                        const int32_t *__restrict__ pos) {
  __shared__ __align__(16) float cs[128], sn[128];
  const int64_t row = blockIdx.x;
  const int p = pos[row];
  if (p < 0) return;
  const uint16_t *src = x + row * xs;
  uint16_t *dst = y + row * ys;
  auto turns = [&]() {
    row_turns(rdim / 2, amp, cs, sn, [&](int i, float &c, float &s) { turn_by((double)p * freqs[i], c, s); });
  };
  if (WIDE) {
    turn_row<INTERLEAVED>(src, dst, heads, D, rdim, cs, sn, turns);
  } else {
    turns();
    turn_row_by_values(src, dst, heads, D, rdim, INTERLEAVED, cs, sn);
  }
}

}  // namespace

hipError_t launch_rope_rows(const ods_rope &r, const uint16_t *x, int64_t xs, uint16_t *y, int64_t ys, int rows,
                            int heads, const int32_t *pos, hipStream_t s) {
  if (rows <= 0 || heads <= 0) return hipSuccess;
  const bool wide = turns_wide(r.rotary_dim, r.interleaved);
  const auto kern = r.interleaved ? (wide ? rope_rows_kernel<true, true> : rope_rows_kernel<false, true>)
                                  : (wide ? rope_rows_kernel<true, false> : rope_rows_kernel<false, false>);
  for (int64_t at = 0; at < rows; at += kMaxGridX) {
    const int n = (int)std::min<int64_t>(rows - at, kMaxGridX);
    hipLaunchKernelGGL(kern, dim3(n), dim3(256), 0, s, x + at * xs, xs, y + at * ys, ys, heads, r.head_dim, r.rotary_dim, r.freqs,
                       r.amplitude, pos + at);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace ods
