// Rotary positions of arbitrary rows (ods_rope_rows): y = x turned to each
// row's position, half or interleaved pairs, part of the head, frequencies
// from a table of doubles. The same of heads that are normalised first, and of
// positions with several axes (ods_head_rows).
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

// `per` rows a block (kHeadRows at most). Bound by memory, and by what the block waits for before its first row: positions,
// then frequencies, then fp64 angles. Several rows a block share that wait, and all but the first items of a thread are loaded
// without it (8192 rows of 32 + 8 heads of 128, 168 MB: a row a block 42 us, four 38, 4.4 TB/s; a copy takes 33; 4097 rows of
// 36 heads, half of each turned: 33 and 20).
constexpr int kHeadRows = 8, kHeadThreads = 512;
template <int KIND>
__global__ __launch_bounds__(kHeadThreads) void head_rows_kernel(const HeadRowsArgs a, int rows, int per) {
  __shared__ __align__(16) float cs[kHeadRows * 128], sn[kHeadRows * 128];
  __shared__ __align__(16) float exchange[KIND == kAny ? 8 * kHeadThreads : 4];
  __shared__ int go[kHeadRows];
  const int64_t row0 = (int64_t)blockIdx.x * per;
  const int n = (int)min((int64_t)per, rows - row0), np = a.turn.rdim / 2, NT = blockDim.x;
  const int32_t *pos = a.pos + row0 * a.n_axes;
  auto turns = [&]() {
    if (threadIdx.x < n) {
      bool all = true;
      for (int i = 0; i < a.n_axes; ++i) all = all && pos[threadIdx.x * a.n_axes + i] >= 0;
      go[threadIdx.x] = all;
    }
    for (int t = threadIdx.x; t < n * np; t += NT) {
      const int r = t / np, i = t - r * np;
      const int axis = a.axis ? min(max(a.axis[i], 0), a.n_axes - 1) : 0;
      float c, s;
      turn_by((double)pos[r * a.n_axes + axis] * a.freqs[i], c, s);
      cs[t] = c * a.amp;
      sn[t] = s * a.amp;
    }
    __syncthreads();
  };
  turn_heads<KIND, 1>(
      a.turn, n, NT, [&](int r) { return a.x + (row0 + r) * a.xs; }, [&](int r) { return a.y + (row0 + r) * a.ys; },
      [&](int r) { return go[r] != 0; }, cs, sn, exchange, turns);
}

}  // namespace

hipError_t launch_head_rows(const HeadRowsArgs &args, int rows, hipStream_t s) {
  if (rows <= 0 || args.turn.heads <= 0) return hipSuccess;
  const HeadKind kind = head_kind(args.turn.rdim, args.turn.interleaved);
  const auto kern = kind == kHalves ? head_rows_kernel<kHalves> : kind == kPairs ? head_rows_kernel<kPairs> : head_rows_kernel<kAny>;
  const int64_t of_row = (int64_t)args.turn.heads << head_lanes_log2(head_items(kind, args.turn.D, args.turn.rdim));
  // Four rows, or more of few heads; fewer where that would leave fewer than two blocks for each of 256 compute units.
  const int64_t per_most = args.turn.heads < 1 << 13 ? kHeadRows : 1;  // turn_heads divides in fp32
  const int per = (int)std::min<int64_t>({per_most, std::max<int64_t>(4, kHeadThreads / of_row), std::max(1, rows / 512)});
  const int threads = (int)std::min<int64_t>(kHeadThreads, (per * of_row + kWave - 1) / kWave * kWave);
  HeadRowsArgs a = args;
  const int64_t most = ((int64_t)kMaxGridX * 256 / kHeadThreads) * per;  // rows of a launch
  for (int64_t at = 0; at < rows; at += most) {
    const int n = (int)std::min<int64_t>(rows - at, most);
    a.x = args.x + at * a.xs;
    a.y = args.y + at * a.ys;
    a.pos = args.pos + at * a.n_axes;
    hipLaunchKernelGGL(kern, dim3((n + per - 1) / per), dim3(threads), 0, s, a, n, per);
    if (const hipError_t e = hipGetLastError(); e != hipSuccess) return e;
  }
  return hipSuccess;
}

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
