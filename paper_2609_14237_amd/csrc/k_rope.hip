// Rotary positions of arbitrary rows (ods_rope_rows): y = x turned to each
// row's position, half or interleaved pairs, part of the head, frequencies
// from a table of doubles.
#include "common.hpp"
#include "kernels.hpp"

namespace ods {

namespace {

// (a, b) -> (a c - b s, b c + a s); the amplitude is in c and s.
__device__ __forceinline__ void turn2(float &a, float &b, float c, float s) {
  const float t = a * c - b * s;
  b = b * c + a * s;
  a = t;
}

// One block per row. Memory-bound: every value is read once and written once.
__global__ __launch_bounds__(256) void rope_rows_kernel(const uint16_t *x, int64_t xs, uint16_t *y, int64_t ys,
                                                        int heads, int D, int rdim, int interleaved,
                                                        const double *__restrict__ freqs, float amp,
                                                        const int32_t *__restrict__ pos) {
  __shared__ float cs[128], sn[128];
  const int64_t row = blockIdx.x;
  const int p = pos[row];
  if (p < 0) return;
  const int np = rdim / 2;
  if (threadIdx.x < np) {
    float c, s;
    turn_by((double)p * freqs[threadIdx.x], c, s);
    cs[threadIdx.x] = c * amp;
    sn[threadIdx.x] = s * amp;
  }
  __syncthreads();
  const uint16_t *src = x + row * xs;
  uint16_t *dst = y + row * ys;
  for (int t = threadIdx.x; t < heads * np; t += 256) {
    const int i = t % np, at = t / np * D + (interleaved ? 2 * i : i), mate = at + (interleaved ? 1 : np);
    float a = bf2f(src[at]), b = bf2f(src[mate]);
    turn2(a, b, cs[i], sn[i]);
    dst[at] = f2bf(a);
    dst[mate] = f2bf(b);
  }
  if (src != dst) {
    const int rest = D - rdim;
    for (int t = threadIdx.x; t < heads * rest; t += 256) {
      const int at = t / rest * D + rdim + t % rest;
      dst[at] = src[at];
    }
  }
}

}  // namespace

hipError_t launch_rope_rows(const ods_rope &r, const uint16_t *x, int64_t xs, uint16_t *y, int64_t ys, int rows,
                            int heads, const int32_t *pos, hipStream_t s) {
  if (rows <= 0 || heads <= 0) return hipSuccess;
  hipLaunchKernelGGL(rope_rows_kernel, dim3(rows), dim3(256), 0, s, x, xs, y, ys, heads, r.head_dim, r.rotary_dim,
                     r.interleaved, r.freqs, r.amplitude, pos);
  return hipGetLastError();
}

}  // namespace ods
