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

// cos and sin of position p times each frequency, by the first threads of the block.
__device__ __forceinline__ void turns(int p, int np, const double *__restrict__ freqs, float amp, float *cs, float *sn) {
  if (threadIdx.x < np) {
    float c, s;
    turn_by((double)p * freqs[threadIdx.x], c, s);
    cs[threadIdx.x] = c * amp;
    sn[threadIdx.x] = s * amp;
  }
  __syncthreads();
}

// One block per row, 16 bytes a load: an item is eight pairs of the half layout (two loads, half a head apart), four of the
// interleaved one, or, where y is not x, eight values that pass through. Bound by memory: a value is read once and written
// once. A thread's loads are made before the angles, whose double products and sincosf they cover. 8192 rows of 40 heads,
// half of each turned, 168 MB: 32 us, 5.2 TB/s, what a copy reaches (two
// bytes a load: 61 us).
template <bool INTERLEAVED>
__global__ __launch_bounds__(256) void rope_rows_wide_kernel(const uint16_t *x, int64_t xs, uint16_t *y, int64_t ys,
                                                             int heads, int D, int rdim, const double *__restrict__ freqs,
                                                             float amp, const int32_t *__restrict__ pos) {
  constexpr int U = INTERLEAVED ? 4 : 2;  // items of a thread in flight
  __shared__ __align__(16) float cs[128], sn[128];
  const int64_t row = blockIdx.x;
  const int p = pos[row];
  if (p < 0) return;
  const int np = rdim / 2, turned = INTERLEAVED ? rdim / 8 : np / 8;
  const int per = turned + (x == y ? 0 : (D - rdim) / 8), items = heads * per;
  const uint16_t *src = x + row * xs;
  uint16_t *dst = y + row * ys;
  for (int t0 = 0; t0 < items; t0 += 256 * U) {
    u32x4 a[U], b[U];
    int at[U], pair[U];  // first dim in the row; first pair, -1: none
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = min(t0 + u * 256 + (int)threadIdx.x, items - 1);  // past the last: it again, not stored
      const int h = t / per, i = t - h * per;
      pair[u] = i >= turned ? -1 : INTERLEAVED ? i * 4 : i * 8;
      at[u] = h * D + (i < turned ? i * 8 : rdim + (i - turned) * 8);
      a[u] = *(const u32x4 *)(src + at[u]);
      if (!INTERLEAVED) b[u] = *(const u32x4 *)(src + at[u] + (i < turned ? np : 0));
    }
    if (t0 == 0) turns(p, np, freqs, amp, cs, sn);
#pragma unroll
    for (int u = 0; u < U; ++u) {
      if (t0 + u * 256 + (int)threadIdx.x >= items) break;
      if (pair[u] >= 0) {
        constexpr int N = INTERLEAVED ? 4 : 8;
        float c[N], s[N];
#pragma unroll
        for (int k = 0; k < N; k += 4) {
          *(f32x4 *)(c + k) = *(const f32x4 *)(cs + pair[u] + k);
          *(f32x4 *)(s + k) = *(const f32x4 *)(sn + pair[u] + k);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          float lo = bf2f((uint16_t)a[u][k]), hi = bf2f((uint16_t)(a[u][k] >> 16));
          if (INTERLEAVED) {
            turn2(lo, hi, c[k], s[k]);
          } else {
            float lo2 = bf2f((uint16_t)b[u][k]), hi2 = bf2f((uint16_t)(b[u][k] >> 16));
            turn2(lo, lo2, c[2 * k], s[2 * k]);
            turn2(hi, hi2, c[2 * k + 1], s[2 * k + 1]);
            b[u][k] = pack2(lo2, hi2);
          }
          a[u][k] = pack2(lo, hi);
        }
        if (!INTERLEAVED) *(u32x4 *)(dst + at[u] + np) = b[u];
      }
      *(u32x4 *)(dst + at[u]) = a[u];
    }
  }
}

// Pairs that do not come in whole 16 bytes (rotary dims that are no multiple of 8, of 16 in the half layout): value by value.
__global__ __launch_bounds__(256) void rope_rows_kernel(const uint16_t *x, int64_t xs, uint16_t *y, int64_t ys,
                                                        int heads, int D, int rdim, int interleaved,
                                                        const double *__restrict__ freqs, float amp,
                                                        const int32_t *__restrict__ pos) {
  __shared__ float cs[128], sn[128];
  const int64_t row = blockIdx.x;
  const int p = pos[row];
  if (p < 0) return;
  const int np = rdim / 2;
  turns(p, np, freqs, amp, cs, sn);
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
  if (r.rotary_dim % (r.interleaved ? 8 : 16) == 0)
    hipLaunchKernelGGL(r.interleaved ? rope_rows_wide_kernel<true> : rope_rows_wide_kernel<false>, dim3(rows), dim3(256), 0, s,
                       x, xs, y, ys, heads, r.head_dim, r.rotary_dim, r.freqs, r.amplitude, pos);
  else
    hipLaunchKernelGGL(rope_rows_kernel, dim3(rows), dim3(256), 0, s, x, xs, y, ys, heads, r.head_dim, r.rotary_dim,
                       r.interleaved, r.freqs, r.amplitude, pos);
  return hipGetLastError();
}

}  // namespace ods
