// Turning the heads of one row, by the 256 threads of a block.
#pragma once
#include "common.hpp"

namespace ods {

// (a, b) -> (a c - b s, b c + a s); the amplitude is in c and s.
__device__ __forceinline__ void turn2(float &a, float &b, float c, float s) {
  const float t = a * c - b * s;
  b = b * c + a * s;
  a = t;
}

// The row's turns, by the first threads of the block: angle(i, cos, sin) of each pair times the amplitude. Ends with a
// barrier.
template <typename Angle>
__device__ __forceinline__ void row_turns(int np, float amp, float *cs, float *sn, Angle angle) {
  if (threadIdx.x < np) {
    float c, s;
    angle(threadIdx.x, c, s);
    cs[threadIdx.x] = c * amp;
    sn[threadIdx.x] = s * amp;
  }
  __syncthreads();
}

// dst = src turned, 16 bytes a load: an item is eight pairs of the half layout (two loads, half a rotary part apart), four
// of the interleaved one, or, where dst is not src, eight values that pass through. rdim is a multiple of 16, or 8. A
// thread's first loads are made before `turns`, which fills cs and sn: its sines come under them.
template <bool INTERLEAVED, typename Turns>
__device__ __forceinline__ void turn_row(const uint16_t *src, uint16_t *dst, int heads, int D, int rdim, const float *cs,
                                         const float *sn, Turns turns) {
  constexpr int U = INTERLEAVED ? 4 : 2;  // items of a thread in flight
  const int np = rdim / 2, turned = INTERLEAVED ? rdim / 8 : np / 8;
  const int per = turned + (src == dst ? 0 : (D - rdim) / 8), items = heads * per;
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
    if (t0 == 0) turns();
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

// The same for pairs that do not come in whole 16 bytes, value by value, cs and sn filled. 8192 rows of 40 heads of 128, 24 of
// a half layout turned: 71 us, 2.4 TB/s, where turn_row takes 32 for parts it can do; the pass-through dims go this way too.
__device__ __forceinline__ void turn_row_by_values(const uint16_t *src, uint16_t *dst, int heads, int D, int rdim,
                                                   int interleaved, const float *cs, const float *sn) {
  const int np = rdim / 2;
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

// Whether turn_row takes it.
__host__ __device__ inline bool turns_wide(int rdim, int interleaved) { return rdim % (interleaved ? 8 : 16) == 0; }

}  // namespace ods
