// Turning the heads of a row, by the 256 threads of a block, and of several rows whose heads are normalised first, by up to 512
// (turn_heads).
#pragma once
#include <type_traits>

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

// ---------------------------------------------------------------- heads normalised before they turn
//
// y = R(pos) (x inv gain), inv = (mean(x^2) + eps)^-1/2 over the head, rounded once, at the end. A head lies on L
// neighbouring lanes of one wave (L a power of two, 32 at most), so its sum of squares is a reduction over lanes and a value
// is read once and written once.
struct HeadTurn {
  int heads, n_q, D, rdim, interleaved;
  const uint16_t *gain_q, *gain_k;  // null: no norm
  float eps;
};

enum HeadKind {
  kHalves,  // half layout, rdim % 16 == 0: an item is 16 bytes of first values and the 16 of their mates, or 16 that pass through
  kPairs,   // interleaved, rdim % 8 == 0: an item is four pairs
  kAny      // else an item is 8 values, whose mates come from the neighbouring lanes by way of LDS
};
__host__ __device__ inline HeadKind head_kind(int rdim, int interleaved) {
  return rdim % (interleaved ? 8 : 16) != 0 ? kAny : interleaved ? kPairs : kHalves;
}
__host__ __device__ inline int head_items(HeadKind kind, int D, int rdim) {
  return kind == kHalves ? rdim / 16 + (D - rdim) / 8 : D / 8;
}
// log2 of the lanes of a head
__host__ __device__ inline int head_lanes_log2(int items) {
  int log = 0;
  while (1 << log < items) ++log;
  return log;
}

// Sum over groups of 1 << log neighbouring lanes, in every lane of the group: partners within rows of sixteen lanes by the
// data path of the vector unit, the two rows of 32 lanes by a shuffle.
__device__ __forceinline__ float lanes_sum(float v, int log) {
  auto with = [](float x, float y) { return x + y; };
  auto moved = [](float x, auto ctrl) {
    return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, x), decltype(ctrl)::value, 0xf, 0xf, true));
  };
  if (log > 0) v = with(v, moved(v, std::integral_constant<int, 0xb1>()));   // lane ^ 1
  if (log > 1) v = with(v, moved(v, std::integral_constant<int, 0x4e>()));   // lane ^ 2
  if (log > 2) v = with(v, moved(v, std::integral_constant<int, 0x141>()));  // 7 - lane of eight: the other four, alike by now
  if (log > 3) v = with(v, moved(v, std::integral_constant<int, 0x140>()));  // 15 - lane of sixteen
  if (log > 4) v = with(v, __shfl_xor(v, 16, kWave));
  return v;
}

__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {  // one conversion for both
  typedef float f32x2 __attribute__((ext_vector_type(2)));
  typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), bf16x2));
}

// Heads of `rows` rows by the NT threads of a block, U items of each in flight; src(r) and dst(r) are a row's first value
// (they may be the same). A thread's first loads are made before `turns`, which fills cs and sn (row r's cosines start at
// cs + r * rdim / 2) and what go(r), whether row r is done at all, looks at: its sines come under them. exchange: 8 NT floats
// of LDS, kAny only.
template <int KIND, int U, typename Src, typename Dst, typename Go, typename Turns>
__device__ __forceinline__ void turn_heads(const HeadTurn &p, int rows, int NT, Src src, Dst dst, Go go, const float *cs,
                                           const float *sn, float *exchange, Turns turns) {
  const int np = p.rdim / 2, turned = np / 8, items = head_items((HeadKind)KIND, p.D, p.rdim);
  const int log = head_lanes_log2(items), lanes = 1 << log, total = rows * p.heads << log;
  const float inv_d = 1.f / (float)p.D, inv_heads = 1.f / (float)p.heads;
  for (int t0 = 0; t0 < total; t0 += NT * U) {
    u32x4 a[U], b[U], ga[U], gb[U];
    int row[U], head[U], at[U];  // at: first dim of the item, -1: none
    bool pair[U];                // kHalves: the item has mates
#pragma unroll
    for (int u = 0; u < U; ++u) {
      const int t = t0 + u * NT + (int)threadIdx.x, h = min(t >> log, rows * p.heads - 1), i = t & (lanes - 1);
      row[u] = rows == 1 ? 0 : (int)(((float)h + 0.5f) * inv_heads);  // h / heads, exact: eight rows of less than 2^13 heads (one
                                                                      // row of more)
      head[u] = h - row[u] * p.heads;
      pair[u] = KIND == kHalves && i < turned;
      at[u] = t >= total || i >= items ? -1 : KIND != kHalves || i < turned ? i * 8 : p.rdim + (i - turned) * 8;
      a[u] = b[u] = u32x4{0u, 0u, 0u, 0u};
      if (at[u] < 0) continue;
      const uint16_t *x = src(row[u]) + head[u] * p.D + at[u];
      a[u] = *(const u32x4 *)x;
      if (pair[u]) b[u] = *(const u32x4 *)(x + np);
    }
    if (p.gain_q || p.gain_k) {
#pragma unroll
      for (int u = 0; u < U; ++u) {
        const uint16_t *g = (head[u] < p.n_q ? p.gain_q : p.gain_k) + max(at[u], 0);
        ga[u] = *(const u32x4 *)g;
        gb[u] = pair[u] ? *(const u32x4 *)(g + np) : ga[u];
      }
    }
    if (t0 == 0) turns();
#pragma unroll
    for (int u = 0; u < U; ++u) {
      float v[8], w[8];  // the item's values, and their mates (kHalves)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        v[2 * k] = bf_lo(a[u][k]);
        v[2 * k + 1] = bf_hi(a[u][k]);
        w[2 * k] = bf_lo(b[u][k]);
        w[2 * k + 1] = bf_hi(b[u][k]);
      }
      if (p.gain_q || p.gain_k) {
        float sum = sumsq8(a[u]);
        if (KIND == kHalves) sum += sumsq8(b[u]);
        const float inv = rsqrtf(lanes_sum(sum, log) * inv_d + p.eps);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          v[2 * k] *= inv * bf_lo(ga[u][k]);
          v[2 * k + 1] *= inv * bf_hi(ga[u][k]);
          if (KIND != kHalves) continue;
          w[2 * k] *= inv * bf_lo(gb[u][k]);
          w[2 * k + 1] *= inv * bf_hi(gb[u][k]);
        }
      }
      const float *c = cs + row[u] * np, *s = sn + row[u] * np;
      if (KIND == kHalves && pair[u]) {
        float cv[8], sv[8];
#pragma unroll
        for (int k = 0; k < 8; k += 4) {
          *(f32x4 *)(cv + k) = *(const f32x4 *)(c + at[u] + k);
          *(f32x4 *)(sv + k) = *(const f32x4 *)(s + at[u] + k);
        }
#pragma unroll
        for (int k = 0; k < 8; ++k) turn2(v[k], w[k], cv[k], sv[k]);
      } else if (KIND == kPairs && at[u] >= 0 && at[u] < p.rdim) {
        const f32x4 cv = *(const f32x4 *)(c + at[u] / 2), sv = *(const f32x4 *)(s + at[u] / 2);
#pragma unroll
        for (int k = 0; k < 4; ++k) turn2(v[2 * k], v[2 * k + 1], cv[k], sv[k]);
      } else if (KIND == kAny) {
        float *mine = exchange + threadIdx.x * 8;
        *(f32x4 *)mine = f32x4{v[0], v[1], v[2], v[3]};
        *(f32x4 *)(mine + 4) = f32x4{v[4], v[5], v[6], v[7]};
        // A wave's LDS operations are done in order: the writes above and those of the next item need no wait, only to stay
        // where they are.
        __builtin_amdgcn_wave_barrier();
        asm volatile("" ::: "memory");
        const float *first = exchange + (threadIdx.x & ~(lanes - 1)) * 8;  // the head's dim 0
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const int d = at[u] + k;
          if (at[u] < 0 || d >= p.rdim) continue;
          const bool low = p.interleaved ? !(d & 1) : d < np;
          const int j = p.interleaved ? d >> 1 : low ? d : d - np;
          const float mate = first[p.interleaved ? d ^ 1 : low ? d + np : d - np];
          v[k] = low ? v[k] * c[j] - mate * s[j] : v[k] * c[j] + mate * s[j];
        }
        asm volatile("" ::: "memory");
        __builtin_amdgcn_wave_barrier();
      }
      if (at[u] < 0 || !go(row[u])) continue;
      uint16_t *y = dst(row[u]) + head[u] * p.D + at[u];
      *(u32x4 *)y = u32x4{pack_bf16(v[0], v[1]), pack_bf16(v[2], v[3]), pack_bf16(v[4], v[5]), pack_bf16(v[6], v[7])};
      if (pair[u]) *(u32x4 *)(y + np) = u32x4{pack_bf16(w[0], w[1]), pack_bf16(w[2], w[3]), pack_bf16(w[4], w[5]), pack_bf16(w[6], w[7])};
    }
  }
}

// Whether turn_row takes it.
__host__ __device__ inline bool turns_wide(int rdim, int interleaved) { return rdim % (interleaved ? 8 : 16) == 0; }

}  // namespace ods
