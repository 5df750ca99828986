// Verification of drafted tokens (ods_draft_verify): each sequence's tree is
// walked along its accepted path, then the token after the path is drawn from
// what is left of the target's probabilities there.
#include <string.h>

#include "draft.hpp"
#include "kernels.hpp"

namespace ods {

namespace {

// W after k children of a row were refused, at one token of its probability p (and proposal q): W_0 = p,
// W_i+1 = max(W_i - Z_i q, 0). A sum over 2^17 tokens loses in fp32 what decides at the border of two of them; the sums and
// all that is compared with them are fp64. It costs no time: five such operations per 8 bytes read.
__device__ __forceinline__ double left_of(float p, float q, const double *z, int k) {
  double w = p;
  for (int i = 0; i < k; ++i) w = fmax(w - z[i] * (double)q, 0.0);
  return w;
}

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(uint16_t v) { return bf2f(v); }
// Negative or not finite: 0.
__device__ __forceinline__ float positive(float v) { return v > 0.f && v < INFINITY ? v : 0.f; }
template <typename T>
__device__ __forceinline__ float prob(const T *row, int t) { return positive(to_float(row[t])); }

// N values from e on, those past `end` as 0. Rows start anywhere: the loads need the alignment of a value only.
template <int N, typename T>
__device__ __forceinline__ void load_probs(const T *__restrict__ row, int e, int end, float (&v)[N]) {
  constexpr int PER = 16 / sizeof(T);
  if (e + N <= end) {
#pragma unroll
    for (int i = 0; i < N; i += PER) {
      T w[PER];
      memcpy(w, row + e + i, 16);
#pragma unroll
      for (int j = 0; j < PER; ++j) v[i + j] = positive(to_float(w[j]));
    }
  } else {
#pragma unroll
    for (int i = 0; i < N; ++i) v[i] = e + i < end ? prob(row, e + i) : 0.f;
  }
}

__device__ __forceinline__ double wave_sum_f64(double v) {
#pragma unroll
  for (int o = 32; o >= 1; o >>= 1) v += __shfl_xor(v, o, kWave);
  return v;
}

// Where a sequence's walk ended.
struct VerifyHead {
  int row;    // of the live buffers; -1: the sequence has none
  int k;      // children refused there
  int pad[2];
};
static_assert(sizeof(VerifyHead) == 16, "workspace layout");

struct VerifyArgs {
  int B, rows, max_rows, vocab, chunks, path_cols;
  const int32_t *row_off, *tokens, *parent;
  const float *accept_u, *next_u;
  const void *target, *proposal;
  int64_t target_stride, proposal_stride;
  int32_t *path, *path_len, *next_token;
  VerifyHead *head;  // [B]
  double *list;      // [B][ODS_DRAFT_MAX_ROWS]: the Z_i of the last row, or (int32) its refused tokens
  double *sums;      // [B][chunks]
};

// What is left at the row a walk ended with: k refused tokens, or k sums of the proposal.
template <typename T, bool DRAWN>
struct Rest {
  const T *p, *q;
  int k, vocab;
  const double *z;  // LDS or global
  const int32_t *gone;
  // Values [e, e + N); uniform k.
  template <int N>
  __device__ __forceinline__ void load(int e, double (&w)[N]) const {
    float a[N], b[N];
    load_probs<N>(p, e, vocab, a);
    if (DRAWN && k > 0) {
      load_probs<N>(q, e, vocab, b);
#pragma unroll
      for (int i = 0; i < N; ++i) w[i] = left_of(a[i], b[i], z, k);
      return;
    }
#pragma unroll
    for (int i = 0; i < N; ++i) w[i] = a[i];
    if (!DRAWN) {
      for (int j = 0; j < k; ++j) {
        const int at = gone[j] - e;
#pragma unroll
        for (int i = 0; i < N; ++i)
          if (at == i) w[i] = 0.0;
      }
    }
  }
};

constexpr int kPer = kVerifyChunk / kWave;  // values of a lane in a chunk

template <typename T, bool DRAWN>
__device__ __forceinline__ Rest<T, DRAWN> rest_of(const VerifyArgs &a, int row, int k, const double *z, const int32_t *gone) {
  Rest<T, DRAWN> r;
  r.p = (const T *)a.target + (int64_t)row * a.target_stride;
  r.q = DRAWN ? (const T *)a.proposal + (int64_t)row * a.proposal_stride : nullptr;
  r.k = k;
  r.vocab = a.vocab;
  r.z = z;
  r.gone = gone;
  return r;
}

// Sum of a chunk, by a wave.
template <typename T, bool DRAWN>
__device__ __forceinline__ double chunk_sum(const Rest<T, DRAWN> &r, int chunk) {
  constexpr int V = 16 / sizeof(T);
  double sum = 0.0;
#pragma unroll
  for (int i = 0; i < kPer / V; ++i) {
    double w[V];
    r.load(chunk * kVerifyChunk + (i * kWave + (int)(threadIdx.x & 63)) * V, w);
#pragma unroll
    for (int j = 0; j < V; ++j) sum += w[j];
  }
  return wave_sum_f64(sum);
}

// One block per sequence, whose first wave walks: a row's token, parent and probabilities are fetched for all rows at once, a
// test is a few operations. Bound by latency, 3 us of which are these fetches. Only a second test of drawn siblings needs the
// sum over the vocabulary of what the first one left; the whole block makes it (200 trees of up to 10 rows, 50257 tokens:
// with 256 threads 60 us, with 1024 22).
template <typename T, bool DRAWN, int THREADS>
__global__ __launch_bounds__(THREADS) void verify_walk_kernel(const VerifyArgs a) {
  constexpr int M = ODS_DRAFT_MAX_ROWS, WAVES = THREADS / kWave;
  __shared__ int s_token[M], s_gone[M];
  __shared__ float s_p[M], s_q[M], s_u[M];
  __shared__ double s_z[M], s_sum[WAVES];
  __shared__ int s_cur, s_k, s_more;
  const int b = blockIdx.x, tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int first = a.row_off[b], last = a.row_off[b + 1];
  const int n = first < 0 || first >= a.rows || last <= first ? 0 : min(min(last, a.rows) - first, a.max_rows);
  int32_t *path = a.path + (int64_t)b * a.path_cols;
  if (n == 0) {
    if (tid == 0) {
      a.path_len[b] = 0;
      a.next_token[b] = -1;
      a.head[b].row = -1;
    }
    for (int i = tid; i < a.path_cols; i += THREADS) path[i] = -1;
    return;
  }
  int of[M / kWave];  // parents of rows lane, lane + 64, ...; -1: passed over
  if (wave == 0) {
#pragma unroll
    for (int i = 0; i < M / kWave; ++i) {
      const int j = i * kWave + lane;
      of[i] = -1;
      if (j == 0 || j >= n) continue;
      const int up = a.parent[first + j], x = a.tokens[first + j];
      if (up < 0 || up >= j || x < 0 || x >= a.vocab) continue;
      of[i] = up;
      s_token[j] = x;
      s_u[j] = a.accept_u[first + j];
      s_p[j] = prob((const T *)a.target + (int64_t)(first + up) * a.target_stride, x);
      if (DRAWN) s_q[j] = prob((const T *)a.proposal + (int64_t)(first + up) * a.proposal_stride, x);
    }
  }
  __syncthreads();
  // The walk, as far as it goes without a sum: every lane of the first wave takes every step.
  int cur = 0, len = 1, k = 0, at = 0;
  double z = 1.0;
  bool stale = false;  // z is not yet the sum of what is left
  if (tid == 0) path[0] = 0;
  for (;;) {
    if (wave == 0) {
      bool more = false;
      while (len < a.path_cols) {
        int j = M;  // the next child of cur behind `at`
#pragma unroll
        for (int i = M / kWave - 1; i >= 0; --i) {
          const uint64_t m = __ballot(of[i] == cur && i * kWave + lane > at);
          if (m) j = i * kWave + __builtin_ctzll(m);
        }
        if (j == M) break;
        if (DRAWN && stale) {
          more = true;
          break;
        }
        at = j;
        const int x = s_token[j];
        double w = s_p[j], least = z * (double)s_u[j];
        if (DRAWN) {
          for (int i = 0; i < k; ++i) w = fmax(w - s_z[i] * (double)s_q[j], 0.0);
          least *= (double)s_q[j];
        } else {
          for (int i = 0; i < k; ++i)
            if (s_gone[i] == x) w = 0.0;
        }
        if (w > 0.0 && least < w) {
          if (lane == 0) path[len] = j;
          cur = j;
          ++len;
          k = 0;
          z = 1.0;
          stale = false;
        } else if (DRAWN) {
          s_z[k++] = z;
          stale = true;
        } else {
          s_gone[k++] = x;
          z -= w;
        }
      }
      if (lane == 0) {
        s_cur = cur;
        s_k = k;
        s_more = more;
      }
    }
    __syncthreads();
    if (!DRAWN || !s_more) break;
    const auto r = rest_of<T, DRAWN>(a, first + s_cur, s_k, s_z, s_gone);
    double mine = 0.0;
#pragma unroll 2
    for (int e = tid * 8; e < a.vocab; e += THREADS * 8) {
      double w[8];
      r.load(e, w);
#pragma unroll
      for (int i = 0; i < 8; ++i) mine += w[i];
    }
    mine = wave_sum_f64(mine);
    if (lane == 0) s_sum[wave] = mine;
    __syncthreads();
    z = 0.0;
    for (int w = 0; w < WAVES; ++w) z += s_sum[w];
    stale = false;
  }
  if (wave == 0) {
    for (int i = len + lane; i < a.path_cols; i += kWave) path[i] = -1;
    if (lane == 0) {
      a.path_len[b] = len;
      a.head[b].row = first + cur;
      a.head[b].k = k;
    }
  }
  for (int i = tid; i < s_k; i += THREADS) {
    if (DRAWN) a.list[(int64_t)b * M + i] = s_z[i];
    else ((int32_t *)(a.list + (int64_t)b * M))[i] = s_gone[i];
  }
}

// Sums of chunks of what is left, a wave each. Bound by memory: every value is read once.
template <typename T, bool DRAWN>
__global__ __launch_bounds__(256) void verify_sums_kernel(const VerifyArgs a) {
  const int b = blockIdx.y, chunk = blockIdx.x * 4 + (threadIdx.x >> 6);
  const VerifyHead h = a.head[b];
  if (h.row < 0 || chunk >= a.chunks) return;
  const double *list = a.list + (int64_t)b * ODS_DRAFT_MAX_ROWS;
  const double sum = chunk_sum(rest_of<T, DRAWN>(a, h.row, h.k, list, (const int32_t *)list), chunk);
  if ((threadIdx.x & 63) == 0) a.sums[(int64_t)b * a.chunks + chunk] = sum;
}

// Inclusive sums over the lanes below.
__device__ __forceinline__ double wave_scan_f64(double v) {
#pragma unroll
  for (int o = 1; o < kWave; o <<= 1) {
    const double up = __shfl_up(v, o, kWave);
    if ((int)(threadIdx.x & 63) >= o) v += up;
  }
  return v;
}

// The first token whose running sum exceeds next_u of the whole, a wave per sequence: its chunk by the chunks' sums, then
// the chunk. Where the rounding of the two sums leaves none, the last token of some probability.
template <typename T, bool DRAWN>
__global__ __launch_bounds__(64) void verify_pick_kernel(const VerifyArgs a) {
  const int b = blockIdx.x, lane = threadIdx.x;
  VerifyHead h = a.head[b];
  if (h.row < 0) return;
  double *sums = a.sums + (int64_t)b * a.chunks;
  const int per = (a.chunks + kWave - 1) / kWave, c0 = min(lane * per, a.chunks), c1 = min(c0 + per, a.chunks);
  auto of_lane = [&]() {
    double s = 0.0;
    for (int c = c0; c < c1; ++c) s += sums[c];
    return s;
  };
  double mine = of_lane();
  if (!__any(mine > 0.0) && h.k > 0) {  // nothing is left: the target itself
    h.k = 0;
    const auto r = rest_of<T, DRAWN>(a, h.row, 0, nullptr, nullptr);
    for (int c = 0; c < a.chunks; ++c) {
      const double s = chunk_sum(r, c);
      if (lane == 0) sums[c] = s;
      if (c >= c0 && c < c1) mine += s;
    }
    __threadfence();  // the wave reads them below
  }
  const double upto = wave_scan_f64(mine), total = __shfl(upto, kWave - 1, kWave);
  if (!(total > 0.0)) {
    if (lane == 0) a.next_token[b] = -1;
    return;
  }
  const double aim = (double)a.next_u[b] * total;
  double run = upto - mine, before = 0.0;
  int found = -1, any = -1;  // this lane's first chunk past the aim, its last one of some probability
  for (int c = c0; c < c1; ++c) {
    const double s = sums[c];
    if (s > 0.0) any = c;
    if (found < 0 && s > 0.0 && run + s > aim) {
      found = c;
      before = run;
    }
    run += s;
  }
  const uint64_t hit = __ballot(found >= 0);
  int chunk;
  if (hit) {
    const int l = __builtin_ctzll(hit);
    chunk = __shfl(found, l, kWave);
    before = __shfl(before, l, kWave);
  } else {
    chunk = __shfl(any, 63 - __builtin_clzll(__ballot(any >= 0)), kWave);
    before = INFINITY;  // its last token
  }
  const double *list = a.list + (int64_t)b * ODS_DRAFT_MAX_ROWS;
  const auto r = rest_of<T, DRAWN>(a, h.row, h.k, list, (const int32_t *)list);
  const int e0 = chunk * kVerifyChunk + lane * kPer;
  double w[kPer], sum = 0.0;
  r.load(e0, w);
#pragma unroll
  for (int i = 0; i < kPer; ++i) sum += w[i];
  run = before + (wave_scan_f64(sum) - sum);
  int first = -1, last = -1;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    run += w[i];
    if (w[i] > 0.0) {
      last = e0 + i;
      if (first < 0 && run > aim && hit) first = e0 + i;
    }
  }
  const uint64_t ahead = __ballot(first >= 0), some = __ballot(last >= 0);
  int token = -1;
  if (ahead) token = __shfl(first, __builtin_ctzll(ahead), kWave);
  else if (some) token = __shfl(last, 63 - __builtin_clzll(some), kWave);
  if (lane == 0) a.next_token[b] = token;
}

template <typename T, bool DRAWN>
hipError_t go_verify(const VerifyArgs &a, hipStream_t s) {
  constexpr int WALK = DRAWN ? 1024 : 64;
  hipLaunchKernelGGL((verify_walk_kernel<T, DRAWN, WALK>), dim3(a.B), dim3(WALK), 0, s, a);
  hipLaunchKernelGGL((verify_sums_kernel<T, DRAWN>), dim3((a.chunks + 3) / 4, a.B), dim3(256), 0, s, a);
  hipLaunchKernelGGL((verify_pick_kernel<T, DRAWN>), dim3(a.B), dim3(64), 0, s, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_verify(int batch, const ods_draft &draft, const ods_verify &v, hipStream_t s) {
  const VerifyWs w = verify_ws(batch, v.vocab);
  VerifyArgs a{};
  a.B = batch; a.rows = draft.rows; a.max_rows = draft.max_rows; a.vocab = v.vocab; a.chunks = w.chunks;
  a.path_cols = v.path_cols;
  a.row_off = draft.row_off; a.tokens = v.tokens; a.parent = v.parent;
  a.accept_u = v.accept_u; a.next_u = v.next_u;
  a.target = v.target; a.proposal = v.proposal;
  a.target_stride = v.target_stride; a.proposal_stride = v.proposal_stride;
  a.path = v.path; a.path_len = v.path_len; a.next_token = v.next_token;
  a.head = (VerifyHead *)((uint8_t *)v.ws + w.head);
  a.list = (double *)((uint8_t *)v.ws + w.list);
  a.sums = (double *)((uint8_t *)v.ws + w.sums);
  if (v.dtype == ODS_PROBS_BF16) return v.proposal ? go_verify<uint16_t, true>(a, s) : go_verify<uint16_t, false>(a, s);
  return v.proposal ? go_verify<float, true>(a, s) : go_verify<float, false>(a, s);
}

}  // namespace ods
