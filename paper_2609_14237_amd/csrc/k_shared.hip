// Attention of drafted rows where groups of sequences share a prefix of the
// cache: one launch over the groups' prefixes (every K/V tile for all rows of a
// group) and what each sequence has beyond them, and one that joins the two.
#include "tree_attention.hpp"

namespace ods {

namespace {

// For a row whose sequence's group shares tokens [0, P): with (m, l, acc) the maximum, the denominator and the sums of a
// softmax over some tokens, o = sum_i 2^(m_i - M) acc_i / sum_i 2^(m_i - M) l_i over the pieces of its prefix task and of its
// tail task. Prefix tasks are bound by the matrix units (their columns are the rows of a whole group), tail tasks by memory
// (few columns a byte). Both are ranges of one grid, so that the two kinds share compute units: the ranges are split
// between them by their expected times, which every workgroup works out from the same metadata.
// LDS: five integers of a group, four of a sequence, three to end lists.
inline size_t shared_meta_bytes(int groups, int B) { return ((5 * (size_t)groups + 4 * (size_t)B + 4) * 4 + 15) / 16 * 16; }

template <int D, int NQP, int NQT, int QW, bool STREAM>
__global__ __launch_bounds__(64 * QW) __attribute__((amdgpu_waves_per_eu(2))) void shared_attention_kernel(
    const DraftArgs a, const int min_tiles, const int max_qt, const float tile_cost, const float scale_log2, const TreeOut prefix_out,
    const TreeOut tail_out) {
  constexpr int THREADS = 64 * QW, QTP = NQP * QW, QTT = NQT * QW, RS = QTP > QTT ? QTP : QTT;
  extern __shared__ __align__(16) int smem[];
  const int N = a.shared.n_groups, B = a.B, group = a.n_q / a.n_kv, tid = threadIdx.x;
  TreeSeqs p{}, t{};
  p.count = N;
  p.first = smem;             // [N + 1]: a group's first sequence, in this launch's numbers
  p.pre = p.first + N + 1;
  p.n = p.pre + N + 1;
  p.r0 = p.n + N;
  p.rows = p.r0 + N;
  t.count = B;
  t.pre = p.rows + N;
  t.first = t.pre + B + 1;
  t.n = t.first + B;
  t.key = t.n + B;
  uint8_t *const slots = (uint8_t *)smem + ((5 * N + 4 * B + 3) * 4 + 15) / 16 * 16;
  __shared__ int s_units[QW][2];

  // Groups, as far as their sequences are this launch's; the rows and tokens of the sequences.
  for (int g = tid; g <= N; g += THREADS) {
    const int s0 = min(max(a.shared.group_off[g] - a.base, 0), B);
    p.first[g] = s0;
    if (g == N) break;
    const int s1 = min(max(a.shared.group_off[g + 1] - a.base, s0), B);
    // Whole tiles, fewer tokens than the table holds, and none in a group of one.
    const int tokens = s1 - s0 < 2 ? 0 : max(0, min(a.shared.tokens[g], a.cols * kPage - 1)) / kTile;
    const int r0 = a.row_off[s0], e = a.row_off[s1];
    const int rows = r0 < 0 || r0 >= a.rows || e <= r0 ? 0 : min(e, a.rows) - r0;
    p.r0[g] = r0;
    p.rows[g] = rows;
    p.n[g] = rows > 0 ? tokens : 0;
    p.pre[g] = p.n[g] > 0 ? a.n_kv * ((rows * group + QTP - 1) / QTP) : 0;
  }
  for (int b = tid; b < B; b += THREADS) {
    const DraftSeq s = draft_seq(a.row_off, a.ctx_lens, b, a.rows, a.max_rows, a.cols, a.ring);
    t.pre[b] = s.n;
    t.first[b] = s.ctx;
    t.n[b] = s.end;
    t.key[b] = s.r0;
  }
  __syncthreads();
  int units[2] = {0, 0};
  for (int b = tid; b < B; b += THREADS) {
    const int rows = t.pre[b], ctx = t.first[b], end = t.n[b], r0 = t.key[b];
    int g = 0, hi = N;  // the last group that begins at b or before
    while (hi - g > 1) {
      const int mid = (g + hi) >> 1;
      if (p.first[mid] <= b) g = mid; else hi = mid;
    }
    // Its group's tiles cover a sequence that has them all cached, tokens of its own behind them, and its rows among theirs.
    const int first = p.n[g];
    const bool covered = first > 0 && b >= p.first[g] && b < p.first[g + 1] && ctx >= first * kTile && end > first * kTile &&
                         r0 >= p.r0[g] && r0 + rows <= p.r0[g] + p.rows[g];
    t.first[b] = covered ? first : 0;
    t.key[b] = covered ? p.r0[g] * group : -1;
    t.n[b] = end == 0 ? 0 : (end - 1) / kTile + 1 - t.first[b];
    t.pre[b] = end == 0 ? 0 : a.n_kv * ((rows * group + QTT - 1) / QTT);
    units[1] += t.n[b] * t.pre[b];
  }
  for (int g = tid; g < N; g += THREADS) units[0] += p.n[g] * p.pre[g];
  for (int i = 0; i < 2; ++i) {
    const int sum = wave_scan(units[i], [](int x, int y) { return x + y; });
    if ((tid & 63) == 63) s_units[tid >> 6][i] = sum;
  }
  __syncthreads();
  units[0] = units[1] = 0;
  for (int w = 0; w < QW; ++w)
    for (int i = 0; i < 2; ++i) units[i] += s_units[w][i];
  const int G = gridDim.x, r = blockIdx.x;
  const float cost = (float)units[0] * tile_cost, all = cost + (float)units[1];
  int of_prefix = units[0] == 0 ? 0 : max(1, min(G - 1, (int)((float)G * cost / all + 0.5f)));
  of_prefix = __builtin_amdgcn_readfirstlane(of_prefix);
  if (r < of_prefix)
    tree_work<D, NQP, QW, false, kPrefix, RS>(a, p, slots, r, of_prefix, r, min_tiles, 2, 0, 0, scale_log2, prefix_out);
  else
    tree_work<D, NQT, QW, STREAM, kTail, RS>(a, t, slots, r - of_prefix, G - of_prefix, r, min_tiles, max_qt, 1, 0, scale_log2, tail_out);
}

// One wave per column of a tail task: the pieces of its prefix task, then its own. Bound by latency where there are few
// columns (the descriptors, then all records at once), by memory where there are many. Also writes the zeros of sequences
// that are left alone.
template <int D>
__global__ __launch_bounds__(256) void shared_join_kernel(const DraftArgs a, const int qtp, const int qtt, const int stride, const int max_qt,
                                                          const TreeOut prefix_out, const TreeOut tail_out) {
  constexpr int LPR = D / 4, RPW = kWave / LPR, PRE = 4;  // lanes per record, records a wave reads at once, trips in flight
  const int lane = threadIdx.x & 63, at = blockIdx.y * 4 + (threadIdx.x >> 6);
  const int group = a.n_q / a.n_kv, task = blockIdx.x, qt = task % max_qt, b = task / max_qt / a.n_kv;
  const TreeDesc e = tail_out.desc[task];  // of a task without units: what an earlier call left
  if (task % (max_qt * a.n_kv) == 0 && blockIdx.y == 0) zero_left_alone(a, b, 256);
  const DraftSeq s = draft_seq(a.row_off, a.ctx_lens, b, a.rows, a.max_rows, a.cols, a.ring);
  const int col = qt * qtt + at;
  if (s.end == 0 || at >= qtt || col >= s.n * group || (e.pieces == 1 && e.key < 0)) return;
  const int row = s.r0 + col / group, head = e.head;
  const int64_t to = (int64_t)row * a.n_q + head * group + col % group;
  const int rel = e.key < 0 ? 0 : s.r0 * group + col - e.key, first = rel / qtp * qtp;
  const int2 p = e.key < 0 ? make_int2(0, 0) : prefix_out.prefix[(int64_t)head * a.rows * group + e.key + first];
  const int pieces = p.x + e.pieces;
  const int d = (lane % LPR) * 4, sub = lane / LPR;
  float M = kNoScore, sum = 0.f;
  f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int i0 = 0; i0 < pieces; i0 += PRE * RPW) {
    f32x4 x[PRE];
    float2 ml[PRE];
#pragma unroll
    for (int k = 0; k < PRE; ++k) {
      const int i = min(i0 + sub + k * RPW, pieces - 1);  // past the last: again, with weight 0
      const bool shared = i < p.x;
      const TreeOut &from = shared ? prefix_out : tail_out;
      const int n = shared ? p.x : e.pieces, j = shared ? i : i - p.x, rec = shared ? p.y : e.rec;
      // whole tasks left a state of the row and head; pieces a record in each of their ranges
      const int64_t idx = n == 1 ? to : (int64_t)(j == 0 ? rec : (rec & ~1) + 2 * j) * stride + (shared ? rel - first : at);
      ml[k] = (n == 1 ? from.state_ml : from.rec_ml)[idx];
      x[k] = *(const f32x4 *)((n == 1 ? from.state_acc : from.rec_acc) + idx * D + d);
    }
    float top = M;
#pragma unroll
    for (int k = 0; k < PRE; ++k) top = fmaxf(top, ml[k].x);
    const float old = __builtin_amdgcn_exp2f(M - top);
    M = top;
    sum *= old;
    acc *= old;
#pragma unroll
    for (int k = 0; k < PRE; ++k) {
      const float w = i0 + sub + k * RPW < pieces ? __builtin_amdgcn_exp2f(ml[k].x - top) : 0.f;
      sum += w * ml[k].y;
      if (w != 0.f) acc += w * x[k];
    }
  }
  float top = M;
#pragma unroll
  for (int o = LPR; o < kWave; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, kWave));
  const float w = __builtin_amdgcn_exp2f(M - top);
  float l = sum * w;
  f32x4 v = acc * w;
#pragma unroll
  for (int o = LPR; o < kWave; o <<= 1) {
    l += __shfl_xor(l, o, kWave);
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] += __shfl_xor(v[i], o, kWave);
  }
  if (lane >= LPR) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  u32x2 out;
  out[0] = pack_pair(v[0] * inv, v[1] * inv);
  out[1] = pack_pair(v[2] * inv, v[3] * inv);
  *(u32x2 *)(a.o + to * D + d) = out;
}

template <int D, int NQP, int NQT, int QW, bool STREAM>
hipError_t go_shared(DraftArgs a, const SharedPlan &plan, void *ws, hipStream_t s) {
  using Shape = TreeShape<D, NQP, QW>;
  static std::atomic<uint64_t> lds_set{0};  // devices whose LDS limit is raised
  const size_t tiles = (size_t)Shape::kSlots * Shape::kTileBytes;
  const auto kern = shared_attention_kernel<D, NQP, NQT, QW, STREAM>;
  const int most = QW == 8 ? kSharedSmall : kSharedBatch;
  const size_t limit = tiles + shared_meta_bytes(QW == 8 ? kSharedSmall : ODS_SHARED_GROUPS, most);
  if (hipError_t e = ensure_lds_limit((const void *)kern, limit, lds_set); e != hipSuccess) return e;
  static_assert(sizeof(TreeDesc) <= kTreeDescBytes, "descriptor size");
  const int N = a.shared.n_groups;
  const SharedWs w = shared_ws(plan, a.batch, a.rows, a.n_q, a.n_kv, D);
  auto at = [&](size_t offset) { return (uint8_t *)ws + offset; };
  TreeOut prefix{}, tail{};
  prefix.rec_acc = tail.rec_acc = (float *)at(w.rec_acc);
  prefix.rec_ml = tail.rec_ml = (float2 *)at(w.rec_ml);
  prefix.state_acc = (float *)at(w.state[0]);
  tail.state_acc = (float *)at(w.state[1]);
  prefix.state_ml = (float2 *)at(w.state_ml[0]);
  tail.state_ml = (float2 *)at(w.state_ml[1]);
  prefix.prefix = (int2 *)at(w.prefix);
  tail.desc = (TreeDesc *)at(w.desc);
  const float scale = (float)(1.4426950408889634 / sqrt((double)D));
  const int B = a.B, stride = plan.qtp > plan.qtt ? plan.qtp : plan.qtt;
  const int columns = a.max_rows * (a.n_q / a.n_kv) < plan.qtt ? a.max_rows * (a.n_q / a.n_kv) : plan.qtt;
  for (int b0 = 0; b0 < B; b0 += most) {  // a group on both sides of a border is two, each of which reads the prefix
    a.B = B - b0 < most ? B - b0 : most;
    a.base = b0;
    hipLaunchKernelGGL(kern, dim3(plan.grid), dim3(64 * QW), tiles + shared_meta_bytes(N, a.B), s, a, plan.min_tiles, plan.max_qt,
                       plan.tile_cost, scale, prefix, tail);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL(shared_join_kernel<D>, dim3(a.B * a.n_kv * plan.max_qt, (columns + 3) / 4), dim3(256), 0, s, a, plan.qtp, plan.qtt,
                       stride, plan.max_qt, prefix, tail);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    a.row_off += a.B;
    a.ctx_lens += a.B;
    a.table += (int64_t)a.B * a.cols;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_shared_attention(const DraftArgs &a, const SharedPlan &plan, void *ws, hipStream_t s) {
  auto of = [&](auto d, auto stream) {
    constexpr int D = decltype(d)::value;
    constexpr bool STREAM = decltype(stream)::value;
    if (plan.waves == 8)
      return plan.qtt == 256 ? go_shared<D, 32, 32, 8, STREAM>(a, plan, ws, s) : go_shared<D, 32, 16, 8, STREAM>(a, plan, ws, s);
    if (plan.qtt == 128) return go_shared<D, 32, 32, 4, STREAM>(a, plan, ws, s);
    return plan.qtp == 128 ? go_shared<D, 32, 16, 4, STREAM>(a, plan, ws, s) : go_shared<D, 16, 16, 4, STREAM>(a, plan, ws, s);
  };
  using D64 = std::integral_constant<int, 64>;
  using D128 = std::integral_constant<int, 128>;
  if (plan.stream) return a.D == 128 ? of(D128(), std::true_type()) : of(D64(), std::true_type());
  return a.D == 128 ? of(D128(), std::false_type()) : of(D64(), std::false_type());
}

}  // namespace ods
