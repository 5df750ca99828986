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
// LDS: six integers of a group, four of a sequence, three to end lists.
inline size_t shared_meta_bytes(int groups, int B) { return ((6 * (size_t)groups + 4 * (size_t)B + 3) * 4 + 15) / 16 * 16; }

// A workgroup has KW waves. Prefix ranges are one workgroup's work; tail ranges of up to 32 columns (WT: waves of a range)
// are one wave's each: with few columns a tile is a chain of latencies, and such chains side by side reach the memory's rate.
template <int D, int NQP, int NQT, int WT, int KW>
__global__ __launch_bounds__(64 * KW) __attribute__((amdgpu_waves_per_eu(2))) void shared_attention_kernel(
    const DraftArgs a, const SharedCost cost, const float scale_log2, const TreeOut prefix_out, const TreeOut tail_out) {
  constexpr int THREADS = 64 * KW, QTP = NQP * KW, QTT = NQT * WT, RPB = KW / WT;  // RPB: tail ranges of a workgroup
  constexpr int TILE = TreeShape<D, NQP, KW>::kTileBytes, NS = TreeShape<D, NQP, KW>::kSlots;
  extern __shared__ __align__(16) int smem[];
  const int N = a.shared.n_groups, B = a.B, group = a.n_q / a.n_kv, tid = threadIdx.x;
  TreeSeqs p{}, t{};
  p.count = N;
  int *const bound = smem;    // [N + 1]: a group's first sequence, in this launch's numbers
  p.first = bound + N + 1;    // the sequence by whose table its prefix is read
  p.pre = p.first + N;
  p.n = p.pre + N + 1;
  p.r0 = p.n + N;
  p.rows = p.r0 + N;
  t.count = B;
  t.pre = p.rows + N;
  t.first = t.pre + B + 1;
  t.n = t.first + B;
  t.key = t.n + B;
  uint8_t *const slots = (uint8_t *)smem + ((6 * N + 4 * B + 3) * 4 + 15) / 16 * 16;
  __shared__ int s_sums[KW][4];
  __shared__ float s_units[KW];

  // Groups, as far as their sequences are this launch's; the rows and tokens of the sequences.
  // Whatever the arrays hold, the tasks counted are those of disjoint groups of disjoint rows: where offsets of groups or of
  // rows descend, nothing is shared.
  auto here = [&](int off) { return (int)min(max((int64_t)off - a.base, (int64_t)0), (int64_t)B); };
  bool descends = false;
  float tiles = 0.f;
  for (int g = tid; g <= N; g += THREADS) {
    const int s0 = here(a.shared.group_off[g]);
    bound[g] = s0;
    if (g == N) break;
    p.first[g] = B;
    descends = descends || a.shared.group_off[g] > a.shared.group_off[g + 1];
    const int s1 = max(here(a.shared.group_off[g + 1]), s0);
    // Whole tiles, fewer tokens than the table holds, and none in a group of one.
    const int tokens = s1 - s0 < 2 ? 0 : max(0, min(a.shared.tokens[g], a.cols * kPage - 1)) / kTile;
    const int r0 = a.row_off[s0], e = a.row_off[s1];
    const int rows = r0 < 0 || r0 >= a.rows || e <= r0 ? 0 : min(e, a.rows) - r0;
    p.r0[g] = r0;
    p.rows[g] = rows;
    p.n[g] = rows > 0 ? tokens : 0;
    p.pre[g] = p.n[g] > 0 ? a.n_kv * ((rows * group + QTP - 1) / QTP) : 0;
    tiles += (float)p.n[g] * (float)p.pre[g];
  }
  tiles = wave_sum(tiles);
  if ((tid & 63) == 0) s_units[tid >> 6] = tiles;
  for (int b = tid; b < B; b += THREADS) {
    const DraftSeq s = draft_seq(a.row_off, a.ctx_lens, b, a.rows, a.max_rows, a.cols, a.ring);
    t.pre[b] = s.n;
    t.first[b] = s.ctx;
    t.n[b] = s.end;
    t.key[b] = s.r0;
    descends = descends || a.row_off[b] > a.row_off[b + 1];
  }
  const bool none = __syncthreads_or(descends);
  tiles = 0.f;
  for (int w = 0; w < KW; ++w) tiles += s_units[w];
  if (none || tiles > 1.07e9f) {  // 2^30
    for (int g = tid; g < N; g += THREADS) p.n[g] = p.pre[g] = 0;
    __syncthreads();
  }
  int sums[4] = {0, 0, 0, 0};  // units and tasks of prefixes, of tails
  for (int b = tid; b < B; b += THREADS) {
    const int rows = t.pre[b], ctx = t.first[b], end = t.n[b], r0 = t.key[b];
    int g = 0, hi = N;  // the last group that begins at b or before
    while (hi - g > 1) {
      const int mid = (g + hi) >> 1;
      if (bound[mid] <= b) g = mid; else hi = mid;
    }
    // Its group's tiles cover a sequence that has them all cached, tokens of its own behind them, and its rows among theirs.
    // They are read by the table of the first such one: others (left alone, released, shorter) may name no pages there.
    const int first = p.n[g];
    const bool covered = first > 0 && b >= bound[g] && b < bound[g + 1] && ctx >= first * kTile && end > first * kTile &&
                         r0 >= p.r0[g] && r0 + rows <= p.r0[g] + p.rows[g];
    if (covered) atomicMin(&p.first[g], b);
    t.first[b] = covered ? first : 0;
    t.key[b] = covered ? p.r0[g] * group : -1;
    t.n[b] = end == 0 ? 0 : (end - 1) / kTile + 1 - t.first[b];
    t.pre[b] = end == 0 ? 0 : a.n_kv;
    sums[2] += t.n[b] * t.pre[b];
    sums[3] += t.pre[b];
  }
  __syncthreads();
  for (int g = tid; g < N; g += THREADS) {
    if (p.first[g] == B) p.n[g] = p.pre[g] = 0;  // covers none
    sums[0] += p.n[g] * p.pre[g];
    sums[1] += p.pre[g];
  }
  for (int i = 0; i < 4; ++i) {
    const int sum = wave_scan(sums[i], [](int x, int y) { return x + y; });
    if ((tid & 63) == 63) s_sums[tid >> 6][i] = sum;
  }
  __syncthreads();
  for (int i = 0; i < 4; ++i) {
    sums[i] = 0;
    for (int w = 0; w < KW; ++w) sums[i] += s_sums[w][i];
  }
  const int G = gridDim.x, r = blockIdx.x;
  for (int b = r; b < B; b += G) {  // what no range writes: zeros of sequences left alone, tasks that are none
    zero_left_alone(a, b, THREADS);
    if (t.n[b] != 0) continue;
    for (int i = tid; i < a.n_kv; i += THREADS) tail_out.desc[(int64_t)b * a.n_kv + i].pieces = 0;
  }
  const float of_p = (float)sums[0] * cost.prefix_tile + (float)sums[1] * cost.prefix_task;
  const float of_t = (float)sums[2] * cost.tail_tile + (float)sums[3] * cost.tail_task;
  int split = sums[0] == 0 ? 0 : max(1, min(G - 1, (int)((float)G * of_p / (of_p + of_t) + 0.5f)));
  split = __builtin_amdgcn_readfirstlane(split);
  if (r < split) {
    tree_work<D, NQP, KW, NS, false, kPrefix, 1>(a, p, slots, r, split, cost.prefix_least, cost.prefix_slack, 2, 0, 0, scale_log2, prefix_out);
  } else {
    constexpr int NT = NS / RPB > 0 ? NS / RPB : 1;
    static_assert(NT * RPB * TILE <= NS * TILE, "tiles of the tail ranges");
    const int of_wave = RPB > 1 ? __builtin_amdgcn_readfirstlane(tid >> 6) : 0;
    // Tails that are more than the last-level cache holds (256 MB) go past the caches, where prefixes are to stay.
    const bool past = (float)sums[2] * (float)TILE > 256e6f;
    tree_work<D, NQT, WT, NT, false, kTail, RPB>(a, t, slots, (r - split) * RPB + of_wave, (G - split) * RPB, cost.tail_least, cost.tail_slack, 1, 1, 0,
                                                  scale_log2, tail_out, past);
  }
}

// JOIN waves per column of a tail task, which take turns at the pieces of its prefix task and then its own. Bound by latency
// where there are few columns (the two descriptors, then all records at once), by memory where there are many.
template <int D, int JOIN>
__global__ __launch_bounds__(256) void shared_join_kernel(const DraftArgs a, const int qtp, const int qtt, const int ranges, const TreeOut prefix_out,
                                                          const TreeOut tail_out) {
  constexpr int LPR = D / 4, RPW = kWave / LPR, PRE = 4;  // lanes per record, records a wave reads at once, trips in flight
  __shared__ float s_m[4], s_l[4];
  __shared__ f32x4 s_v[4][LPR];
  const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part = wave % JOIN;
  const int at = blockIdx.y * (4 / JOIN) + wave / JOIN;
  const int group = a.n_q / a.n_kv;
  const TreeDesc e = tail_out.desc[blockIdx.x];
  const int col = e.col0 + at;
  const bool live = !(e.pieces == 0 || at >= qtt || col >= e.cols || (e.pieces == 1 && e.key < 0));
  const int row = e.r0 + col / group, head = e.head;
  const int64_t to = (int64_t)row * a.n_q + head * group + col % group;
  const int rel = e.key < 0 ? 0 : e.r0 * group + col - e.key, first = rel / qtp * qtp;
  const int2 p = !live || e.key < 0 ? make_int2(0, 0) : prefix_out.prefix[(int64_t)head * a.rows * group + e.key + first];
  // Records of the launch, whatever was left where a group's rows are not ascending.
  const bool none = !live || p.x < 0 || p.y < 0 || (int64_t)(p.y | 1) + 2 * ((int64_t)p.x - 1) >= 2 * ranges;
  if (JOIN == 1 && none) return;
  const int pieces = none ? 0 : p.x + e.pieces;
  const int d = (lane % LPR) * 4, sub = lane / LPR;
  float M = kNoScore, sum = 0.f;
  f32x4 acc = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int i0 = part * PRE * RPW; i0 < pieces; i0 += JOIN * PRE * RPW) {
    f32x4 x[PRE];
    float2 ml[PRE];
#pragma unroll
    for (int k = 0; k < PRE; ++k) {
      const int i = min(i0 + sub + k * RPW, pieces - 1);  // past the last: again, with weight 0
      const bool shared = i < p.x;
      const TreeOut &from = shared ? prefix_out : tail_out;
      const int n = shared ? p.x : e.pieces, j = shared ? i : i - p.x, rec = shared ? p.y : e.rec;
      // whole tasks left a state of the row and head; pieces a record in each of their ranges
      const int64_t idx = n == 1 ? to : (int64_t)(j == 0 ? rec : (rec & ~1) + 2 * j) * (shared ? qtp : qtt) + (shared ? rel - first : at);
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
  if (JOIN > 1) {
    if (lane == 0) s_m[wave] = top, s_l[wave] = l;
    if (lane < LPR) s_v[wave][lane] = v;
    __syncthreads();
    if (part > 0) return;
#pragma unroll
    for (int i = 1; i < JOIN; ++i) {
      const float other = s_m[wave + i], both = fmaxf(top, other);
      const float x = __builtin_amdgcn_exp2f(top - both), y = __builtin_amdgcn_exp2f(other - both);
      l = l * x + s_l[wave + i] * y;
      v = v * x + s_v[wave + i][lane % LPR] * y;
      top = both;
    }
  }
  if ((JOIN > 1 && none) || lane >= LPR) return;
  const float inv = l == 0.f ? 0.f : 1.f / l;
  u32x2 out;
  out[0] = pack_pair(v[0] * inv, v[1] * inv);
  out[1] = pack_pair(v[2] * inv, v[3] * inv);
  *(u32x2 *)(a.o + to * D + d) = out;
}

template <int D, int NQP, int NQT, int WT, int KW>
hipError_t go_shared(DraftArgs a, const SharedPlan &plan, void *ws, hipStream_t s) {
  using Shape = TreeShape<D, NQP, KW>;
  static std::atomic<uint64_t> lds_set{0};  // devices whose LDS limit is raised
  if (plan.waves != KW || plan.qtp != NQP * KW || plan.qtt != NQT * WT) return hipErrorInvalidValue;  // what the workspace is cut for
  if (a.max_rows * (a.n_q / a.n_kv) > NQT * WT || a.max_rows > 32) return hipErrorInvalidValue;  // one query tile, masks of 32 bits
  const size_t tiles = (size_t)Shape::kSlots * Shape::kTileBytes;
  const auto kern = shared_attention_kernel<D, NQP, NQT, WT, KW>;
  if (hipError_t e = ensure_lds_limit((const void *)kern, tiles + shared_meta_bytes(ODS_SHARED_GROUPS, kSharedBatch), lds_set); e != hipSuccess)
    return e;
  static_assert(sizeof(TreeDesc) <= kTreeDescBytes, "descriptor size");
  const SharedWs w = shared_ws(plan, a.batch, a.rows, a.n_q, a.n_kv, D);
  TreeOut out[2] = {};  // prefix, tail
  for (int i = 0; i < 2; ++i) {
    auto at = [&](size_t offset) { return (uint8_t *)ws + offset; };
    out[i].rec_acc = (float *)at(w.rec_acc[i]);
    out[i].rec_ml = (float2 *)at(w.rec_ml[i]);
    out[i].state_acc = (float *)at(w.state[i]);
    out[i].state_ml = (float2 *)at(w.state_ml[i]);
    out[i].prefix = (int2 *)at(w.prefix);
    out[i].desc = (TreeDesc *)at(w.desc);
  }
  const float scale = (float)(1.4426950408889634 / sqrt((double)D));
  const int B = a.B, most = a.max_rows * (a.n_q / a.n_kv), columns = most < plan.qtt ? most : plan.qtt;
  // Four waves a column where one each is fewer than the chip runs at once (64 tokens over 8192, 2048 columns: 45.2 us with one,
  // 43.9; 4 over 32768: 49.5, 40.2), one where they are more than enough (4096 columns: 56, 58; seven groups: 107, 119).
  const int waves = (int64_t)a.rows * a.n_q <= 2048 ? 4 : 1;
  const auto join = waves == 4 ? shared_join_kernel<D, 4> : shared_join_kernel<D, 1>;
  for (int b0 = 0; b0 < B; b0 += kSharedBatch) {  // a group on both sides of a border is two, each of which reads the prefix
    a.B = B - b0 < kSharedBatch ? B - b0 : kSharedBatch;
    a.base = b0;
    hipLaunchKernelGGL(kern, dim3(plan.grid), dim3(64 * KW), tiles + shared_meta_bytes(a.shared.n_groups, a.B), s, a, plan.cost,
                       scale, out[0], out[1]);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    hipLaunchKernelGGL(join, dim3(a.B * a.n_kv, (columns * waves + 3) / 4), dim3(256), 0, s, a, plan.qtp, plan.qtt, plan.grid, out[0],
                       out[1]);
    if (hipError_t e = hipGetLastError(); e != hipSuccess) return e;
    a.row_off += a.B;
    a.ctx_lens += a.B;
    a.table += (int64_t)a.B * a.cols;
  }
  return hipSuccess;
}

}  // namespace

hipError_t launch_shared_attention(const DraftArgs &a, const SharedPlan &plan, void *ws, hipStream_t s) {
  auto of = [&](auto d) {
    constexpr int D = decltype(d)::value;
    if (plan.waves == 8) switch (plan.qtt) {
        case 16: return go_shared<D, 32, 16, 1, 8>(a, plan, ws, s);
        case 32: return go_shared<D, 32, 32, 1, 8>(a, plan, ws, s);
      }
    else switch (plan.qtt) {
        case 16: return go_shared<D, 32, 16, 1, 4>(a, plan, ws, s);
        case 64: return go_shared<D, 32, 16, 4, 4>(a, plan, ws, s);
      }
    return hipErrorInvalidValue;
  };
  return a.D == 128 ? of(std::integral_constant<int, 128>()) : of(std::integral_constant<int, 64>());
}

}  // namespace ods
