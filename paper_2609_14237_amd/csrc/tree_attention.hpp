// Attention of drafted rows over the paged cache: the kernels of k_tree.hip
// (every sequence by itself) and k_shared.hip (prefixes that several sequences
// share, and what each has beyond them).
#pragma once
#include <math.h>

#include <type_traits>

#include "draft.hpp"
#include "kernels.hpp"

namespace ods {

namespace {

// o = softmax(q k^T / sqrt(D)) v of each drafted row over the cached tokens in
// its window and the drafted tokens of its mask. The query vectors of a
// sequence that share a KV head (its drafted rows times the query heads of the
// group) are columns of one problem, and up to QT of them (a query tile) share
// every K/V byte read. Bound by memory up to about 128 columns (64 sequences of
// 9216 tokens, 4 rows of 32 heads on 8: 362 us, 6.9 TB/s; 16 rows 366), by the
// matrix and vector units past that (64 sequences of 8192, 64 rows: 620 us, 0.89
// PFLOP/s, the matrix cores busy for 45% of the cycles and the vector unit for 41%;
// more rows take as many passes over K and V of that kind: 256 rows 2640 us), by
// latency where there is little to read (one sequence of 3000, 16
// rows: 17 us).
//
// Work split: a task is a (sequence, KV head, query tile), its units are tiles of
// 32 tokens. Every workgroup gets a range of units, in one of three ways, which
// each works out from the same metadata:
//   - one whole task, where there are no more tasks than workgroups and the
//     longest is not much longer than an even share;
//   - up to four whole tasks, dealt out by length (longest first, every second
//     round backwards), where the longest range that gives is not much longer;
//   - else the units are numbered in order and cut into equal ranges, which may
//     end inside a task. Such a task leaves a record (sums, running maximum,
//     running denominator) per range, and a second kernel joins them.
// What records cost (written, read, one more change of tasks) is kSplitTiles
// units' time. Through the caches: 32 sequences of 3600 to 4096 tokens, 24 rows,
// 8 heads: whole 110 us, cut 126; of 2048 to 4096 (32 tiles more than even) 111
// and 112; 64 ragged sequences of 512 to 4096: dealt 140 us, cut 157 (past the
// caches, as such a batch now is, dealt 129).
//
// A workgroup is QW waves over one stream of tiles. The tiles (keys and values
// of two pages) are fetched direct-to-LDS, up to seven ahead; each wave holds NQ
// of the tile's QT = QW * NQ columns in registers and reads every tile once:
//   S = K Q^T      16x16x32, twice: 16 tokens by 16 query vectors. Row 4 r + i of
//                  product h is token 8 r + 4 h + i of the tile, so lane quad r
//                  ends with the eight scores of tokens 8 r .. 8 r + 7;
//   softmax        a lane's eight scores of its column. The reference point m is
//                  moved only when a score exceeds it by 2^8: a probability then
//                  is at most 2^8 instead of 1, which no fp32 sum or bf16
//                  rounding feels, and the maximum across lanes and the rescale
//                  of the sums are skipped for most tiles;
//   O += V^T P     16x16x32 over both pages: the k index of lane quad r is tokens
//                  8 r .. 8 r + 7, which is how S leaves P in registers, and one
//                  16-byte read of a dim's slots in the dim-major V, so P never
//                  moves.
// P is rounded to bf16 for the product: the matrix cores multiply equal types, and
// the values are bf16. A probability is off by 2^-8 of itself at most, an output by
// 2^-8 of sum p |v| / sum p: no more than its own rounding to bf16 where the values
// have one sign (over normal values the outputs are 0.0023 off the 64-bit ones in
// the mean square, 0.0017 with fp32 probabilities). P in two bf16 halves would
// double the products of V. Its sum, the maximum and the outputs before their
// store are fp32.
//
// Tiles with a drafted token, a window edge, the end of the sequence or a page
// outside the pool are masked score by score. In these a value that is not
// finite is taken out of the product (0 * NaN would reach rows that may not
// see it) and added only to the columns that see it.

// Parts: a sequence is one problem (kWhole), or two where its group shares a prefix. kPrefix: a "sequence" is a group, its
// columns are those of all the group's drafted rows, its tokens the shared ones, none of them masked. kTail: a sequence's
// tokens behind those its group shares. What either computes of a row and query head is joined by shared_join_kernel.
enum TreePart { kWhole, kPrefix, kTail };

typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef __bf16 bf16x2 __attribute__((ext_vector_type(2)));
__device__ __forceinline__ uint32_t pack_pair(float lo, float hi) {  // one conversion for both
  return __builtin_bit_cast(uint32_t, __builtin_convertvector((f32x2{lo, hi}), bf16x2));
}

constexpr int kTile = 32;   // tokens per tile: two pages
constexpr float kSlack = 8.f;
constexpr float kNoScore = -1.7e38f;  // reference point before the first score: any score moves it, and 2^(kNoScore - m) is 0

// Tiles of a sequence: [first, first + n). n = 0: nothing to do; the window of
// a context past the page table may hold no token, one masked tile then.
__device__ __forceinline__ void tiles_of(const DraftSeq &s, int window, int &first, int &n) {
  first = n = 0;
  if (s.end == 0) return;
  const int last = (s.end - 1) / kTile;
  if (window > 0) first = min(max(0, s.ctx - window + 1) / kTile, last);
  n = last - first + 1;
}

__device__ __forceinline__ uint32_t bits_between(int lo, int hi) {  // bits [lo, hi) of 32
  lo = max(lo, 0);
  hi = min(hi, 32);
  if (lo >= hi) return 0u;
  return (hi == 32 ? 0xffffffffu : (1u << hi) - 1u) & ~((1u << lo) - 1u);
}

// Bits [j0, j0 + 32) of a row's mask (zeros before and after it).
__device__ __forceinline__ uint32_t mask_window(const uint64_t *__restrict__ m, int words, int j0) {
  if (j0 <= -32 || j0 >= words * 64) return 0u;
  if (j0 < 0) return (uint32_t)(m[0] << -j0);
  const int w = j0 / 64, sh = j0 % 64;
  uint64_t v = m[w] >> sh;
  if (sh > 32 && w + 1 < words) v |= m[w + 1] << (64 - sh);
  return (uint32_t)v;
}

// op of this lane's value and those of the lanes below it; op(x, 0) is x.
template <typename Op>
__device__ __forceinline__ int wave_scan(int x, Op op) {
  // within rows of sixteen lanes, then from row to row; a lane without a source takes 0
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x111, 0xf, 0xf, false));
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x112, 0xf, 0xf, false));
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x114, 0xf, 0xf, false));
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x118, 0xf, 0xf, false));
  x = op(x, __builtin_amdgcn_update_dpp(0, x, 0x142, 0xa, 0xf, false));
  return op(x, __builtin_amdgcn_update_dpp(0, x, 0x143, 0xc, 0xf, false));
}

// The two bf16 halves of a dword as weights of what is not finite: 1 for +inf, 64 for -inf, 4096 for NaN, else 0. one: 1 in
// bf16, of which 64 and 4096 are other exponents.
__device__ __forceinline__ uint32_t nonfinite_weight(uint32_t w, uint32_t one) {
  auto of = [=](uint32_t h) {
    return (h & 0x7f80u) != 0x7f80u ? 0u : (h & 0x7fu) ? one + 0x600u : (h & 0x8000u) ? one + 0x300u : one;
  };
  return of(w & 0xffffu) | of(w >> 16) << 16;
}

// Non-finite bf16 halves of a dword are cleared.
__device__ __forceinline__ void drop_nonfinite(uint32_t &w) {
  if ((w & 0x7f80u) == 0x7f80u) w &= 0xffff0000u;
  if ((w & 0x7f800000u) == 0x7f800000u) w &= 0x0000ffffu;
}

// A task that begins in a range and ends in a later one.
struct TreeDesc {
  int pieces;      // ranges it lies in (0: none such)
  int rec;         // record of its first piece; piece i's is slot 0 of range i further on
  int r0;          // first drafted row of its sequence
  int col0, cols;  // first column of its query tile, columns of the sequence
  int head;        // KV head
  int key;         // kTail: first column of its group's rows (of all drafted rows), -1: its group shares nothing
};

// What a workgroup knows of its sequences, in LDS.
struct TreeSeqs {
  int count;
  int *pre;          // [count + 1] units before (of whole tasks: tasks before)
  int *first, *n;    // first tile (kPrefix: the sequence whose table counts), tiles
  int *r0, *rows;    // kPrefix: rows of the group
  int *key;          // kTail: as TreeDesc::key
};

// Where results that are joined go.
struct TreeOut {
  float *rec_acc;    // records: sums [..][stride][D], maximum and denominator [..][stride]
  float2 *rec_ml;
  TreeDesc *desc;    // of each range, or of each task of the batch
  float *state_acc;  // of tasks in one piece: sums [rows * n_q][D], maximum and denominator [rows * n_q]
  float2 *state_ml;
  int2 *prefix;      // kPrefix: (pieces, record) of a query tile, at [head][its first column of all drafted rows]
};

// Outputs of a sequence that is left alone; `threads` of them.
__device__ __forceinline__ void zero_left_alone(const DraftArgs &a, int b, int threads) {
  if (a.ctx_lens[b] >= 0) return;
  const DraftSeq s = draft_seq(a.row_off, a.ctx_lens, b, a.rows, a.max_rows, a.cols, a.ring);
  const int64_t n = (int64_t)s.n * a.n_q * a.D / 8;
  u32x4 *dst = (u32x4 *)(a.o + (int64_t)s.r0 * a.n_q * a.D);
  for (int64_t i = threadIdx.x; i < n; i += threads) dst[i] = u32x4{0u, 0u, 0u, 0u};
}

template <int D, int NQ, int QW>
struct TreeShape {
  static constexpr int QT = NQ * QW;
  static constexpr int kTileBytes = kTile * D * 2 * 2;
  // Tiles in LDS: 128 KB of them, or 64 or 32 for each of the smaller workgroups that share a compute unit.
  static constexpr int kSlots = QW == 1 ? 2 : QW <= 4 ? 4 : 8;
  static constexpr int kChunks = kTileBytes / 1024;   // 1 KB direct-to-LDS loads of a tile
  static constexpr int kPerWave = kChunks / QW;
};

// Range r of G of a launch's tasks, by QW waves. The sequences of kPrefix and kTail are known already, seqs.pre holding the
// tasks of each. Ranges are whole tasks where the longest is at most `slack` tiles more than an even share. WPB > 1: a
// workgroup is that many waves of one range each (QW is 1), with tiles of their own. K and V go past the caches with STREAM
// (kTail: with `past`).
template <int D, int NQ, int QW, int NS, bool STREAM, TreePart PART, int WPB>
__device__ __forceinline__ void tree_work(const DraftArgs &a, const TreeSeqs &seqs, uint8_t *const all_slots, const int r, const int G,
                                          const int min_tiles, const int slack, const int max_qt, const int by_task, const int no_cut,
                                          const float scale_log2, const TreeOut &out, const bool past = false) {
  static_assert(WPB == 1 || QW == 1, "waves of a range, or ranges of a wave");
  using Shape = TreeShape<D, NQ, QW>;
  constexpr int KK = D / 32, NB = D / 16, CB = NQ / 16, QT = Shape::QT;
  constexpr int LPT = Shape::kPerWave, THREADS = 64 * QW * WPB;
  constexpr bool EARLY = PART == kTail && QW == 1;  // a tile's slot is filled again as soon as the tile is in registers
  constexpr int PB = kPage * D * 2;  // bytes of one page block of a head
  constexpr int DEAL = PART == kWhole && NQ == 16 ? 4 : 1;  // most whole tasks of a range; wider waves have no registers left for a list
  const int B = seqs.count, group = a.n_q / a.n_kv;
  int *const s_pre = seqs.pre, *const s_first = seqs.first, *const s_n = seqs.n;
  const int window = PART == kWhole ? a.window : 0, ring = PART == kWhole ? a.ring : 0;  // groups are of full attention
  TreeDesc *const desc = out.desc;
  __shared__ int s_tot[QW * WPB][3], s_ids[THREADS], s_ord[DEAL > 1 ? THREADS : 1], s_lists[WPB][DEAL][4], s_most;

  const int tid = threadIdx.x, lane = tid & 63;
  const int of_block = __builtin_amdgcn_readfirstlane(tid >> 6), wave = WPB > 1 ? 0 : of_block;
  const int at_list = WPB > 1 ? lane : tid;  // among the threads of the range
  const bool lead = at_list == 0;
  uint8_t *const slots = all_slots + (WPB > 1 ? of_block * NS * Shape::kTileBytes : 0);
  auto &s_list = s_lists[WPB > 1 ? of_block : 0];
  const int hl = lane & 15, rq = lane >> 4;
  const int col0 = NQ * wave;  // this wave's columns of a query tile
  // c / group and c % group of a column, c < 2^13: exact, (c + 1/2) / group is 1/32 off an integer at least
  const float inv_group = 1.f / (float)group;
  auto row_of = [&](int c) { return PART == kPrefix ? c / group : (int)(((float)c + 0.5f) * inv_group); };

  auto uniform = [](int v) { return __builtin_amdgcn_readfirstlane(v); };
  // last i with s_pre[i] <= u
  auto find = [&](int u) {
    int i = 0, hi = B;
    while (hi - i > 1) {
      const int mid = (i + hi) >> 1;
      if (s_pre[mid] <= u) i = mid; else hi = mid;
    }
    return i;
  };

  if (PART == kWhole && !by_task && tid == 0) desc[r].pieces = 0;
  if (PART == kWhole && no_cut)  // no second launch
    for (int b = r; b < B; b += G) zero_left_alone(a, b, THREADS);
  int total = 0, all_tasks = 0, most = 0, S, each;
  bool whole = false, dealt = false;  // ranges are lists of whole tasks; dealt out by length
  int cut = 0, tile0 = 0;             // or each is a piece of one task, of about `cut` tiles; its first tile
  // The tasks of a sequence: its heads' in turn, of each all query tiles; of a prefix its query tiles' in turn, of each all
  // heads. Those that read the same tokens are then a multiple of n_kv ranges apart, with eight heads on the same XCD, whose
  // L2 has what the first has read (two query tiles: 64 tokens over 8192 44.3 us, 43.2; 128 rows over 8192 56.4, 53.5).
  // Task of round j of range x.
  auto deal = [&](int x, int j) { return j & 1 ? (j + 1) * G - 1 - x : j * G + x; };
  {
    const int per = (B + THREADS - 1) / THREADS;
    const int b0 = min(B, tid * per), b1 = min(B, b0 + per);
    int loc = 0, tasks = 0;
    for (int b = b0; b < b1; ++b) {
      int first, n, of_seq;
      if (PART == kWhole) {
        const DraftSeq s = draft_seq(a.row_off, a.ctx_lens, b, a.rows, a.max_rows, a.cols, ring);
        tiles_of(s, window, first, n);
        s_first[b] = first;
        s_n[b] = n;
        of_seq = n == 0 ? 0 : a.n_kv * ((s.n * group + QT - 1) / QT);
        s_pre[b] = of_seq;
      } else {
        n = s_n[b];
        of_seq = s_pre[b];
      }
      loc += n * of_seq;
      tasks += of_seq;
      most = max(most, n);
    }
    auto plus = [](int x, int y) { return x + y; };
    const int inc = wave_scan(loc, plus), inc_tasks = wave_scan(tasks, plus);
    most = wave_scan(most, [](int x, int y) { return max(x, y); });
    if (lane == 63) s_tot[of_block][0] = inc, s_tot[of_block][1] = inc_tasks, s_tot[of_block][2] = most;
    __syncthreads();
    int run = inc - loc, run_tasks = inc_tasks - tasks;
    most = 0;
    for (int w = 0; w < QW * WPB; ++w) {
      if (w < of_block) run += s_tot[w][0], run_tasks += s_tot[w][1];
      total += s_tot[w][0];
      all_tasks += s_tot[w][1];
      most = max(most, s_tot[w][2]);
    }
    total = uniform(total);
    all_tasks = uniform(all_tasks);
    S = max(min_tiles, (total + G - 1) / G);
    each = (all_tasks + G - 1) / G;
    whole = each == 1 && uniform(most) <= S + slack;  // then s_pre counts tasks, not units
    if (DEAL > 1 && each > 1 && each <= DEAL && B <= THREADS) {  // s_ord: sequences by length; s_pre: tasks before each of them
      const int n = tid < B ? s_n[tid] : 0, of_seq = tid < B ? s_pre[tid] : 0;
      s_ids[tid] = of_seq;
      if (tid == 0) s_most = 0;
      __syncthreads();
      int rank = 0, before = 0;  // sequences that are longer, and their tasks
      for (int b = 0; b < B; ++b) {
        const int m = s_n[b];
        if (m > n || (m == n && b < tid)) ++rank, before += s_ids[b];
      }
      if (tid < B) {
        s_ord[rank] = tid;
        s_pre[rank] = before;
      }
      __syncthreads();
      // The longest range has the first or the last task of some sequence.
      for (int k = before, i = 0; i < 2 && of_seq > 0; k = before + of_seq - 1, ++i) {
        const int j = k / G, x = j & 1 ? (j + 1) * G - 1 - k : k - j * G;
        int load = 0;
        for (int y = 0; y < each; ++y)
          if (deal(x, y) < all_tasks) load += s_n[s_ord[find(deal(x, y))]];
        atomicMax(&s_most, load);
      }
      __syncthreads();
      whole = dealt = uniform(s_most) <= S + slack;
      if (!dealt && tid < B) s_pre[tid] = of_seq;  // per is 1
    }
    // Equal ranges end inside tasks and begin others, each change of which costs a range a few tiles' time and a second
    // record. Prefix tasks are few and long: each is cut into pieces of its own instead, where lengths of at most `slack`
    // tiles more make no more pieces than ranges (64 sequences over one prefix of 8192 tokens: 46 us with equal ranges, 37).
    if (PART == kPrefix && !whole && B <= 64) {
      const int length = S + min(lane, slack);
      const float inv = 1.f / (float)length;
      float ranges = 0.f;
      for (int b = 0; b < B; ++b)  // at least the pieces of each task: the quotient is never rounded below them
        ranges += (float)s_pre[b] * truncf((float)(s_n[b] + length - 1) * inv * 1.000001f + 0.001f);
      const uint64_t fits = __ballot(ranges <= (float)G);
      if (fits) cut = __shfl(length, __builtin_ctzll(fits), kWave);
      cut = uniform(cut);
      __syncthreads();  // s_pre is read above
    }
    if (PART == kPrefix && cut > 0) {  // s_pre: ranges before
      run = 0;
      for (int b = b0; b < b1; ++b) run += s_pre[b] * ((s_n[b] + cut - 1) / cut);
      const int upto = wave_scan(run, plus);  // B is 64 at most: one wave's
      run = upto - run;
      for (int b = b0; b < b1; ++b) {
        const int of_seq = s_pre[b] * ((s_n[b] + cut - 1) / cut);
        s_pre[b] = run;
        run += of_seq;
      }
      if (tid == min(B, THREADS) - 1) s_pre[B] = run;
    } else {
      if (!dealt)
        for (int b = b0; b < b1; ++b) {
          const int of_seq = s_pre[b];
          s_pre[b] = whole ? run_tasks : run;
          run += s_n[b] * of_seq;
          run_tasks += of_seq;
        }
      if (tid == 0) s_pre[B] = whole ? all_tasks : total;
    }
    __syncthreads();
  }
  int u0 = 0, n_w, pieces = 0;
  if (PART == kPrefix && cut > 0) {
    if (r >= s_pre[B]) return;
    const int b = find(r), n = s_n[b];
    pieces = uniform((n + cut - 1) / cut);
    const int each_piece = (n + pieces - 1) / pieces, off = r - s_pre[b], task = off / pieces;
    tile0 = uniform((off - task * pieces) * each_piece);
    n_w = uniform(min(n - tile0, each_piece));
    whole = true;
    each = 1;
    if (tid == 0) {
      s_list[0][0] = b;
      s_list[0][1] = task;
      s_list[0][2] = n_w;
      s_list[0][3] = task % a.n_kv;
    }
    __syncthreads();
    if (n_w <= 0) return;
  } else if (whole) {
    if (at_list < each) {
      const int k = deal(r, at_list), i = k < all_tasks ? find(k) : 0, b = dealt ? s_ord[i] : i;
      const int rows = PART == kPrefix ? 0 : draft_seq(a.row_off, a.ctx_lens, b, a.rows, a.max_rows, a.cols, ring).n;
      s_list[at_list][0] = b;
      s_list[at_list][1] = k - s_pre[i];
      s_list[at_list][2] = k < all_tasks ? s_n[b] : 0;
      s_list[at_list][3] = PART == kPrefix ? (k - s_pre[i]) % a.n_kv : (k - s_pre[i]) / max(1, (rows * group + QT - 1) / QT);
    }
    __syncthreads();
    n_w = 0;
    for (int i = 0; i < each; ++i) n_w += uniform(s_list[i][2]);
    if (n_w == 0) return;
  } else {
    if ((int64_t)r * S >= total) return;
    u0 = r * S;
    n_w = min(total - u0, S);
  }

  // The page window: of units [t0, t0 + 32) of the range lane l knows page l % 2 of unit t0 + l / 2 and the unit's KV head.
  // entry: where in the table that page stands (-1: nowhere), from LDS alone.
  auto entry = [&](int t0, int &head) -> int64_t {
    const int t = t0 + (lane >> 1);
    head = 0;
    if (t >= n_w) return -1;
    int b, off = t;
    if (whole) {
      int i = 0;
      if (DEAL > 1)
        while (i + 1 < each && off >= s_list[i][2]) off -= s_list[i++][2];
      b = s_list[i][0];
      head = s_list[i][3];
      if (PART == kPrefix) off += tile0;
    } else {
      b = find(u0 + t);
      const int n = s_n[b];
      off = u0 + t - s_pre[b];
      head = off / n;
      off -= head * n;
      if (PART == kPrefix) head %= a.n_kv;
      else if (max_qt > 1) head /= (s_pre[b + 1] - s_pre[b]) / (n * a.n_kv);
    }
    const int lp = 2 * ((PART == kPrefix ? 0 : s_first[b]) + off) + (lane & 1);
    if (ring <= 0 && lp >= a.cols) return -1;
    return (int64_t)(PART == kPrefix ? s_first[b] : b) * a.cols + (ring > 0 ? lp % ring : lp);
  };
  constexpr int64_t blk = (int64_t)kPage * D;
  int it = 0, islot = 0;   // next unit to fetch, and its slot
  uint32_t ok_bits = 0;    // two bits per fetched unit, the next one to be consumed lowest
  // The next window's pages come to LDS like the tiles, 32 units before they are used: nothing waits for them, where a wait
  // for a register would drain the tiles in flight.
  int page_cur, head_cur, head_nxt;
  bool has_nxt;
  int *const ids = s_ids + of_block * 64;
  auto fetch_window = [&](int t0) {
    const int64_t e = entry(t0, head_nxt);
    has_nxt = e >= 0;
    __builtin_amdgcn_global_load_lds((const void *)(a.table + (has_nxt ? e : 0)),
                                     (__attribute__((address_space(3))) void *)ids, 4, 0, 0);
  };
  auto next_window = [&]() {  // before the fetch of every 32nd unit
    page_cur = has_nxt ? ids[lane] : -1;
    head_cur = head_nxt;
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): read before it is overwritten
    fetch_window(it + 32);
  };
  {
    const int64_t e = entry(0, head_cur);
    page_cur = e >= 0 ? a.table[e] : -1;
    fetch_window(32);
  }
  // Fetching unit `it` (past the range: the first page of the pool, so that every fetch makes LPT loads and the waits can
  // count them) in two steps: where its pages are, and the loads. Chunk c of the tile, 1 KB each: 2 KK of keys, then KK of
  // values of either page; a wave takes LPT neighbouring ones. Keys: lane l brings the 16 bytes it reads as its fragment
  // of product h, K[token 8 (l % 16 / 4) + 4 h + l % 4][kk * 32 + l / 16 * 8 ..]. Values: 32 dims, the first eight slots of
  // each, then the last eight, so that sixteen lanes read 256 neighbouring bytes (as they lie in the page, every other 16:
  // half the banks).
  const uint32_t stride = (uint32_t)(a.n_kv * blk * 4), head_bytes = (uint32_t)(blk * 2);  // of a page, of a head in it
  const uint32_t pages = (uint32_t)min(a.pool_pages, (int64_t)0x7fffffff);
  uint32_t chunk_off[LPT];  // this lane's bytes of a chunk, from its page's head
  bool chunk_p1[LPT];       // and whether that is the second page
#pragma unroll
  for (int i = 0; i < LPT; ++i) {
    const int c = wave * LPT + i;
    const bool keys = c < 2 * KK;
    chunk_off[i] = keys ? (uint32_t)(c / KK * (4 * D * 2) + c % KK * 64 + (((hl & 4) * 2 + (hl & 3)) * D + rq * 8) * 2)
                        : (uint32_t)(stride / 2 + c % KK * 1024 + (lane & 31) * 32 + (lane >> 5) * 16);
    chunk_p1[i] = keys ? hl >= 8 : c >= 3 * KK;
  }
  const uint8_t *base0 = nullptr, *base1 = nullptr;
  uint32_t ok_next = 0;
  auto find_pages = [&]() {
    const int at = (it & 31) * 2;
    const uint32_t p0 = __builtin_amdgcn_readlane(page_cur, at), p1 = __builtin_amdgcn_readlane(page_cur, at + 1);
    const uint32_t g = __builtin_amdgcn_readlane(head_cur, at);
    const uint32_t most = it < n_w ? pages : 0u;
    const bool ok0 = p0 < most, ok1 = p1 < most;
    ok_next = (ok0 ? 1u : 0u) | (ok1 ? 2u : 0u);
    const uint32_t q0 = ok0 ? p0 : 0u, q1 = ok1 ? p1 : q0;
    const uint8_t *pool = (const uint8_t *)a.pool + (uint64_t)g * head_bytes;
    base0 = pool + (uint64_t)q0 * stride;
    base1 = pool + (uint64_t)q1 * stride;
    ++it;
  };
  auto issue = [&](int age) {
    ok_bits |= ok_next << (2 * age);
    uint8_t *const dst = slots + islot * Shape::kTileBytes;
#define ODS_TILE_LOADS(aux)                                                                                            \
  _Pragma("unroll") for (int i = 0; i < LPT; ++i)                                                                      \
      __builtin_amdgcn_global_load_lds((const void *)((chunk_p1[i] ? base1 : base0) + chunk_off[i]),                   \
                                       (__attribute__((address_space(3))) void *)(dst + (wave * LPT + i) * 1024), 16, 0, aux)
    if (PART == kTail && past) {
      ODS_TILE_LOADS(2);  // nt
    } else {
      ODS_TILE_LOADS(STREAM ? 2 : 0);
    }
#undef ODS_TILE_LOADS
    islot = islot + 1 == NS ? 0 : islot + 1;
  };

  // ---- the task being accumulated
  int cb_seq, ct, c_n, c_first, c_qts, c_key = -1, item = 0;  // sequence, task in it, its tiles; where in the list
  int tile;                                                                          // next tile of the task
  DraftSeq seq;
  bool busy;                          // this wave has columns in it
  int head, qt, seg_first;            // KV head, query tile, first tile of this range's piece
  bool first_piece = true;
  u32x4 q[CB][KK];
  f32x4 acc[CB][NB];
  u32x4 kf[2][KK], vf[NB], p[CB];     // operands of the next products: keys, values and probabilities
  f32x4 s[CB][2];
  float m[CB], l[CB];
  int col_lo[CB];                     // first visible token of this lane's columns
  // Their rows' masks, or, where those are of several words, the rows themselves; groups have 32 columns a sequence at most.
  std::conditional_t<PART == kWhole, uint64_t, uint32_t> col_mask[CB];

  auto task_id = [&]() { return ((int64_t)cb_seq * a.n_kv + head) * max_qt + qt; };
  auto load_seq = [&]() {
    c_n = uniform(s_n[cb_seq]);
    if (PART == kPrefix) {
      c_first = 0;
      seq.r0 = uniform(seqs.r0[cb_seq]);
      seq.n = uniform(seqs.rows[cb_seq]);
      seq.ctx = seq.end = seq.cap = c_n * kTile;
    } else {
      c_first = uniform(s_first[cb_seq]);
      const DraftSeq s = draft_seq((ConstInts)a.row_off, (ConstInts)a.ctx_lens, cb_seq, a.rows, a.max_rows, a.cols, ring);
      seq.r0 = uniform(s.r0);
      seq.n = uniform(s.n);
      seq.ctx = uniform(s.ctx);
      seq.end = uniform(s.end);
      seq.cap = s.cap;
    }
    if (PART == kTail) c_key = uniform(seqs.key[cb_seq]);
    c_qts = max_qt > 1 ? (seq.n * group + QT - 1) / QT : 1;
  };
  auto open_task = [&]() {
    head = PART == kPrefix ? ct % a.n_kv : max_qt > 1 ? ct / c_qts : ct;
    qt = PART == kPrefix ? ct / a.n_kv : max_qt > 1 ? ct % c_qts : 0;
    seg_first = tile;
    const int cols = seq.n * group;
    busy = qt * QT + col0 < cols;
    const int64_t row_elems = (int64_t)(a.n_q + 2 * a.n_kv) * D;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      const int c = min(qt * QT + col0 + cb * 16 + hl, cols - 1);  // columns past the last repeat it, unwritten
      const int j = row_of(c);
      const uint16_t *src = a.qkv + (seq.r0 + j) * row_elems + (head * group + c - j * group) * D + rq * 8;
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) q[cb][kk] = *(const u32x4 *)(src + kk * 32);
      col_mask[cb] = PART == kPrefix ? 0 : PART == kTail || a.max_rows <= 64 ? a.mask[seq.r0 + j] : (uint64_t)(seq.r0 + j);
      col_lo[cb] = window > 0 ? max(0, seq.ctx + clamp_depth(a.depth[seq.r0 + j], a.max_rows) - window + 1) : 0;
      m[cb] = kNoScore;
      l[cb] = 0.f;
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) acc[cb][nb] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) p[cb] = u32x4{0u, 0u, 0u, 0u};  // the first products add nothing
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) vf[nb] = u32x4{0u, 0u, 0u, 0u};
    // The q rows wait here, once per task: waited for at their first use, the compiler would drain the tiles in flight
    // in every step.
    __builtin_amdgcn_s_waitcnt(0x0f70);  // vmcnt(0)
  };
  // Output or record of the task's piece [seg_first, last tile so far]; `whole`: the piece is all of the task.
  auto close_task = [&](bool whole) {
    const int cols = seq.n * group;
    const int rec = 2 * r + (first_piece ? 0 : 1);
    const int hl = made_here(lane) & 15, rq = made_here(lane) >> 4;
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
      float sum = l[cb];
      sum += __shfl_xor(sum, 16, kWave);
      sum += __shfl_xor(sum, 32, kWave);
      const int at = col0 + cb * 16 + hl, c = qt * QT + at;
      const int j = row_of(min(c, cols - 1));
      const int64_t to = (int64_t)(seq.r0 + j) * a.n_q + head * group + c - j * group, at_rec = (int64_t)rec * QT + at;
      const bool mine = c < cols, state = whole && (PART == kPrefix || (PART == kTail && c_key >= 0));
      if (mine && whole && !state) {
        const float inv = sum == 0.f ? 0.f : 1.f / sum;
        uint16_t *dst = a.o + to * D + rq * 4;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          u32x2 w;
          w[0] = pack_pair(acc[cb][nb][0] * inv, acc[cb][nb][1] * inv);
          w[1] = pack_pair(acc[cb][nb][2] * inv, acc[cb][nb][3] * inv);
          *(u32x2 *)(dst + nb * 16) = w;
        }
      }
      if (mine && (state || !whole)) {
        float *dst = (state ? out.state_acc + to * D : out.rec_acc + at_rec * D) + rq * 4;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) *(f32x4 *)(dst + nb * 16) = acc[cb][nb];
      }
      if (mine && (state || !whole) && rq == 0) *(state ? out.state_ml + to : out.rec_ml + at_rec) = make_float2(m[cb], sum);
    }
  };

  // The task that began in this range lies in `pieces` ranges. By one thread.
  auto describe = [&](int pieces) {
    const int rec = 2 * r + (first_piece ? 0 : 1);
    if (PART == kPrefix)
      out.prefix[((int64_t)head * a.rows + seq.r0) * group + qt * QT] = make_int2(pieces, rec);
    else
      desc[PART == kTail || by_task ? task_id() : r] = TreeDesc{pieces, rec, seq.r0, qt * QT, seq.n * group, head, c_key};
  };

  // ---- the phases of a tile
  auto key = [&](const uint8_t *src, int half, int kk) { return *(const u32x4 *)(src + half * PB + kk * 1024 + lane * 16); };
  auto value = [&](const uint8_t *src, int nb) {
    return *(const u32x4 *)(src + (2 + (rq >> 1)) * PB + (nb >> 1) * 1024 + (rq & 1) * 512 + ((nb & 1) * 16 + hl) * 16);
  };
  // O += V^T P; S = K Q^T. NEXT: an operand is replaced right after its last product, by this tile's values at src_v and
  // the next one's keys at src_k, so the reads run under the products.
  auto values = [&](auto next, const uint8_t *src_v) {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
#pragma unroll
      for (int cb = 0; cb < CB; ++cb)
        acc[cb][nb] = mfma_16x16x32(__builtin_bit_cast(bf16x8, vf[nb]), __builtin_bit_cast(bf16x8, p[cb]), acc[cb][nb]);
      if (decltype(next)::value) vf[nb] = value(src_v, nb);
    }
  };
  auto scores = [&](auto next, const uint8_t *src_k) {
#pragma unroll
    for (int kk = 0; kk < KK; ++kk) {  // the products of a sum lie apart: each waits for the one before
#pragma unroll
      for (int half = 0; half < 2; ++half) {
#pragma unroll
        for (int cb = 0; cb < CB; ++cb)
          s[cb][half] = mfma_16x16x32(__builtin_bit_cast(bf16x8, kf[half][kk]), __builtin_bit_cast(bf16x8, q[cb][kk]),
                                      kk == 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : s[cb][half]);
        if (decltype(next)::value) kf[half][kk] = key(src_k, half, kk);
      }
    }
  };
  // Scores of tokens [t0, t0 + 32) to probabilities. EDGE: masked score by score.
  auto softmax = [&](auto edge, int t0, bool ok0, bool ok1) {
    constexpr bool EDGE = decltype(edge)::value;
    uint32_t vis[CB];  // of this lane's eight tokens
    if (EDGE) {
      const int rq = made_here(lane) >> 4;
      const int words = (a.max_rows + 63) / 64, seen_end = min(seq.ctx, seq.cap);
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
        const int j0 = t0 - seq.ctx;  // drafted token of the tile's first slot (below 0: cached ones come first)
        constexpr int BITS = 8 * sizeof(col_mask[0]);
        uint32_t v = PART == kPrefix ? 0u : PART == kTail || words == 1 ? (j0 < 0 ? (j0 > -32 ? (uint32_t)(col_mask[cb] << -j0) : 0u)
                                          : j0 < BITS ? (uint32_t)(col_mask[cb] >> j0) : 0u)
                                : mask_window(a.mask + (int64_t)col_mask[cb] * words, words, j0);
        v &= bits_between(-j0, seq.end - t0);
        v = v >> (rq * 8) & 0xffu;
        if (window > 0 && window < a.max_rows) {  // not the drafted tokens `window` positions or more before the row
          int depth[8];
#pragma unroll
          for (int i = 0; i < 8; ++i) depth[i] = v >> i & 1 ? a.depth[seq.r0 + j0 + rq * 8 + i] : 0;
#pragma unroll
          for (int i = 0; i < 8; ++i)
            if (seq.ctx + clamp_depth(depth[i], a.max_rows) < col_lo[cb]) v &= ~(1u << i);
        }
        v |= bits_between(col_lo[cb] - t0, seen_end - t0) >> (rq * 8);
        vis[cb] = (rq < 2 ? ok0 : ok1) ? v & 0xffu : 0u;
#pragma unroll
        for (int i = 0; i < 8; ++i)
          if (!(vis[cb] >> i & 1)) s[cb][i / 4][i % 4] = -INFINITY;
      }
    }
    float e[CB][8];
    bool move = false;
    auto exponents = [&]() {
#pragma unroll
      for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int i = 0; i < 8; ++i) e[cb][i] = s[cb][i / 4][i % 4] * scale_log2 - m[cb];
    };
    auto most = [](const float *x) {
      return fmaxf(fmaxf(fmaxf(x[0], x[1]), fmaxf(x[2], x[3])), fmaxf(fmaxf(x[4], x[5]), fmaxf(x[6], x[7])));
    };
    exponents();
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) move |= most(e[cb]) > kSlack;
    if (__any(move)) {  // move the reference points of whole columns
#pragma unroll
      for (int cb = 0; cb < CB; ++cb) {
#pragma unroll
        for (int i = 0; i < 8; ++i) e[cb][i] = s[cb][i / 4][i % 4] * scale_log2;
        float to = fmaxf(m[cb], most(e[cb]));
        to = fmaxf(to, __shfl_xor(to, 16, kWave));
        to = fmaxf(to, __shfl_xor(to, 32, kWave));
        const float alpha = __builtin_amdgcn_exp2f(m[cb] - to);
        m[cb] = to;
        l[cb] *= alpha;
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) acc[cb][nb] *= alpha;
      }
      exponents();
    }
#pragma unroll
    for (int cb = 0; cb < CB; ++cb) {
#pragma unroll
      for (int i = 0; i < 8; ++i) e[cb][i] = __builtin_amdgcn_exp2f(e[cb][i]);
      l[cb] += ((e[cb][0] + e[cb][1]) + (e[cb][2] + e[cb][3])) + ((e[cb][4] + e[cb][5]) + (e[cb][6] + e[cb][7]));
#pragma unroll
      for (int i = 0; i < 4; ++i) p[cb][i] = pack_pair(e[cb][2 * i], e[cb][2 * i + 1]);
    }
    if (!EDGE) return;
    // Zeros times the values tell whether all of them are finite.
    f32x4 zero[2] = {f32x4{0.f, 0.f, 0.f, 0.f}, f32x4{0.f, 0.f, 0.f, 0.f}};
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
      zero[nb & 1] = mfma_16x16x32(__builtin_bit_cast(bf16x8, vf[nb]), __builtin_bit_cast(bf16x8, u32x4{0u, 0u, 0u, 0u}), zero[nb & 1]);
    const f32x4 nan = zero[0] + zero[1];
    if (__any(!(nan[0] + nan[1] + nan[2] + nan[3] == 0.f))) {
      // Rare. What is not finite leaves the product and is added to the columns that see it: how many +inf, -inf and NaN
      // of each dim they see, 32 at most of each, as one product: weights 1, 64 and 4096 times the column's visible tokens.
      const uint32_t one = made_here(0x3f80u);
      const float not_a_number = made_here(NAN);
      u32x4 see[CB];
#pragma unroll
      for (int cb = 0; cb < CB; ++cb)
#pragma unroll
        for (int i = 0; i < 4; ++i)
          see[cb][i] = (vis[cb] >> (2 * i) & 1 ? one : 0u) | (vis[cb] >> (2 * i) & 2 ? one << 16 : 0u);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        u32x4 v = vf[nb];
        const f32x4 of = mfma_16x16x32(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, u32x4{0u, 0u, 0u, 0u}), f32x4{0.f, 0.f, 0.f, 0.f});
        if (!__any(!(of[0] + of[1] + of[2] + of[3] == 0.f))) continue;  // these dims are finite
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          uint32_t w = v[i];
          drop_nonfinite(w);
          vf[nb][i] = w;
          v[i] = nonfinite_weight(v[i], one);
        }
#pragma unroll
        for (int cb = 0; cb < CB; ++cb) {
          const f32x4 n = mfma_16x16x32(__builtin_bit_cast(bf16x8, v), __builtin_bit_cast(bf16x8, see[cb]), f32x4{0.f, 0.f, 0.f, 0.f});
#pragma unroll
          for (int d = 0; d < 4; ++d) {
            const int c = (int)n[d];
            if (c & 63) acc[cb][nb][d] += INFINITY;
            if (c & (63 << 6)) acc[cb][nb][d] -= INFINITY;
            if (c >> 12) acc[cb][nb][d] = not_a_number;
          }
        }
        __builtin_amdgcn_sched_barrier(0);
      }
    }
  };

  if (whole) {
    cb_seq = uniform(s_list[0][0]);
    ct = uniform(s_list[0][1]);
    tile = tile0;
    load_seq();
  } else {
    cb_seq = uniform(find(u0));
    load_seq();
    const int off = u0 - uniform(s_pre[cb_seq]);
    ct = off / c_n;
    tile = off % c_n;
  }
  constexpr int LEAD = QW == 1 ? NS : NS - 1;  // tiles fetched before the first is used
#pragma unroll
  for (int i = 0; i < LEAD; ++i) {
    find_pages();
    issue(i);
  }
  open_task();  // ends with a wait for every load
  int t = 0;
  // A tile takes two phases: products (the last tile's values, then this one's scores; each operand is replaced from LDS
  // after its last use) and softmax, which also fetches a tile.
  //  - Softmax of tile t fetches into the slot of tile t - 1, whose last reads were made in products t - 1.
  //  - Two or four waves meet once a tile, after its softmax; where a compute unit runs two workgroups, the other fills the
  //    gaps. Products of tile t read its keys first, so one tile fewer has to have landed (24 rows x 64 sequences: 123 us with
  //    the keys read a tile ahead, 112).
  //  - Eight waves have a compute unit to themselves. Their products read the next tile's keys, so that the reads run under
  //    the products: everyone's loads of t + 1 have landed before products t. The two waves of a SIMD run half a tile apart
  //    and all meet after either phase: while one is at its products the other is at its softmax. In step they queue for
  //    the matrix cores and for the vector unit in turn (64 sequences x 8192 tokens x 64 rows: 680 us, apart 630; at 16
  //    columns a wave the two do not differ).
  //    The later half's products t are the earlier half's softmax t: what the products of t + 1 read (tile t + 2) has to
  //    have landed when anyone's products t end.
  //  - One wave alone has no barrier; it reads a tile when it starts on it.
  constexpr bool PING = QW == 8;
  // Keys are read a tile ahead. Not where prefixes and tails are one kernel, which spilled 32 registers with them when that was
  // tried (128 x 4 rows over 32768: 300 us, without either 312), one of them read back by the lanes of an inner branch alone.
  constexpr bool AHEAD = QW == 8 && PART == kWhole;
  int slot = 0;
  auto next_slot = [](int x) { return x + 1 == NS ? 0 : x + 1; };
  auto at_slot = [&](int x) { return (const uint8_t *)(slots + x * Shape::kTileBytes); };
  // At most `tiles` of this wave's fetches are outstanding; `reads`: its LDS reads are done. Then a barrier.
  auto meet = [&](auto tiles, bool reads) {
    constexpr int n = decltype(tiles)::value * LPT;
    __builtin_amdgcn_sched_barrier(0);
    if (reads) __builtin_amdgcn_s_waitcnt((n & 15) | 7 << 4 | 0 << 8 | n >> 4 << 14);
    else __builtin_amdgcn_s_waitcnt((n & 15) | 7 << 4 | 15 << 8 | n >> 4 << 14);
    asm volatile("s_barrier" ::: "memory");
    __builtin_amdgcn_sched_barrier(0);
  };
  using All = std::integral_constant<int, 63 / LPT>;  // as many as the counter holds: no wait
  using Prod = std::integral_constant<int, PING ? NS - 4 : 63 / LPT>;
  using Soft = std::integral_constant<int, PING || QW == 1 ? 63 / LPT : AHEAD ? NS - 3 : NS - 2>;
  auto first_keys = [&]() {
#pragma unroll
    for (int half = 0; half < 2; ++half)
#pragma unroll
      for (int kk = 0; kk < KK; ++kk) kf[half][kk] = key(at_slot(slot), half, kk);
  };
  if (QW > 1) {
    asm volatile("s_barrier" ::: "memory");
    if (AHEAD) first_keys();
  }
  if (PING && wave >= 4) meet(All(), true);
  auto products = [&]() {
    if (QW > 1) {
      if (busy) {
        if (!AHEAD) first_keys();
        values(std::true_type(), at_slot(slot));
        scores(std::integral_constant<bool, AHEAD>(), at_slot(next_slot(slot)));
        if (!AHEAD) __builtin_amdgcn_sched_group_barrier(0x100, 2 * KK, 0);
#pragma unroll
        for (int i = 0; i < (AHEAD ? NB + 2 * KK : NB); ++i) {  // a read after the products of an operand
          __builtin_amdgcn_sched_group_barrier(0x8, CB, 0);
          __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
        }
      }
      if (PING) meet(Prod(), false);
    } else {
      asm volatile("s_waitcnt vmcnt(%0)" ::"n"((NS - 1) * LPT) : "memory");
      first_keys();
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) vf[nb] = value(at_slot(slot), nb);
      if (EARLY) {
        asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
        __builtin_amdgcn_sched_barrier(0);
        find_pages();
        ok_bits >>= 2;
        issue(NS - 1);
      }
      scores(std::false_type(), nullptr);
    }
  };
  auto to_softmax = [&](auto edge, int t0, bool ok0, bool ok1) {
    if (!EARLY) {
      find_pages();
      if (QW > 1) issue(NS - 1);
      ok_bits >>= 2;
    }
    if (busy) softmax(edge, t0, ok0, ok1);
    if (QW == 1) {
      values(std::false_type(), nullptr);
      if (!EARLY) issue(NS - 1);
    } else {
      meet(Soft(), true);
    }
    slot = next_slot(slot);
    ++tile;
    ++t;
  };
  while (t < n_w) {
    if ((it & 31) == 0) next_window();
    __builtin_amdgcn_s_waitcnt(0xc07f);  // lgkmcnt(0): what is pending here is not waited for in every product phase below
    // Tiles that need no mask, up to the next page window: all of it cached tokens that every row sees, pages in the pool.
    const int lo_most = window > 0 ? seq.ctx + a.max_rows - window : 0;
    const int full_end = min(seq.ctx, seq.cap) / kTile - c_first, full_begin = (max(lo_most, 0) + kTile - 1) / kTile - c_first;
    const int run = tile < full_begin ? 0 : min(min(n_w - t, full_end - tile), 32 - (it & 31));
    int done = 0;
    for (; done < run && (ok_bits & 3) == 3; ++done) {
      products();
      to_softmax(std::false_type(), 0, true, true);
    }
    if (done == 0) {
      const bool ok0 = ok_bits & 1, ok1 = ok_bits & 2;
      products();
      to_softmax(std::true_type(), (c_first + tile) * kTile, ok0, ok1);
    }
    if (tile == c_n) {  // the task ends here
      if (PING && wave < 4) meet(All(), true);  // the halves change tasks together
      if (QW > 1) values(std::false_type(), nullptr);
      close_task(seg_first == 0);
      if (PART == kWhole) {
        if (by_task && lead && seg_first == 0) desc[task_id()].pieces = 1;
      } else if (lead && seg_first == 0) {
        describe(1);
      }
      first_piece = false;
      tile = 0;
      if (t < n_w) {
        if (DEAL > 1 && whole) {
          ++item;
          cb_seq = uniform(s_list[item][0]);
          ct = uniform(s_list[item][1]);
          load_seq();
        } else if (++ct == c_qts * a.n_kv) {
          ct = 0;
          ++cb_seq;
          while (uniform(s_pre[cb_seq + 1]) == uniform(s_pre[cb_seq])) ++cb_seq;
          load_seq();
        }
        open_task();
        if (AHEAD) first_keys();  // the last products did not read them if this wave had no columns there
      }
      if (PING && wave >= 4) meet(All(), true);
    }
  }
  if (PING && wave < 4) meet(All(), true);  // as many barriers as the other half
  if (QW > 1 && tile > 0) values(std::false_type(), nullptr);
  // No load may still be writing LDS when the workgroup retires.
  asm volatile("s_waitcnt vmcnt(0)" ::: "memory");
  if (tile > 0) {  // the range ends inside a task
    close_task(false);
    if (lead && seg_first == 0) {  // ... that began in it: this range names the records to join
      const int begin = uniform(s_pre[cb_seq]) + ct * c_n, end = begin + c_n;
      describe(pieces > 0 ? pieces : (end - 1) / S - r + 1);
    }
  }
}

template <int D, int NQ, int QW, bool STREAM>
__global__ __launch_bounds__(64 * QW) __attribute__((amdgpu_waves_per_eu(2))) void tree_attention_kernel(
    const DraftArgs a, const int min_tiles, const int max_qt, const int by_task, const int no_cut, const float scale_log2,
    const TreeOut out) {
  extern __shared__ __align__(16) int smem[];
  TreeSeqs seqs{};
  seqs.count = a.B;
  seqs.pre = smem;  // units before, first tile, tiles of a sequence
  seqs.first = smem + a.B + 1;
  seqs.n = seqs.first + a.B;
  tree_work<D, NQ, QW, TreeShape<D, NQ, QW>::kSlots, STREAM, kWhole, 1>(a, seqs, (uint8_t *)smem + ((3 * a.B + 1) * 4 + 15) / 16 * 16,
                                                                        blockIdx.x, gridDim.x, min_tiles, kSplitTiles, max_qt, by_task, no_cut,
                                                                        scale_log2, out);
}

// Joins the records of tasks that lie in several ranges: o[d] = sum_i
// 2^(m_i - M) acc_i[d] / sum_i 2^(m_i - M) l_i, D / 4 lanes per record. Bound by
// latency: the descriptor, then all of a column's first records and weights in
// one trip. SPLIT: a column is four waves' work, a quarter of its records each
// (few tasks of many records); otherwise a wave joins four columns at a time
// (many tasks of two or three). Block x is task x of the batch, or, where there
// are more tasks than ranges, the task that begins in range x. Also writes the
// zeros of sequences that are left alone.
template <int D, bool SPLIT>
__global__ __launch_bounds__(256) void tree_join_kernel(const DraftArgs a, const int QT, const int max_qt, const int by_task,
                                                        const float *__restrict__ rec_acc,
                                                        const float2 *__restrict__ rec_ml,
                                                        const TreeDesc *__restrict__ desc) {
  constexpr int LPR = D / 4, RPW = kWave / LPR;                 // lanes per record, records a wave reads at once
  constexpr int NC = SPLIT ? 1 : 4, G = SPLIT ? 4 * RPW : RPW;  // columns of a wave, records of a column at once
  constexpr int PRE = SPLIT ? 4 : 2;                            // trips in flight
  __shared__ float part[SPLIT ? 4 * (D + 4) : 1];
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int group = a.n_q / a.n_kv;
  const TreeDesc e = desc[blockIdx.x];
  bool zero = blockIdx.y == 0;
  int b0 = blockIdx.x, step = gridDim.x;
  if (by_task) {  // the descriptor of a task without units was not written
    b0 = blockIdx.x / (a.n_kv * max_qt);
    step = a.B;
    zero = zero && blockIdx.x % (a.n_kv * max_qt) == 0;
  }
  if (zero) {
    for (int b = b0; b < a.B; b += step) zero_left_alone(a, b, 256);
  }
  if (by_task) {
    const DraftSeq s = draft_seq(a.row_off, a.ctx_lens, b0, a.rows, a.max_rows, a.cols, a.ring);
    if (s.end == 0 || (int)(blockIdx.x % max_qt) * QT >= s.n * group) return;
  }
  const int at0 = SPLIT ? blockIdx.y : (blockIdx.y * 4 + wave) * NC;  // first column of the tile this wave joins
  if (e.pieces <= 1 || e.col0 + at0 >= e.cols) return;
  const int d = (lane % LPR) * 4, sub = (SPLIT ? wave * RPW : 0) + lane / LPR;
  // Columns past the last one read the records' unwritten rows and are not stored; every index is inside the records.
  auto rec = [&](int i, int c) { return (int64_t)(i == 0 ? e.rec : (e.rec & ~1) + 2 * i) * QT + at0 + c; };
  float M[NC], sum[NC];
  f32x4 acc[NC];
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    M[c] = kNoScore;
    sum[c] = 0.f;
    acc[c] = f32x4{0.f, 0.f, 0.f, 0.f};
  }
  for (int i0 = 0; i0 < e.pieces; i0 += PRE * G) {
    f32x4 x[PRE][NC];
    float2 ml[PRE][NC];
#pragma unroll
    for (int k = 0; k < PRE; ++k)
#pragma unroll
      for (int c = 0; c < NC; ++c) {
        const int64_t at = rec(min(i0 + sub + k * G, e.pieces - 1), c);  // past the last: again, with weight 0
        ml[k][c] = rec_ml[at];
        x[k][c] = *(const f32x4 *)(rec_acc + at * D + d);
      }
#pragma unroll
    for (int c = 0; c < NC; ++c) {
      float top = M[c];
#pragma unroll
      for (int k = 0; k < PRE; ++k) top = fmaxf(top, ml[k][c].x);
      const float old = __builtin_amdgcn_exp2f(M[c] - top);
      M[c] = top;
      sum[c] *= old;
      acc[c] *= old;
#pragma unroll
      for (int k = 0; k < PRE; ++k) {
        const float w = i0 + sub + k * G < e.pieces ? __builtin_amdgcn_exp2f(ml[k][c].x - top) : 0.f;
        sum[c] += w * ml[k][c].y;
        if (w != 0.f) acc[c] += w * x[k][c];
      }
    }
  }
#pragma unroll
  for (int c = 0; c < NC; ++c) {
    float top = M[c];
#pragma unroll
    for (int o = LPR; o < kWave; o <<= 1) top = fmaxf(top, __shfl_xor(top, o, kWave));
    const float w = __builtin_amdgcn_exp2f(M[c] - top);
    float l = sum[c] * w;
    f32x4 v = acc[c] * w;
#pragma unroll
    for (int o = LPR; o < kWave; o <<= 1) {
      l += __shfl_xor(l, o, kWave);
#pragma unroll
      for (int i = 0; i < 4; ++i) v[i] += __shfl_xor(v[i], o, kWave);
    }
    if (SPLIT) {
      if (lane < LPR) *(f32x4 *)(part + wave * (D + 4) + d) = v;
      if (lane == 0) *(float2 *)(part + wave * (D + 4) + D) = make_float2(top, l);
      __syncthreads();
      if (wave > 0) return;
      top = kNoScore;
#pragma unroll
      for (int w4 = 0; w4 < 4; ++w4) top = fmaxf(top, part[w4 * (D + 4) + D]);
      l = 0.f;
      v = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w4 = 0; w4 < 4; ++w4) {
        const float u = __builtin_amdgcn_exp2f(part[w4 * (D + 4) + D] - top);
        l += u * part[w4 * (D + 4) + D + 1];
        v += u * *(const f32x4 *)(part + w4 * (D + 4) + d);
      }
    }
    const int col = e.col0 + at0 + c;
    if (lane >= LPR || col >= e.cols) continue;
    const float inv = l == 0.f ? 0.f : 1.f / l;
    u32x2 out;
    out[0] = pack_pair(v[0] * inv, v[1] * inv);
    out[1] = pack_pair(v[2] * inv, v[3] * inv);
    *(u32x2 *)(a.o + ((int64_t)(e.r0 + col / group) * a.n_q + e.head * group + col % group) * D + d) = out;
  }
}

}  // namespace

}  // namespace ods
