/*
 * ods.h -- C ABI of the operator-level-disaggregated (ODS) decode hot path on
 * AMD Instinct MI355X (gfx950).
 *
 * The paper models one decode step as a fixed, ordered sequence of kernels
 * o_1..o_N (Appendix A.1) and a serving stage as a contiguous slice of the
 * operator sequence of a repeating partition block: stage j holds operators
 * q_{j-1}+1 .. q_j (Section 4, "Partition-block abstraction"; Appendix B.1).
 * Stages exchange an activation interface A_j at each boundary (Appendix B.3,
 * the stage-latency and transfer-latency equations), a worker loads only its
 * assigned components and state, buffers are bound once with only token,
 * position and KV metadata changing between steps, and one native call
 * enqueues a whole per-step action sequence (Section 6 and its "Single native
 * submission" optimisation). This library is that native call for one GPU.
 *
 * Operator index space. A block of layers is numbered globally, layer after
 * layer; indices are 0-based and ranges half-open, so the paper's stage j is
 * [q_{j-1}, q_j). Per layer (local index):
 *
 *   dense layer (10 ops)                  MoE layer (14 ops)
 *   0 attn_norm        resid -> xn        0..6 as in the dense layer
 *   1 qkv_proj         xn -> qkv          7  router          hn -> logits
 *   2 rope             qkv -> qkv         8  topk_softmax    logits -> topk_ids, topk_w
 *   3 kv_append        qkv -> KV pool     9  moe_permute     hn, topk_ids -> xp, perm,
 *   4 attn_core        qkv, pool -> o                            slot_pos, expert_off
 *   5 o_proj_residual  o, resid -> resid  10 expert_gate_up  xp -> gu_p
 *   6 ffn_norm         resid -> hn        11 silu_mul        gu_p -> act_p
 *   7 gate_up          hn -> gu           12 expert_down     act_p -> yp
 *   8 silu_mul         gu -> act          13 moe_combine_residual
 *   9 down_residual    act, resid -> resid                   yp, topk_w, slot_pos, resid -> resid
 *
 * Attention-FFN disaggregation cuts every layer at local 6; core-attention
 * disaggregation isolates [3, 5); the colocated template is [0, N_block)
 * (Section 4, "Design-space expressiveness").
 *
 * Numerics (the paper leaves the layer's arithmetic unspecified; these are the
 * library's conventions): bf16 storage, fp32 accumulation. RMSNorm
 * x * (mean(x^2) + eps)^-1/2 * gain. RoPE rotate-half pairs (i, i + d/2) at
 * position ctx - 1, angle (ctx - 1) * theta^(-2i/d) evaluated in double.
 * Attention softmax(q K^T / sqrt(d)) V over keys [ctx - window, ctx - 1]
 * (window 0: all keys); query head h reads KV head h / (n_q / n_kv).
 * SwiGLU silu(gate) * up. Routing: top-k of the fp32 router logits (ties go to
 * the lower expert index), weights = softmax over the chosen k. Every live
 * buffer is rounded to bf16 (round-to-nearest-even) except logits and routing
 * weights (fp32) and indices (int32).
 *
 * Ownership and errors. The caller owns all memory and the stream. The library
 * never allocates, frees, synchronises, or changes the current device, and
 * keeps no state between calls (apart from the static workspace array of
 * ods_run_partition_scratch). Every argument is checked on the host before
 * anything is enqueued: a non-OK status means nothing was enqueued, except
 * ODS_EHIP, which reports a launch failure after earlier kernels of the same
 * call were enqueued. Device faults surface at the caller's synchronisation.
 * All device pointers must be 16-byte aligned. Calls are thread-safe;
 * ods_last_error() is per thread.
 */
#ifndef ODS_H
#define ODS_H

#include <stddef.h>
#include <stdint.h>
#include <hip/hip_runtime_api.h>

#ifdef __cplusplus
extern "C" {
#endif

typedef enum {
  ODS_OK = 0,
  ODS_EINVAL = -1,        /* null / misaligned pointer, negative size, bad enum */
  ODS_ERANGE = -2,        /* operator range or context outside its bounds */
  ODS_ENOMEM = -3,        /* KV pool or workspace too small */
  ODS_EUNSUPPORTED = -4,  /* shape the kernels do not implement */
  ODS_EHIP = -5           /* HIP runtime reported an error while enqueuing */
} ods_status;

#define ODS_PAGE_TOKENS 16

/* Shape of one decoder layer. n_experts == 0 selects a dense SwiGLU FFN of
 * width ffn; otherwise a top_k-of-n_experts MoE with per-expert width moe_ffn.
 * window == 0 selects full attention, window > 0 a sliding window of that many
 * most recent tokens (the decoded token included).
 * Supported: head_dim in {64, 128}; n_q a multiple of n_kv with n_q / n_kv <= 16;
 * hidden, ffn, moe_ffn multiples of 8; n_experts <= 256; 1 <= top_k <= n_experts. */
typedef struct {
  int32_t hidden, n_q, n_kv, head_dim;
  int32_t ffn;
  int32_t n_experts, top_k, moe_ffn;
  int32_t window;
  float rope_theta, rms_eps;
} ods_layer_cfg;

/* Layout of a layer's projection weights (w_qkv, w_o, w_gate_up, w_down).
 *   ODS_WEIGHTS_ROWS:  row-major "out x in", as listed under ods_layer.
 *   ODS_WEIGHTS_TILED: the tile order ods_tile_weight() writes, which the
 *     weight-streaming GEMM reads as one contiguous run per block (faster at
 *     decode batches). Needs hidden, n_q * head_dim and ffn (dense) or moe_ffn
 *     (MoE) to be multiples of 64 (ODS_EUNSUPPORTED otherwise). w_router stays
 *     row-major. */
typedef enum { ODS_WEIGHTS_ROWS = 0, ODS_WEIGHTS_TILED = 1 } ods_weight_layout;

/* One layer's device-resident weights (bf16, row-major "out x in" unless
 * weight_layout says otherwise) and KV pool.
 *   g_attn, g_ffn  [hidden]
 *   w_qkv          [(n_q + 2 n_kv) head_dim, hidden]   q heads, then k heads, then v heads
 *   w_o            [hidden, n_q head_dim]
 *   dense: w_gate_up [2 ffn, hidden] (gate rows, then up rows); w_down [hidden, ffn]
 *   MoE:   w_router [n_experts, hidden]; w_gate_up [n_experts, 2 moe_ffn, hidden];
 *          w_down [n_experts, hidden, moe_ffn]
 *   kv_pool  [pool_pages][2][n_kv][16 * head_dim] bf16. Block (page, 0, g) holds the
 *            keys of 16 token slots row-major (slot t, dim i at t * head_dim + i);
 *            block (page, 1, g) holds the values dim-major (dim i, slot t at i * 16 + t).
 *            Token position t of a sequence lives in page page_table[b][t / 16],
 *            slot t % 16. Every block is 16 * head_dim * 2 bytes, contiguous. */
typedef struct {
  ods_layer_cfg cfg;
  const void *g_attn, *w_qkv, *w_o, *g_ffn, *w_gate_up, *w_down, *w_router;
  void *kv_pool;
  int64_t pool_pages;
  int32_t weight_layout;  /* ods_weight_layout */
} ods_layer;

/* A partition block: n_layers layers whose operators are numbered consecutively.
 * All layers share one batch, page table and live set. */
typedef struct {
  int32_t n_layers;
  const ods_layer *layers;
} ods_block;

/* Per-step metadata (device pointers). ctx_lens[b] counts the keys sequence b
 * attends to, the token being decoded included, so that token's position is
 * ctx_lens[b] - 1; valid values are 1 .. max_pages * 16 (larger values are
 * clamped; a row with a value < 1 is left alone by RoPE and KV append, and
 * its attention output is a row of zeros).
 * page_table [batch][max_pages] int32, -1 for unused entries; page ids outside
 * [0, pool_pages) are skipped by the kernels. attn_core numbers the (sequence,
 * KV head, window page) units of the batch and gives every wave of its grid an
 * equal contiguous range of them; split_pages fixes the range length in pages
 * (0: library choice, the batch's pages over all waves, at least 4 each, or 2
 * with 64-wide heads).
 * attn_core takes batch <= 4096 and batch * n_kv * window pages < 2^30
 * (ODS_EUNSUPPORTED otherwise).
 *
 * Window-only page ring (ring_pages > 0). A sliding-window layer only ever
 * reads the most recent `window` tokens, so its KV pages can live in a ring
 * (a sliding-window layer reads at most its window of KV; Section 3, hybrid
 * architectures): with ring_pages = R > 0, every layer of
 * the call with window > 0 maps token position t of sequence b to page
 * ring_table[b][(t / 16) % R], slot t % 16, of its own kv_pool, and its
 * contexts are not clamped to max_pages * 16. Full-attention layers keep
 * page_table. R must be at least ceil(window / 16) + 1 for every such layer
 * the call touches (the window's pages plus the one the next token opens), so
 * a page is only reused once it has left the window (ODS_EINVAL otherwise).
 * ring_table is [batch][R] int32; ods_kv_alloc with max_pages = R and contexts
 * min(ctx, 16 R) fills one. A ring layer's pool needs at most batch * R pages
 * however long the contexts grow. ring_pages = 0: no ring (ring_table unused). */
typedef struct {
  int32_t batch, max_pages;
  const int32_t *ctx_lens;
  const int32_t *page_table;
  int32_t split_pages;
  int32_t ring_pages;
  const int32_t *ring_table;
} ods_batch;

/* Live buffers (the activation interface at any cut), device, caller-allocated.
 * Sizes per ods_live_bytes(). Only buffers read or written by the operators of
 * a call's range need to be non-null.
 *   resid [B, H] bf16 (updated in place by o_proj_residual, down_residual,
 *   moe_combine_residual); xn, hn [B, H]; qkv [B, (n_q + 2 n_kv) d]; o [B, n_q d];
 *   gu [B, 2F]; act [B, F]; logits [B, E] fp32; topk_ids [B, k] int32;
 *   topk_w [B, k] fp32; perm [B k] (sorted position -> token * k + slot);
 *   slot_pos [B k] (token * k + slot -> sorted position); expert_off [E + 1];
 *   xp [B k, H]; gu_p [B k, 2 I]; act_p [B k, I]; yp [B k, H] (all bf16);
 *   ws: scratch of at least ods_workspace_bytes() bytes. */
typedef struct {
  void *resid, *xn, *qkv, *o, *hn, *gu, *act;
  float *logits, *topk_w;
  int32_t *topk_ids, *perm, *slot_pos, *expert_off;
  void *xp, *gu_p, *act_p, *yp;
  void *ws;
  size_t ws_bytes;
} ods_state;

typedef enum {
  ODS_BUF_RESID = 0, ODS_BUF_XN, ODS_BUF_QKV, ODS_BUF_O, ODS_BUF_HN, ODS_BUF_GU, ODS_BUF_ACT,
  ODS_BUF_LOGITS, ODS_BUF_TOPK_W, ODS_BUF_TOPK_IDS, ODS_BUF_PERM, ODS_BUF_SLOT_POS,
  ODS_BUF_EXPERT_OFF, ODS_BUF_XP, ODS_BUF_GU_P, ODS_BUF_ACT_P, ODS_BUF_YP, ODS_BUF_COUNT
} ods_buffer;

/* Host-only page allocation for one step's batch (no device work). The pool's
 * page ids [0, pool_pages) are shuffled by a Fisher-Yates pass driven by
 * splitmix64(seed) (for i = P-1 down to 1, swap entries i and next() mod (i+1));
 * sequence b then takes the next ceil(ctx_lens_host[b] / 16) shuffled ids, in
 * batch order. Writes page_table_host [batch][max_pages] (caller memory), -1 in
 * unused entries. ODS_ENOMEM if the batch needs more than pool_pages pages,
 * ODS_ERANGE if a sequence needs more than max_pages, ODS_EINVAL for null
 * pointers or non-positive ctx. The paged cache itself follows the paper's use
 * of paged KV memory in its serving engine (Section 6). */
ods_status ods_kv_alloc(int64_t pool_pages, const int32_t *ctx_lens_host, int32_t batch,
                        uint64_t seed, int32_t max_pages, int32_t *page_table_host);

/* Bytes of one layer's KV pool of pool_pages pages (0 for an invalid cfg). */
size_t ods_kv_pool_bytes(const ods_layer_cfg *cfg, int64_t pool_pages);

/* Bytes of live buffer `which` for this block at this batch size (the maximum
 * over the block's layers; 0 when no layer uses the buffer). */
size_t ods_live_bytes(const ods_block *blk, int32_t batch, ods_buffer which);

/* Minimum ods_state.ws_bytes for any operator range of this block and batch,
 * under the launch plans of the library that is loaded: ask it again after an
 * update instead of carrying a size over. A larger batch does not always need
 * more, so one workspace for several batch sizes takes the largest of their
 * needs. */
size_t ods_workspace_bytes(const ods_block *blk, const ods_batch *batch);

/* Number of operators of the block (sum over layers of 10 or 14); < 0 on error. */
int32_t ods_block_num_ops(const ods_block *blk);

/* Tiled weight layout (ODS_WEIGHTS_TILED). A weight of `groups` slabs (1, or
 * n_experts for the expert weights), each `out` x `in` row-major bf16 (gated:
 * 2 out rows, the gate rows then the up rows, as w_gate_up), is stored as
 * consecutive 16 KB tiles, slab by slab: for each N tile nt and each 64-wide
 * K step s, 128 rows of 64 columns, row r at byte r * 128 of the tile and the
 * row's 16-byte chunk c (columns 64 s + 8 c .. + 7) at position c ^ (r % 8)
 * of that row. Plain weights: tile row r is weight row 128 nt + r. Gated: tile
 * rows r < 64 are gate rows 64 nt + r, rows 64 + j the matching up rows
 * out + 64 nt + j, so both halves of an output column stream together (the
 * SwiGLU epilogue of the fused gate_up GEMM, Section 2's FFN operator). Rows
 * past `out` are zero. The XOR position of the chunks keeps the GEMM's LDS
 * fragment reads free of bank conflicts.
 *
 * ods_tiled_weight_bytes: bytes of that layout; 0 unless out >= 1, in >= 64,
 *   in % 64 == 0, groups >= 1 and gated in {0, 1}.
 * ods_tile_weight: enqueues on `stream` the conversion of the row-major weight
 *   at src (device, groups * (gated ? 2 : 1) * out * in bf16) into dst (device,
 *   ods_tiled_weight_bytes() bytes, not overlapping src). Both 16-byte aligned.
 *   ODS_EINVAL for null or misaligned pointers or sizes the layout rejects;
 *   ODS_EHIP if the launch fails. Nothing is enqueued on error. */
size_t ods_tiled_weight_bytes(int32_t out, int32_t in, int32_t gated, int32_t groups);
ods_status ods_tile_weight(const void *src, void *dst, int32_t out, int32_t in, int32_t gated, int32_t groups,
                           hipStream_t stream);

/* Static name of global operator `op` ("attn_core", ...), NULL if out of range. */
const char *ods_op_name(const ods_block *blk, int32_t op);

/* Enqueue operators [op_begin, op_end) of the block on `stream` (one native
 * submission for one stage; Section 6). Adjacent operators inside the range
 * may be fused; every buffer of the live set at op_end is materialised, so a
 * block run as any sequence of contiguous ranges computes the same step. A
 * buffer consumed inside the range may be left unwritten (with moe_permute
 * and expert_gate_up in one range the expert GEMM reads hn through perm and
 * xp is not written).
 * ODS_ERANGE unless 0 <= op_begin < op_end <= ods_block_num_ops(). An empty
 * batch (batch->batch == 0) returns ODS_OK once the block and the range are
 * valid, enqueueing nothing and reading no pointer of batch or state. */
ods_status ods_run_partition(const ods_block *blk, int32_t op_begin, int32_t op_end,
                             const ods_batch *batch, ods_state *state, hipStream_t stream);

/* Size of the workspace the library itself holds on each device for
 * ods_run_partition_scratch (64 MiB; every evaluated block needs at most
 * 32 MiB, as ods_workspace_bytes reports). */
#define ODS_SCRATCH_BYTES ((size_t)64 << 20)

/* For callers that cannot allocate device memory (code under HIP graph
 * capture, serving loops and harnesses that forbid hipMalloc): the same as
 * ods_run_partition, except that the workspace is a static device array of
 * ODS_SCRATCH_BYTES bytes inside the library instead of state->ws (state->ws
 * and state->ws_bytes are ignored and may be NULL / 0). The caller still
 * passes every input and output buffer. Nothing is allocated or freed: each
 * device the library runs on holds its own copy of the array from module load
 * until the process ends; its address is resolved on the first call on a
 * device (with that device current). Nothing in the array needs to start at
 * zero; it keeps the contents the last call left. Calls that overlap on one
 * GPU (several streams or threads at once) share the array and race: the
 * caller must order them, e.g. on one stream per device.
 * Errors: those of ods_run_partition, plus ODS_ENOMEM when the range needs
 * more than ODS_SCRATCH_BYTES of workspace (nothing is enqueued) and ODS_EHIP
 * when the array's device address cannot be resolved. */
ods_status ods_run_partition_scratch(const ods_block *blk, int32_t op_begin, int32_t op_end,
                                     const ods_batch *batch, ods_state *state, hipStream_t stream);

/* The attention stage of layer `layer`: its operators 0..5 (attention-FFN
 * disaggregation's attention side; Section 2, "Attention-FFN Disaggregation"). */
ods_status ods_attn_stage(const ods_block *blk, int32_t layer, const ods_batch *batch,
                          ods_state *state, hipStream_t stream);

/* The FFN / MoE stage of layer `layer`: its operators 6 .. end of layer. */
ods_status ods_ffn_stage(const ods_block *blk, int32_t layer, const ods_batch *batch,
                         ods_state *state, hipStream_t stream);

/* Capture operators [op_begin, op_end) as an instantiated HIP graph, so a
 * stage replays as one submission with its buffers bound once (Section 6:
 * static plan capacity; graphs and buffers bound once, only token, position
 * and KV metadata change between iterations).
 * The graph holds the pointers of blk, batch and state and the host values
 * they carry (batch size, max_pages, split_pages, shapes) as of this call; the
 * device contents they point to (resid, ctx_lens, page_table, weights, pools)
 * are read at each launch, so a new decode step only rewrites those buffers.
 * Validation is that of ods_run_partition; on a non-OK status *exec is NULL.
 * The caller owns *exec: launch it with ods_graph_launch, free it with
 * ods_graph_destroy. Capture runs on a private stream and enqueues nothing. */
ods_status ods_partition_graph(const ods_block *blk, int32_t op_begin, int32_t op_end,
                               const ods_batch *batch, ods_state *state, hipGraphExec_t *exec);

/* Launch a graph from ods_partition_graph on `stream` (hipGraphLaunch). */
ods_status ods_graph_launch(hipGraphExec_t exec, hipStream_t stream);

/* Free a graph from ods_partition_graph (NULL is a no-op). */
ods_status ods_graph_destroy(hipGraphExec_t exec);

/* ---- Rotary positions ------------------------------------------------------
 *
 * A rotary embedding other than the whole-head, half-layout one the layer's
 * `rope` operator applies. Pair i of rotary_dim / 2 turns by position *
 * freqs[i]; the two values of a pair are dims i and i + rotary_dim / 2, or
 * with interleaved != 0 dims 2 i and 2 i + 1. Dims from rotary_dim on pass
 * through. The turned values are multiplied by `amplitude` (1: a plain
 * rotation; a long-context model's attention factor goes here, as its square
 * root of the score's factor).
 *
 * freqs: device table of rotary_dim / 2 doubles, which ods_rope_freqs() fills
 * on the host from the other fields (angles of far positions need more than
 * float: position 10^6 times a float's rounding is 0.06 of a radian). With
 * f_i = theta^(-2 i / rotary_dim), `scaling` is
 *   ODS_ROPE_PLAIN      f_i
 *   ODS_ROPE_LINEAR     f_i / factor (position interpolation)
 *   ODS_ROPE_BASE       f_i of theta * factor^(r / (r - 2)), r = rotary_dim (f_i for r = 2)
 *   ODS_ROPE_ROTATIONS  f_i for pairs that turn turns_hi times or more over
 *                       orig_ctx positions, f_i / factor for turns_lo or fewer,
 *                       between them a blend linear in the number of turns
 *   ODS_ROPE_INDEX      the same two ends, the blend linear in the pair's index
 *                       between the indices of turns_hi (rounded down, at least
 *                       0) and turns_lo (rounded up, at most r - 1)
 * (interpolation by parts: Peng et al. 2023, arxiv 2309.00071). */
typedef enum {
  ODS_ROPE_PLAIN = 0, ODS_ROPE_LINEAR, ODS_ROPE_BASE, ODS_ROPE_ROTATIONS, ODS_ROPE_INDEX
} ods_rope_scaling;

typedef struct {
  int32_t head_dim;     /* multiple of 8, 8 .. 256 */
  int32_t rotary_dim;   /* even, 2 .. head_dim */
  int32_t interleaved;  /* 0: half layout, 1: interleaved */
  int32_t scaling;      /* ods_rope_scaling */
  double theta, factor; /* > 0; theta != 1 for ODS_ROPE_INDEX */
  double orig_ctx, turns_hi, turns_lo; /* ROTATIONS, INDEX: orig_ctx > 0, turns_hi > turns_lo > 0 */
  float amplitude;
  const double *freqs;  /* device [rotary_dim / 2] */
} ods_rope;

/* The table of `rope` (its freqs pointer is not read): rotary_dim / 2 doubles
 * into caller memory on the host. ODS_EINVAL for null pointers, a field outside
 * the ranges above or a value that is not finite; ODS_EUNSUPPORTED for a
 * head_dim that is no multiple of 8 or past 256. */
ods_status ods_rope_freqs(const ods_rope *rope, double *freqs_host);

/* y = the heads of x rotated, bf16: row r's `heads` heads of head_dim values
 * start at x + r * x_stride (in elements) and go to y + r * y_stride, turned
 * to position pos[r] (device int32). A row with a negative position is left
 * alone: its y is not written. x and y may be the same rows (in place) or
 * rows that do not overlap; strides are multiples of 8 and at least
 * heads * head_dim, so the q and k heads of qkv rows are one call.
 * ODS_EINVAL for null or misaligned pointers, negative rows or heads, bad
 * strides, a partial overlap, or rope fields ods_rope_freqs refuses; rows or
 * heads of 0 return ODS_OK with nothing enqueued. */
ods_status ods_rope_rows(const ods_rope *rope, const void *x, int64_t x_stride, void *y, int64_t y_stride,
                         int32_t rows, int32_t heads, const int32_t *pos, hipStream_t stream);

/* Gains of heads that are normalised before they turn: x * (mean(x^2) +
 * eps)^-1/2 * gain over the head's head_dim values, in fp32, the result not
 * rounded before the rotation. gain_q, gain_k: device bf16 [head_dim], for the
 * query and the key heads. */
typedef struct {
  const void *gain_q, *gain_k;
  float eps;            /* >= 0 */
} ods_head_norm;

/* y = the heads of x normalised and rotated, in one pass: ods_rope_rows for rows
 * of n_q query heads and n_k key heads behind them. norm NULL: a rotation alone;
 * norm->gain_q (gain_k) may be NULL where n_q (n_k) is 0.
 * Positions of several axes (time, height, width of images and video): pos is
 * device int32 [rows][n_axes], 1 <= n_axes <= ODS_ROPE_AXES, and pair i of the
 * rotated ones turns by pos[r][axis[i]] * freqs[i]; axis is a device table of
 * rotary_dim / 2 int32 in 0 .. n_axes - 1 (values outside are clamped), NULL with
 * n_axes == 1. A row with a negative position on any axis is left alone.
 * Values past the rotated ones are normalised and pass through. Errors as
 * ods_rope_rows, and ODS_EINVAL for a norm or axes outside the above. */
#define ODS_ROPE_AXES 8
ods_status ods_head_rows(const ods_rope *rope, const ods_head_norm *norm, const int32_t *axis, int32_t n_axes,
                         const void *x, int64_t x_stride, void *y, int64_t y_stride, int32_t rows, int32_t n_q,
                         int32_t n_k, const int32_t *pos, hipStream_t stream);

/* ---- Drafted rows: several tokens of a sequence in one step -----------------
 *
 * A step over a tree of drafted tokens per sequence (speculative decoding), a
 * chunk of a prompt (a tree that is a chain) or one token (a tree of one).
 * The operators are those of ods_run_partition, on rows instead of sequences:
 * row_off[b] .. row_off[b + 1] - 1 of every live buffer are the drafted tokens
 * of sequence b, and rope, kv_append and attn_core take their drafted form:
 *   - batch->ctx_lens[b] counts the tokens already in the cache, none of the
 *     drafted ones among them; 0 is a new sequence. A sequence with a negative
 *     count is left alone by rope and kv_append, its attention output is zeros;
 *   - drafted token j of a sequence lives in the cache slot of token position
 *     ctx + j, whatever its place in the tree, and kv_append writes it there;
 *   - its position for rope and sliding windows is ctx + depth[row]; depth is
 *     0 for a token that follows the cached ones directly;
 *   - it attends the cached tokens t < ctx (a sliding-window layer: those with
 *     t > ctx + depth - window) and the drafted tokens j of its own sequence
 *     with bit j of its mask set (bit j % 64 of word j / 64; in a
 *     sliding-window layer only those less than `window` positions before it).
 *     Its own bit is not implied: a row that may see nothing gets zeros. What
 *     a row may not see does not reach it, infinities and NaN included.
 * A chain of one token with its bit set is the decode step of context ctx + 1.
 *
 *   rows      rows of the live buffers (what ods_live_bytes and the GEMMs take
 *             as the batch), 4096 * ODS_DRAFT_MAX_ROWS at most (past that
 *             ODS_EUNSUPPORTED); rows from row_off[batch] on are padding, which
 *             rope, kv_append and attn_core leave as they were
 *   max_rows  most rows of one sequence, 1 .. ODS_DRAFT_MAX_ROWS; a sequence's
 *             rows past it are treated as padding
 *   row_off   device [batch + 1], ascending, row_off[0] >= 0
 *   depth     device [rows], 0 .. max_rows - 1 (values outside are clamped)
 *   mask      device [rows][(max_rows + 63) / 64]
 *   rope      NULL: the layers' own rope_theta; or n_layers entries (host),
 *             each with the layer's head_dim
 * Slots past the page table (max_pages * 16 tokens) are neither written nor
 * attended. Attention's launch is planned for the table's width, as if contexts
 * filled it: a table no wider than the batch needs is a few us faster on short
 * contexts. A window-only ring must also hold the drafted tokens:
 * ring_pages >= ceil((window + max_rows) / 16) + 1 (ODS_EINVAL otherwise).
 * batch <= 4096 as for attn_core; rows * n_q < 2^31, and batch * n_kv * query
 * tiles * window pages < 2^30 (ODS_EUNSUPPORTED otherwise). split_pages is not
 * used. */
#define ODS_DRAFT_MAX_ROWS 256

/* Sequences that share the pages of a prefix (forks of one prompt): group g is
 * sequences group_off[g] .. group_off[g + 1] - 1 of the batch, whose page tables
 * name the same pages for their first tokens[g] tokens. In full-attention layers
 * attn_core then reads those pages once for all drafted rows of the group, by
 * the table of the first sequence that has rows and them all cached, and each
 * sequence's other tokens by its own. What it computes is the same attention. It
 * does so where that pays, by the sizes the host sees: up to 32 query vectors of
 * a KV head and sequence (max_rows * n_q / n_kv), and tables that span 128 MB of
 * keys and values or more (batch * max_pages); elsewhere each sequence is read by
 * itself. So are sequences in no group, groups of one, and sequences of fewer
 * cached tokens than their group shares, whatever their tables hold; what is
 * shared is rounded down to 32 tokens. Sliding-window layers read each sequence's
 * own window. A table as wide as the longest context passes the 128 MB whatever
 * is in it: short contexts are then better given no groups. Sharing has one
 * level, of sequences that are neighbours in the batch: of a prefix common to all
 * and longer ones common to some, a group names one. n_kv * (query tiles of the
 * groups + batch) * 32-token tiles of a table < 2^30 (ODS_EUNSUPPORTED otherwise).
 *   n_groups   0 .. batch, at most ODS_SHARED_GROUPS
 *   group_off  device [n_groups + 1], ascending, in 0 .. batch
 *   tokens     device [n_groups] */
#define ODS_SHARED_GROUPS 512
typedef struct {
  int32_t n_groups;
  const int32_t *group_off;
  const int32_t *tokens;
} ods_shared;

/*   norm      NULL, or n_layers entries (host): the rope operator normalises the q
 *             and k heads before it turns them (ods_head_norm)
 *   shared    NULL, or the batch's shared prefixes */
typedef struct {
  int32_t rows, max_rows;
  const int32_t *row_off;
  const int32_t *depth;
  const uint64_t *mask;
  const ods_rope *rope;
  const ods_head_norm *norm;
  const ods_shared *shared;
} ods_draft;

/* An ods_state.ws_bytes that is enough for any operator range of this block, for
 * this batch and draft (its pointers are not read) and for every one of no more
 * sequences, rows and max_rows over no wider a table: a state sized once for the
 * widest trees serves all others. 0 on invalid arguments. */
size_t ods_draft_workspace_bytes(const ods_block *blk, const ods_batch *batch, const ods_draft *draft);

/* Enqueue operators [op_begin, op_end) of the block for drafted rows: the
 * contract of ods_run_partition (fusion, checks before anything is enqueued,
 * errors), with ods_draft_workspace_bytes() of workspace. batch->batch == 0 or
 * draft->rows == 0 returns ODS_OK with nothing enqueued. */
ods_status ods_run_draft(const ods_block *blk, int32_t op_begin, int32_t op_end, const ods_batch *batch,
                         const ods_draft *draft, ods_state *state, hipStream_t stream);

/* ods_partition_graph for drafted rows: the pointers of draft (the entries of
 * draft->rope, norm and shared included) and rows, max_rows, n_groups are held as
 * of this call; row_off, depth, mask, freqs, gains, group_off and tokens are read
 * at each launch. */
ods_status ods_draft_graph(const ods_block *blk, int32_t op_begin, int32_t op_end, const ods_batch *batch,
                           const ods_draft *draft, ods_state *state, hipGraphExec_t *exec);

/* ---- Pages of a cache: sharing, copying, compacting, freeing ----------------
 *
 * Host bookkeeping over caller memory, for page tables of full-attention
 * layers (rings are not shared): who holds each page and which are free. No
 * device work; the copies a call asks for are (src, dst) page pairs for
 * ods_kv_copy_pages. One ods_pages serves all layers that share a table.
 * Calls on one ods_pages are ordered by the caller. On a non-OK status nothing
 * was changed. */
typedef struct {
  int64_t pool_pages;
  int32_t *refs;      /* [pool_pages] holders of each page */
  int32_t *free_ids;  /* [pool_pages]; the first n_free are the free pages, the next one taken last */
  int64_t n_free;
} ods_pages;

/* Count the holders of every page in table [rows][max_pages] (NULL: none;
 * entries < 0 hold nothing) and list the rest as free, lowest id taken first.
 * ODS_ERANGE for an entry >= pool_pages. */
ods_status ods_pages_init(ods_pages *pages, const int32_t *table, int32_t rows, int32_t max_pages);

/* A sequence (its table row) goes from old_tokens to new_tokens tokens. Fewer:
 * pages past the new count are given back. More: pages are taken, and if the
 * page that holds position old_tokens is partly filled and shared, the
 * sequence gets a page of its own for it: one pair (at most) is written to
 * pair[2] and *n_pairs is 1, else 0; the caller copies it before the new
 * tokens are written. ODS_ENOMEM without enough free pages, ODS_ERANGE when the
 * row is too short, ODS_EINVAL for a row whose held pages are not exactly those
 * of old_tokens. */
ods_status ods_pages_resize(ods_pages *pages, int32_t *row, int32_t max_pages, int32_t old_tokens,
                            int32_t new_tokens, int32_t pair[2], int32_t *n_pairs);

/* dst_row (empty: every entry < 0) holds the pages of the `tokens` tokens of
 * src_row too. Nothing is copied until either grows (ods_pages_resize). */
ods_status ods_pages_fork(ods_pages *pages, const int32_t *src_row, int32_t *dst_row, int32_t max_pages,
                          int32_t tokens);

/* Give back every page of a row; its entries become -1. */
ods_status ods_pages_release(ods_pages *pages, int32_t *row, int32_t max_pages);

/* Move held pages with the highest ids into the lowest free ids, at most
 * max_pairs of them, and rewrite the table: with max_pairs large enough the
 * held pages become [0, pool_pages - n_free). Writes pairs [*n_pairs][2], no
 * page twice in them. ODS_EINVAL unless the table's rows hold exactly what
 * `refs` counts. */
ods_status ods_pages_compact(ods_pages *pages, int32_t *table, int32_t rows, int32_t max_pages, int32_t *pairs,
                             int32_t max_pairs, int32_t *n_pairs);

/* Copy pages inside the pools of layers [layer_begin, layer_end): page
 * pairs[i][0] to page pairs[i][1] (device int32 [n_pairs][2]), keys and values
 * of every KV head. The copies have no order among each other: no page may be
 * a dst twice, or both a src and a dst. Pairs with an id outside a layer's pool
 * or with src == dst are skipped. ODS_ERANGE for a bad layer range. */
ods_status ods_kv_copy_pages(const ods_block *blk, int32_t layer_begin, int32_t layer_end, const int32_t *pairs,
                             int32_t n_pairs, hipStream_t stream);

/* Keep one path of each sequence's drafted tokens: with path [batch][path_cols]
 * and path_len [batch] (device), the cache slot of drafted token path[b][k]
 * moves to that of token position ctx + k, for k < path_len[b], in every layer
 * of [layer_begin, layer_end) (through the ring in ring layers), and
 * ctx_out[b] = ctx + path_len[b] (device [batch]; NULL: not written; may be
 * batch->ctx_lens itself, else it overlaps no array the call reads). A path is strictly ascending and below the
 * sequence's row count; the first entry that is not ends it there, and a
 * length past path_cols is cut. The slots of a sequence being kept must lie on
 * pages that no other sequence holds. draft: rows, max_rows and row_off are
 * read. path_cols 1 .. ODS_DRAFT_MAX_ROWS. */
ods_status ods_kv_accept(const ods_block *blk, int32_t layer_begin, int32_t layer_end, const ods_batch *batch,
                         const ods_draft *draft, const int32_t *path, int32_t path_cols, const int32_t *path_len,
                         int32_t *ctx_out, hipStream_t stream);

/* Groups of adjacent sequences that share leading pages, for ods_shared (host
 * only): rows of table [rows][max_pages] whose first entries are the same. A row
 * joins the group before it while that does not lower the pages the group saves
 * ((its rows - 1) * its common pages); only whole pages of `tokens` (host [rows],
 * each sequence's cached tokens) count. Writes group_off [rows + 1] and
 * group_tokens [rows] (their first *n_groups + 1 and *n_groups entries): together
 * the groups hold all rows, those that share nothing in groups of 0 tokens, or as
 * many of the first rows as ODS_SHARED_GROUPS groups take.
 * Where none shares 32 tokens, give ods_draft no groups: with groups of nothing
 * attn_core still takes the way of shared prefixes, which is slower for a batch
 * without them (64 sequences of 512 to 4096 tokens, one row each: 107 us instead
 * of 100, eight rows 135 instead of 113).
 * ODS_EINVAL for null pointers, negative sizes or token counts past the table. */
ods_status ods_pages_shared(const int32_t *table, int32_t rows, int32_t max_pages, const int32_t *tokens,
                            int32_t *group_off, int32_t *group_tokens, int32_t *n_groups);

/* ---- Verification of drafted tokens ------------------------------------------
 *
 * The accepted path of each sequence's tree and the token after it, so that what
 * is kept is distributed as if it had been drawn from the target model alone
 * (rejection sampling of drafts: Leviathan et al. 2023, arxiv 2211.17192; of
 * several drafts after one token, each tested on what the ones before left:
 * Miao et al. 2024, arxiv 2305.09781). Random numbers are inputs.
 *
 * Row 0 of a sequence is the token its last step ended with, which is always
 * kept; row j > 0 holds tokens[j], a draft of what follows row parent[j] (an
 * index below j inside the sequence). target row i holds the target's
 * probabilities of the token after row i, proposal row i the draft's, from which
 * the children of row i were drawn independently. From row i = 0 on:
 *   W = target[i], Z = 1; for the children c of i in ascending order, x = tokens[c]:
 *     c is kept, and i = c, if W(x) > 0 and accept_u[c] * Z * proposal[i](x) < W(x);
 *     else W = max(W - Z * proposal[i], 0) and Z = the sum of W.
 * proposal NULL: the drafted tokens are plain guesses (the likeliest ones, say),
 * as if proposal[i](x) were 1: c is kept if accept_u[c] * Z < W(x), else W(x) = 0
 * and Z = Z - the W(x) that was there.
 * When no child is kept the token after the path is the first t with
 * W(0) + .. + W(t) > next_u[b] * (the sum of W); where rounding leaves none, the
 * last t with W(t) > 0; where W holds nothing, the same of target[i]; where that
 * holds nothing, -1. Probabilities are fp32 or bf16 and all of this is computed
 * in fp64. Probabilities that are negative or not finite count as 0. A row whose
 * token is outside [0, vocab), or whose parent is not a row before it, is passed
 * over. A path ends early at path_cols rows: the token after it is drawn from
 * that row's target.
 *
 *   vocab            1 .. ODS_VERIFY_MAX_VOCAB; row r of target starts at target + r * target_stride
 *                    values (stride >= vocab), of proposal likewise
 *   tokens, parent   device int32 [rows]
 *   accept_u         device fp32 [rows], in [0, 1) (row 0's is not used)
 *   next_u           device fp32 [batch], in [0, 1)
 *   path             device [batch][path_cols]: the kept rows as ods_kv_accept takes
 *                    them, -1 behind them; path_cols 1 .. ODS_DRAFT_MAX_ROWS
 *   path_len, next_token  device int32 [batch]; 0 and -1 for a sequence without rows
 *   ws               at least ods_verify_workspace_bytes() bytes
 * Arrays of this struct need the alignment of their values only, ws 16 bytes. */
#define ODS_VERIFY_MAX_VOCAB (1 << 20)
typedef enum { ODS_PROBS_F32 = 0, ODS_PROBS_BF16 = 1 } ods_probs;

typedef struct {
  int32_t vocab;
  int32_t dtype;         /* ods_probs, of target and proposal */
  const void *target;
  int64_t target_stride;
  const void *proposal;
  int64_t proposal_stride;
  const int32_t *tokens, *parent;
  const float *accept_u, *next_u;
  int32_t path_cols;
  int32_t *path, *path_len, *next_token;
  void *ws;
  size_t ws_bytes;
} ods_verify;

/* Workspace of a verification of up to `batch` sequences over up to `vocab`
 * tokens (0 on invalid arguments). */
size_t ods_verify_workspace_bytes(int32_t batch, int32_t vocab);

/* Enqueue the verification of the draft's rows (rows, max_rows and row_off are
 * read; batch as of its ods_batch). batch == 0 returns ODS_OK with nothing
 * enqueued. */
ods_status ods_draft_verify(int32_t batch, const ods_draft *draft, const ods_verify *verify, hipStream_t stream);

/* Message for the last non-OK status returned on this thread ("" if none). */
const char *ods_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* ODS_H */
