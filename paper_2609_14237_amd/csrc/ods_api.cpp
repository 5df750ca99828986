// HIP side of the ODS decode library: the operator-range dispatcher that
// enqueues the launches ods_host.cpp plans for a stage [op_begin, op_end) of a
// partition block on one stream (one native submission per stage, no
// allocation, no synchronisation), graph capture of a stage, the on-device
// weight tiling, and the library-held workspace of the scratch entry point.
// Validation, sizing, the allocator and every launch-shape choice are in the
// HIP-free ods_host.cpp.
#include <stdlib.h>
#include <stdio.h>

#include <mutex>
#include <string>

#include "../../include/ods.h"
#include "kernels.hpp"

using namespace ods;

namespace {

bool trace_on() {
  const char *e = getenv("ODS_TRACE");
  return e && e[0] && e[0] != '0';
}

bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }

hipError_t execute(const Launch &L, hipStream_t s) {
  switch (L.kind) {
    case LK_RMSNORM: return launch_rmsnorm(L.x, L.gain, L.out, L.rows, L.width, L.eps, s);
    case LK_GEMM: return launch_gemm(L.gemm, s);
    case LK_SKINNY:
      return launch_gemm_skinny_fused(L.gemm, L.gain, L.eps, L.out, L.has_rope ? &L.rope : nullptr, s);
    case LK_NONE: return hipSuccess;
    case LK_GEMM_NORM: {
      const hipError_t e = launch_gemm(L.gemm, s);
      if (e != hipSuccess) return e;
      return launch_reduce_norm(L.gemm.partial, L.gemm.splits, L.gemm.M, L.gemm.N, (uint16_t *)L.gemm.C, L.gain, L.eps,
                                L.out, s);
    }
    case LK_QKV_ROPE:
    case LK_ROPE_APPEND: {
      if (L.kind == LK_QKV_ROPE) {
        const hipError_t e = launch_gemm(L.gemm, s);
        if (e != hipSuccess) return e;
      }
      const RopeArgs &r = L.rope;
      return launch_rope_append(r.qkv, r.B, r.n_q, r.n_kv, r.D, r.theta, r.ctx_lens, r.table, r.cols, r.ring, r.pool,
                                r.pool_pages, r.do_rope, r.do_append, s, r.partial, r.splits);
    }
    case LK_ATTENTION: {
      const AttnArgs &a = L.attn;
      return launch_attention(a.qkv, a.B, a.n_q, a.n_kv, a.D, a.window, a.ctx_lens, a.table, a.cols, a.ring, a.pool,
                              a.pool_pages, a.plan, a.ws, a.o, s);
    }
    case LK_SILU: return launch_silu_mul(L.x, L.out, L.rows, L.width, s);
    case LK_TOPK: return launch_topk(L.logits, L.rows, L.E, L.k, L.ids, L.weights, s);
    case LK_ROUTER_TOPK: {
      const hipError_t e = launch_gemm(L.gemm, s);
      if (e != hipSuccess) return e;
      return launch_topk(nullptr, L.rows, L.E, L.k, L.ids, L.weights, s, L.topk_partial, L.topk_splits, L.logits_out);
    }
    case LK_PERMUTE: {
      const hipError_t e = launch_permute(L.ids, L.rows, L.k, L.E, L.perm, L.slot_pos, L.expert_off, s);
      if (e != hipSuccess || !L.xp) return e;  // no xp: the expert GEMM that follows gathers its rows
      return launch_gather_rows(L.x, L.perm, L.expert_off + L.E, L.rows * L.k, L.k, L.width, L.xp, s);
    }
    case LK_COMBINE: return launch_moe_combine(L.x, L.weights, L.slot_pos, L.rows, L.k, L.width, L.out, s);
  }
  return hipErrorInvalidValue;
}

}  // namespace

// Workspace held by the library for callers that cannot allocate device
// memory (ods_run_partition_scratch). Each device the library runs on holds
// its own copy, zero-filled at load, until the process ends. In host code
// this name is a host-side stand-in, never a device address: the address is
// resolved per device with hipGetSymbolAddress and only that pointer is
// passed to kernels.
static __device__ __align__(256) uint8_t scratch[ODS_SCRATCH_BYTES];

namespace {

constexpr int kMaxScratchDevices = 64;
std::mutex g_scratch_mu;
void *g_scratch_ptr[kMaxScratchDevices] = {};

// Device address of `scratch` on the current device, resolved on the first
// call per device (with that device current) and cached.
ods_status scratch_ptr(void **out) {
  int dev = -1;
  hipError_t e = hipGetDevice(&dev);
  if (e != hipSuccess) return set_error(ODS_EHIP, "hipGetDevice: %s", hipGetErrorString(e));
  if (dev < 0 || dev >= kMaxScratchDevices)
    return set_error(ODS_EUNSUPPORTED, "device %d: the library scratch supports device ids below %d", dev,
                kMaxScratchDevices);
  std::lock_guard<std::mutex> lock(g_scratch_mu);
  if (!g_scratch_ptr[dev]) {
    void *p = nullptr;
    e = hipGetSymbolAddress(&p, HIP_SYMBOL(scratch));
    if (e != hipSuccess || !p)
      return set_error(ODS_EHIP, "hipGetSymbolAddress(scratch) on device %d: %s", dev, hipGetErrorString(e));
    g_scratch_ptr[dev] = p;
  }
  *out = g_scratch_ptr[dev];
  return ODS_OK;
}

// Enqueues a validated range.
ods_status run_rows(const ods_block *blk, int op_begin, int op_end, const ods_batch *batch, const ods_state *st, int cus,
                    bool trace, hipStream_t stream) {
  for (int i = 0; i < op_end - op_begin;) {
    Launch L;
    plan_launch(blk, op_begin, op_end, i, batch, st, cus, &L);
    const hipError_t e = execute(L, stream);
    if (trace) fprintf(stderr, "[ods] layer %d %s B=%d -> %s\n", L.layer, L.what, batch->batch, hipGetErrorString(e));
    if (e != hipSuccess)
      return set_error(ODS_EHIP, "launch of %s (layer %d) failed: %s", L.what, L.layer, hipGetErrorString(e));
    i += L.n_ops;
  }
  return ODS_OK;
}

// Captures what `enqueue` puts on a private stream as an instantiated graph.
template <typename F>
ods_status capture(hipGraphExec_t *exec, F enqueue) {
  if (!exec) return set_error(ODS_EINVAL, "exec is null");
  *exec = nullptr;
  hipStream_t s = nullptr;
  hipError_t e = hipStreamCreateWithFlags(&s, hipStreamNonBlocking);
  if (e != hipSuccess) return set_error(ODS_EHIP, "hipStreamCreate: %s", hipGetErrorString(e));
  e = hipStreamBeginCapture(s, hipStreamCaptureModeThreadLocal);
  if (e != hipSuccess) {
    hipStreamDestroy(s);
    return set_error(ODS_EHIP, "hipStreamBeginCapture: %s", hipGetErrorString(e));
  }
  const ods_status rc = enqueue(s);
  std::string msg = rc == ODS_OK ? "" : error_text();
  hipGraph_t graph = nullptr;
  e = hipStreamEndCapture(s, &graph);
  hipStreamDestroy(s);
  if (rc != ODS_OK) {
    if (graph) hipGraphDestroy(graph);
    return set_error(rc, "%s", msg.c_str());
  }
  if (e != hipSuccess || !graph) return set_error(ODS_EHIP, "hipStreamEndCapture: %s", hipGetErrorString(e));
  e = hipGraphInstantiate(exec, graph, nullptr, nullptr, 0);
  hipGraphDestroy(graph);
  if (e != hipSuccess) {
    *exec = nullptr;
    return set_error(ODS_EHIP, "hipGraphInstantiate: %s", hipGetErrorString(e));
  }
  clear_error();
  return ODS_OK;
}

DraftArgs draft_args(const ods_block *blk, int layer, const ods_batch *batch, const ods_draft *draft,
                     const ods_state *st) {
  const ods_layer &L = blk->layers[layer];
  const ods_layer_cfg &c = L.cfg;
  const KvMap m = kv_map(c, batch);
  DraftArgs a{};
  a.qkv = (uint16_t *)st->qkv;
  a.o = (uint16_t *)st->o;
  a.B = batch->batch; a.rows = draft->rows; a.max_rows = draft->max_rows;
  a.n_q = c.n_q; a.n_kv = c.n_kv; a.D = c.head_dim; a.window = c.window;
  a.row_off = draft->row_off; a.depth = draft->depth; a.ctx_lens = batch->ctx_lens; a.mask = draft->mask;
  a.table = m.table; a.cols = m.cols; a.ring = m.ring;
  a.pool = (uint16_t *)L.kv_pool; a.pool_pages = L.pool_pages;
  a.theta = c.rope_theta;
  if (draft->rope) {
    const ods_rope &r = draft->rope[layer];
    a.freqs = r.freqs; a.rdim = r.rotary_dim; a.interleaved = r.interleaved; a.amp = r.amplitude;
  }
  return a;
}

// Calls go(pools, n) for layers [begin, end), at most kPoolSet at a time.
template <typename F>
hipError_t each_pool_set(const ods_block *blk, int begin, int end, const ods_batch *batch, F go) {
  for (int l0 = begin; l0 < end; l0 += kPoolSet) {
    PoolSet set{};
    const int n = end - l0 < kPoolSet ? end - l0 : kPoolSet;
    for (int i = 0; i < n; ++i) {
      const ods_layer &L = blk->layers[l0 + i];
      PoolRef &r = set.p[i];
      r.pool = (uint16_t *)L.kv_pool;
      r.pages = L.pool_pages;
      r.n_kv = L.cfg.n_kv;
      r.D = L.cfg.head_dim;
      r.page_elems = (int64_t)2 * r.n_kv * ODS_PAGE_TOKENS * r.D;
      if (!batch) continue;
      const KvMap m = kv_map(L.cfg, batch);
      r.table = m.table; r.cols = m.cols; r.ring = m.ring;
    }
    if (const hipError_t e = go(set, n); e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace

extern "C" {

size_t ods_workspace_bytes(const ods_block *blk, const ods_batch *batch) {
  if (check_block(blk) != ODS_OK || !batch || batch->batch < 0 || batch->max_pages <= 0) return 0;
  return block_ws_bytes(blk, batch, num_cus());
}

ods_status ods_run_partition(const ods_block *blk, int32_t op_begin, int32_t op_end, const ods_batch *batch,
                             ods_state *st, hipStream_t stream) {
  const int cus = num_cus();
  const ods_status rc = validate_range(blk, op_begin, op_end, batch, st, cus);
  if (rc != ODS_OK) return rc;
  if (batch->batch == 0) {
    clear_error();
    return ODS_OK;
  }
  const ods_status done = run_rows(blk, op_begin, op_end, batch, st, cus, trace_on(), stream);
  if (done == ODS_OK) clear_error();
  return done;
}

ods_status ods_run_partition_scratch(const ods_block *blk, int32_t op_begin, int32_t op_end,
                                     const ods_batch *batch, ods_state *state, hipStream_t stream) {
  ods_status rc = check_block(blk);
  if (rc != ODS_OK) return rc;
  if (!batch || !state) return set_error(ODS_EINVAL, "null batch or state");
  const int n_ops = num_ops(blk);
  if (op_begin < 0 || op_end > n_ops || op_begin >= op_end)
    return set_error(ODS_ERANGE, "operator range [%d, %d) outside [0, %d) or empty", op_begin, op_end, n_ops);
  if (batch->batch < 0 || batch->split_pages < 0 || batch->ring_pages < 0)
    return set_error(ODS_EINVAL, "negative batch, split_pages or ring_pages");
  ods_state st = *state;
  st.ws = nullptr;
  st.ws_bytes = 0;
  if (batch->batch == 0) return ods_run_partition(blk, op_begin, op_end, batch, &st, stream);
  const size_t need = range_ws_bytes(blk, op_begin, op_end, batch, num_cus());
  if (need > ODS_SCRATCH_BYTES)
    return set_error(ODS_ENOMEM, "operators [%d, %d) need %zu bytes of workspace; the library scratch holds %zu",
                     op_begin, op_end, need, (size_t)ODS_SCRATCH_BYTES);
  rc = scratch_ptr(&st.ws);
  if (rc != ODS_OK) return rc;
  st.ws_bytes = ODS_SCRATCH_BYTES;
  return ods_run_partition(blk, op_begin, op_end, batch, &st, stream);
}

ods_status ods_tile_weight(const void *src, void *dst, int32_t out, int32_t in, int32_t gated, int32_t groups,
                           hipStream_t stream) {
  const size_t bytes = ods_tiled_weight_bytes(out, in, gated, groups);
  if (!bytes) return set_error(ODS_EINVAL, "ods_tile_weight: out %d, in %d, gated %d, groups %d", out, in, gated, groups);
  if (!src || !dst) return set_error(ODS_EINVAL, "ods_tile_weight: null pointer");
  if (!aligned16(src) || !aligned16(dst)) return set_error(ODS_EINVAL, "ods_tile_weight: pointers must be 16-byte aligned");
  const size_t src_bytes = (size_t)groups * (gated ? 2 : 1) * out * in * 2;
  const uintptr_t s0 = (uintptr_t)src, d0 = (uintptr_t)dst;
  if (s0 < d0 + bytes && d0 < s0 + src_bytes) return set_error(ODS_EINVAL, "ods_tile_weight: src and dst overlap");
  const hipError_t e = launch_tile_weight((const uint16_t *)src, (uint16_t *)dst, out, in, gated != 0, groups, stream);
  if (e != hipSuccess) return set_error(ODS_EHIP, "ods_tile_weight: %s", hipGetErrorString(e));
  clear_error();
  return ODS_OK;
}

ods_status ods_attn_stage(const ods_block *blk, int32_t layer, const ods_batch *batch, ods_state *state,
                          hipStream_t stream) {
  ods_status rc = check_block(blk);
  if (rc != ODS_OK) return rc;
  if (layer < 0 || layer >= blk->n_layers) return set_error(ODS_ERANGE, "layer %d outside [0, %d)", layer, blk->n_layers);
  const int off = layer_offset(blk, layer);
  return ods_run_partition(blk, off, off + 6, batch, state, stream);
}

ods_status ods_ffn_stage(const ods_block *blk, int32_t layer, const ods_batch *batch, ods_state *state,
                         hipStream_t stream) {
  ods_status rc = check_block(blk);
  if (rc != ODS_OK) return rc;
  if (layer < 0 || layer >= blk->n_layers) return set_error(ODS_ERANGE, "layer %d outside [0, %d)", layer, blk->n_layers);
  const int off = layer_offset(blk, layer);
  return ods_run_partition(blk, off + 6, off + layer_num_ops(blk->layers[layer].cfg), batch, state, stream);
}

ods_status ods_partition_graph(const ods_block *blk, int32_t op_begin, int32_t op_end, const ods_batch *batch,
                               ods_state *state, hipGraphExec_t *exec) {
  return capture(exec, [&](hipStream_t s) { return ods_run_partition(blk, op_begin, op_end, batch, state, s); });
}

ods_status ods_draft_graph(const ods_block *blk, int32_t op_begin, int32_t op_end, const ods_batch *batch,
                           const ods_draft *draft, ods_state *state, hipGraphExec_t *exec) {
  return capture(exec, [&](hipStream_t s) { return ods_run_draft(blk, op_begin, op_end, batch, draft, state, s); });
}

ods_status ods_graph_launch(hipGraphExec_t exec, hipStream_t stream) {
  if (!exec) return set_error(ODS_EINVAL, "exec is null");
  const hipError_t e = hipGraphLaunch(exec, stream);
  if (e != hipSuccess) return set_error(ODS_EHIP, "hipGraphLaunch: %s", hipGetErrorString(e));
  clear_error();
  return ODS_OK;
}

ods_status ods_graph_destroy(hipGraphExec_t exec) {
  if (!exec) return ODS_OK;
  const hipError_t e = hipGraphExecDestroy(exec);
  if (e != hipSuccess) return set_error(ODS_EHIP, "hipGraphExecDestroy: %s", hipGetErrorString(e));
  clear_error();
  return ODS_OK;
}

ods_status ods_rope_rows(const ods_rope *rope, const void *x, int64_t x_stride, void *y, int64_t y_stride,
                         int32_t rows, int32_t heads, const int32_t *pos, hipStream_t stream) {
  const ods_status rc = check_rope_rows(rope, x, x_stride, y, y_stride, rows, heads, pos);
  if (rc != ODS_OK) return rc;
  const hipError_t e = launch_rope_rows(*rope, (const uint16_t *)x, x_stride, (uint16_t *)y, y_stride, rows, heads, pos,
                                        stream);
  if (e != hipSuccess) return set_error(ODS_EHIP, "ods_rope_rows: %s", hipGetErrorString(e));
  clear_error();
  return ODS_OK;
}

size_t ods_draft_workspace_bytes(const ods_block *blk, const ods_batch *batch, const ods_draft *draft) {
  if (check_block(blk) != ODS_OK || check_draft_sizes(blk, 0, num_ops(blk), batch, draft) != ODS_OK) return 0;
  return draft_ws_most(blk, batch, draft, num_cus());
}

ods_status ods_run_draft(const ods_block *blk, int32_t op_begin, int32_t op_end, const ods_batch *batch,
                         const ods_draft *draft, ods_state *st, hipStream_t stream) {
  const int cus = num_cus();
  ods_status rc = validate_draft(blk, op_begin, op_end, batch, draft, st, cus);
  if (rc != ODS_OK) return rc;
  if (batch->batch == 0 || draft->rows == 0) {
    clear_error();
    return ODS_OK;
  }
  const bool trace = trace_on();
  const ods_batch rb = row_batch(batch, draft);
  for (int g = op_begin; g < op_end;) {
    const DraftStep step = draft_step(blk, g, op_end);
    g = step.end;
    if (step.rows_only) {
      if ((rc = run_rows(blk, step.begin, step.end, &rb, st, cus, trace, stream)) != ODS_OK) return rc;
      continue;
    }
    const OpRef op = op_at(blk, step.begin);
    const DraftArgs a = draft_args(blk, op.layer, batch, draft, st);
    const hipError_t e =
        step.attn ? launch_tree_attention(a, tree_plan(blk->layers[op.layer].cfg, batch, draft, cus), st->ws, stream)
                  : launch_draft_rope_append(a, step.rope, step.append, stream);
    const char *what = step.rope && step.append ? "rope+kv_append" : op_kind_name(op.kind);
    if (trace)
      fprintf(stderr, "[ods] layer %d drafted %s B=%d rows=%d -> %s\n", op.layer, what, a.B, a.rows, hipGetErrorString(e));
    if (e != hipSuccess)
      return set_error(ODS_EHIP, "launch of drafted %s (layer %d) failed: %s", what, op.layer, hipGetErrorString(e));
  }
  clear_error();
  return ODS_OK;
}

ods_status ods_kv_copy_pages(const ods_block *blk, int32_t layer_begin, int32_t layer_end, const int32_t *pairs,
                             int32_t n_pairs, hipStream_t stream) {
  const ods_status rc = check_pools(blk, layer_begin, layer_end, "ods_kv_copy_pages");
  if (rc != ODS_OK) return rc;
  if (n_pairs < 0) return set_error(ODS_EINVAL, "ods_kv_copy_pages: %d pairs", n_pairs);
  if (n_pairs > 0) {
    if (!pairs || !aligned16(pairs)) return set_error(ODS_EINVAL, "ods_kv_copy_pages: pairs is null or not 16-byte aligned");
    const hipError_t e = each_pool_set(blk, layer_begin, layer_end, nullptr, [&](const PoolSet &set, int n) {
      return launch_copy_pages(set, n, pairs, n_pairs, stream);
    });
    if (e != hipSuccess) return set_error(ODS_EHIP, "ods_kv_copy_pages: %s", hipGetErrorString(e));
  }
  clear_error();
  return ODS_OK;
}

ods_status ods_kv_accept(const ods_block *blk, int32_t layer_begin, int32_t layer_end, const ods_batch *batch,
                         const ods_draft *draft, const int32_t *path, int32_t path_cols, const int32_t *path_len,
                         int32_t *ctx_out, hipStream_t stream) {
  const ods_status rc = check_accept(blk, layer_begin, layer_end, batch, draft, path, path_cols, path_len, ctx_out);
  if (rc != ODS_OK) return rc;
  if (batch->batch > 0) {
    AcceptArgs a{};
    a.B = batch->batch; a.rows = draft->rows; a.max_rows = draft->max_rows; a.path_cols = path_cols;
    a.row_off = draft->row_off; a.ctx_lens = batch->ctx_lens; a.path = path; a.path_len = path_len;
    int max_kv = 0;
    for (int l = layer_begin; l < layer_end; ++l) max_kv = blk->layers[l].cfg.n_kv > max_kv ? blk->layers[l].cfg.n_kv : max_kv;
    const bool in_place = ctx_out == batch->ctx_lens;
    int32_t *out = in_place ? nullptr : ctx_out;  // written by the first set's launch
    hipError_t e = each_pool_set(blk, layer_begin, layer_end, batch, [&](const PoolSet &set, int n) {
      const hipError_t rc = launch_accept(a, set, n, max_kv, out, stream);
      out = nullptr;
      return rc;
    });
    if (e == hipSuccess && in_place) e = launch_accept_ctx(a, ctx_out, stream);
    if (e != hipSuccess) return set_error(ODS_EHIP, "ods_kv_accept: %s", hipGetErrorString(e));
  }
  clear_error();
  return ODS_OK;
}

}  // extern "C"
