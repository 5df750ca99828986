// Host side of rotary positions, drafted rows and the page operators: the
// frequency table, argument checks, workspace sizing, and the cut of a drafted
// operator range into row-wise runs and drafted KV operators. Plain C++, free
// of HIP calls; nothing here allocates.
#include <math.h>

#include <algorithm>

#include "plan.hpp"

namespace ods {

namespace {

bool aligned16(const void *p) { return ((uintptr_t)p & 15u) == 0; }
bool positive(double v) { return v > 0.0 && std::isfinite(v); }

ods_status check_ptr(const void *p, const char *who, const char *name) {
  if (!p) return set_error(ODS_EINVAL, "%s: %s is null", who, name);
  if (!aligned16(p)) return set_error(ODS_EINVAL, "%s: %s is not 16-byte aligned", who, name);
  return ODS_OK;
}

// Batch and draft fields that need no operator: counts, and what the kernels index by.
ods_status check_counts(const ods_batch *batch, const ods_draft *draft) {
  if (batch->batch < 0 || batch->ring_pages < 0) return set_error(ODS_EINVAL, "negative batch or ring_pages");
  if (draft->rows < 0) return set_error(ODS_EINVAL, "negative draft rows");
  if (draft->max_rows < 1 || draft->max_rows > ODS_DRAFT_MAX_ROWS)
    return set_error(ODS_EINVAL, "draft max_rows %d (need 1 .. %d)", draft->max_rows, ODS_DRAFT_MAX_ROWS);
  if (batch->batch > kMaxAttnBatch)
    return set_error(ODS_EUNSUPPORTED, "drafted rows support batch <= %d, got %d", kMaxAttnBatch, batch->batch);
  // all that the sequences can have; the row-wise operators' launches hold fewer than 2^24 workgroups
  if (draft->rows > kMaxAttnBatch * ODS_DRAFT_MAX_ROWS)
    return set_error(ODS_EUNSUPPORTED, "draft rows %d (at most %d)", draft->rows, kMaxAttnBatch * ODS_DRAFT_MAX_ROWS);
  return ODS_OK;
}

// The page table a layer's drafted KV operators use, and its ring.
ods_status check_table(const ods_layer &L, int layer, const ods_batch *batch, const ods_draft *draft) {
  const KvMap m = kv_map(L.cfg, batch);
  if (m.cols <= 0) return set_error(ODS_EINVAL, "max_pages must be positive");
  if ((int64_t)m.cols * ODS_PAGE_TOKENS > INT32_MAX) return set_error(ODS_ERANGE, "max_pages too large");
  if (m.ring > 0) {
    const int64_t need = ((int64_t)L.cfg.window + draft->max_rows + ODS_PAGE_TOKENS - 1) / ODS_PAGE_TOKENS + 1;
    if (m.ring < need)
      return set_error(ODS_EINVAL, "layer %d: ring_pages %d < ceil((window + max_rows) / 16) + 1 = %lld", layer, m.ring,
                       (long long)need);
  }
  const ods_status rc = check_ptr(m.table, "draft", m.ring > 0 ? "ring_table" : "page_table");
  if (rc != ODS_OK) return rc;
  if (L.pool_pages <= 0) return set_error(ODS_EINVAL, "layer %d: pool_pages <= 0", layer);
  return check_ptr(L.kv_pool, "draft", "kv_pool");
}

}  // namespace

// ---------------------------------------------------------------- rotary positions

ods_status check_rope(const ods_rope *r, const char *who, bool need_freqs) {
  if (!r) return set_error(ODS_EINVAL, "%s: null rope", who);
  if (r->head_dim <= 0) return set_error(ODS_EINVAL, "%s: head_dim %d", who, r->head_dim);
  if (r->head_dim % 8 != 0 || r->head_dim > 256)
    return set_error(ODS_EUNSUPPORTED, "%s: head_dim %d (supported: multiples of 8 up to 256)", who, r->head_dim);
  if (r->rotary_dim < 2 || r->rotary_dim > r->head_dim || r->rotary_dim % 2 != 0)
    return set_error(ODS_EINVAL, "%s: rotary_dim %d (need even, 2 .. head_dim %d)", who, r->rotary_dim, r->head_dim);
  if (r->interleaved != 0 && r->interleaved != 1) return set_error(ODS_EINVAL, "%s: interleaved %d", who, r->interleaved);
  if (r->scaling < ODS_ROPE_PLAIN || r->scaling > ODS_ROPE_INDEX)
    return set_error(ODS_EINVAL, "%s: scaling %d", who, r->scaling);
  if (!positive(r->theta) || !std::isfinite(r->amplitude))
    return set_error(ODS_EINVAL, "%s: theta must be positive and amplitude finite", who);
  if (r->scaling != ODS_ROPE_PLAIN && !positive(r->factor)) return set_error(ODS_EINVAL, "%s: factor must be positive", who);
  if (r->scaling == ODS_ROPE_ROTATIONS || r->scaling == ODS_ROPE_INDEX) {
    if (!positive(r->orig_ctx) || !positive(r->turns_lo) || !std::isfinite(r->turns_hi) || !(r->turns_hi > r->turns_lo))
      return set_error(ODS_EINVAL, "%s: need orig_ctx > 0 and turns_hi > turns_lo > 0", who);
    if (r->scaling == ODS_ROPE_INDEX && r->theta == 1.0)
      return set_error(ODS_EINVAL, "%s: theta 1 has no index scale", who);
  }
  if (need_freqs) return check_ptr(r->freqs, who, "freqs");
  return ODS_OK;
}

ods_status check_rope_rows(const ods_rope *r, const void *x, int64_t xs, const void *y, int64_t ys, int rows, int heads,
                           const int32_t *pos) {
  const char *who = "ods_rope_rows";
  ods_status rc = check_rope(r, who, true);
  if (rc != ODS_OK) return rc;
  if (rows < 0 || heads < 0) return set_error(ODS_EINVAL, "%s: rows %d, heads %d", who, rows, heads);
  if (rows == 0 || heads == 0) return ODS_OK;
  if ((rc = check_ptr(x, who, "x")) != ODS_OK || (rc = check_ptr(y, who, "y")) != ODS_OK) return rc;
  if (!pos || ((uintptr_t)pos & 3u)) return set_error(ODS_EINVAL, "%s: pos is null or not 4-byte aligned", who);
  const int64_t width = (int64_t)heads * r->head_dim;
  if (width > INT32_MAX) return set_error(ODS_EUNSUPPORTED, "%s: rows of %lld values", who, (long long)width);
  if (xs % 8 != 0 || ys % 8 != 0 || xs < width || ys < width)
    return set_error(ODS_EINVAL, "%s: strides %lld, %lld (need multiples of 8, at least %lld)", who, (long long)xs,
                     (long long)ys, (long long)width);
  if (xs > INT64_MAX / 4 / rows || ys > INT64_MAX / 4 / rows) return set_error(ODS_EINVAL, "%s: strides too large", who);
  const uintptr_t a = (uintptr_t)x, b = (uintptr_t)y;
  if (a == b && (xs == ys || rows == 1)) return ODS_OK;
  const uintptr_t ax = a + (uintptr_t)(((int64_t)(rows - 1) * xs + width) * 2);
  const uintptr_t bx = b + (uintptr_t)(((int64_t)(rows - 1) * ys + width) * 2);
  if (a < bx && b < ax) {  // the spans meet: fine only as columns of the same rows that lie beside each other
    const int64_t gap = (a > b ? (int64_t)(a - b) : (int64_t)(b - a)) / 2 % xs;
    if (xs != ys || gap < width || gap > xs - width) return set_error(ODS_EINVAL, "%s: x and y overlap", who);
  }
  return ODS_OK;
}

// ---------------------------------------------------------------- drafted ranges

DraftStep draft_step(const ods_block *blk, int begin, int op_end) {
  DraftStep s{};
  s.begin = begin;
  s.end = begin + 1;
  const OpKind k = op_at(blk, begin).kind;
  if (!is_kv_op(k)) {
    s.rows_only = true;
    while (s.end < op_end && !is_kv_op(op_at(blk, s.end).kind)) ++s.end;
    return s;
  }
  s.rope = k == K_ROPE;
  s.append = k == K_KV_APPEND;
  s.attn = k == K_ATTN_CORE;
  if (s.rope && s.end < op_end) {  // kv_append follows rope in every layer: one launch
    s.append = true;
    ++s.end;
  }
  return s;
}

TreePlan tree_plan(const ods_layer_cfg &c, const ods_batch *batch, const ods_draft *draft, int cus) {
  TreePlan p;
  const int64_t nq = (int64_t)draft->max_rows * (c.n_q / c.n_kv);
  p.qt = 16;
  while (p.qt < nq && p.qt < 256) p.qt *= 2;
  p.max_qt = (int)((nq + p.qt - 1) / p.qt);
  // Tokens of a sequence a layer may read: the table's, or a window with the drafted rows. The host sees no contexts, so a
  // table wider than they need is planned for as if they filled it: right, but of the rules below no_cut needs a table of 864
  // tokens at most (4 sequences of 128 tokens: 7.9 us up to 54 pages, 9.9 at 64, 10.7 at 2048), and a wide one reads past the
  // caches what they would hold (64 sequences of 300 tokens, 4 rows: 18.9 us in 19 pages, 21.0 in 2048).
  int64_t tokens = (int64_t)kv_map(c, batch).cols * ODS_PAGE_TOKENS;
  if (c.window > 0) tokens = std::min(tokens, (int64_t)c.window + draft->max_rows + 64);
  const int64_t units = (int64_t)batch->batch * c.n_kv * p.max_qt * ((tokens + 31) / 32 + 1);
  p.units_ok = units < (int64_t)1 << 30;
  // One sequence of 3000 tokens, us at 2, 4 and 6: 16 rows 17.3, 16.8, 17.0, 32 rows 24.7, 23.8, 24.1. Nearly level: what a
  // shorter range saves in tiles its record costs.
  p.min_tiles = 4;
  cus = std::max(cus, 1);
  // 128 columns as four waves of 32: half the LDS reads of eight waves of 16, which read every tile once each. It pays
  // where the tasks are nearly equal and need no dealing (64 sequences of 2304 tokens, 24 rows: 112 us with two workgroups a
  // compute unit, eight waves 139), and a window makes them so (32 sequences, 1024 tokens of each: 42 to 45 us, eight waves
  // 44). Contexts that differ are better dealt out to workgroups of eight (64 of 512 to 4096: 129 us, 139). A compute unit
  // runs one such workgroup, with half its LDS, until per_cu below is 2.
  p.equal = p.qt == 128 && c.window > 0;
  // Workgroups per compute unit. Up to 16 columns are one wave's work, and two have room (64 sequences of up to 4096
  // tokens, 4 rows, us at 1, 2 and 4: D = 128 124, 121, 126; D = 64 at 4 and 8 68). The workgroups of two or four waves
  // fit twice, which pays once a range is long, 64 units with both (64 sequences of 2304 tokens, 16 rows: 102 us, one each 119;
  // 8 of 2000 to 8000, 12 rows: 44 and 42; behind a window of 1024 with 8 heads from 114 sequences on: 128 of them 129 us, 64
  // with one each 83). Eight waves have all the LDS.
  const bool small = p.qt <= 64 || p.equal;
  int per_cu = p.qt <= 16 ? 256 / c.head_dim : 1;
  if (p.qt > 16 && small && units >= (int64_t)2 * cus * 64) per_cu = 2;
  p.grid = (int)std::max<int64_t>(1, std::min<int64_t>((int64_t)cus * per_cu, (units + p.min_tiles - 1) / p.min_tiles));
  // Each tile is read once, and all of them are more than the last-level cache holds (256 MB): past the caches (64
  // sequences of 9216 tokens, 4 rows: 362 us, through them 402; 64 ragged ones 129, 138). What fits may still be there
  // (16 sequences of 1000 to 2000 tokens, read again: 32 us, 34 past the caches), and query tiles read the same tiles again.
  p.stream = p.max_qt == 1 && units * 32 * c.head_dim * 4 > (int64_t)256 << 20;
  // One task a range, none long enough to be cut, whatever the contexts (4 short sequences: 7 us, with the second launch
  // 10). Longer tasks may still all be whole (32 behind a window of 1024: 36 tiles at most), or dealt out: then the
  // second launch finds nothing to join, 3 to 4 us.
  const int64_t tasks = (int64_t)batch->batch * c.n_kv * p.max_qt;
  p.no_cut = tasks <= p.grid && (tokens + 31) / 32 + 1 <= p.min_tiles + kSplitTiles;
  // Joining a task of many ranges by quarters of a column (one sequence: 18 us, by whole waves 23), or of few by whole waves
  // (64 ragged sequences cut into even ranges: 157 us, by quarters 173).
  p.split_join = p.grid > 6 * (int64_t)batch->batch * c.n_kv * p.max_qt;
  return p;
}

// Per range: a descriptor, and two records of qt columns (maximum and denominator, then the sums).
size_t tree_ws_bytes(const TreePlan &p, int D) {
  return (size_t)p.grid * kTreeDescBytes + (size_t)2 * p.grid * p.qt * (D + 2) * sizeof(float);
}

ods_batch row_batch(const ods_batch *batch, const ods_draft *draft) {
  ods_batch b = *batch;
  b.batch = draft->rows;
  b.split_pages = 0;
  return b;
}

size_t draft_ws_bytes(const ods_block *blk, int op_begin, int op_end, const ods_batch *batch, const ods_draft *draft,
                      int cus) {
  const ods_batch rb = row_batch(batch, draft);
  size_t w = std::max<size_t>(256, range_ws_bytes(blk, op_begin, op_end, &rb, cus, false));
  for (int g = op_begin; g < op_end; ++g) {
    const OpRef op = op_at(blk, g);
    const ods_layer_cfg &c = blk->layers[op.layer].cfg;
    if (op.kind == K_ATTN_CORE) w = std::max(w, tree_ws_bytes(tree_plan(c, batch, draft, cus), c.head_dim));
  }
  return w;
}

size_t draft_ws_most(const ods_block *blk, const ods_batch *batch, const ods_draft *draft, int cus) {
  size_t w = std::max<size_t>(256, rows_ws_most(blk, draft->rows));
  for (int l = 0; l < blk->n_layers; ++l) {
    const ods_layer_cfg &c = blk->layers[l].cfg;
    auto take = [&](int max_rows) {
      ods_draft d = *draft;
      d.max_rows = max_rows;
      w = std::max(w, tree_ws_bytes(tree_plan(c, batch, &d, cus), c.head_dim));
    };
    // A query tile's width times the grid may be more for a narrower tree, of which more workgroups share a compute unit; of
    // the trees of one width the longest needs most.
    for (int qt = 16; qt <= 256; qt *= 2)
      if (qt / (c.n_q / c.n_kv) >= 1) take(std::min(draft->max_rows, qt / (c.n_q / c.n_kv)));
    take(draft->max_rows);
  }
  return w;
}

ods_status check_draft_sizes(const ods_block *blk, int op_begin, int op_end, const ods_batch *batch,
                             const ods_draft *draft) {
  if (!batch || !draft) return set_error(ODS_EINVAL, "null batch or draft");
  const ods_status rc = check_counts(batch, draft);
  if (rc != ODS_OK) return rc;
  for (int g = op_begin; g < op_end; ++g) {
    const OpRef op = op_at(blk, g);
    const ods_layer_cfg &c = blk->layers[op.layer].cfg;
    if (is_kv_op(op.kind) && (int64_t)draft->rows * c.n_q > INT32_MAX)
      return set_error(ODS_EUNSUPPORTED, "layer %d: draft rows * n_q exceeds 2^31", op.layer);
    if (op.kind == K_ATTN_CORE && !tree_plan(c, batch, draft, 1).units_ok)
      return set_error(ODS_EUNSUPPORTED, "layer %d: batch * n_kv * query tiles * window pages exceeds 2^30", op.layer);
  }
  return ODS_OK;
}

ods_status validate_draft(const ods_block *blk, int op_begin, int op_end, const ods_batch *batch, const ods_draft *draft,
                          const ods_state *st, int cus) {
  ods_status rc = check_block(blk);
  if (rc != ODS_OK) return rc;
  if (!batch || !draft || !st) return set_error(ODS_EINVAL, "null batch, draft or state");
  const int n_ops = num_ops(blk);
  if (op_begin < 0 || op_end > n_ops || op_begin >= op_end)
    return set_error(ODS_ERANGE, "operator range [%d, %d) outside [0, %d) or empty", op_begin, op_end, n_ops);
  if ((rc = check_draft_sizes(blk, op_begin, op_end, batch, draft)) != ODS_OK) return rc;
  if (batch->batch == 0 || draft->rows == 0) return ODS_OK;
  const ods_batch rb = row_batch(batch, draft);
  size_t need = 0;  // of the whole range: worked out once, at its first attention
  for (int g = op_begin; g < op_end;) {
    const DraftStep s = draft_step(blk, g, op_end);
    g = s.end;
    if (s.rows_only) {
      if ((rc = validate_range(blk, s.begin, s.end, &rb, st, cus, false)) != ODS_OK) return rc;
      continue;
    }
    const int layer = op_at(blk, s.begin).layer;
    const ods_layer &L = blk->layers[layer];
    const ods_layer_cfg &c = L.cfg;
    const char *who = op_kind_name(op_at(blk, s.begin).kind);
    if ((rc = check_ptr(st->qkv, who, "qkv")) != ODS_OK || (rc = check_ptr(batch->ctx_lens, who, "ctx_lens")) != ODS_OK ||
        (rc = check_ptr(draft->row_off, who, "row_off")) != ODS_OK)
      return rc;
    if ((s.rope || s.attn) && (rc = check_ptr(draft->depth, who, "depth")) != ODS_OK) return rc;
    if (s.rope && draft->rope) {
      if ((rc = check_rope(&draft->rope[layer], who, true)) != ODS_OK) return rc;
      if (draft->rope[layer].head_dim != c.head_dim)
        return set_error(ODS_EINVAL, "layer %d: rope of head_dim %d for heads of %d", layer, draft->rope[layer].head_dim,
                         c.head_dim);
    }
    if ((s.append || s.attn) && (rc = check_table(L, layer, batch, draft)) != ODS_OK) return rc;
    if (s.attn) {
      if ((rc = check_ptr(draft->mask, who, "mask")) != ODS_OK || (rc = check_ptr(st->o, who, "o")) != ODS_OK ||
          (rc = check_ptr(st->ws, who, "ws")) != ODS_OK)
        return rc;
      if (need == 0) need = draft_ws_bytes(blk, op_begin, op_end, batch, draft, cus);
      if (st->ws_bytes < need) return set_error(ODS_ENOMEM, "workspace %zu bytes < required %zu", st->ws_bytes, need);
    }
  }
  return ODS_OK;
}

// ---------------------------------------------------------------- page operators

ods_status check_pools(const ods_block *blk, int layer_begin, int layer_end, const char *who) {
  ods_status rc = check_block(blk);
  if (rc != ODS_OK) return rc;
  if (layer_begin < 0 || layer_end > blk->n_layers || layer_begin >= layer_end)
    return set_error(ODS_ERANGE, "%s: layers [%d, %d) outside [0, %d) or empty", who, layer_begin, layer_end,
                     blk->n_layers);
  for (int l = layer_begin; l < layer_end; ++l) {
    if ((rc = check_ptr(blk->layers[l].kv_pool, who, "kv_pool")) != ODS_OK) return rc;
    if (blk->layers[l].pool_pages <= 0) return set_error(ODS_EINVAL, "%s: layer %d: pool_pages <= 0", who, l);
  }
  return ODS_OK;
}

ods_status check_accept(const ods_block *blk, int layer_begin, int layer_end, const ods_batch *batch,
                        const ods_draft *draft, const int32_t *path, int path_cols, const int32_t *path_len,
                        const int32_t *ctx_out) {
  const char *who = "ods_kv_accept";
  ods_status rc = check_pools(blk, layer_begin, layer_end, who);
  if (rc != ODS_OK) return rc;
  if (!batch || !draft) return set_error(ODS_EINVAL, "%s: null batch or draft", who);
  if ((rc = check_counts(batch, draft)) != ODS_OK) return rc;
  if (path_cols < 1 || path_cols > ODS_DRAFT_MAX_ROWS)
    return set_error(ODS_EINVAL, "%s: path_cols %d (need 1 .. %d)", who, path_cols, ODS_DRAFT_MAX_ROWS);
  if (batch->batch == 0) return ODS_OK;
  if ((rc = check_ptr(path, who, "path")) != ODS_OK || (rc = check_ptr(path_len, who, "path_len")) != ODS_OK ||
      (rc = check_ptr(batch->ctx_lens, who, "ctx_lens")) != ODS_OK ||
      (rc = check_ptr(draft->row_off, who, "row_off")) != ODS_OK ||
      (ctx_out && (rc = check_ptr(ctx_out, who, "ctx_out")) != ODS_OK))
    return rc;
  const uintptr_t out = (uintptr_t)ctx_out, out_end = out + (uintptr_t)batch->batch * 4;
  auto meets = [&](const int32_t *p, int64_t count) {
    return ctx_out && out < (uintptr_t)p + (uintptr_t)(count * 4) && (uintptr_t)p < out_end;
  };
  if ((ctx_out != batch->ctx_lens && meets(batch->ctx_lens, batch->batch)) || meets(path_len, batch->batch) ||
      meets(path, (int64_t)batch->batch * path_cols) || meets(draft->row_off, (int64_t)batch->batch + 1))
    return set_error(ODS_EINVAL, "%s: ctx_out overlaps an array the call reads", who);
  for (int l = layer_begin; l < layer_end; ++l)
    if ((rc = check_table(blk->layers[l], l, batch, draft)) != ODS_OK) return rc;
  return ODS_OK;
}

}  // namespace ods

// ---------------------------------------------------------------- C ABI (host-only entry points)

using namespace ods;

extern "C" {

ods_status ods_rope_freqs(const ods_rope *rope, double *freqs_host) {
  const ods_status rc = check_rope(rope, "ods_rope_freqs", false);
  if (rc != ODS_OK) return rc;
  if (!freqs_host) return set_error(ODS_EINVAL, "ods_rope_freqs: null table");
  const int d = rope->rotary_dim;
  const double turn = 6.283185307179586;
  double theta = rope->theta;
  if (rope->scaling == ODS_ROPE_BASE && d > 2) theta *= pow(rope->factor, (double)d / (d - 2));
  // pair index (of d / 2, fractional) whose angle turns n times over the first context
  auto pair_of = [&](double n) { return d * log(rope->orig_ctx / (n * turn)) / (2.0 * log(rope->theta)); };
  double lo = 0.0, hi = 0.0;
  if (rope->scaling == ODS_ROPE_INDEX) {
    lo = std::max(floor(pair_of(rope->turns_hi)), 0.0);
    hi = std::min(ceil(pair_of(rope->turns_lo)), d - 1.0);
  }
  for (int i = 0; i < d / 2; ++i) {
    const double f = pow(theta, -2.0 * i / d);
    double keep = 1.0;  // share of the unscaled frequency
    if (rope->scaling == ODS_ROPE_LINEAR) keep = 0.0;
    if (rope->scaling == ODS_ROPE_ROTATIONS)
      keep = (rope->orig_ctx * f / turn - rope->turns_lo) / (rope->turns_hi - rope->turns_lo);
    if (rope->scaling == ODS_ROPE_INDEX) keep = 1.0 - (i - lo) / std::max(hi - lo, 0.001);
    keep = std::min(1.0, std::max(0.0, keep));
    freqs_host[i] = keep == 1.0 ? f : f * keep + f / rope->factor * (1.0 - keep);
  }
  clear_error();
  return ODS_OK;
}

}  // extern "C"
