// Host side of the verification of drafted tokens: argument checks,
// workspace. Plain C++, free of HIP calls.
#include "plan.hpp"

namespace ods {

VerifyWs verify_ws(int batch, int vocab) {
  VerifyWs w;
  w.chunks = (vocab + kVerifyChunk - 1) / kVerifyChunk;
  w.head = 0;
  w.list = (size_t)batch * 16;
  w.sums = w.list + (size_t)batch * ODS_DRAFT_MAX_ROWS * sizeof(double);
  w.bytes = w.sums + (size_t)batch * w.chunks * sizeof(double);
  return w;
}

ods_status check_verify(int batch, const ods_draft *draft, const ods_verify *v) {
  const char *who = "ods_draft_verify";
  if (!draft || !v) return set_error(ODS_EINVAL, "%s: null draft or verify", who);
  if (batch < 0 || draft->rows < 0) return set_error(ODS_EINVAL, "%s: batch %d, rows %d", who, batch, draft->rows);
  if (batch > kMaxAttnBatch) return set_error(ODS_EUNSUPPORTED, "%s: batch %d (at most %d)", who, batch, kMaxAttnBatch);
  if (draft->max_rows < 1 || draft->max_rows > ODS_DRAFT_MAX_ROWS)
    return set_error(ODS_EINVAL, "%s: max_rows %d (need 1 .. %d)", who, draft->max_rows, ODS_DRAFT_MAX_ROWS);
  if (draft->rows > kMaxAttnBatch * ODS_DRAFT_MAX_ROWS)
    return set_error(ODS_EUNSUPPORTED, "%s: rows %d (at most %d)", who, draft->rows, kMaxAttnBatch * ODS_DRAFT_MAX_ROWS);
  if (v->vocab < 1 || v->vocab > ODS_VERIFY_MAX_VOCAB)
    return set_error(ODS_EINVAL, "%s: vocab %d (need 1 .. %d)", who, v->vocab, ODS_VERIFY_MAX_VOCAB);
  if (v->dtype != ODS_PROBS_F32 && v->dtype != ODS_PROBS_BF16) return set_error(ODS_EINVAL, "%s: dtype %d", who, v->dtype);
  if (v->path_cols < 1 || v->path_cols > ODS_DRAFT_MAX_ROWS)
    return set_error(ODS_EINVAL, "%s: path_cols %d (need 1 .. %d)", who, v->path_cols, ODS_DRAFT_MAX_ROWS);
  if (batch == 0) return ODS_OK;
  const uintptr_t one = v->dtype == ODS_PROBS_F32 ? 3u : 1u;
  const struct { const char *name; const void *p; uintptr_t low; bool need; } arrays[] = {
      {"row_off", draft->row_off, 15u, true},
      {"target", v->target, one, draft->rows > 0}, {"proposal", v->proposal, one, false},
      {"tokens", v->tokens, 3u, draft->rows > 0}, {"parent", v->parent, 3u, draft->rows > 0},
      {"accept_u", v->accept_u, 3u, draft->rows > 0}, {"next_u", v->next_u, 3u, true},
      {"path", v->path, 3u, true}, {"path_len", v->path_len, 3u, true}, {"next_token", v->next_token, 3u, true},
      {"ws", v->ws, 15u, true}};
  for (const auto &a : arrays) {
    if (!a.p && a.need) return set_error(ODS_EINVAL, "%s: %s is null", who, a.name);
    if ((uintptr_t)a.p & a.low) return set_error(ODS_EINVAL, "%s: %s is not aligned", who, a.name);
  }
  const int64_t most = INT64_MAX / 8 / (draft->rows > 0 ? draft->rows : 1);
  if (v->target_stride < v->vocab || v->target_stride > most)
    return set_error(ODS_EINVAL, "%s: target_stride %lld for %d tokens", who, (long long)v->target_stride, v->vocab);
  if (v->proposal && (v->proposal_stride < v->vocab || v->proposal_stride > most))
    return set_error(ODS_EINVAL, "%s: proposal_stride %lld for %d tokens", who, (long long)v->proposal_stride, v->vocab);
  const size_t need = verify_ws(batch, v->vocab).bytes;
  if (v->ws_bytes < need) return set_error(ODS_ENOMEM, "%s: workspace %zu bytes < required %zu", who, v->ws_bytes, need);
  return ODS_OK;
}

}  // namespace ods

extern "C" {

size_t ods_verify_workspace_bytes(int32_t batch, int32_t vocab) {
  using namespace ods;
  if (batch < 0 || batch > kMaxAttnBatch || vocab < 1 || vocab > ODS_VERIFY_MAX_VOCAB) return 0;
  const size_t bytes = verify_ws(batch, vocab).bytes;
  return bytes > 16 ? bytes : 16;
}

}  // extern "C"
