// Attention of drafted rows where groups of sequences share a prefix of the
// cache: the prefix for all rows of a group at once, then each sequence's own
// tokens on top of it.
#include "tree_attention.hpp"

namespace ods {

hipError_t launch_shared_attention(const DraftArgs &a, const SharedPlan &plan, void *ws, hipStream_t s) {
  TreeState state;
  state.acc = (float *)ws;
  state.ml = (float2 *)(state.acc + (size_t)a.rows * a.n_q * a.D);
  void *const records = (uint8_t *)ws + shared_state_bytes(a.rows, a.n_q, a.D);
  const hipError_t e = launch_part<kPrefix, false>(a, plan.prefix, records, state, s);
  if (e != hipSuccess) return e;
  return plan.tail.stream ? launch_part<kTail, true>(a, plan.tail, records, state, s)
                          : launch_part<kTail, false>(a, plan.tail, records, state, s);
}

}  // namespace ods
