// What the host checks of a drafted range cost and how its workspace is sized,
// for a build under AddressSanitizer and UndefinedBehaviorSanitizer. Device
// pointers are aligned addresses that are never dereferenced. Prints
// "draft_sizes_check OK".
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
#include <chrono>
#include <vector>

#include "../../paper_2609_14237_amd/csrc/plan.hpp"

using namespace ods;

#define CHECK(c)                                                                              \
  do {                                                                                        \
    if (!(c)) {                                                                               \
      fprintf(stderr, "CHECK failed at %s:%d: %s (%s)\n", __FILE__, __LINE__, #c, ods_last_error()); \
      exit(1);                                                                                \
    }                                                                                         \
  } while (0)

static void *const kFake = (void *)0x100000;

static ods_layer layer(ods_layer_cfg c, bool tiled) {
  ods_layer L;
  memset(&L, 0, sizeof(L));
  L.cfg = c;
  L.g_attn = L.w_qkv = L.w_o = L.g_ffn = L.w_gate_up = L.w_down = L.w_router = kFake;
  L.kv_pool = kFake;
  L.pool_pages = 1 << 20;
  L.weight_layout = tiled ? ODS_WEIGHTS_TILED : ODS_WEIGHTS_ROWS;
  return L;
}

static ods_state state(size_t ws_bytes) {
  ods_state st;
  memset(&st, 0, sizeof(st));
  st.resid = st.xn = st.qkv = st.o = st.hn = st.gu = st.act = st.xp = st.gu_p = st.act_p = st.yp = st.ws = kFake;
  st.logits = st.topk_w = (float *)kFake;
  st.topk_ids = st.perm = st.slot_pos = st.expert_off = (int32_t *)kFake;
  st.ws_bytes = ws_bytes;
  return st;
}

static ods_batch batch_of(int B, int pages) { return ods_batch{B, pages, (int32_t *)kFake, (int32_t *)kFake, 0, 0, nullptr}; }
static ods_draft draft_of(int rows, int max_rows) {
  return ods_draft{rows, max_rows, (int32_t *)kFake, (int32_t *)kFake, (uint64_t *)kFake, nullptr};
}

template <typename F>
static double best_us(F f) {
  double best = 1e30;
  for (int i = 0; i < 7; ++i) {
    const auto t0 = std::chrono::steady_clock::now();
    f();
    best = std::min(best, std::chrono::duration<double, std::micro>(std::chrono::steady_clock::now() - t0).count());
  }
  return best;
}

// A deep block's drafted range costs a small multiple of what the decode step's checks do, whatever the depth: the
// workspace is worked out once a call. (Worked out at every attention operator: 63 times as long at 80 layers.)
static void check_cost_of_a_deep_block() {
  const ods_layer_cfg c{4096, 32, 8, 128, 14336, 0, 0, 0, 0, 1e4f, 1e-6f};
  std::vector<ods_layer> ls(80, layer(c, true));
  const ods_block blk{(int)ls.size(), ls.data()};
  const int n = num_ops(&blk);
  const ods_state st = state((size_t)1 << 40);
  const ods_batch b = batch_of(64, 256);
  const ods_draft d = draft_of(512, 8);
  const double decode = best_us([&] { CHECK(validate_range(&blk, 0, n, &b, &st, 256) == ODS_OK); });
  const double drafted = best_us([&] { CHECK(validate_draft(&blk, 0, n, &b, &d, &st, 256) == ODS_OK); });
  CHECK(drafted < 12 * decode);
}

// The need of the whole range counts wherever in it the attention stands, and not for a range without a GEMM or attention.
static void check_short_workspaces() {
  const ods_layer_cfg c{2048, 16, 8, 128, 8192, 0, 0, 0, 0, 1e4f, 1e-6f};
  std::vector<ods_layer> ls(2, layer(c, false));
  const ods_block blk{2, ls.data()};
  const ods_batch b = batch_of(8, 40);
  const ods_draft d = draft_of(40, 5);
  for (int a = 0; a < 20; ++a)
    for (int e = a + 1; e <= 20; ++e) {
      const size_t need = draft_ws_bytes(&blk, a, e, &b, &d, 256);
      ods_state st = state(need);
      CHECK(validate_draft(&blk, a, e, &b, &d, &st, 256) == ODS_OK);
      bool attn = false;
      for (int g = a; g < e; ++g) attn |= op_at(&blk, g).kind == K_ATTN_CORE;
      st.ws_bytes = need - 1;
      if (attn) CHECK(validate_draft(&blk, a, e, &b, &d, &st, 256) == ODS_ENOMEM);
      st = state(0);
      st.ws = nullptr;
      if (e - a == 1 && (op_at(&blk, a).kind == K_ROPE || op_at(&blk, a).kind == K_KV_APPEND || op_at(&blk, a).kind == K_ATTN_NORM))
        CHECK(validate_draft(&blk, a, e, &b, &d, &st, 256) == ODS_OK);
    }
}

int main() {
  check_cost_of_a_deep_block();
  check_short_workspaces();
  printf("draft_sizes_check OK\n");
  return 0;
}
