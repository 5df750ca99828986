// Exercises the HIP-free host parts of rotary positions, drafted rows and the
// page bookkeeping for a build under AddressSanitizer and
// UndefinedBehaviorSanitizer. Device pointers are aligned addresses that are
// never dereferenced. Prints "draft_check OK".
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <random>
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

static ods_layer layer(int n_q, int n_kv, int D, int window, int experts) {
  ods_layer L;
  memset(&L, 0, sizeof(L));
  L.cfg = ods_layer_cfg{256, n_q, n_kv, D, experts ? 0 : 512, experts, experts ? 2 : 0, experts ? 128 : 0, window, 1e4f, 1e-6f};
  L.g_attn = L.w_qkv = L.w_o = L.g_ffn = L.w_gate_up = L.w_down = L.w_router = kFake;
  L.kv_pool = kFake;
  L.pool_pages = 1 << 20;
  return L;
}

static void drafted_ranges() {
  ods_state st;
  memset(&st, 0, sizeof(st));
  st.resid = st.xn = st.qkv = st.o = st.hn = st.gu = st.act = st.xp = st.gu_p = st.act_p = st.yp = st.ws = kFake;
  st.logits = st.topk_w = (float *)kFake;
  st.topk_ids = st.perm = st.slot_pos = st.expert_off = (int32_t *)kFake;
  for (int D : {64, 128})
    for (int n_kv : {1, 2, 8})
      for (int group : {1, 4, 16}) {
        std::vector<ods_layer> ls = {layer(n_kv * group, n_kv, D, 0, 0), layer(n_kv * group, n_kv, D, 100, 4)};
        const ods_block blk{2, ls.data()};
        const int n = num_ops(&blk);
        CHECK(n == 24);
        for (int B : {1, 3, 64, 4096})
          for (int max_rows : {1, 5, 64, 65, 256})
            for (int pages : {1, 40, 2048}) {
              const int64_t want = (int64_t)B * max_rows;
              const int rows = (int)(want < 20000 ? want : 20000);
              const ods_batch b{B, pages, (int32_t *)kFake, (int32_t *)kFake, 0, 0, nullptr};
              const ods_draft d{rows, max_rows, (int32_t *)kFake, (int32_t *)kFake, (uint64_t *)kFake, nullptr};
              for (int cus : {1, 256}) {
                const size_t ws = draft_ws_bytes(&blk, 0, n, &b, &d, cus);
                CHECK(ws >= 256);
                st.ws_bytes = ws;
                for (int a = 0; a < n; ++a)
                  for (int e = a + 1; e <= n; ++e) {
                    const ods_status rc = validate_draft(&blk, a, e, &b, &d, &st, cus);
                    CHECK(rc == ODS_OK || rc == ODS_EUNSUPPORTED);
                    int at = a;
                    while (at < e) {  // the steps tile the range, each of one kind
                      const DraftStep s = draft_step(&blk, at, e);
                      CHECK(s.begin == at && s.end > at && s.end <= e);
                      CHECK(s.rows_only + (s.rope || s.append) + s.attn == 1);
                      for (int g = s.begin; g < s.end; ++g) CHECK(is_kv_op(op_at(&blk, g).kind) != s.rows_only);
                      at = s.end;
                    }
                  }
              }
            }
      }
}

static void rope_tables() {
  for (int scaling = 0; scaling <= 4; ++scaling)
    for (int hd : {8, 64, 256})
      for (int rd = 2; rd <= hd; rd += 2) {
        ods_rope r{hd, rd, 0, scaling, 1e4, 8.0, 4096.0, 32.0, 1.0, 1.f, nullptr};
        std::vector<double> f(rd / 2, -1.0);
        CHECK(ods_rope_freqs(&r, f.data()) == ODS_OK);
        for (double v : f) CHECK(v > 0.0 && v <= 1.0);
      }
}

static void pages() {
  std::mt19937 rng(7);
  const int rows = 5, cols = 6, pool = 17;
  std::vector<int32_t> refs(pool), ids(pool), table(rows * cols, -1), tokens(rows, 0), pairs(2 * pool);
  ods_pages p{pool, refs.data(), ids.data(), 0};
  CHECK(ods_pages_init(&p, nullptr, 0, 0) == ODS_OK && p.n_free == pool);
  for (int i = 0; i < 20000; ++i) {
    const int b = rng() % rows, op = rng() % 5;
    int32_t *row = &table[b * cols], pair[2], n = -1;
    if (op < 2) {
      const int want = rng() % (cols * 16 + 4);
      const ods_status rc = ods_pages_resize(&p, row, cols, tokens[b], want, pair, &n);
      CHECK(rc == ODS_OK || rc == ODS_ENOMEM || (rc == ODS_ERANGE && want > cols * 16));
      if (rc == ODS_OK) tokens[b] = want;
    } else if (op == 2) {
      const int c = rng() % rows;
      const ods_status rc = ods_pages_fork(&p, &table[c * cols], row, cols, tokens[c]);
      CHECK((rc == ODS_OK) == (tokens[b] == 0));
      if (rc == ODS_OK) tokens[b] = tokens[c];
    } else if (op == 3) {
      CHECK(ods_pages_release(&p, row, cols) == ODS_OK);
      tokens[b] = 0;
    } else {
      CHECK(ods_pages_compact(&p, table.data(), rows, cols, pairs.data(), rng() % (pool + 1), &n) == ODS_OK);
    }
    int64_t held = 0;
    std::vector<int32_t> count(pool, 0);
    for (int32_t v : table)
      if (v >= 0) ++count[v];
    for (int v = 0; v < pool; ++v) {
      CHECK(count[v] == refs[v]);
      held += refs[v] > 0;
    }
    CHECK(held + p.n_free == pool);
  }
}

int main() {
  drafted_ranges();
  rope_tables();
  pages();
  printf("draft_check OK\n");
  return 0;
}
