// Exercises the HIP-free host parts of normalised heads, shared prefixes and the
// verification of drafted tokens for a build under AddressSanitizer and
// UndefinedBehaviorSanitizer. Device pointers are aligned addresses that are
// never dereferenced. Prints "serve_check OK".
#include <stdio.h>
#include <stdlib.h>
#include <string.h>

#include <algorithm>
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

// Plans of every shape: the kernels that launch them exist, parts of the workspace follow each other and fit.
static void shared_plans() {
  int taken = 0;
  for (int hd : {64, 128})
    for (int n_kv : {1, 2, 8})
      for (int group : {1, 3, 4, 16})
        for (int batch : {1, 2, 64, 512, 513, 4096})
          for (int max_rows : {1, 2, 4, 5, 16, 64, 65, 256})
            for (int pages : {1, 20, 2048})
              for (int groups : {1, 2, std::min(batch, 512)}) {
                if (groups > batch) continue;
                ods_layer L;
                memset(&L, 0, sizeof(L));
                L.cfg = ods_layer_cfg{256, n_kv * group, n_kv, hd, 512, 0, 0, 0, 0, 1e4f, 1e-6f};
                L.g_attn = L.w_qkv = L.w_o = L.g_ffn = L.w_gate_up = L.w_down = kFake;
                L.kv_pool = kFake;
                L.pool_pages = 1 << 20;
                const ods_block blk{1, &L};
                ods_batch b;
                memset(&b, 0, sizeof(b));
                b.batch = batch;
                b.max_pages = pages;
                b.ctx_lens = b.page_table = (int32_t *)kFake;
                const ods_shared shared{groups, (int32_t *)kFake, (int32_t *)kFake};
                ods_draft d;
                memset(&d, 0, sizeof(d));
                d.rows = batch * max_rows;
                d.max_rows = max_rows;
                d.row_off = d.depth = (int32_t *)kFake;
                d.mask = (uint64_t *)kFake;
                d.shared = &shared;
                const size_t need = draft_ws_bytes(&blk, 4, 5, &b, &d, 256);
                CHECK(draft_ws_most(&blk, &b, &d, 256) >= need);
                const bool takes = takes_shared(L.cfg, &b, &d);
                CHECK(takes == (max_rows * group <= 32 && (int64_t)batch * pages * 16 * n_kv * hd * 4 >= 128 << 20));
                taken += takes;
                if (!takes) {
                  d.shared = nullptr;
                  CHECK(!takes_shared(L.cfg, &b, &d) && draft_ws_bytes(&blk, 4, 5, &b, &d, 256) == need);
                  continue;
                }
                const SharedPlan p = shared_plan(L.cfg, &b, &d, 256);
                if (!p.units_ok) continue;
                CHECK(p.waves == 4 || p.waves == 8);
                CHECK(p.qtp == 32 * p.waves);
                CHECK(p.qtt == 16 || p.qtt == (p.waves == 8 ? 32 : 64));
                CHECK(p.qtt >= max_rows * group && p.grid >= 2 && p.grid <= 512);
                const SharedWs w = shared_ws(p, batch, d.rows, n_kv * group, n_kv, hd);
                const size_t at[] = {w.state[0], w.state_ml[0], w.state[1], w.state_ml[1], w.prefix, w.desc,
                                     w.rec_ml[0], w.rec_acc[0], w.rec_ml[1], w.rec_acc[1], w.bytes};
                for (size_t i = 0; i + 1 < sizeof(at) / sizeof(at[0]); ++i) CHECK(at[i] < at[i + 1] && at[i] % 16 == 0);
                CHECK(need >= w.bytes);
                ods_state st;
                memset(&st, 0, sizeof(st));
                st.qkv = st.o = st.ws = kFake;
                st.ws_bytes = need;
                CHECK(validate_draft(&blk, 4, 5, &b, &d, &st, 256) == ODS_OK);
                st.ws_bytes = need - 1;
                CHECK(validate_draft(&blk, 4, 5, &b, &d, &st, 256) == ODS_ENOMEM);
              }
  CHECK(taken > 100);
}

// Groups of random tables against what they promise.
static void groups() {
  std::mt19937 rng(1);
  for (int round = 0; round < 2000; ++round) {
    const int rows = rng() % 40, pages = 1 + rng() % 6;
    std::vector<int32_t> table((size_t)rows * pages), tokens(rows), off(rows + 1, -7), shared(std::max(rows, 1), -7);
    for (auto &x : table) x = (int)(rng() % 3) - (rng() % 8 == 0);
    for (auto &x : tokens) x = rng() % (pages * 16 + 1);
    int32_t n = -1;
    CHECK(ods_pages_shared(table.data(), rows, pages, tokens.data(), off.data(), shared.data(), &n) == ODS_OK);
    CHECK(n >= 0 && n <= rows && off[0] == 0 && off[n] == rows);
    for (int g = 0; g < n; ++g) {
      CHECK(off[g] < off[g + 1] && shared[g] >= 0 && shared[g] % 16 == 0);
      for (int r = off[g]; r < off[g + 1] && shared[g] > 0; ++r) {
        CHECK(tokens[r] >= shared[g]);
        for (int j = 0; j < shared[g] / 16; ++j)
          CHECK(table[(size_t)r * pages + j] >= 0 && table[(size_t)r * pages + j] == table[(size_t)off[g] * pages + j]);
      }
    }
  }
  const int rows = 3 * ODS_SHARED_GROUPS;  // pairs that share, a row between them: more groups than a call takes
  std::vector<int32_t> table(rows), tokens(rows, 16), off(rows + 1), shared(rows);
  for (int r = 0; r < rows; ++r) table[r] = r % 3 == 2 ? r : r / 3 * 3;
  int32_t n;
  CHECK(ods_pages_shared(table.data(), rows, 1, tokens.data(), off.data(), shared.data(), &n) == ODS_OK);
  CHECK(n == ODS_SHARED_GROUPS && off[n] < rows);
}

static void verify() {
  for (int batch : {1, 7, 4096})
    for (int vocab : {1, 1023, 1024, 1025, 128000, ODS_VERIFY_MAX_VOCAB}) {
      const VerifyWs w = verify_ws(batch, vocab);
      CHECK(w.head < w.list && w.list < w.sums && w.sums < w.bytes && w.list % 8 == 0 && w.sums % 8 == 0);
      CHECK((int64_t)w.chunks * kVerifyChunk >= vocab && ods_verify_workspace_bytes(batch, vocab) == w.bytes);
      ods_draft d;
      memset(&d, 0, sizeof(d));
      d.rows = batch * 4;
      d.max_rows = 4;
      d.row_off = (int32_t *)kFake;
      ods_verify v;
      memset(&v, 0, sizeof(v));
      v.vocab = vocab;
      v.target = kFake;
      v.target_stride = vocab;
      v.tokens = v.parent = (int32_t *)kFake;
      v.accept_u = v.next_u = (float *)kFake;
      v.path = v.path_len = v.next_token = (int32_t *)kFake;
      v.path_cols = 4;
      v.ws = kFake;
      v.ws_bytes = w.bytes;
      CHECK(check_verify(batch, &d, &v) == ODS_OK);
      --v.ws_bytes;
      CHECK(check_verify(batch, &d, &v) == ODS_ENOMEM);
    }
}

int main() {
  shared_plans();
  groups();
  verify();
  printf("serve_check OK\n");
  return 0;
}
