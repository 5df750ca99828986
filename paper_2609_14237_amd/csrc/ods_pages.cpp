// Page bookkeeping of the shared KV cache: holders, free list, growth with
// copy-on-write, forks and compaction. Host only, over caller memory (two
// scratch arrays of a compaction aside). Every call checks before it changes
// anything.
#include <algorithm>
#include <new>
#include <vector>

#include "plan.hpp"

using namespace ods;

namespace {

ods_status check_pages(const ods_pages *p, const char *who) {
  if (!p || !p->refs || !p->free_ids) return set_error(ODS_EINVAL, "%s: null pages", who);
  if (p->pool_pages < 1 || p->pool_pages > INT32_MAX)
    return set_error(ODS_EINVAL, "%s: pool_pages %lld", who, (long long)p->pool_pages);
  if (p->n_free < 0 || p->n_free > p->pool_pages)
    return set_error(ODS_EINVAL, "%s: n_free %lld of %lld pages", who, (long long)p->n_free, (long long)p->pool_pages);
  return ODS_OK;
}

int64_t pages_of(int32_t tokens) { return ((int64_t)tokens + ODS_PAGE_TOKENS - 1) / ODS_PAGE_TOKENS; }

// The row holds exactly the pages of `tokens` tokens: valid, held ids, then only empty entries.
ods_status check_row(const ods_pages *p, const int32_t *row, int32_t max_pages, int32_t tokens, const char *who) {
  if (!row || max_pages < 1 || tokens < 0) return set_error(ODS_EINVAL, "%s: null row, max_pages %d or tokens %d", who, max_pages, tokens);
  const int64_t n = pages_of(tokens);
  if (n > max_pages) return set_error(ODS_ERANGE, "%s: %d tokens need %lld pages > max_pages %d", who, tokens, (long long)n, max_pages);
  for (int64_t j = 0; j < max_pages; ++j) {
    if (j >= n ? row[j] >= 0 : row[j] < 0 || row[j] >= p->pool_pages || p->refs[row[j]] < 1)
      return set_error(ODS_EINVAL, "%s: entry %lld of the row is %d, with %d tokens held", who, (long long)j, row[j], tokens);
  }
  return ODS_OK;
}

void give_back(ods_pages *p, int32_t id) {
  if (--p->refs[id] == 0) p->free_ids[p->n_free++] = id;
}

int32_t take(ods_pages *p) {
  const int32_t id = p->free_ids[--p->n_free];
  p->refs[id] = 1;
  return id;
}

// Lists the unheld pages, the lowest last (taken first).
void list_free(ods_pages *p) {
  p->n_free = 0;
  for (int64_t i = p->pool_pages - 1; i >= 0; --i)
    if (p->refs[i] == 0) p->free_ids[p->n_free++] = (int32_t)i;
}

}  // namespace

extern "C" {

ods_status ods_pages_init(ods_pages *p, const int32_t *table, int32_t rows, int32_t max_pages) {
  const char *who = "ods_pages_init";
  if (!p || !p->refs || !p->free_ids || p->pool_pages < 1 || p->pool_pages > INT32_MAX)
    return set_error(ODS_EINVAL, "%s: null pages or pool_pages", who);
  if (rows < 0 || max_pages < 0) return set_error(ODS_EINVAL, "%s: rows %d, max_pages %d", who, rows, max_pages);
  const int64_t n = table ? (int64_t)rows * max_pages : 0;
  for (int64_t i = 0; i < n; ++i)
    if (table[i] >= p->pool_pages)
      return set_error(ODS_ERANGE, "%s: page id %d of %lld pages", who, table[i], (long long)p->pool_pages);
  std::fill(p->refs, p->refs + p->pool_pages, 0);
  for (int64_t i = 0; i < n; ++i)
    if (table[i] >= 0) ++p->refs[table[i]];
  list_free(p);
  clear_error();
  return ODS_OK;
}

ods_status ods_pages_resize(ods_pages *p, int32_t *row, int32_t max_pages, int32_t old_tokens, int32_t new_tokens,
                            int32_t pair[2], int32_t *n_pairs) {
  const char *who = "ods_pages_resize";
  ods_status rc = check_pages(p, who);
  if (rc != ODS_OK) return rc;
  if (!pair || !n_pairs) return set_error(ODS_EINVAL, "%s: null pair", who);
  if ((rc = check_row(p, row, max_pages, old_tokens, who)) != ODS_OK) return rc;
  if (new_tokens < 0) return set_error(ODS_EINVAL, "%s: %d tokens", who, new_tokens);
  const int64_t had = pages_of(old_tokens), want = pages_of(new_tokens);
  if (want > max_pages)
    return set_error(ODS_ERANGE, "%s: %d tokens need %lld pages > max_pages %d", who, new_tokens, (long long)want, max_pages);
  const int64_t part = old_tokens / ODS_PAGE_TOKENS;  // page of the first new token
  const bool own = new_tokens > old_tokens && old_tokens % ODS_PAGE_TOKENS != 0 && p->refs[row[part]] > 1;
  if (std::max<int64_t>(0, want - had) + (own ? 1 : 0) > p->n_free)
    return set_error(ODS_ENOMEM, "%s: %d tokens need %lld more pages, %lld are free", who, new_tokens,
                     (long long)(std::max<int64_t>(0, want - had) + (own ? 1 : 0)), (long long)p->n_free);
  *n_pairs = 0;
  if (own) {
    pair[0] = row[part];
    --p->refs[row[part]];  // others hold it: it does not become free
    pair[1] = row[part] = take(p);
    *n_pairs = 1;
  }
  for (int64_t j = had; j < want; ++j) row[j] = take(p);
  for (int64_t j = had - 1; j >= want; --j) {
    give_back(p, row[j]);
    row[j] = -1;
  }
  clear_error();
  return ODS_OK;
}

ods_status ods_pages_fork(ods_pages *p, const int32_t *src_row, int32_t *dst_row, int32_t max_pages, int32_t tokens) {
  const char *who = "ods_pages_fork";
  ods_status rc = check_pages(p, who);
  if (rc != ODS_OK) return rc;
  if (!src_row || max_pages < 1 || tokens < 0) return set_error(ODS_EINVAL, "%s: null row, max_pages %d or tokens %d", who, max_pages, tokens);
  const int64_t n = pages_of(tokens);
  if (n > max_pages) return set_error(ODS_ERANGE, "%s: %d tokens need %lld pages > max_pages %d", who, tokens, (long long)n, max_pages);
  for (int64_t j = 0; j < n; ++j)
    if (src_row[j] < 0 || src_row[j] >= p->pool_pages || p->refs[src_row[j]] < 1 || p->refs[src_row[j]] == INT32_MAX)
      return set_error(ODS_EINVAL, "%s: entry %lld of the source row is %d", who, (long long)j, src_row[j]);
  if ((rc = check_row(p, dst_row, max_pages, 0, who)) != ODS_OK) return rc;
  for (int64_t j = 0; j < n; ++j) {
    ++p->refs[src_row[j]];
    dst_row[j] = src_row[j];
  }
  clear_error();
  return ODS_OK;
}

ods_status ods_pages_release(ods_pages *p, int32_t *row, int32_t max_pages) {
  const char *who = "ods_pages_release";
  const ods_status rc = check_pages(p, who);
  if (rc != ODS_OK) return rc;
  if (!row || max_pages < 0) return set_error(ODS_EINVAL, "%s: null row or max_pages %d", who, max_pages);
  for (int j = 0; j < max_pages; ++j)
    if (row[j] >= p->pool_pages || (row[j] >= 0 && p->refs[row[j]] < 1))
      return set_error(ODS_EINVAL, "%s: entry %d of the row is %d, which is not held", who, j, row[j]);
  for (int j = 0; j < max_pages; ++j) {
    if (row[j] >= 0 && p->refs[row[j]] > 0) give_back(p, row[j]);
    row[j] = -1;
  }
  clear_error();
  return ODS_OK;
}

ods_status ods_pages_shared(const int32_t *table, int32_t rows, int32_t max_pages, const int32_t *tokens,
                            int32_t *group_off, int32_t *group_tokens, int32_t *n_groups) {
  const char *who = "ods_pages_shared";
  if (!group_off || !group_tokens || !n_groups || (rows > 0 && (!table || !tokens)))
    return set_error(ODS_EINVAL, "%s: null pointer", who);
  if (rows < 0 || max_pages < 1) return set_error(ODS_EINVAL, "%s: rows %d, max_pages %d", who, rows, max_pages);
  for (int32_t r = 0; r < rows; ++r)
    if (tokens[r] < 0 || pages_of(tokens[r]) > max_pages)
      return set_error(ODS_EINVAL, "%s: row %d of %d tokens in %d pages", who, r, tokens[r], max_pages);
  int32_t n = 0;
  group_off[0] = 0;
  for (int32_t r = 0; r < rows && n < ODS_SHARED_GROUPS;) {
    const int32_t *first = table + (int64_t)r * max_pages;
    int64_t common = tokens[r] / ODS_PAGE_TOKENS;  // whole pages of the rows so far
    int32_t end = r + 1;
    for (; end < rows; ++end) {
      const int32_t *row = table + (int64_t)end * max_pages;
      const int64_t most = std::min<int64_t>(common, tokens[end] / ODS_PAGE_TOKENS);
      int64_t same = 0;
      while (same < most && row[same] >= 0 && row[same] == first[same]) ++same;
      const int64_t saved = (end - r - 1) * common, then = (end - r) * same;
      if (then == 0 || then < saved) break;
      common = same;
    }
    const int32_t of_group = end - r > 1 ? (int32_t)(common * ODS_PAGE_TOKENS) : 0;
    if (of_group == 0 && n > 0 && group_tokens[n - 1] == 0) --n;  // with the row before, which shares nothing either
    group_tokens[n] = of_group;
    group_off[++n] = end;
    r = end;
  }
  *n_groups = n;
  clear_error();
  return ODS_OK;
}

ods_status ods_pages_compact(ods_pages *p, int32_t *table, int32_t rows, int32_t max_pages, int32_t *pairs,
                             int32_t max_pairs, int32_t *n_pairs) {
  const char *who = "ods_pages_compact";
  const ods_status rc = check_pages(p, who);
  if (rc != ODS_OK) return rc;
  if (!table || rows < 0 || max_pages < 0 || !n_pairs || max_pairs < 0 || (max_pairs > 0 && !pairs))
    return set_error(ODS_EINVAL, "%s: null table or pairs, rows %d, max_pages %d, max_pairs %d", who, rows, max_pages, max_pairs);
  const int64_t n = (int64_t)rows * max_pages;
  try {
    std::vector<int32_t> seen((size_t)p->pool_pages, 0);
    for (int64_t i = 0; i < n; ++i) {
      if (table[i] >= p->pool_pages) return set_error(ODS_EINVAL, "%s: page id %d of %lld pages", who, table[i], (long long)p->pool_pages);
      if (table[i] >= 0) ++seen[(size_t)table[i]];
    }
    if (!std::equal(seen.begin(), seen.end(), p->refs))
      return set_error(ODS_EINVAL, "%s: the table's rows are not the holders the pages count", who);
    // seen becomes the new id of every page
    int64_t low = 0, high = p->pool_pages - 1, moved = 0;
    for (int64_t i = 0; i < p->pool_pages; ++i) seen[(size_t)i] = (int32_t)i;
    while (moved < max_pairs) {
      while (low < high && p->refs[low] != 0) ++low;
      while (high > low && p->refs[high] == 0) --high;
      if (low >= high) break;
      pairs[2 * moved] = (int32_t)high;
      pairs[2 * moved + 1] = seen[(size_t)high] = (int32_t)low;
      p->refs[low] = p->refs[high];
      p->refs[high] = 0;
      ++moved;
    }
    for (int64_t i = 0; i < n; ++i)
      if (table[i] >= 0) table[i] = seen[(size_t)table[i]];
    list_free(p);
    *n_pairs = (int32_t)moved;
  } catch (const std::bad_alloc &) {  // before anything was changed: `seen` is the only allocation
    return set_error(ODS_ENOMEM, "%s: no host memory for %lld pages", who, (long long)p->pool_pages);
  }
  clear_error();
  return ODS_OK;
}

}  // extern "C"
