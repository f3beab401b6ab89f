// Books over the pages of a pool (host only): rows of page ids that grow, share pages after a fork, shrink and are packed
// together.  What has to be copied on the device is handed to the caller as (source, destination) pairs for
// lsk_kv_copy_pages.
#include <algorithm>
#include <functional>
#include <new>
#include <vector>

#include "../../include/lemix_serve.h"
#include "common.h"

struct ls_pages {
  int n_pages, page, max_rows, max_pages;
  std::vector<int32_t> table;   // [max_rows][max_pages]
  std::vector<int32_t> count;   // pages of each row
  std::vector<int32_t> users;   // rows that hold each page
  std::vector<int32_t> free;    // min-heap: the lowest free page is handed out first
  std::vector<int32_t> moved;   // scratch of ls_pages_compact
};

namespace {

int32_t take(ls_pages* p) {
  std::pop_heap(p->free.begin(), p->free.end(), std::greater<int32_t>());
  const int32_t id = p->free.back();
  p->free.pop_back();
  p->users[id] = 1;
  return id;
}

void drop(ls_pages* p, int32_t id) {
  if (--p->users[id] > 0) return;
  p->free.push_back(id);   // within the capacity set aside at creation
  std::push_heap(p->free.begin(), p->free.end(), std::greater<int32_t>());
}

ls_status check_row(const char* who, const ls_pages* p, int row) {
  LS_REQUIRE(p, "%s: null argument", who);
  LS_REQUIRE(row >= 0 && row < p->max_rows, "%s: row %d outside 0..%d", who, row, p->max_rows - 1);
  return LS_OK;
}

}  // namespace

extern "C" {

ls_status ls_pages_create(int n_pages, int page_size, int max_rows, int max_pages_per_row, ls_pages** out) {
  LS_REQUIRE(out, "pages_create: null argument");
  LS_REQUIRE(n_pages > 0 && page_size > 0 && max_rows > 0 && max_pages_per_row > 0, "pages_create: non-positive size");
  ls_pages* p = nullptr;
  try {
    p = new ls_pages();
    p->n_pages = n_pages;
    p->page = page_size;
    p->max_rows = max_rows;
    p->max_pages = max_pages_per_row;
    p->table.assign((size_t)max_rows * max_pages_per_row, 0);
    p->count.assign(max_rows, 0);
    p->users.assign(n_pages, 0);
    p->moved.assign(n_pages, -1);
    p->free.resize(n_pages);
    for (int i = 0; i < n_pages; ++i) p->free[i] = i;   // rising: a heap already
  } catch (const std::exception&) {
    delete p;
    ls_set_error("pages_create: host allocation failed");
    return LS_ENOMEM;
  }
  *out = p;
  return LS_OK;
}

void ls_pages_destroy(ls_pages* p) { delete p; }

int ls_pages_available(const ls_pages* p) { return p ? (int)p->free.size() : 0; }

ls_status ls_pages_row(const ls_pages* p, int row, int32_t* ids, int* n) {
  LS_TRY(check_row("pages_row", p, row));
  if (ids) std::copy_n(p->table.begin() + (size_t)row * p->max_pages, p->max_pages, ids);
  if (n) *n = p->count[row];
  return LS_OK;
}

ls_status ls_pages_grow(ls_pages* p, int row, int written_from, int n_tokens, int32_t* src, int32_t* dst, int* n_copies) {
  LS_TRY(check_row("pages_grow", p, row));
  LS_REQUIRE(src && dst && n_copies, "pages_grow: null argument");
  LS_REQUIRE(written_from >= 0 && written_from <= n_tokens, "pages_grow: tokens %d.. of %d", written_from, n_tokens);
  const long need = ((long)n_tokens + p->page - 1) / p->page;
  LS_REQUIRE(need <= p->max_pages, "pages_grow: %d tokens need %ld pages, a row holds %d", n_tokens, need, p->max_pages);
  int32_t* ids = p->table.data() + (size_t)row * p->max_pages;
  const int have = p->count[row], first = written_from < n_tokens ? written_from / p->page : have;   // nothing written: none shared
  // pages that tokens written_from .. n_tokens - 1 lie on
  long fresh = need > have ? need - have : 0;
  for (int j = first; j < have && j < need; ++j) fresh += p->users[ids[j]] > 1;
  if (fresh > (long)p->free.size()) {
    ls_set_error("pages_grow: %ld pages needed, %zu free", fresh, p->free.size());
    return LS_ENOMEM;
  }
  *n_copies = 0;
  for (int j = first; j < have && j < need; ++j) {
    if (p->users[ids[j]] == 1) continue;
    const int32_t id = take(p);
    if ((long)j * p->page < written_from) {   // tokens before the written ones stay; later pages are written anew
      src[*n_copies] = ids[j];
      dst[(*n_copies)++] = id;
    }
    --p->users[ids[j]];   // shared, so it keeps a user
    ids[j] = id;
  }
  for (int j = have; j < need; ++j) ids[j] = take(p);
  if (need > have) p->count[row] = (int32_t)need;
  return LS_OK;
}

ls_status ls_pages_fork(ls_pages* p, int from, int to, int n_tokens) {
  LS_TRY(check_row("pages_fork", p, from));
  LS_TRY(check_row("pages_fork", p, to));
  LS_REQUIRE(from != to && p->count[to] == 0, "pages_fork: row %d is in use", to);
  LS_REQUIRE(n_tokens >= 0, "pages_fork: negative number of tokens");
  const long need = ((long)n_tokens + p->page - 1) / p->page;
  LS_REQUIRE(need <= p->count[from], "pages_fork: %d tokens lie on %ld pages, row %d has %d", n_tokens, need, from, p->count[from]);
  const int32_t* a = p->table.data() + (size_t)from * p->max_pages;
  int32_t* b = p->table.data() + (size_t)to * p->max_pages;
  for (int j = 0; j < need; ++j) {
    b[j] = a[j];
    ++p->users[a[j]];
  }
  p->count[to] = (int32_t)need;
  return LS_OK;
}

ls_status ls_pages_truncate(ls_pages* p, int row, int n_tokens) {
  LS_TRY(check_row("pages_truncate", p, row));
  LS_REQUIRE(n_tokens >= 0, "pages_truncate: negative number of tokens");
  const long keep = ((long)n_tokens + p->page - 1) / p->page;
  int32_t* ids = p->table.data() + (size_t)row * p->max_pages;
  while (p->count[row] > keep) {
    const int j = --p->count[row];
    drop(p, ids[j]);
    ids[j] = 0;
  }
  return LS_OK;
}

ls_status ls_pages_compact(ls_pages* p, int32_t* src, int32_t* dst, int* n_moves) {
  LS_REQUIRE(p && src && dst && n_moves, "pages_compact: null argument");
  *n_moves = 0;
  const int used = p->n_pages - (int)p->free.size();
  // every used page from `used` on finds a free one below: as many as there are
  int lo = 0;
  for (int id = used; id < p->n_pages; ++id) {
    if (p->users[id] == 0) continue;
    while (p->users[lo] > 0) ++lo;
    src[*n_moves] = id;
    dst[(*n_moves)++] = lo;
    p->users[lo] = p->users[id];
    p->users[id] = 0;
    p->moved[id] = lo;
  }
  if (*n_moves == 0) return LS_OK;
  for (int row = 0; row < p->max_rows; ++row) {
    int32_t* ids = p->table.data() + (size_t)row * p->max_pages;
    for (int j = 0; j < p->count[row]; ++j)
      if (p->moved[ids[j]] >= 0) ids[j] = p->moved[ids[j]];
  }
  for (int i = 0; i < *n_moves; ++i) p->moved[src[i]] = -1;
  for (size_t i = 0; i < p->free.size(); ++i) p->free[i] = used + (int32_t)i;
  return LS_OK;
}

}  // extern "C"
