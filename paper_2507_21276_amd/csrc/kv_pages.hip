// Moving cached K/V inside the pool: whole pages of all layers (forks and compaction), and the accepted rows of a drafted
// tree to the end of the context.  Pure byte movement: results are bit-exact, and the floor is one read and one write of
// every byte moved.
#include <algorithm>
#include <new>

#include "common.h"

namespace {

constexpr int kPairs = 256;   // page pairs passed by value to one launch
struct Pairs { int32_t src[kPairs], dst[kPairs]; };

// One workgroup per (pair, K / V and layer, piece of 16 KB of the page): 256 pages of 2 MB 214 us, 5.0 TB/s read and written
// together, where a copy of 1 GB reaches 5.2.  Pairs come by value: no buffer to fill before the launch, and a captured call keeps
// them.
__global__ __launch_bounds__(256) void copy_pages_kernel(char* k_pool, char* v_pool, Pairs pr, size_t page_bytes,
                                                         size_t slab_bytes, int piece_bytes) {
  const int l = blockIdx.y >> 1;
  char* pool = ((blockIdx.y & 1) ? v_pool : k_pool) + (size_t)l * slab_bytes;
  const char* src = pool + (size_t)pr.src[blockIdx.x] * page_bytes;
  char* dst = pool + (size_t)pr.dst[blockIdx.x] * page_bytes;
  const size_t lo = (size_t)blockIdx.z * piece_bytes, hi = lo + piece_bytes < page_bytes ? lo + piece_bytes : page_bytes;
  for (size_t i = lo + (size_t)threadIdx.x * 16; i < hi; i += 256 * 16) *(u32x4*)(dst + i) = *(const u32x4*)(src + i);
}

// Rows ctx + path[i] -> ctx + i of one request, all layers and heads.  A thread owns one 16-byte column of the row and walks
// the path itself: nodes rise along it, so path[i] >= i, no row is read after it was overwritten, and no order between
// threads matters.  Eight nodes at a time, whose path entries, page ids and rows are each asked for together: one node after
// the other is three round trips each (paths of up to five nodes, 32 requests, two layers of 32 heads x 128: 8.2 -> 5.9 us).
// One workgroup per (256 columns, K / V and layer, request).
__global__ __launch_bounds__(256) void move_rows_kernel(char* k_pool, char* v_pool, const int32_t* block_table,
                                                        const int32_t* ctx_len, const int32_t* path, int max_path,
                                                        const int32_t* n_path, int h, int page, int row_bytes, int max_pages,
                                                        int n_pages, size_t slab_bytes) {
  constexpr int N = 8;
  const int b = blockIdx.z, l = blockIdx.y >> 1, per = row_bytes / 16;
  const int col = blockIdx.x * 256 + threadIdx.x;
  if (col >= h * per) return;
  char* pool = ((blockIdx.y & 1) ? v_pool : k_pool) + (size_t)l * slab_bytes;
  const int32_t* row = block_table + (size_t)b * max_pages;
  const int32_t* nodes = path + (size_t)b * max_path;
  const int ctx = ctx_len[b], n = min(n_path[b], max_path);
  if (ctx < 0) return;
  // the slot's place in a head's column of its page; the page's id comes from the table
  auto within = [&](int slot) { return ((size_t)(col / per) * page + slot % page) * row_bytes + (col % per) * 16; };
  const size_t page_bytes = (size_t)h * page * row_bytes;
  const long room = (long)max_pages * page;
  int prev = -1;
  for (int i0 = 0; i0 < n; i0 += N) {
    int node[N], from[N], to[N];
#pragma unroll
    for (int i = 0; i < N; ++i) node[i] = i0 + i < n ? nodes[i0 + i] : -1;
    int live = 0;   // nodes of the eight that belong to the path: it ends at the first that does not rise or has no slot
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const bool ok = live == i && node[i] > prev && (long)ctx + node[i] < room;
      live += ok;
      if (ok) prev = node[i];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) {
      const bool moves = i < live && node[i] != i0 + i;
      from[i] = moves ? row[(ctx + node[i]) / page] : -1;
      to[i] = moves ? row[(ctx + i0 + i) / page] : -1;
    }
    u32x4 v[N];
#pragma unroll
    for (int i = 0; i < N; ++i)
      if ((unsigned)from[i] < (unsigned)n_pages) v[i] = *(const u32x4*)(pool + from[i] * page_bytes + within(ctx + node[i]));
#pragma unroll
    for (int i = 0; i < N; ++i)
      if ((unsigned)from[i] < (unsigned)n_pages && (unsigned)to[i] < (unsigned)n_pages)
        *(u32x4*)(pool + to[i] * page_bytes + within(ctx + i0 + i)) = v[i];
    if (live < N) return;
  }
}

ls_status check_pool(const char* who, const ls_config* c, const ls_kv* kv) {
  LS_REQUIRE(c && kv && kv->k_pool && kv->v_pool, "%s: null argument", who);
  LS_REQUIRE(c->mma_dtype == LS_F32 || c->mma_dtype == LS_BF16 || c->mma_dtype == LS_F16, "%s: unknown dtype %d", who,
             c->mma_dtype);
  LS_REQUIRE(c->n_layers > 0 && c->n_layers <= 32767 && c->n_heads > 0 && c->head_dim > 0 && c->page_size > 0 && kv->n_pages > 0,
             "%s: non-positive size of the pool", who);
  LS_REQUIRE(((uintptr_t)kv->k_pool | (uintptr_t)kv->v_pool) % 16 == 0 && c->head_dim * dtype_size(c->mma_dtype) % 16 == 0,
             "%s: pools and rows of a head must be multiples of 16 bytes", who);
  return LS_OK;
}

}  // namespace

extern "C" {

ls_status lsk_kv_copy_pages(const ls_config* c, const ls_kv* kv, const int32_t* src, const int32_t* dst, int n, void* stream) {
  LS_TRY(check_pool("kv_copy_pages", c, kv));
  LS_REQUIRE(n >= 0, "kv_copy_pages: negative number of pages");
  if (n == 0) return LS_OK;
  LS_REQUIRE(src && dst, "kv_copy_pages: null argument");
  for (int i = 0; i < n; ++i)
    LS_REQUIRE(src[i] >= 0 && src[i] < kv->n_pages && dst[i] >= 0 && dst[i] < kv->n_pages,
               "kv_copy_pages: pair %d (%d to %d) outside the pool's %d pages", i, src[i], dst[i], kv->n_pages);
  int32_t* sorted = new (std::nothrow) int32_t[(size_t)n];
  if (!sorted) { ls_set_error("kv_copy_pages: host allocation failed"); return LS_ENOMEM; }
  std::copy(dst, dst + n, sorted);
  std::sort(sorted, sorted + n);
  const bool twice = std::adjacent_find(sorted, sorted + n) != sorted + n;
  int both = -1;
  for (int i = 0; i < n && both < 0; ++i)
    if (std::binary_search(sorted, sorted + n, src[i])) both = src[i];
  delete[] sorted;
  LS_REQUIRE(!twice, "kv_copy_pages: a page is written twice");
  LS_REQUIRE(both < 0, "kv_copy_pages: page %d is read and written by one call", both);
  const size_t page_bytes = (size_t)c->n_heads * c->page_size * c->head_dim * dtype_size(c->mma_dtype);
  const int piece = 16384;
  const unsigned pieces = (unsigned)((page_bytes + piece - 1) / piece);
  LS_REQUIRE(pieces <= 65535, "kv_copy_pages: a page of %zu bytes is too large", page_bytes);
  for (int at = 0; at < n; at += kPairs) {
    const int m = n - at < kPairs ? n - at : kPairs;
    Pairs pr;
    std::copy(src + at, src + at + m, pr.src);
    std::copy(dst + at, dst + at + m, pr.dst);
    copy_pages_kernel<<<dim3(m, 2 * c->n_layers, pieces), 256, 0, (hipStream_t)stream>>>(
        (char*)kv->k_pool, (char*)kv->v_pool, pr, page_bytes, (size_t)kv->n_pages * page_bytes, piece);
    LS_CHECK_LAUNCH();
  }
  return LS_OK;
}

ls_status lsk_kv_move_rows(const ls_config* c, const ls_kv* kv, int B, const int32_t* path, int max_path, const int32_t* n_path,
                           void* stream) {
  LS_TRY(check_pool("kv_move_rows", c, kv));
  LS_REQUIRE(kv->block_table && kv->ctx_len && path && n_path, "kv_move_rows: null argument");
  LS_REQUIRE(B > 0 && B <= 65535, "kv_move_rows: %d requests, not 1..65535", B);
  LS_REQUIRE(max_path > 0 && kv->max_pages_per_req > 0, "kv_move_rows: non-positive size");
  const int row_bytes = c->head_dim * (int)dtype_size(c->mma_dtype);
  const long cols = (long)c->n_heads * (row_bytes / 16);
  LS_REQUIRE(cols <= 0x7fffff00L, "kv_move_rows: rows are too wide");
  const size_t slab = (size_t)kv->n_pages * c->n_heads * c->page_size * row_bytes;
  move_rows_kernel<<<dim3((unsigned)((cols + 255) / 256), 2 * c->n_layers, B), 256, 0, (hipStream_t)stream>>>(
      (char*)kv->k_pool, (char*)kv->v_pool, kv->block_table, kv->ctx_len, path, max_path, n_path, c->n_heads, c->page_size,
      row_bytes, kv->max_pages_per_req, kv->n_pages, slab);
  LS_CHECK_LAUNCH();
  return LS_OK;
}

}  // extern "C"
