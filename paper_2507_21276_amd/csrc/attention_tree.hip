// Attention of a tree of drafted tokens over the paged cache (speculative decoding: several continuations of a context are
// verified by one forward).  The rows of a request are the nodes of its tree; their K and V rows lie in the pages behind the
// ctx cached tokens, in node order, and node i attends to all cached tokens and to the nodes that its mask names (itself and
// its ancestors).
#include "common.h"

namespace {

constexpr int kMaxNodes = 256;

// pos, slot, request and ancestor mask of every node, from the parents: one workgroup per request, the last one marks the
// rows behind the last tree.  A node's ancestors come before it, so a walk up the parents ends after at most its index.
__global__ __launch_bounds__(256) void tree_index_kernel(const int32_t* parent, const int32_t* start, const int32_t* ctx_len,
                                                         int B, int T, int max_nodes, int words, int32_t* pos, int32_t* slot,
                                                         int32_t* req, uint64_t* mask) {
  __shared__ int s_parent[kMaxNodes];
  const int b = blockIdx.x;
  if (b == B) {
    for (int t = max(start[B], 0) + threadIdx.x; t < T; t += 256) {
      pos[t] = 0;
      slot[t] = 0;
      req[t] = -1;
      for (int w = 0; w < words; ++w) mask[(size_t)t * words + w] = 0;
    }
    return;
  }
  const int first = start[b], last = min(start[b + 1], T), n = min(last - first, max_nodes), i = threadIdx.x;
  if (first < 0) return;
  if (i < n) {
    const int p = parent[first + i];
    s_parent[i] = p < i ? p : -1;
  }
  __syncthreads();
  for (int t = first + max(n, 0) + i; t < last; t += 256) {   // more nodes than max_nodes: no request's rows
    pos[t] = 0;
    slot[t] = 0;
    req[t] = -1;
    for (int w = 0; w < words; ++w) mask[(size_t)t * words + w] = 0;
  }
  if (i >= n) return;
  uint64_t seen[kMaxNodes / 64] = {0, 0, 0, 0};
  int depth = -1;
  for (int j = i; j >= 0; j = s_parent[j]) {
#pragma unroll
    for (int w = 0; w < kMaxNodes / 64; ++w)
      if (j >> 6 == w) seen[w] |= 1ull << (j & 63);
    ++depth;
  }
  const int t = first + i, ctx = ctx_len[b];
  pos[t] = ctx + depth;
  slot[t] = ctx + i;
  req[t] = b;
#pragma unroll
  for (int w = 0; w < kMaxNodes / 64; ++w)
    if (w < words) mask[(size_t)t * words + w] = seen[w];
}

struct Tree {
  const int32_t *start, *ctx_len;
  const uint64_t* mask;
  int B, T, max_nodes, words;
  const int32_t* block_table;
  int max_pages, page, n_pages;
};

// The request of row t: the last one whose first row is not behind it
__device__ __forceinline__ int request_of(const int32_t* start, int B, int t) {
  int lo = 0, hi = B;   // start[lo] <= t < start[hi]
  while (hi - lo > 1) {
    const int mid = (lo + hi) / 2;
    if (start[mid] <= t) lo = mid;
    else hi = mid;
  }
  return lo;
}

// Any type and head size: a workgroup of four wavefronts per (row, head).  A wavefront takes 64 keys at a time, a lane one
// key for the scores and a column (of up to four) for the outputs; the softmax is online per wavefront, the four are joined
// through LDS.  Keys that the row does not see are left out of both products, whatever their rows hold.
template <class T>
__global__ __launch_bounds__(256) void tree_attn_any_kernel(const T* q, long ldq, T* o, long ldo, const T* k_pool,
                                                            const T* v_pool, Tree tr, int h, int hk, int dh, float scale_log2) {
  __shared__ float s_q[256], s_p[4][64], s_o[4][256], s_m[4], s_l[4];
  const int t = blockIdx.x, head = blockIdx.y, wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  if (t >= tr.start[tr.B] || t < tr.start[0]) return;
  const int b = request_of(tr.start, tr.B, t);
  const int ctx = max(tr.ctx_len[b], 0), nodes = min(tr.start[b + 1] - tr.start[b], tr.max_nodes);
  if (t - tr.start[b] >= nodes) return;
  const long room = (long)tr.max_pages * tr.page;
  const int nkeys = (int)min((long)ctx + nodes, room), kvh = head / (h / hk);
  for (int c = threadIdx.x; c < dh; c += 256) s_q[c] = to_f(q[(long)t * ldq + (long)head * dh + c]) * scale_log2;
  __syncthreads();
  float m = -INFINITY, l = 0.f, acc[4] = {0.f, 0.f, 0.f, 0.f};
  for (int k0 = wave * 64; k0 < nkeys; k0 += 256) {
    const int key = k0 + lane;
    long at = -1;
    if (key < nkeys) {
      const int id = tr.block_table[(long)b * tr.max_pages + key / tr.page], node = key - ctx;
      const bool seen = node < 0 || (tr.mask[(size_t)t * tr.words + (node >> 6)] >> (node & 63) & 1);
      if (seen && (unsigned)id < (unsigned)tr.n_pages) at = (((long)id * hk + kvh) * tr.page + key % tr.page) * dh;
    }
    float s = -INFINITY;
    if (at >= 0) {
      s = 0.f;
      for (int c = 0; c < dh; ++c) s = fmaf(s_q[c], to_f(k_pool[at + c]), s);
    }
    const float m_new = fmaxf(m, wave_max(s)), ref = m_new == -INFINITY ? 0.f : m_new;
    const float alpha = __builtin_amdgcn_exp2f(m - ref), p = __builtin_amdgcn_exp2f(s - ref);
    m = m_new;
    l = l * alpha + p;
#pragma unroll
    for (int i = 0; i < 4; ++i) acc[i] *= alpha;
    s_p[wave][lane] = p;
    for (uint64_t todo = __ballot(at >= 0); todo; todo &= todo - 1) {
      const int j = __ffsll((unsigned long long)todo) - 1;
      const float pj = s_p[wave][j];
      const long aj = __shfl(at, j, 64);
#pragma unroll
      for (int i = 0; i < 4; ++i)
        if (lane + 64 * i < dh) acc[i] = fmaf(pj, to_f(v_pool[aj + lane + 64 * i]), acc[i]);
    }
  }
  l = wave_sum(l);
  if (lane == 0) { s_m[wave] = m; s_l[wave] = l; }
#pragma unroll
  for (int i = 0; i < 4; ++i) s_o[wave][lane + 64 * i] = acc[i];
  __syncthreads();
  const float mm = fmaxf(fmaxf(s_m[0], s_m[1]), fmaxf(s_m[2], s_m[3])), ref = mm == -INFINITY ? 0.f : mm;
  for (int c = threadIdx.x; c < dh; c += 256) {
    float ll = 0.f, oo = 0.f;
#pragma unroll
    for (int w = 0; w < 4; ++w) {
      const float f = __builtin_amdgcn_exp2f(s_m[w] - ref);
      ll += s_l[w] * f;
      oo += s_o[w][c] * f;
    }
    o[(long)t * ldo + (long)head * dh + c] = from_f<T>(ll == 0.f ? 0.f : oo / ll);   // a row that sees nothing: zeros
  }
}

}  // namespace

extern "C" {

ls_status lsk_tree_index(const int32_t* parent, const int32_t* start, const int32_t* ctx_len, int B, int T, int max_nodes,
                         int32_t* pos, int32_t* slot, int32_t* req, uint64_t* mask, void* stream) {
  LS_REQUIRE(parent && start && ctx_len && pos && slot && req && mask, "tree_index: null argument");
  LS_REQUIRE(B > 0 && T > 0, "tree_index: non-positive size (B %d, T %d)", B, T);
  LS_REQUIRE(max_nodes > 0 && max_nodes <= kMaxNodes, "tree_index: max_nodes %d outside 1..%d", max_nodes, kMaxNodes);
  tree_index_kernel<<<(unsigned)B + 1, 256, 0, (hipStream_t)stream>>>(parent, start, ctx_len, B, T, max_nodes,
                                                                     (max_nodes + 63) / 64, pos, slot, req, mask);
  LS_CHECK_LAUNCH();
  return LS_OK;
}

size_t lsk_attn_tree_scratch_floats(int T, int B, int h, int hk, int dh, int max_nodes, int max_ctx) {
  return 0;
}

ls_status lsk_attn_tree(const void* q, long ldq, int dt, int T, int B, int max_nodes, int h, int hk, int dh,
                        const int32_t* start, const int32_t* ctx_len, const uint64_t* mask, const void* k_pool,
                        const void* v_pool, const int32_t* block_table, int max_pages, int page, int n_pages, int max_ctx,
                        void* o, long ldo, float* scratch, size_t scratch_floats, void* stream) {
  LsTimed timed(LSK_TIMED_DECODE_ATTN, stream);
  LS_REQUIRE(q && start && ctx_len && mask && k_pool && v_pool && block_table && o, "attn_tree: null argument");
  LS_REQUIRE(dt == LS_F32 || dt == LS_BF16 || dt == LS_F16, "attn_tree: unknown dtype %d", dt);
  LS_REQUIRE(T > 0 && B > 0 && h > 0 && hk > 0 && max_pages > 0 && page > 0 && n_pages > 0 && max_ctx >= 0,
             "attn_tree: non-positive size");
  LS_REQUIRE(h % hk == 0 && h <= 65535, "attn_tree: %d query heads do not share %d key heads evenly", h, hk);
  LS_REQUIRE(dh > 0 && dh <= 256, "attn_tree: head_dim %d outside 1..256", dh);
  LS_REQUIRE(max_nodes > 0 && max_nodes <= kMaxNodes, "attn_tree: max_nodes %d outside 1..%d", max_nodes, kMaxNodes);
  LS_REQUIRE(ldq >= (long)h * dh && ldo >= (long)h * dh, "attn_tree: rows overlap (ldq %ld, ldo %ld)", ldq, ldo);
  const Tree tr = {start, ctx_len, mask, B, T, max_nodes, (max_nodes + 63) / 64, block_table, max_pages, page, n_pages};
  const float scale_log2 = 1.4426950408889634f / sqrtf((float)dh);
  hipStream_t st = (hipStream_t)stream;
  auto any = [&](auto* one) {
    typedef std::remove_pointer_t<decltype(one)> T_;
    tree_attn_any_kernel<T_><<<dim3((unsigned)T, h), 256, 0, st>>>((const T_*)q, ldq, (T_*)o, ldo, (const T_*)k_pool,
                                                                  (const T_*)v_pool, tr, h, hk, dh, scale_log2);
  };
  if (dt == LS_F32) any((float*)nullptr);
  else if (dt == LS_BF16) any((bf16_t*)nullptr);
  else any((f16_t*)nullptr);
  LS_CHECK_LAUNCH();
  return LS_OK;
}

}  // extern "C"
