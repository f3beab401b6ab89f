// Attention of a tree of drafted tokens over the paged cache (speculative decoding: several continuations of a context are
// verified by one forward).  The rows of a request are the nodes of its tree; their K and V rows lie in the pages behind the
// ctx cached tokens, in node order, and node i attends to all cached tokens and to the nodes that its mask names (itself and
// its ancestors).
#include <algorithm>
#include <type_traits>

#include "common.h"

namespace {

constexpr int kMaxNodes = 256;
// Workgroups of 256 along x at most: a launch's work-items along one dimension are counted in 32 bits, and a larger grid wraps
// without an error.
constexpr long kGridX = (1 << 24) - 1;

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
  int order_bit;   // the requests' order is that of their lengths in this bit and the five below it; -1: as they come
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

// Any type, head size, page size and alignment: a workgroup of four wavefronts per (row, head), so that every row reads the keys
// for itself, through the caches.  A wavefront takes 64 keys at a time, a lane one key for the scores and a column (of up to four)
// for the outputs; the softmax is online per wavefront, the four are joined through LDS.  Keys that the row does not see are left
// out of both products, whatever their rows hold.  16 trees of 8 nodes, 8 heads of 256, 1024 tokens, 16 bits: 510 us.
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

// ---- 16-bit matrix-core kernel ------------------------------------------------------------------
//
// A workgroup of four wavefronts owns 16 NT RW rows (node, query head of one key head) of one request, one key head and one
// part of the keys: RW wavefronts have 16 NT rows each, and KW = 4 / RW such sets share out the part's tiles of 32 keys.
// S^T = K Q^T (16x16x32) leaves a row's scores in one lane column; the lane's eight keys of a tile are 4 q .. 4 q + 3 and
// 16 + 4 q .. + 3 (q = lane / 16), and O^T += V^T P^T takes P from these very registers when V^T is fed in the same order of
// keys, which two transposing LDS reads per 16 head dimensions do.
//   RW = 1 (up to 32 rows): bound by the K and V bytes.  Each is loaded by one wavefront; K goes straight to registers as the
//   first product's operand, V to the wavefront's own LDS buffer: no barrier in the loop.  64 trees of 8 nodes, 32 heads of 128,
//   16384 tokens each: 6.7 TB/s; of 128 to 2048 tokens 6.6 (194 us; the requests as they come 216, with K and V read through the caches as
//   well 239; two register sets of a tile and spills 330).
//   RW = 2, 4 (more rows): bound by the exponentials and the products.  K and V tiles are loaded once for the RW wavefronts,
//   straight to two LDS buffers and with one barrier a tile, of 64 keys where all four share it.  12 trees of 40 - 61 nodes, five
//   query heads a key head, 3000 to 16001 tokens, with the join: 525 - 540 TFLOP/s (225 - 232 us by the card; by way of registers, which are 32 more, 16
//   us longer; before that a wavefront with 64 rows of its own, which spills, 489; tiles of 32 keys 326); 64 of 64 nodes, 4096 tokens
//   each, 467 us, by way of registers 500.  No single part sets the pace: of 238 us that a call alone took, 228 without the
//   exponentials, 197 without the loads, 206 without the second product.
template <class T> struct Mma16;
template <> struct Mma16<bf16_t> {
  typedef bf16x8 V8;
  static __device__ __forceinline__ f32x4 run(V8 a, V8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0); }
  static constexpr uint32_t kExp = 0x7f80u;   // exponent bits: all set in infinities and NaN
  static constexpr float kLift = 0.f;
};
template <> struct Mma16<f16_t> {
  typedef f16x8 V8;
  static __device__ __forceinline__ f32x4 run(V8 a, V8 b, f32x4 c) { return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0); }
  static constexpr uint32_t kExp = 0x7c00u;
  static constexpr float kLift = 6.f;
};

typedef short s16x4 __attribute__((ext_vector_type(4)));

// Byte offset of 16-byte piece c of row r in a V tile.  A transposing read takes 32 bytes of each of 16 rows: pairs of pieces
// are spread over the banks by the row.
template <int DH> __device__ __forceinline__ int v_at(int r, int c) {
  constexpr int PAIRS = DH / 16;
  const int x = DH == 128 ? r & 7 : DH == 64 ? (r >> 1) & 3 : (r >> 2) & 1;
  return r * (DH * 2) + (((c >> 1) ^ (x & (PAIRS - 1))) << 5) + ((c & 1) << 4);
}
// The same in a K tile, where 16 lanes read the same piece of 16 rows
template <int DH> __device__ __forceinline__ int k_at(int r, int c) {
  const int x = DH == 128 ? r & 15 : DH == 64 ? (r >> 1) & 7 : (r >> 2) & 3;
  return r * (DH * 2) + ((c ^ x) << 4);
}

// Over the four quads of lanes that hold a row's scores: lane permutations without LDS
__device__ __forceinline__ float quads_max(float v) {
  auto a = __builtin_amdgcn_permlane16_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  v = fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
  a = __builtin_amdgcn_permlane32_swap(__float_as_uint(v), __float_as_uint(v), false, false);
  return fmaxf(__uint_as_float(a[0]), __uint_as_float(a[1]));
}

struct Parts {
  int n, keys;       // parts of a context, keys of each (the last takes the rest)
  int row_blocks;
  float* partial;    // [T][h][n][dh + 4]: output, maximum (base 2), sum
};

// A workgroup's rows: of request rows first .., `rows` (node, query head) pairs of key head kvh, from pair row0 on
struct Rows { int first, rows, row0, kvh, g, h, used, part; };

// Joins the 4 / RW sets of wavefronts, 16 rows of each wavefront at a time, through LDS, and stores the rows or the part's results.
// oacc[n][j][i] is dimension 16 j + 4 quad + i of row 16 n + col, m_run and l_run its reference (base 2) and the lane's sum.
template <class T, int DH, int NT, int RW>
__device__ __forceinline__ void store_rows(const f32x4 (&oacc)[NT][DH / 16], const float (&m_run)[NT], const float (&l_run)[NT],
                                           char* smem, float (&s_m)[4][NT * 16], float (&s_l)[4][NT * 16], const Rows& rw,
                                           const Parts& parts, T* o, long ldo) {
  constexpr int KW = 4 / RW, DT = DH / 16;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    float l = l_run[n] + __shfl_xor(l_run[n], 16, 64);
    l += __shfl_xor(l, 32, 64);
    if (quad == 0) { s_m[wave][n * 16 + col] = m_run[n]; s_l[wave][n * 16 + col] = l; }
  }
  float* so = (float*)smem;   // [wave][row][DH + 4]
  constexpr int TPR = 16 / RW;   // threads a row
  const int r = threadIdx.x / TPR, jw = r >> 4, jr = r & 15;
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    __syncthreads();
#pragma unroll
    for (int j = 0; j < DT; ++j) *(f32x4*)(so + (wave * 16 + col) * (DH + 4) + 16 * j + 4 * quad) = oacc[n][j];
    __syncthreads();
    const int row = rw.row0 + (jw * NT + n) * 16 + jr;
    if (row < rw.rows) {
      float mm = -INFINITY, f[KW], l = 0.f;
#pragma unroll
      for (int w = 0; w < KW; ++w) mm = fmaxf(mm, s_m[w * RW + jw][n * 16 + jr]);
      const float ref = mm == -INFINITY ? 0.f : mm;
#pragma unroll
      for (int w = 0; w < KW; ++w) {
        f[w] = __builtin_amdgcn_exp2f(s_m[w * RW + jw][n * 16 + jr] - ref);   // a set without a tile: weight 0 and zeros
        l += s_l[w * RW + jw][n * 16 + jr] * f[w];
      }
      const long trow = rw.first + row / rw.g, head = rw.kvh * rw.g + row % rw.g;
      const float inv = 1.f / l;
      float* pp = parts.partial + ((trow * rw.h + head) * parts.n + rw.part) * (DH + 4);
      for (int c = (threadIdx.x % TPR) * 4; c < DH; c += 4 * TPR) {
        f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < KW; ++w) v += *(const f32x4*)(so + ((w * RW + jw) * 16 + jr) * (DH + 4) + c) * f[w];
        if (rw.used == 1) {
          typedef T V4 __attribute__((ext_vector_type(4)));
          V4 out;
#pragma unroll
          for (int i = 0; i < 4; ++i) out[i] = from_f<T>(l == 0.f ? 0.f : v[i] * inv);   // a row that sees nothing: zeros
          *(V4*)(o + trow * ldo + head * DH + c) = out;
        } else {
          *(f32x4*)(pp + c) = v;
        }
      }
      if (rw.used > 1 && threadIdx.x % TPR == 0) {
        pp[DH] = mm;
        pp[DH + 1] = l;
      }
    }
  }
}

// Workgroups that do not all fit on the chip at once take the requests of each 64 in falling order of their contexts, so that short
// ones end the launch: bf16, 32 heads of 128, 128 to 2048 tokens, 64 trees of 8 nodes 190 -> 172 us, 32 of 13 115 -> 101.  Every
// wavefront finds its own: one load, then bit by bit of the length the half in which the place-th longest lies; among equal ones
// the order is theirs.
__device__ __forceinline__ int request_at(const Tree& tr, int place) {
  if (tr.order_bit < 0) return place;
  const int base = place & ~63, n = min(64, tr.B - base), lane = threadIdx.x & 63;
  const int len = tr.ctx_len[base + min(lane, n - 1)];
  uint64_t left = n == 64 ? ~0ull : (1ull << n) - 1;
  int k = place & 63;   // of those left
#pragma unroll
  for (int i = 0; i < 6; ++i) {
    if (tr.order_bit < i) break;
    const uint64_t longer = __builtin_amdgcn_ballot_w64(len >> (tr.order_bit - i) & 1) & left;
    const int c = __popcll(longer);
    if (k < c) left = longer;
    else { left &= ~longer; k -= c; }
  }
  const int before = __builtin_amdgcn_mbcnt_hi((uint32_t)(left >> 32), __builtin_amdgcn_mbcnt_lo((uint32_t)left, 0));
  return base + __ffsll((unsigned long long)__builtin_amdgcn_ballot_w64((left >> lane & 1) && before == k)) - 1;
}

// Bits of 64 nodes from node nd0 on of a mask row: whether the row sees the key that lies there.  Below 0 lie cached tokens.
__device__ __forceinline__ uint64_t window(const uint64_t* mask, int words, int nd0) {
  const int w0 = nd0 >> 6, sh = nd0 & 63;
  if (nd0 <= -64) return ~0ull;
  if (nd0 < 0) return mask[0] << -nd0 | ((1ull << -nd0) - 1);
  if (w0 >= words) return 0;
  return mask[w0] >> sh | (sh > 0 && w0 + 1 < words ? mask[w0 + 1] << (64 - sh) : 0);
}

constexpr int tree_halves(int rw) { return rw == 4 ? 2 : 1; }   // of a tile, 32 keys each
template <int DH, int RW> constexpr int tree_lds() {
  constexpr int KW = 4 / RW, tile = tree_halves(RW) * 32 * DH * 2, work = RW == 1 ? 4 * tile : KW * 2 * tile, join = 4 * 16 * (DH + 4) * 4;
  return work > join ? work : join;
}

// head_dim 64 with rows of its own: three workgroups a compute unit (two: 24 nodes 49 us, 64 requests of 1024, 12 heads; three 39)
template <class T, int DH, int NT, int RW>
__global__ __launch_bounds__(256, DH == 64 && RW == 1 ? 3 : 2) void tree_attn_kernel(const T* __restrict__ q, long ldq, T* __restrict__ o, long ldo,
                                                           const T* __restrict__ k_pool, const T* __restrict__ v_pool,
                                                           const int32_t* __restrict__ table,
                                                           const uint64_t* __restrict__ masks, Tree tr, int h, int hk,
                                                           int shift, float scale_log2, Parts parts) {
  typedef typename Mma16<T>::V8 V8;
  constexpr int KW = 4 / RW, ROWS = 16 * NT * RW, H = tree_halves(RW), KEYS = 32 * H;
  constexpr int KS = DH / 32, DT = DH / 16, LPR = DH / 8;   // steps of the first product, of the second; lanes per row loaded
  constexpr int NL = H * DH / 16 / RW;                      // loads of K, and of V, per wavefront and tile
  constexpr int G = 4 * H / RW;                             // groups of eight rows that a wavefront loads
  constexpr int TILE = KEYS * DH * 2;
  // Two objects, so that the compiler knows that reads of one do not wait for the loads that go to the other
  __shared__ __attribute__((aligned(16))) char smem[tree_lds<DH, RW>()];
  __shared__ __attribute__((aligned(16))) char smem2[RW == 1 ? 16 : KW * 2 * TILE];
  __shared__ float s_m[4][NT * 16], s_l[4][NT * 16];
  __shared__ int s_flag[2][KW][RW];   // of the tile in a buffer: groups of rows on no page, and values that are not finite

  // Blocks of rows that read the same keys follow each other on one XCD (workgroups go round the eight of them)
  const int slot8 = blockIdx.x >> 3, item = (slot8 / parts.row_blocks) * 8 + (blockIdx.x & 7), rb = slot8 % parts.row_blocks;
  if (item >= tr.B * hk) return;
  const int b = request_at(tr, item / hk), kvh = item % hk, part = blockIdx.y, g = h / hk;
  const int first = tr.start[b], nodes = min(min(tr.start[b + 1], tr.T) - first, tr.max_nodes), rows = nodes * g;
  if (first < 0 || rb * ROWS >= rows) return;
  const int ctx = max(tr.ctx_len[b], 0), page = 1 << shift;
  const int nkeys = (int)min((long)ctx + nodes, (long)tr.max_pages * page);
  const int used = min(parts.n, max(1, (nkeys + parts.keys - 1) / parts.keys));   // parts of this request
  if (part >= used) return;
  const int k_lo = part * parts.keys, k_hi = part == used - 1 ? nkeys : k_lo + parts.keys;
  const int t_lo = k_lo / KEYS, t_hi = (k_hi + KEYS - 1) / KEYS;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4;
  const int rw = wave % RW, kw = wave / RW, row0 = rb * ROWS + rw * 16 * NT;
  const int32_t* bt = table + (long)b * tr.max_pages;

  V8 qf[NT][KS];
  int node[NT];      // of the lane's row; rows past the last repeat it
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int r = min(row0 + n * 16 + col, rows - 1);
    node[n] = r / g;
    const T* qr = q + (long)(first + node[n]) * ldq + (long)(kvh * g + r % g) * DH;
#pragma unroll
    for (int s = 0; s < KS; ++s) qf[n][s] = *(const V8*)(qr + s * 32 + quad * 8);
  }
  // Q has arrived before any tile is asked for: its first use in the loop would otherwise wait for the newest loads as well
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int s = 0; s < KS; ++s) asm volatile("" : "+v"(qf[n][s]));
  f32x4 oacc[NT][DT];
  float m_run[NT], l_run[NT];

  // A tile's rows lie in groups of eight on one page each: the ids of the pages of the wavefront's groups, read a tile before
  // they are needed, then the groups' offsets in the pools and which of them lie on no page (bits of the tile's groups)
  struct Ids { int v[G]; };
  struct Where { long at[G]; int bad; };
  const int last_page = (nkeys - 1) >> shift;
  auto look_up = [&](int t) {
    Ids ids;
#pragma unroll
    for (int i = 0; i < G; ++i) ids.v[i] = bt[min((t * KEYS + (rw * G + i) * 8) >> shift, last_page)];
    return ids;
  };
  auto find = [&](int t, const Ids& ids) {
    Where w;
    w.bad = 0;
#pragma unroll
    for (int i = 0; i < G; ++i) {
      int id = ids.v[i];
      if ((unsigned)id >= (unsigned)tr.n_pages) { id = 0; w.bad |= 1 << (rw * G + i); }
      w.at[i] = ((((long)id * hk + kvh) << shift) + ((t * KEYS + (rw * G + i) * 8) & (page - 1))) * DH;
    }
    return w;
  };
  // loads of a tile in registers (RW = 1): K as the lane's operand of the first product, V in whole rows
  struct Set { V8 k[2 * KS], v[NL]; int bad; };
  // Loads of whole rows: 64 lanes read 512 elements, 512 / DH rows, from one group of eight rows (head_dim 32: from two).  The
  // group's offset is the wavefront's, the lane's place in it 8 lane elements.
  auto row_of = [&](int j) { return (rw * NL + j) * (64 / LPR) + lane / LPR; };
  auto rows_at = [&](const T* pool, const Where& w, int j) {
    const int r = j * (64 / LPR);
    if constexpr (DH == 32) {
      const long lo = w.at[r >> 3], hi = w.at[(r >> 3) + 1];
      return pool + (lane < 32 ? lo : hi) + (lane & 31) * 8;
    } else {
      return pool + w.at[r >> 3] + (r & 7) * DH + lane * 8;
    }
  };
  // K and V that one workgroup reads are read past the caches
  auto load = [&](const T* p) { return __builtin_nontemporal_load((const V8*)p); };
  auto fetch_k = [&](const Where& w, Set& set) {
#pragma unroll
    for (int c = 0; c < 2; ++c) {
      const long a0 = w.at[2 * c], a1 = w.at[2 * c + 1];
      const T* kr = k_pool + ((lane >> 3) & 1 ? a1 : a0) + (lane & 7) * DH + quad * 8;
#pragma unroll
      for (int s = 0; s < KS; ++s) set.k[c * KS + s] = load(kr + s * 32);
    }
  };
  auto fetch_v = [&](const Where& w, Set& set) {
    set.bad = w.bad;
#pragma unroll
    for (int j = 0; j < NL; ++j) set.v[j] = load(rows_at(v_pool, w, j));
  };
  // A lane's byte offsets in the tiles.  Both swizzles are an exclusive or of the piece with row bits that a load, a step of a
  // product or a half of the tile does not touch, or only as a constant: the other offsets follow from these.
  const int v_put = v_at<DH>(lane / LPR, lane % LPR) + rw * NL * 1024;
  const int v_get = v_at<DH>(4 * quad + (col >> 2), (col >> 1) & 1) + (col & 1) * 8, k_get = k_at<DH>(col, quad);
  auto v_put_at = [&](int j) { return (v_put ^ (DH == 128 ? (j & 1) << 7 : 0)) + j * 1024; };
  // Tiles of which all rows see all keys are taken as they are.  There an infinite value times the remainder of a weight (SPLIT below),
  // or times one that fp16 does not hold, is NaN where the weight itself, which is positive, gives infinity: results that are not
  // finite are computed once more, with every tile looked through.  (Finite ones: 0 - 2 % for the registers that the way back takes, 5 %
  // for 24 rows of head_dim 64.  bf16 weights rounded once have fp32's range: nothing to look for.)
  constexpr bool AGAIN = RW == 1 || std::is_same_v<T, f16_t>;
  bool looked = false;
  auto is_plain = [&](int t, int bad) { return !(AGAIN && looked) && (t + 1) * KEYS <= ctx && (t + 1) * KEYS <= k_hi && bad == 0; };
  auto all_finite = [&] {
    float x = 0.f;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int j = 0; j < DT; ++j)
#pragma unroll
        for (int i = 0; i < 4; ++i) x = fmaf(oacc[n][j][i], 0.f, x);
    return x == 0.f;
  };
  auto clear = [&] {
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      m_run[n] = -INFINITY;
      l_run[n] = 0.f;
#pragma unroll
      for (int j = 0; j < DT; ++j) oacc[n][j] = f32x4{0.f, 0.f, 0.f, 0.f};
    }
  };
  // V to LDS.  In the tiles that some row does not see whole, values that are not finite are left out of the product (0 * x
  // would reach the rows that do not see them); returns whether there were any.
  auto put_v = [&](auto plain_, char* vt, int t, const Set& set) {
    const int bad = set.bad;
    if (decltype(plain_)::value || is_plain(t, bad)) {
#pragma unroll
      for (int j = 0; j < NL; ++j) *(V8*)(vt + v_put_at(j)) = set.v[j];
      return false;
    }
    bool odd = false;
#pragma unroll
    for (int j = 0; j < NL; ++j) {
      const int r = row_of(j);
      u32x4 v = __builtin_bit_cast(u32x4, set.v[j]);
      const bool live = t * KEYS + r < k_hi && !(bad >> (r >> 3) & 1);
      constexpr uint32_t E = Mma16<T>::kExp;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const bool lo = (v[e] & E) == E, hi = (v[e] >> 16 & E) == E;
        odd |= live && (lo || hi);
        v[e] = !live ? 0u : v[e] & (lo ? 0xffff0000u : ~0u) & (hi ? 0x0000ffffu : ~0u);
      }
      *(u32x4*)(vt + v_put_at(j)) = v;
    }
    return __builtin_amdgcn_ballot_w64(odd) != 0;
  };

  f32x4 sacc[NT][2 * H];
  auto first_product = [&](const char* kt, const Set& set) {
    V8 ka[2][KS];   // from LDS 16 keys ahead
    int at = k_get;
    asm volatile("" : "+v"(at));   // the few offsets are made anew: held over the loop they are registers that spill
    auto read_k = [&](int c) {
#pragma unroll
      for (int s = 0; s < KS; ++s) ka[c & 1][s] = *(const V8*)(kt + (at ^ (s << 6)) + c * 16 * DH * 2);
    };
    if constexpr (RW > 1) read_k(0);
#pragma unroll
    for (int c = 0; c < 2 * H; ++c) {
      if constexpr (RW > 1) {
        if (c + 1 < 2 * H) read_k(c + 1);
        __builtin_amdgcn_sched_barrier(0);
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) sacc[n][c] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int s = 0; s < KS; ++s)
#pragma unroll
        for (int n = 0; n < NT; ++n) sacc[n][c] = Mma16<T>::run(RW == 1 ? set.k[c * KS + s] : ka[c & 1][s], qf[n][s], sacc[n][c]);
    }
  };
  // softmax and second product of tile t from the scores in sacc
  auto attend = [&](auto plain_, const char* vt, int t, int bad, bool odd) {
    const int k0 = t * KEYS;
    const bool plain = decltype(plain_)::value || is_plain(t, bad);
    // Operand of the second product: keys 4 quad + (col / 4), head dimensions 16 j + 4 (col % 4) ..: the lane receives its column
    // of the 4 x 16 block.  Those of the first 32 keys are read ahead of the softmax, the others as registers come free.
    constexpr bool EARLY = !(RW == 1 && NT == 2);   // beside two tiles of rows and a tile of K there are no registers for them yet
    V8 vf[DT];
    int at = v_get;
    asm volatile("" : "+v"(at));
    auto read_v = [&](int hf, int j) {
      const char* p0 = vt + (at ^ (j << 5)) + hf * 32 * DH * 2;
      const char* p1 = p0 + 16 * DH * 2;
      const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p0);
      const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)p1);
      vf[j] = __builtin_bit_cast(V8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
    };
#pragma unroll
    for (int j = 0; j < DT; ++j) if (EARLY) read_v(0, j);
    uint64_t seen[NT];   // bit r: the lane's row sees key k0 + r
    if (!plain) {
      uint64_t live = k_hi - k0 >= 64 ? ~0ull : (1ull << (k_hi - k0)) - 1;
#pragma unroll
      for (int i = 0; i < 4 * H; ++i)
        if (bad >> i & 1) live &= ~(0xffull << (8 * i));
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const uint64_t win = window(masks + (size_t)(first + node[n]) * tr.words, tr.words, k0 - ctx);
        seen[n] = win & live;
        const uint64_t mine = seen[n] >> (4 * quad);
#pragma unroll
        for (int c = 0; c < 2 * H; ++c)
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!(mine >> (16 * c + i) & 1)) sacc[n][c][i] = -INFINITY;
      }
    }
    // The weights are the second product's operand, in 16 bits.  Where the bytes of K and V set the pace they come in two parts,
    // rounded and remainder, and the product's error is that of its sums: rounded once, bf16 weights add as much to the result's
    // error as its own rounding does.  Twice the products there cost nothing up to 16 rows and 2 % up to 32; with four wavefronts
    // a tile, where the products count, 253 us would be 400, and each weight is rounded once, by half a step at most.
    constexpr bool SPLIT = RW == 1;
    V8 pf[NT][H], pl[SPLIT ? NT : 1][SPLIT ? H : 1];
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float mc[2 * H];
#pragma unroll
      for (int c = 0; c < 2 * H; ++c) mc[c] = fmaxf(fmaxf(fmaxf(sacc[n][c][0], sacc[n][c][1]), sacc[n][c][2]), sacc[n][c][3]);
      float mx = fmaxf(mc[0], mc[1]);
      if constexpr (H == 2) mx = fmaxf(mx, fmaxf(mc[2], mc[3]));
      mx = quads_max(mx) * scale_log2;
      // The reference of the exponentials follows the maximum only when some row exceeds it by more than 2^8: until then the
      // weights stay at or below 256, inside every format, and nothing has to be rescaled.
      if (__builtin_amdgcn_ballot_w64(mx > m_run[n] + 8.f) != 0) {
        const float m_new = fmaxf(m_run[n], mx);
        const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[n] - m_new);
        l_run[n] *= alpha;
        m_run[n] = m_new;
#pragma unroll
        for (int j = 0; j < DT; ++j) oacc[n][j] *= alpha;
      }
      // fp16 weights are lifted by 2^6, to 2^14 at most: the matrix cores take subnormal operands for zero, and so only
      // weights below 2^-20 of the largest are lost.  The sums carry the same factor, which the division takes out.
      const float ref = (m_run[n] == -INFINITY ? 0.f : m_run[n]) - Mma16<T>::kLift;
#pragma unroll
      for (int c = 0; c < 2 * H; ++c)
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          const float p = __builtin_amdgcn_exp2f(__builtin_fmaf(sacc[n][c][i], scale_log2, -ref));
          sacc[n][c][i] = p;
          const T hi = from_f<T>(p);
          pf[n][c >> 1][4 * (c & 1) + i] = hi;
          if constexpr (SPLIT) pl[n][c >> 1][4 * (c & 1) + i] = from_f<T>(p - to_f(hi));
        }
      float lc[2 * H];
#pragma unroll
      for (int c = 0; c < 2 * H; ++c) lc[c] = (sacc[n][c][0] + sacc[n][c][1]) + (sacc[n][c][2] + sacc[n][c][3]);
      if constexpr (H == 2) l_run[n] += (lc[0] + lc[1]) + (lc[2] + lc[3]);
      else l_run[n] += lc[0] + lc[1];
    }
#pragma unroll
    for (int hf = 0; hf < H; ++hf)
#pragma unroll
      for (int j = 0; j < DT; ++j) {
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          if (!EARLY && n == 0) read_v(0, j);
          oacc[n][j] = Mma16<T>::run(vf[j], pf[n][hf], oacc[n][j]);
          if constexpr (SPLIT) oacc[n][j] = Mma16<T>::run(vf[j], pl[n][hf], oacc[n][j]);
        }
        if (hf + 1 < H) read_v(hf + 1, j);
      }
    if (!plain && odd) {
      // Rare: values of this tile are infinite or NaN.  Key by key, what was left out is read again and added where it is seen.
#pragma unroll 1
      for (int r = 0; r < KEYS; ++r) {
        const int key = k0 + r;
        if (key >= k_hi || (bad >> (r >> 3) & 1)) continue;
        const T* vr = v_pool + ((((long)bt[key >> shift] * hk + kvh) << shift) + (key & (page - 1))) * DH;
        float p[NT];   // the weight of the key in the lane's row: held by the lane of that row and the key's quad
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          float x = 0.f;
#pragma unroll
          for (int c = 0; c < 2 * H; ++c)
#pragma unroll
            for (int i = 0; i < 4; ++i)
              if ((r >> 4) == c && (r & 3) == i) x = to_f(pf[n][c >> 1][4 * (c & 1) + i]);
          x = fmaxf(x, 1e-30f);   // a weight that its 16 bits do not hold is still positive (NaN becomes 1e-30, its sum is NaN)
          p[n] = __shfl(x, ((r >> 2) & 3) * 16 + col, 64);
        }
#pragma unroll
        for (int j = 0; j < DT; ++j)
#pragma unroll
          for (int i = 0; i < 4; ++i) {
            const float v = to_f(vr[16 * j + 4 * quad + i]);
            if (v - v != 0.f) {
#pragma unroll
              for (int n = 0; n < NT; ++n)
                if (seen[n] >> r & 1) oacc[n][j][i] += p[n] * v;
            }
          }
      }
    }
  };

  const std::true_type plain_tile;
  const std::false_type any_tile;
  if constexpr (RW == 1) {
    // The next tile's V is asked for as soon as this one's is in LDS, its K after the first product: a wavefront nearly
    // always has a tile in flight.  The tiles that every row sees whole come first; from the first other one on (behind the
    // context, or on a page that is not there) a second loop takes them all, so that its registers are not the first one's.
    char* vt = smem + wave * TILE;
    for (;;) {
      clear();
      int t = t_lo;
      asm volatile("" : "+s"(t));   // made anew the second time: held over the loop, the first tile's offsets are registers that spill
      t += wave;
      if (t >= t_hi) break;
      Set set;
      Where next = find(t, look_up(t));
      fetch_v(next, set);
      fetch_k(next, set);
      Ids ids = look_up(t + 4);
      auto step = [&](auto plain_) {
        const int bad = set.bad;
        const bool more = t + 4 < t_hi;
        next = find(t + 4, ids);
        ids = look_up(t + 8);
        const bool odd = put_v(plain_, vt, t, set);
        if (more) fetch_v(next, set);
        first_product(nullptr, set);
        if (more) fetch_k(next, set);
        attend(plain_, vt, t, bad, odd);
        t += 4;
      };
      while (t < t_hi && is_plain(t, set.bad)) step(plain_tile);
      while (t < t_hi) step(any_tile);
      if (looked || __builtin_amdgcn_ballot_w64(!all_finite()) == 0) break;
      looked = true;
    }
  } else {
    // whether any page of this part is not there: the flags of plain tiles are not looked at otherwise
    bool gaps = false;
    for (int p = (k_lo >> shift) + threadIdx.x; p <= (k_hi - 1) >> shift; p += 256) gaps |= (unsigned)bt[p] >= (unsigned)tr.n_pages;
    const bool any_gap = __syncthreads_or(gaps);
    // Direct-to-LDS loads.  64 lanes write 1 KB one after the other, so a lane asks for the piece of its row that the swizzle puts
    // in its place: element offsets in the rows of a load, to which a later load adds a constant.
    const int k_lane = (lane / LPR) * DH + ((lane % LPR) ^ ((k_at<DH>(lane / LPR, 0) >> 4) & (LPR - 1))) * 8;
    const int v_lane = (lane / LPR) * DH + ((lane % LPR) ^ ((v_at<DH>(lane / LPR, 0) >> 4) & (LPR - 1))) * 8;
    // Past the caches where one workgroup reads the keys.  head_dim 32 has two wavefronts for any number of rows above 32, so that several
    // workgroups may: through the caches 64 trees of 256 nodes, 16 heads, 4096 tokens 379 us (past them 386), of 50 nodes the same.
    constexpr int PAST = RW < 4 && DH > 32 ? 2 : 0;
    auto issue = [&](char* st, const Where& w) {
      char* kt = st + kw * 2 * TILE + rw * NL * 1024;
#pragma unroll
      for (int j = 0; j < NL; ++j) {
        const int r = j * (64 / LPR);
        long at;
        if constexpr (DH == 32) at = lane < 32 ? w.at[r >> 3] : w.at[(r >> 3) + 1] - 8 * DH;   // lanes count on over the two groups
        else at = w.at[r >> 3] + (r & 7) * DH;
        const int kx = DH == 128 ? (j & 3) << 5 : DH == 64 ? (j & 1) << 5 : 0, vx = DH == 128 ? (j & 1) << 6 : 0;
        const T *kp = k_pool + at + (k_lane ^ kx), *vp = v_pool + at + (v_lane ^ vx);
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)kp,
                                         (__attribute__((address_space(3))) void*)(kt + j * 1024), 16, 0, PAST);
        __builtin_amdgcn_global_load_lds((const __attribute__((address_space(1))) void*)vp,
                                         (__attribute__((address_space(3))) void*)(kt + TILE + j * 1024), 16, 0, PAST);
      }
    };
    int t, bad;
    Ids ids;
    // A tile of each set of wavefronts from `cur`, while the next one's loads go to `nxt`.  Waits are the compiler's own, so that it
    // knows which loads are still under way: it would otherwise wait for `nxt` before it reads `cur`.
    auto step = [&](char* cur, char* nxt, int buf) __attribute__((always_inline)) {
      char* kt = cur + kw * 2 * TILE;
      char* vt = kt + TILE;
      const Where next = find(t + KW, ids);   // of ids that came during the tile before this one
      const bool all = !any_gap && is_plain(t, 0);
      asm volatile("" ::: "memory");
      __builtin_amdgcn_s_waitcnt(0x0070);     // vmcnt(0), lgkmcnt(0): the wavefront's own loads are here
      asm volatile("" ::: "memory");
      if (!all && t < t_hi) {                 // its own rows of V once more through put_v
        Set set;
        set.bad = bad;
#pragma unroll
        for (int j = 0; j < NL; ++j) set.v[j] = *(const V8*)(vt + v_put_at(j));
        const bool odd = put_v(any_tile, vt, t, set);
        if (lane == 0) s_flag[buf][kw][rw] = bad | (int)odd << 8;
        asm volatile("" ::: "memory");
        __builtin_amdgcn_s_waitcnt(0x0070);
      }
      __builtin_amdgcn_s_barrier();           // everyone's are, and everyone is past the tile before this one: `nxt` is free
      asm volatile("" ::: "memory");
      if (t + KW < t_hi) issue(nxt, next);
      bad = next.bad;
      ids = look_up(t + 2 * KW);
      if (t < t_hi && row0 < rows) {
        int flags = 0;
        if (!all) {
#pragma unroll
          for (int w = 0; w < RW; ++w) flags |= s_flag[buf][kw][w];
          flags = __builtin_amdgcn_readfirstlane(flags);
        }
        first_product(kt, Set());
        attend(any_tile, vt, t, flags & 255, flags >> 8);
      }
      t += KW;
    };
    for (;;) {
      clear();
      t = t_lo;
      if constexpr (AGAIN) asm volatile("" : "+s"(t));
      t += kw;
      bad = 0;
      ids = look_up(t);
      if (t < t_hi) {
        const Where w = find(t, ids);
        bad = w.bad;
        issue(smem, w);
      }
      ids = look_up(t + KW);
      for (int i = t_lo; i < t_hi; i += KW) {   // the same number of trips in every wavefront
        step(smem, smem2, 0);
        if ((i += KW) >= t_hi) break;
        step(smem2, smem, 1);
      }
      if (!AGAIN || looked || !__syncthreads_or(!all_finite())) break;
      looked = true;
    }
  }
  store_rows<T, DH, NT, RW>(oacc, m_run, l_run, smem, s_m, s_l, Rows{first, rows, rb * ROWS, kvh, g, h, used, part}, parts, o, ldo);
}

// ---- fp32 matrix-core kernel ---------------------------------------------------------------------
//
// The same split as RW = 1 with 16x16x4 fp32 products: 16 NT rows a workgroup, tiles of 16 keys shared out over the wavefronts.
// A lane's K operand is a quarter of its key's row (the order of the contraction is free, so its four steps' worth are
// contiguous), and the second product's steps take key 4 quad + i from the scores as they lie, V element by element from
// memory, 64 bytes of a row for 16 lanes: nothing goes through LDS before the join.  Bound by the matrix instructions, which
// take 32 cycles for 1024 multiply-adds, from two blocks of rows on, by loads before that: 16 trees of 16 nodes, 12 heads of 64,
// 1024 tokens 26 us (4.0 TB/s), 300 with a workgroup a (row, head); 8 trees of 8, 4 heads of 32, 2048 tokens 14 and 214.
template <int DH, int NT>
__global__ __launch_bounds__(256, 2) void tree_attn_f32_kernel(const float* __restrict__ q, long ldq, float* __restrict__ o, long ldo,
                                                               const float* __restrict__ k_pool, const float* __restrict__ v_pool,
                                                               const int32_t* __restrict__ table, const uint64_t* __restrict__ masks,
                                                               Tree tr, int h, int hk, int shift, float scale_log2, Parts parts) {
  constexpr int ROWS = 16 * NT, DT = DH / 16, NK = DH / 16;   // 16-byte loads of a lane's quarter of a K row
  __shared__ __attribute__((aligned(16))) char smem[4 * 16 * (DH + 4) * 4];
  __shared__ float s_m[4][NT * 16], s_l[4][NT * 16];
  const int slot8 = blockIdx.x >> 3, item = (slot8 / parts.row_blocks) * 8 + (blockIdx.x & 7), rb = slot8 % parts.row_blocks;
  if (item >= tr.B * hk) return;
  const int b = request_at(tr, item / hk), kvh = item % hk, part = blockIdx.y, g = h / hk;
  const int first = tr.start[b], nodes = min(min(tr.start[b + 1], tr.T) - first, tr.max_nodes), rows = nodes * g;
  if (first < 0 || rb * ROWS >= rows) return;
  const int ctx = max(tr.ctx_len[b], 0), page = 1 << shift;
  const int nkeys = (int)min((long)ctx + nodes, (long)tr.max_pages * page);
  const int used = min(parts.n, max(1, (nkeys + parts.keys - 1) / parts.keys));
  if (part >= used) return;
  const int k_lo = part * parts.keys, k_hi = part == used - 1 ? nkeys : k_lo + parts.keys;
  const int t_lo = k_lo / 16, t_hi = (k_hi + 15) / 16;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), lane = threadIdx.x & 63, col = lane & 15, quad = lane >> 4;
  const int32_t* bt = table + (long)b * tr.max_pages;

  f32x4 qf[NT][NK];
  int node[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    const int r = min(rb * ROWS + n * 16 + col, rows - 1);
    node[n] = r / g;
    const float* qr = q + (long)(first + node[n]) * ldq + (long)(kvh * g + r % g) * DH + quad * (DH / 4);
#pragma unroll
    for (int s = 0; s < NK; ++s) qf[n][s] = *(const f32x4*)(qr + 4 * s);
  }
#pragma unroll
  for (int n = 0; n < NT; ++n)
#pragma unroll
    for (int s = 0; s < NK; ++s) asm volatile("" : "+v"(qf[n][s]));   // Q is here before the first tile is asked for
  f32x4 oacc[NT][DT];
  float m_run[NT], l_run[NT];
#pragma unroll
  for (int n = 0; n < NT; ++n) {
    m_run[n] = -INFINITY;
    l_run[n] = 0.f;
#pragma unroll
    for (int j = 0; j < DT; ++j) oacc[n][j] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // the two groups of eight rows of a tile: their offsets in the pools, and which lie on no page
  struct Where { long at[2]; int bad; };
  const int last_page = (nkeys - 1) >> shift;
  struct Ids { int v[2]; };
  auto look_up = [&](int t) { return Ids{{bt[min((t * 16) >> shift, last_page)], bt[min((t * 16 + 8) >> shift, last_page)]}}; };
  auto find = [&](int t, const Ids& ids) {
    Where w;
    w.bad = 0;
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      int id = ids.v[i];
      if ((unsigned)id >= (unsigned)tr.n_pages) { id = 0; w.bad |= 1 << i; }
      w.at[i] = ((((long)id * hk + kvh) << shift) + ((t * 16 + i * 8) & (page - 1))) * DH;
    }
    return w;
  };
  f32x4 kf[NK];
  float vf[DT][4];
  int bad = 0;
  auto fetch_k = [&](const Where& w) {
    const long a0 = w.at[0], a1 = w.at[1];
    const float* kr = k_pool + (col >= 8 ? a1 : a0) + (col & 7) * DH + quad * (DH / 4);
#pragma unroll
    for (int s = 0; s < NK; ++s) kf[s] = *(const f32x4*)(kr + 4 * s);
  };
  auto fetch_v = [&](const Where& w) {
    bad = w.bad;
    const long a0 = w.at[0], a1 = w.at[1];
    const float* vr = v_pool + (quad >= 2 ? a1 : a0) + (4 * quad & 7) * DH + col;
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < DT; ++j) vf[j][i] = vr[i * DH + 16 * j];
  };

  int t = t_lo + wave;
  if (t < t_hi) {
    Where next = find(t, look_up(t));
    fetch_k(next);
    fetch_v(next);
    Ids ids = look_up(t + 4);
    for (; t < t_hi; t += 4) {
      const int k0 = t * 16;
      const bool more = t + 4 < t_hi, plain = k0 + 16 <= ctx && k0 + 16 <= k_hi && bad == 0;   // plain: all rows see all keys
      const int gaps = bad;
      next = find(t + 4, ids);
      ids = look_up(t + 8);
      f32x4 p[NT];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        p[n] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int s = 0; s < NK; ++s)
#pragma unroll
          for (int e = 0; e < 4; ++e) p[n] = __builtin_amdgcn_mfma_f32_16x16x4f32(kf[s][e], qf[n][s][e], p[n], 0, 0, 0);
      }
      if (more) fetch_k(next);
      uint32_t seen[NT];   // bit r: the lane's row sees key k0 + r
      bool odd = false;
      if (!plain) {
        uint32_t live = k_hi - k0 >= 16 ? 0xffffu : (1u << (k_hi - k0)) - 1;
        live &= (gaps & 1 ? 0xff00u : 0xffffu) & (gaps & 2 ? 0x00ffu : 0xffffu);
#pragma unroll
        for (int n = 0; n < NT; ++n) {
          seen[n] = (uint32_t)window(masks + (size_t)(first + node[n]) * tr.words, tr.words, k0 - ctx) & live;
#pragma unroll
          for (int i = 0; i < 4; ++i)
            if (!(seen[n] >> (4 * quad + i) & 1)) p[n][i] = -INFINITY;
        }
        // values that are not finite are left out of the product, and added to the rows that see them afterwards
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
          for (int j = 0; j < DT; ++j) {
            const bool here = live >> (4 * quad + i) & 1, finite = vf[j][i] - vf[j][i] == 0.f;
            odd |= here && !finite;
            if (!here || !finite) vf[j][i] = 0.f;
          }
      }
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const float mx = quads_max(fmaxf(fmaxf(p[n][0], p[n][1]), fmaxf(p[n][2], p[n][3]))) * scale_log2;
        if (__builtin_amdgcn_ballot_w64(mx > m_run[n]) != 0) {
          const float m_new = fmaxf(m_run[n], mx);
          const float alpha = m_new == -INFINITY ? 1.f : __builtin_amdgcn_exp2f(m_run[n] - m_new);
          l_run[n] *= alpha;
          m_run[n] = m_new;
#pragma unroll
          for (int j = 0; j < DT; ++j) oacc[n][j] *= alpha;
        }
        const float ref = m_run[n] == -INFINITY ? 0.f : m_run[n];
#pragma unroll
        for (int i = 0; i < 4; ++i) p[n][i] = __builtin_amdgcn_exp2f(__builtin_fmaf(p[n][i], scale_log2, -ref));
        l_run[n] += (p[n][0] + p[n][1]) + (p[n][2] + p[n][3]);
      }
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < DT; ++j)
#pragma unroll
          for (int n = 0; n < NT; ++n) oacc[n][j] = __builtin_amdgcn_mfma_f32_16x16x4f32(vf[j][i], p[n][i], oacc[n][j], 0, 0, 0);
      if (more) fetch_v(next);
      if (!plain && __builtin_amdgcn_ballot_w64(odd) != 0) {
#pragma unroll 1
        for (int r = 0; r < 16; ++r) {
          const int key = k0 + r;
          if (key >= k_hi || (gaps >> (r >> 3) & 1)) continue;
          const float* vr = v_pool + ((((long)bt[key >> shift] * hk + kvh) << shift) + (key & (page - 1))) * DH;
          float w[NT];
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            const float x = (r & 2) ? ((r & 1) ? p[n][3] : p[n][2]) : ((r & 1) ? p[n][1] : p[n][0]);
            w[n] = __shfl(fmaxf(x, 1e-30f), (r >> 2) * 16 + col, 64);
          }
#pragma unroll
          for (int j = 0; j < DT; ++j)
#pragma unroll
            for (int i = 0; i < 4; ++i) {
              const float v = vr[16 * j + 4 * quad + i];
              if (v - v != 0.f) {
#pragma unroll
                for (int n = 0; n < NT; ++n)
                  if (seen[n] >> r & 1) oacc[n][j][i] += w[n] * v;
              }
            }
        }
      }
    }
  }
  store_rows<float, DH, NT, 1>(oacc, m_run, l_run, smem, s_m, s_l, Rows{first, rows, rb * ROWS, kvh, g, h, used, part}, parts, o, ldo);
}

// Joins the parts of a request's rows, in a fixed order: a wavefront has a (row, head), DH / 4 lanes have a part, four of its
// values each.  `blocks` workgroups belong to a request, so that no wavefront has to search for its own; a lane holds the
// maximum and sum of one part while the outputs are on their way (600 rows x 40 heads of up to eight parts: 22 -> 16 us).
template <class T, int DH>
__global__ __launch_bounds__(256) void tree_merge_kernel(T* __restrict__ o, long ldo, Tree tr, int h, int shift, int blocks,
                                                         Parts parts) {
  constexpr int LP = DH / 4, AT = 64 / LP;
  const int b = blockIdx.x / blocks, lane = threadIdx.x & 63;
  const long item = (long)(blockIdx.x % blocks) * 4 + (threadIdx.x >> 6);   // of the request's nodes x heads
  const int first = tr.start[b], nodes = min(min(tr.start[b + 1], tr.T) - first, tr.max_nodes);
  if (first < 0 || item >= (long)nodes * h) return;
  const int nkeys = (int)min((long)max(tr.ctx_len[b], 0) + nodes, (long)tr.max_pages << shift);
  const int used = min(parts.n, max(1, (nkeys + parts.keys - 1) / parts.keys));
  if (used == 1) return;   // written already
  const long t = first + item / h, head = item % h;
  const float* pp = parts.partial + (t * h + head) * parts.n * (DH + 4);
  float m = -INFINITY, l = 0.f;
  f32x4 v = f32x4{0.f, 0.f, 0.f, 0.f};
  for (int s0 = 0; s0 < used; s0 += 64) {
    const int n = min(64, used - s0);
    const float ms = lane < n ? pp[(long)(s0 + lane) * (DH + 4) + DH] : -INFINITY;
    const float ls = lane < n ? pp[(long)(s0 + lane) * (DH + 4) + DH + 1] : 0.f;
    const float m_new = fmaxf(m, wave_max(ms)), ref = m_new == -INFINITY ? 0.f : m_new, alpha = __builtin_amdgcn_exp2f(m - ref);
    const float f = __builtin_amdgcn_exp2f(ms - ref);
    m = m_new;
    l = l * alpha + wave_sum(ls * f);
    v *= alpha;
    for (int s = 0; s < n; s += 4 * AT) {
      f32x4 x[4];
#pragma unroll
      for (int i = 0; i < 4; ++i) x[i] = *(const f32x4*)(pp + (long)(s0 + min(s + i * AT + lane / LP, n - 1)) * (DH + 4) + (lane % LP) * 4);
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int at = s + i * AT + lane / LP;
        const float fs = __shfl(f, at, 64);
        if (at < n) v += x[i] * fs;
      }
    }
  }
#pragma unroll
  for (int off = LP; off < 64; off <<= 1)
#pragma unroll
    for (int i = 0; i < 4; ++i) v[i] += __shfl_xor(v[i], off, 64);
  if (lane >= LP) return;
  typedef T V4 __attribute__((ext_vector_type(4)));
  V4 out;
#pragma unroll
  for (int i = 0; i < 4; ++i) out[i] = from_f<T>(l == 0.f ? 0.f : v[i] / l);
  *(V4*)(o + t * ldo + head * DH + lane * 4) = out;
}

// Rows of a workgroup (tiles of 16 a wavefront, wavefronts with rows of their own), blocks of rows, parts of the contexts.
// How far the other contexts fall short of the longest is not known here, so a rule has to hold for equal ones and for one
// long one among short ones (up to a sixteenth).  us, equal | one long, 8 nodes, 32 heads of 128 unless said:
//   A split costs a launch (one request of 256 tokens 1/8.5, 2/11.3; 1024 1/15, 8/10.4) and the partial results.  Workgroups
//   fill the chip from about 512 on (4 requests of 4096: 1/68 | 60, 4/50 | 39, 16/55 | 24), with 128 keys or more each.
//   Beyond that only so that one long context is not the last workgroup's for itself: parts of 2048 keys below 512 pairs (4
//   requests of 16384 2/165 | 125, 8/173 | 74; five query heads a key head, 64 nodes, 16 requests 1/636 | 417, 4/542 | 134, 8/562
//   | 114), of 4096 from there on (64 requests of 16384 1/2551 | 277, 4/2737 | 211, 8/2864 | 171; of 4096 1/649 | 74, 2/714 | 71).
struct Plan { int tiles, row_waves, row_blocks, parts; };
Plan plan(int dt, int B, int hk, int g, int dh, int max_nodes, int max_ctx) {
  // head_dim 32: a tile is two loads, for two wavefronts
  const int rows = max_nodes * g, tiles = rows <= 16 ? 1 : 2;
  const int row_waves = rows <= 32 || dt == LS_F32 ? 1 : rows <= 64 || dh == 32 ? 2 : 4;
  Plan p = {tiles, row_waves, (rows + 16 * tiles * row_waves - 1) / (16 * tiles * row_waves), 1};
  const long pairs = (long)B * hk * p.row_blocks, keys = (long)max_ctx + max_nodes;
  if (keys <= 512) return p;
  const long fill = 512 / pairs, most = pairs < 512 ? 2048 : 4096, even = (keys + most / 2) / most;
  long n = fill > even ? fill : even;
  if (n > keys / 128) n = keys / 128;
  if (n > 1) p.parts = n < 4096 ? (int)n : 4096;
  return p;
}

// What a call uses of its scratch at most, 1 GB: partial results grow with rows x heads x parts (4096 rows of 32 heads of 128 in
// eight parts 554 MB, 16384 rows in 32 parts 8.9 GB), and fewer parts are right as well.  Launches that reach the limit have
// thousands of workgroups, so that a split only shortens the last ones.
constexpr size_t kMaxScratch = (size_t)1 << 28;   // floats

bool mma_covers(int dh) { return dh == 32 || dh == 64 || dh == 128; }

// keys of a part, for a context of the longest length: a whole number of tiles for each wavefront
int part_keys(long keys, int parts) { return (int)(((keys + parts - 1) / parts + 127) / 128 * 128); }

}  // namespace

extern "C" {

ls_status lsk_tree_index(const int32_t* parent, const int32_t* start, const int32_t* ctx_len, int B, int T, int max_nodes,
                         int32_t* pos, int32_t* slot, int32_t* req, uint64_t* mask, void* stream) {
  LS_REQUIRE(parent && start && ctx_len && pos && slot && req && mask, "tree_index: null argument");
  LS_REQUIRE(B > 0 && T > 0, "tree_index: non-positive size (B %d, T %d)", B, T);
  LS_REQUIRE(max_nodes > 0 && max_nodes <= kMaxNodes, "tree_index: max_nodes %d outside 1..%d", max_nodes, kMaxNodes);
  LS_REQUIRE(B < kGridX, "tree_index: %d requests are too many", B);
  tree_index_kernel<<<(unsigned)B + 1, 256, 0, (hipStream_t)stream>>>(parent, start, ctx_len, B, T, max_nodes,
                                                                     (max_nodes + 63) / 64, pos, slot, req, mask);
  LS_CHECK_LAUNCH();
  return LS_OK;
}

size_t lsk_attn_tree_scratch_floats(int T, int B, int h, int hk, int dh, int max_nodes, int max_ctx) {
  if (T <= 0 || B <= 0 || h <= 0 || hk <= 0 || h % hk || dh <= 0 || max_nodes <= 0 || max_ctx < 0) return 0;
  const int a = plan(LS_F32, B, hk, h / hk, dh, max_nodes, max_ctx).parts, b = plan(LS_F16, B, hk, h / hk, dh, max_nodes, max_ctx).parts;
  const size_t one = (size_t)T * h * (dh + 4), parts = std::min<size_t>(a > b ? a : b, kMaxScratch / one);
  return parts > 1 && mma_covers(dh) ? one * parts : 0;
}

ls_status lsk_attn_tree(const void* q, long ldq, int dt, int T, int B, int max_nodes, int h, int hk, int dh,
                        const int32_t* start, const int32_t* ctx_len, const uint64_t* mask, const void* k_pool,
                        const void* v_pool, const int32_t* block_table, int max_pages, int page, int n_pages, int max_ctx,
                        void* o, long ldo, float* scratch, size_t scratch_floats, void* stream) {
  LS_REQUIRE(q && start && ctx_len && mask && k_pool && v_pool && block_table && o, "attn_tree: null argument");
  LS_REQUIRE(dt == LS_F32 || dt == LS_BF16 || dt == LS_F16, "attn_tree: unknown dtype %d", dt);
  LS_REQUIRE(T > 0 && B > 0 && h > 0 && hk > 0 && max_pages > 0 && page > 0 && n_pages > 0 && max_ctx >= 0,
             "attn_tree: non-positive size");
  LS_REQUIRE(h % hk == 0 && h <= 65535, "attn_tree: %d query heads do not share %d key heads evenly", h, hk);
  LS_REQUIRE(dh > 0 && dh <= 256, "attn_tree: head_dim %d outside 1..256", dh);
  LS_REQUIRE(max_nodes > 0 && max_nodes <= kMaxNodes, "attn_tree: max_nodes %d outside 1..%d", max_nodes, kMaxNodes);
  LS_REQUIRE(ldq >= (long)h * dh && ldo >= (long)h * dh, "attn_tree: rows overlap (ldq %ld, ldo %ld)", ldq, ldo);
  Tree tr = {start, ctx_len, mask, B, T, max_nodes, (max_nodes + 63) / 64, block_table, max_pages, page, n_pages, -1};
  const float scale_log2 = 1.4426950408889634f / sqrtf((float)dh);
  hipStream_t st = (hipStream_t)stream;
  const int per16 = dt == LS_F32 ? 4 : 8;   // elements of 16 bytes
  if (mma_covers(dh) && page >= 8 && (page & (page - 1)) == 0 && ldq % per16 == 0 && ldo % per16 == 0 &&
      ((uintptr_t)q | (uintptr_t)o | (uintptr_t)k_pool | (uintptr_t)v_pool) % 16 == 0) {
    Plan p = plan(dt, B, hk, h / hk, dh, max_nodes, max_ctx);
    const size_t one = (size_t)T * h * (dh + 4);
    const size_t room = scratch && (uintptr_t)scratch % 16 == 0 ? std::min(scratch_floats, kMaxScratch) / one : 0;
    if ((size_t)p.parts > room) p.parts = room > 1 ? (int)room : 1;
    const long merge = ((long)max_nodes * h + 3) / 4;   // workgroups a request
    if (merge * B > kGridX) p.parts = 1;                // nothing to join
    const long keys = (long)max_ctx + max_nodes;
    LS_REQUIRE(keys <= 0x7fffff00L, "attn_tree: max_ctx %d is too large", max_ctx);
    const Parts parts = {p.parts, part_keys(keys, p.parts), p.row_blocks, scratch};
    const long groups = ((long)B * hk + 7) / 8 * 8 * p.row_blocks;
    LS_REQUIRE(groups <= kGridX, "attn_tree: %d requests of up to %d nodes and %d key heads are too many", B, max_nodes, hk);
    const dim3 grid((unsigned)groups, p.parts);
    if (B > 1 && max_ctx > 0 && groups * p.parts > 512) tr.order_bit = 31 - __builtin_clz(max_ctx);   // two workgroups a compute unit
    const int shift = __builtin_ctz(page);
    auto go = [&](auto* one_, auto dh_, auto nt_, auto rw_) {
      typedef std::remove_pointer_t<decltype(one_)> T_;
      constexpr int DH = decltype(dh_)::value, NT = decltype(nt_)::value, RW = decltype(rw_)::value;
      if constexpr (std::is_same_v<T_, float>)
        tree_attn_f32_kernel<DH, NT><<<grid, 256, 0, st>>>((const float*)q, ldq, (float*)o, ldo, (const float*)k_pool,
                                                         (const float*)v_pool, block_table, mask, tr, h, hk, shift, scale_log2, parts);
      else
        tree_attn_kernel<T_, DH, NT, RW><<<grid, 256, 0, st>>>((const T_*)q, ldq, (T_*)o, ldo, (const T_*)k_pool,
                                                             (const T_*)v_pool, block_table, mask, tr, h, hk, shift, scale_log2,
                                                             parts);
      if (p.parts > 1) tree_merge_kernel<T_, DH><<<(unsigned)(B * merge), 256, 0, st>>>((T_*)o, ldo, tr, h, shift, (int)merge, parts);
    };
    auto rows = [&](auto* one_, auto dh_) {
      constexpr bool f32 = std::is_same_v<std::remove_pointer_t<decltype(one_)>, float>;
      const std::integral_constant<int, 1> c1;
      const std::integral_constant<int, 2> c2;
      const std::integral_constant<int, 4> c4;
      if (p.tiles == 1) go(one_, dh_, c1, c1);
      else if (p.row_waves == 1) go(one_, dh_, c2, c1);
      else if constexpr (!f32) {
        if (p.row_waves == 2) go(one_, dh_, c2, c2);
        else if constexpr (decltype(dh_)::value > 32) go(one_, dh_, c2, c4);
      }
    };
    auto size = [&](auto* one_) {
      if (dh == 32) rows(one_, std::integral_constant<int, 32>());
      else if (dh == 64) rows(one_, std::integral_constant<int, 64>());
      else rows(one_, std::integral_constant<int, 128>());
    };
    LsTimed timed(LSK_TIMED_DECODE_ATTN, stream);   // a refusal launches nothing and is not recorded
    if (dt == LS_F32) size((float*)nullptr);
    else if (dt == LS_BF16) size((bf16_t*)nullptr);
    else size((f16_t*)nullptr);
    LS_CHECK_LAUNCH();
    return LS_OK;
  }
  LS_REQUIRE(T <= kGridX, "attn_tree: %d rows are too many", T);
  auto any = [&](auto* one) {
    typedef std::remove_pointer_t<decltype(one)> T_;
    tree_attn_any_kernel<T_><<<dim3((unsigned)T, h), 256, 0, st>>>((const T_*)q, ldq, (T_*)o, ldo, (const T_*)k_pool,
                                                                  (const T_*)v_pool, tr, h, hk, dh, scale_log2);
  };
  LsTimed timed(LSK_TIMED_DECODE_ATTN, stream);
  if (dt == LS_F32) any((float*)nullptr);
  else if (dt == LS_BF16) any((bf16_t*)nullptr);
  else any((f16_t*)nullptr);
  LS_CHECK_LAUNCH();
  return LS_OK;
}

}  // extern "C"
