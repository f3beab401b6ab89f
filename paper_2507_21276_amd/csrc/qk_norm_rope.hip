// Norms of queries and keys for each head with the rotation in the same pass, its backward, its page-writing form for
// serving, and the tables of angles.
//
// A head vector x of dh elements becomes y = R (g * x r), r = (mean(x^2) + eps)^-1/2: r is one sum over the head's lanes, and
// R turns pairs of the first rot elements by the row's angles.  Backward, with dy the gradient of y: du = R^T dy,
//   dg = sum over rows and heads of du * x r,   dx = r (g du - x r^2 S / dh),   S = sum(g du x).
#include <math.h>

#include <initializer_list>
#include <type_traits>

#include "common.h"

namespace {

struct Shape {
  int T, h, hk, dh, rot;
  int norm;              // 1: RMSNorm, else none
  float eps;
  const void *gain_q, *gain_k;
  int pdt;
  const int32_t* pos;
  const float* table;    // [max_pos][rot / 2][2]
  int max_pos;
};

// Where the K and V rows of a serving batch go
struct Pages {
  void *k_pool, *v_pool;
  const int32_t *req, *slot, *block_table;
  int max_pages, page, n_pages;
};

// element offset of a row's slot in a pool [n_pages][hk][page][dh], head 0; -1: a padded row, or nowhere in the pool
__device__ __forceinline__ long slot_of(const Pages& pg, int t, int hk, int dh) {
  const int r = pg.req[t], s = pg.slot[t];
  if (r < 0 || s < 0 || s / pg.page >= pg.max_pages) return -1;
  const int id = pg.block_table[(size_t)r * pg.max_pages + s / pg.page];
  if ((unsigned)id >= (unsigned)pg.n_pages) return -1;
  return ((long)id * hk * pg.page + s % pg.page) * dh;
}

// Pair p < dh / 2 of a head: two element indexes; pairs from rot / 2 on are not turned.
template <int LAYOUT> __device__ __forceinline__ void pair_at(int p, int rot, int* a, int* b) {
  if (LAYOUT == 0 && p < rot / 2) { *a = p; *b = p + rot / 2; }
  else { *a = 2 * p; *b = 2 * p + 1; }   // neighbours; past the turned part too: rot + 2 (p - rot / 2)
}

__device__ __forceinline__ const float* angles(const Shape& s, int t) {
  const int p = min(max(s.pos[t], 0), s.max_pos - 1);
  return s.table + (size_t)p * s.rot;
}

enum { OUT_ROWS = 0, IN_PLACE = 1, TO_PAGES = 2 };

// Workgroups along x at most: a launch's work-items along one dimension are counted in 32 bits, and a larger grid wraps without
// an error.  More workgroups go on along the next free dimension.
constexpr long kGridX = 1 << 22;

// Any even dh up to 512, any alignment: one wavefront per (row, head), a lane holds up to four pairs.  Two-byte accesses: a
// quarter to a third of the vectorised kernels' rate.
template <int LAYOUT, int MODE>
__global__ __launch_bounds__(256) void norm_rope_any_kernel(const void* in, long ld_in, void* out, long ld_out, int dt, Shape s,
                                                            Pages pg) {
  const int heads = s.h + s.hk + (MODE == IN_PLACE ? 0 : s.hk);
  const long item = ((long)blockIdx.y * gridDim.x + blockIdx.x) * 4 + (threadIdx.x >> 6);
  const int lane = threadIdx.x & 63;
  if (item >= (long)s.T * heads) return;
  const int t = (int)(item / heads), hd = (int)(item % heads);
  const int part = hd < s.h ? 0 : hd < s.h + s.hk ? 1 : 2;
  const size_t src = (size_t)t * ld_in + (size_t)hd * s.dh;
  void* dst_base = out;
  size_t dst = (size_t)t * ld_out + (size_t)hd * s.dh;
  if (MODE == TO_PAGES) {
    if (pg.req[t] < 0) return;
    if (part > 0) {
      const long at = slot_of(pg, t, s.hk, s.dh);
      if (at < 0) return;
      dst_base = part == 1 ? pg.k_pool : pg.v_pool;
      dst = (size_t)at + (size_t)(hd - s.h - (part - 1) * s.hk) * pg.page * s.dh;
    }
  }
  float a[4], b[4], sum = 0.f;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int p = lane + 64 * i;
    a[i] = b[i] = 0.f;
    if (p < s.dh / 2) {
      int ia, ib;
      pair_at<LAYOUT>(p, s.rot, &ia, &ib);
      a[i] = load_as_f(in, src + ia, dt);
      b[i] = load_as_f(in, src + ib, dt);
      sum += a[i] * a[i] + b[i] * b[i];
    }
  }
  const float r = s.norm && part < 2 ? rsqrtf(wave_total(sum) / s.dh + s.eps) : 1.f;
  const void* gain = part == 0 ? s.gain_q : part == 1 ? s.gain_k : nullptr;
  const float* cs = s.rot && part < 2 ? angles(s, t) : nullptr;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int p = lane + 64 * i;
    if (p >= s.dh / 2) break;
    int ia, ib;
    pair_at<LAYOUT>(p, s.rot, &ia, &ib);
    float ua = a[i] * r, ub = b[i] * r;
    if (gain) { ua *= load_as_f(gain, ia, s.pdt); ub *= load_as_f(gain, ib, s.pdt); }
    if (cs && p < s.rot / 2) {
      const float c = cs[2 * p], sn = cs[2 * p + 1], ta = ua * c - ub * sn;
      ub = ua * sn + ub * c;
      ua = ta;
    }
    store_from_f(dst_base, dst + ia, dt, ua);
    store_from_f(dst_base, dst + ib, dt, ub);
  }
}

// Backward for the same shapes.  blockIdx.y: q, k (v rows are copied where din is not dout); a workgroup's wavefronts walk
// the part's (row, head) pairs and keep the gains' gradients of their lanes; the workgroup's sum goes to
// partial[y][blockIdx.x][dh].
template <int LAYOUT>
__global__ __launch_bounds__(256) void norm_rope_bwd_any_kernel(const void* dout, long ld_dout, const void* in, long ld_in,
                                                                void* din, long ld_din, int dt, Shape s, float* partial) {
  __shared__ float s_dg[4][512];
  const int part = blockIdx.y, heads = part == 0 ? s.h : s.hk, first = part == 0 ? 0 : part == 1 ? s.h : s.h + s.hk;
  const int wave = threadIdx.x >> 6, lane = threadIdx.x & 63;
  const void* gain = part == 0 ? s.gain_q : part == 1 ? s.gain_k : nullptr;
  float dga[4] = {0.f, 0.f, 0.f, 0.f}, dgb[4] = {0.f, 0.f, 0.f, 0.f};
  const long items = (long)s.T * heads;
  for (long item = (long)blockIdx.x * 4 + wave; item < items; item += (long)gridDim.x * 4) {
    const int t = (int)(item / heads), hd = first + (int)(item % heads);
    const size_t at = (size_t)hd * s.dh;
    const float* cs = s.rot && part < 2 ? angles(s, t) : nullptr;
    float xa[4], xb[4], da[4], db[4], ga[4], gb[4], sq = 0.f, dot = 0.f;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = lane + 64 * i;
      xa[i] = xb[i] = da[i] = db[i] = 0.f;
      ga[i] = gb[i] = 1.f;
      if (p < s.dh / 2) {
        int ia, ib;
        pair_at<LAYOUT>(p, s.rot, &ia, &ib);
        da[i] = load_as_f(dout, (size_t)t * ld_dout + at + ia, dt);
        db[i] = load_as_f(dout, (size_t)t * ld_dout + at + ib, dt);
        if (cs && p < s.rot / 2) {
          const float c = cs[2 * p], sn = cs[2 * p + 1], ta = da[i] * c + db[i] * sn;
          db[i] = db[i] * c - da[i] * sn;
          da[i] = ta;
        }
        if (gain) { ga[i] = load_as_f(gain, ia, s.pdt); gb[i] = load_as_f(gain, ib, s.pdt); }
        if (s.norm && part < 2) {
          xa[i] = load_as_f(in, (size_t)t * ld_in + at + ia, dt);
          xb[i] = load_as_f(in, (size_t)t * ld_in + at + ib, dt);
          sq += xa[i] * xa[i] + xb[i] * xb[i];
          dot += da[i] * ga[i] * xa[i] + db[i] * gb[i] * xb[i];
        }
      }
    }
    float r = 1.f, back = 0.f;
    if (s.norm && part < 2) {
      r = rsqrtf(wave_total(sq) / s.dh + s.eps);
      back = wave_total(dot) * r * r / s.dh;
    }
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int p = lane + 64 * i;
      if (p >= s.dh / 2) break;
      int ia, ib;
      pair_at<LAYOUT>(p, s.rot, &ia, &ib);
      dga[i] += da[i] * xa[i] * r;
      dgb[i] += db[i] * xb[i] * r;
      store_from_f(din, (size_t)t * ld_din + at + ia, dt, r * (da[i] * ga[i] - xa[i] * back));
      store_from_f(din, (size_t)t * ld_din + at + ib, dt, r * (db[i] * gb[i] - xb[i] * back));
    }
  }
  if (!partial || part == 2) return;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const int p = lane + 64 * i;
    if (p >= s.dh / 2) break;
    int ia, ib;
    pair_at<LAYOUT>(p, s.rot, &ia, &ib);
    s_dg[wave][ia] = dga[i];
    s_dg[wave][ib] = dgb[i];
  }
  __syncthreads();
  for (int c = threadIdx.x; c < s.dh; c += 256)
    partial[((size_t)part * gridDim.x + blockIdx.x) * s.dh + c] = s_dg[0][c] + s_dg[1][c] + s_dg[2][c] + s_dg[3][c];
}

// ---- vectorised kernels: dh <= 256 and rot multiples of 8, rows and bases aligned to four elements ----------------------
//
// LPH lanes have a head, each eight of its elements: four pairs, in two vectors of four.  Pairs are local to a lane in
// either layout, and r takes one sum over the lanes, in lane permutations without LDS.  A lane keeps the angles of its
// row and the gains, which are as many bytes as a head itself, over the heads that it works through.
// Bound by the bytes of the rows, few rows by the round trips of a launch.  4096 rows of 96 heads of 128, 16 bits: forward
// 39 us (5.2 TB/s; a large copy reaches 5.2), backward 44 (6.1); with a wavefront a head 146 and 313.  890 rows of 48 heads to
// their pages 9.3 us, one row of 36 heads of 64 4.8.

template <int LPH> __device__ __forceinline__ float head_sum(float v) {
  v = dpp_add<0xb1, 0xf>(v);                  // lane ^ 1
  v = dpp_add<0x4e, 0xf>(v);                  // lane ^ 2
  if (LPH >= 8) v = dpp_add<0x141, 0xf>(v);   // mirrored in eight
  if (LPH >= 16) v = dpp_add<0x140, 0xf>(v);  // mirrored in sixteen
  if (LPH >= 32) v += __shfl_xor(v, 16, 64);
  return v;
}

template <class T> struct Four { typedef T type __attribute__((ext_vector_type(4))); };

// A lane's place in a head: its two vectors, and what it keeps of its row
template <class T, int LAYOUT> struct Lane {
  typedef typename Four<T>::type V4;
  int oa, ob;
  bool live, turned;
  float c[4], s[4];
  __device__ __forceinline__ Lane(const Shape& sh, int sub) {
    live = 8 * sub < sh.dh;
    turned = 8 * sub < sh.rot;
    oa = LAYOUT == 0 && turned ? 4 * sub : 8 * sub;
    ob = LAYOUT == 0 && turned ? 4 * sub + sh.rot / 2 : 8 * sub + 4;
  }
  __device__ __forceinline__ void row(const Shape& sh, int sub, int t) {
    if (!turned) return;
    const f32x4* cs = (const f32x4*)(angles(sh, t) + 8 * sub);
    const f32x4 x = cs[0], y = cs[1];
    c[0] = x[0]; s[0] = x[1]; c[1] = x[2]; s[1] = x[3];
    c[2] = y[0]; s[2] = y[1]; c[3] = y[2]; s[3] = y[3];
  }
  // element e < 4 of vector a or b of pair p: the half layout has the pair (a[p], b[p]), neighbours are (v[2p], v[2p + 1])
  __device__ __forceinline__ void turn(float (&a)[4], float (&b)[4], float sign) const {
    if (!turned) return;
    if (LAYOUT == 0) {
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        const float sn = sign * s[p], x = a[p] * c[p] - b[p] * sn;
        b[p] = a[p] * sn + b[p] * c[p];
        a[p] = x;
      }
    } else {
#pragma unroll
      for (int p = 0; p < 4; ++p) {
        float& u = p < 2 ? a[2 * p] : b[2 * p - 4];
        float& w = p < 2 ? a[2 * p + 1] : b[2 * p - 3];
        const float sn = sign * s[p], x = u * c[p] - w * sn;
        w = u * sn + w * c[p];
        u = x;
      }
    }
  }
};

__device__ __forceinline__ void load_gain(const void* gain, int pdt, int oa, int ob, bool live, float (&g)[8]) {
#pragma unroll
  for (int e = 0; e < 8; ++e) g[e] = gain && live ? load_as_f(gain, (e < 4 ? oa : ob) + (e & 3), pdt) : 1.f;
}

// Heads of a lane in flight: 96 heads of 128 elements are six for each of a workgroup's 16 groups (4096 rows, forward: 2 59 us,
// 4 50, 6 42, 8 43).  Results are stored past the caches: what is written is as large as what is read, and read by another
// kernel (forward and backward together 100 -> 88 us; a verification step with its attention 194 -> 187).
constexpr int kHeads = 6;

// `per` groups of lanes share a token's heads (a power of two); blockIdx.y takes kHeads of each group
template <class T, int LAYOUT, int LPH, int MODE>
__global__ __launch_bounds__(256) void norm_rope_kernel(const T* in, long ld_in, T* out, long ld_out, Shape s, Pages pg, int per) {
  typedef typename Four<T>::type V4;
  const int sub = threadIdx.x % LPH, grp = threadIdx.x / LPH;
  const long t = ((long)blockIdx.z * gridDim.x + blockIdx.x) * (256 / LPH / per) + grp / per;
  if (t >= s.T) return;
  const int heads = s.h + s.hk + (MODE == IN_PLACE ? 0 : s.hk), first = grp % per + blockIdx.y * per * kHeads;
  if (first >= heads) return;
  Lane<T, LAYOUT> ln(s, sub);
  // the rows are on their way while positions, slots, pages and angles are looked up one from the other
  const T* src = in + t * ld_in;
  V4 a[kHeads], b[kHeads];
#pragma unroll
  for (int u = 0; u < kHeads; ++u) {
    const int hd = first + u * per;
    a[u] = b[u] = V4{};
    if (hd < heads && ln.live) {
      a[u] = *(const V4*)(src + (long)hd * s.dh + ln.oa);
      b[u] = *(const V4*)(src + (long)hd * s.dh + ln.ob);
    }
  }
  long at = 0;
  if (MODE == TO_PAGES) {
    if (pg.req[t] < 0) return;
    at = slot_of(pg, (int)t, s.hk, s.dh);
  }
  if (s.rot) ln.row(s, sub, (int)t);
  float gq[8], gk[8];
  load_gain(s.gain_q, s.pdt, ln.oa, ln.ob, ln.live, gq);
  load_gain(s.gain_k, s.pdt, ln.oa, ln.ob, ln.live, gk);
#pragma unroll
  for (int u = 0; u < kHeads; ++u) {
    const int hd = first + u * per;
    if (hd >= heads) break;
    const int part = hd < s.h ? 0 : hd < s.h + s.hk ? 1 : 2;
    float x[4], y[4], sq = 0.f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      x[e] = to_f(a[u][e]);
      y[e] = to_f(b[u][e]);
      sq += x[e] * x[e] + y[e] * y[e];
    }
    if (part < 2) {
      const float r = s.norm ? rsqrtf(head_sum<LPH>(sq) / s.dh + s.eps) : 1.f;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        x[e] = x[e] * r * (part == 0 ? gq[e] : gk[e]);
        y[e] = y[e] * r * (part == 0 ? gq[e + 4] : gk[e + 4]);
      }
      ln.turn(x, y, 1.f);
#pragma unroll
      for (int e = 0; e < 4; ++e) { a[u][e] = from_f<T>(x[e]); b[u][e] = from_f<T>(y[e]); }
    }
    if (!ln.live) continue;
    T* dst = out + t * ld_out + (long)hd * s.dh;
    if (MODE == TO_PAGES && part > 0) {
      if (at < 0) continue;
      dst = (T*)(part == 1 ? pg.k_pool : pg.v_pool) + at + (long)(hd - s.h - (part - 1) * s.hk) * pg.page * s.dh;
    }
    __builtin_nontemporal_store(a[u], (V4*)(dst + ln.oa));
    __builtin_nontemporal_store(b[u], (V4*)(dst + ln.ob));
  }
}

// Backward: a workgroup walks tokens, its lanes keep the gains' gradients of their elements and the workgroup's sum goes to
// partial[part][blockIdx.x][dh].  Both sums over a head, of x^2 and of g du x, are taken before r is needed.  Two heads of a lane
// in flight (four: 95 us instead of 88 for both directions at 4096 rows), 1024 workgroups (512: 92, 2048: 91).
template <class T, int LAYOUT, int LPH>
__global__ __launch_bounds__(256) void norm_rope_bwd_kernel(const T* dout, long ld_dout, const T* in, long ld_in, T* din,
                                                            long ld_din, Shape s, int per, int copy_v, float* partial) {
  typedef typename Four<T>::type V4;
  __shared__ float s_dg[256 * 8];
  constexpr int U = 2;
  const int sub = threadIdx.x % LPH, grp = threadIdx.x / LPH, tokens = 256 / LPH / per, g0 = grp % per;
  Lane<T, LAYOUT> ln(s, sub);
  float gain[2][8], dg[2][8];
  load_gain(s.gain_q, s.pdt, ln.oa, ln.ob, ln.live, gain[0]);
  load_gain(s.gain_k, s.pdt, ln.oa, ln.ob, ln.live, gain[1]);
#pragma unroll
  for (int e = 0; e < 8; ++e) dg[0][e] = dg[1][e] = 0.f;
  for (long t = (long)blockIdx.x * tokens + grp / per; t < s.T; t += (long)gridDim.x * tokens) {
    if (s.rot) ln.row(s, sub, (int)t);
    const T *dy = dout + t * ld_dout, *xr = in + t * ld_in;
    T* dx = din + t * ld_din;
#pragma unroll
    for (int part = 0; part < 2; ++part) {
      const int lo = part == 0 ? 0 : s.h, n = part == 0 ? s.h : s.hk;
      for (int h0 = g0; h0 < n; h0 += per * U) {
        V4 da[U], db[U], xa[U], xb[U];
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int hd = h0 + u * per;
          const long at = (long)(lo + hd) * s.dh;
          da[u] = db[u] = xa[u] = xb[u] = V4{};
          if (hd < n && ln.live) {
            da[u] = *(const V4*)(dy + at + ln.oa);
            db[u] = *(const V4*)(dy + at + ln.ob);
            if (s.norm) {
              xa[u] = *(const V4*)(xr + at + ln.oa);
              xb[u] = *(const V4*)(xr + at + ln.ob);
            }
          }
        }
#pragma unroll
        for (int u = 0; u < U; ++u) {
          const int hd = h0 + u * per;
          if (hd >= n) break;
          float w[4], z[4], sq = 0.f, dot = 0.f;
#pragma unroll
          for (int e = 0; e < 4; ++e) { w[e] = to_f(da[u][e]); z[e] = to_f(db[u][e]); }
          ln.turn(w, z, -1.f);
          if (s.norm) {
            float x[4], y[4];
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              x[e] = to_f(xa[u][e]);
              y[e] = to_f(xb[u][e]);
              sq += x[e] * x[e] + y[e] * y[e];
              dot += w[e] * gain[part][e] * x[e] + z[e] * gain[part][e + 4] * y[e];
            }
            const float r = rsqrtf(head_sum<LPH>(sq) / s.dh + s.eps), back = head_sum<LPH>(dot) * r * r / s.dh;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              dg[part][e] += w[e] * x[e] * r;
              dg[part][e + 4] += z[e] * y[e] * r;
              w[e] = r * (w[e] * gain[part][e] - x[e] * back);
              z[e] = r * (z[e] * gain[part][e + 4] - y[e] * back);
            }
          }
          if (!ln.live) continue;
          const long at = (long)(lo + hd) * s.dh;
          V4 oa, ob;
#pragma unroll
          for (int e = 0; e < 4; ++e) { oa[e] = from_f<T>(w[e]); ob[e] = from_f<T>(z[e]); }
          __builtin_nontemporal_store(oa, (V4*)(dx + at + ln.oa));
          __builtin_nontemporal_store(ob, (V4*)(dx + at + ln.ob));
        }
      }
    }
    if (copy_v && ln.live)
      for (int hd = g0; hd < s.hk; hd += per) {
        const long at = (long)(s.h + s.hk + hd) * s.dh;
        const V4 va = *(const V4*)(dy + at + ln.oa), vb = *(const V4*)(dy + at + ln.ob);
        __builtin_nontemporal_store(va, (V4*)(dx + at + ln.oa));
        __builtin_nontemporal_store(vb, (V4*)(dx + at + ln.ob));
      }
  }
  if (!partial) return;
#pragma unroll
  for (int part = 0; part < 2; ++part) {
    __syncthreads();
    if (ln.live) {
#pragma unroll
      for (int e = 0; e < 8; ++e) s_dg[grp * (LPH * 8) + (e < 4 ? ln.oa + e : ln.ob + e - 4)] = dg[part][e];
    }
    __syncthreads();
    for (int c = threadIdx.x; c < s.dh; c += 256) {
      float v = 0.f;
      for (int g = 0; g < 256 / LPH; ++g) v += s_dg[g * (LPH * 8) + c];
      partial[((size_t)part * gridDim.x + blockIdx.x) * s.dh + c] = v;
    }
  }
}

// dgain (+)= alpha * sum over the workgroups, in a fixed order; 16 columns of one part a workgroup, 64 rows at a time, four
// loads of a thread in flight (1024 rows of 128: 3.2 us; 17 with one row of 64 columns a wavefront, one after the other)
__global__ __launch_bounds__(1024) void gain_sum_kernel(const float* partial, int blocks, int dh, float* dgq, float* dgk,
                                                        int accumulate, const float* alpha) {
  __shared__ float s_sum[64][17];
  const int part = blockIdx.y, row = threadIdx.x >> 4, lane = threadIdx.x & 15, c = blockIdx.x * 16 + lane;
  const float* src = partial + (size_t)part * blocks * dh + c;
  float v = 0.f;
  if (c < dh) {
    int b = row;
    for (; b + 192 < blocks; b += 256) {   // four loads in flight
      const float v0 = src[(size_t)b * dh], v1 = src[(size_t)(b + 64) * dh], v2 = src[(size_t)(b + 128) * dh],
                  v3 = src[(size_t)(b + 192) * dh];
      v += (v0 + v1) + (v2 + v3);
    }
    for (; b < blocks; b += 64) v += src[(size_t)b * dh];
  }
  s_sum[row][lane] = v;
  __syncthreads();
  if (threadIdx.x >= 64) return;
  v = 0.f;
#pragma unroll
  for (int i = 0; i < 16; ++i) v += s_sum[(threadIdx.x >> 4) * 16 + i][lane];
  v += __shfl_xor(v, 16, 64);
  v += __shfl_xor(v, 32, 64);
  if (threadIdx.x >= 16 || c >= dh) return;
  if (alpha) v *= alpha[0];
  float* out = part == 0 ? dgq : dgk;
  out[c] = accumulate ? out[c] + v : v;
}

// Workgroups of the backward pass: the sums over rows are kept by that many
int bwd_blocks(long rows_heads) {
  const long n = (rows_heads + 3) / 4;
  return (int)(n < 1024 ? n : 1024);
}

constexpr int kMaxHalf = 256;   // frequencies passed by value
struct Freqs { double f[kMaxHalf]; };

// table[p][i] = mag * (cos, sin)(p f_i).  A thread takes one frequency and kRun positions: the angle of the first by sincos,
// the next ones by turning it one step further, in 64 bits (each turn adds less than 2^-52 of error: far below the half step
// 2^-25 that the result is rounded by), so that the pass is bound by its writes and not by sincos of 64-bit angles: 131072
// positions of 64 frequencies 12.3 us, 5.5 TB/s.
constexpr int kRun = 16;
__global__ __launch_bounds__(256) void rope_table_kernel(float* table, int n_pos, int half, Freqs fr, double mag) {
  const long idx = (long)blockIdx.x * 256 + threadIdx.x;
  const int i = (int)(idx % half);
  const long p0 = idx / half * kRun;
  if (p0 >= n_pos) return;
  double c, s, c1, s1;
  sincos((double)p0 * fr.f[i], &s, &c);
  sincos(fr.f[i], &s1, &c1);
  const int n = (int)(n_pos - p0 < kRun ? n_pos - p0 : kRun);
  for (int k = 0; k < n; ++k) {
    float* at = table + ((size_t)(p0 + k) * half + i) * 2;
    at[0] = (float)(mag * c);
    at[1] = (float)(mag * s);
    const double t = c * c1 - s * s1;
    s = s * c1 + c * s1;
    c = t;
  }
}

ls_status check_shape(const char* who, int dt, const Shape& s, int layout) {
  LS_REQUIRE(dt == LS_F32 || dt == LS_BF16 || dt == LS_F16, "%s: unknown dtype %d", who, dt);
  LS_REQUIRE(s.T > 0 && s.h > 0 && s.hk > 0, "%s: non-positive size (T %d, heads %d, %d)", who, s.T, s.h, s.hk);
  LS_REQUIRE(s.h <= 65535, "%s: %d heads, at most 65535", who, s.h);
  LS_REQUIRE(s.h % s.hk == 0, "%s: %d query heads do not share %d key heads evenly", who, s.h, s.hk);
  LS_REQUIRE(s.dh >= 2 && s.dh <= 512 && s.dh % 2 == 0, "%s: head_dim %d is not even or outside 2..512", who, s.dh);
  LS_REQUIRE((long)s.T * (s.h + 2L * s.hk) <= 0x7fffffffL * 4, "%s: too many (row, head) pairs", who);
  LS_REQUIRE(s.norm == -1 || s.norm == 1, "%s: kind %d is neither -1 (no norm) nor 1 (RMSNorm)", who, s.norm);
  LS_REQUIRE(s.norm == 1 || (!s.gain_q && !s.gain_k), "%s: gains without a norm", who);
  LS_REQUIRE(s.norm == -1 || s.eps > 0, "%s: eps must be positive", who);
  LS_REQUIRE(s.pdt == LS_F32 || s.pdt == LS_BF16 || s.pdt == LS_F16, "%s: unknown dtype %d of the gains", who, s.pdt);
  LS_REQUIRE(s.rot >= 0 && s.rot <= s.dh && s.rot % 2 == 0, "%s: %d rotated elements of %d", who, s.rot, s.dh);
  LS_REQUIRE(s.rot == 0 || (s.pos && s.table && s.max_pos > 0), "%s: rotation without positions or table", who);
  LS_REQUIRE(layout == LSK_ROPE_HALF || layout == LSK_ROPE_NEIGHBOURS, "%s: unknown layout %d", who, layout);
  return LS_OK;
}

Shape make_shape(int T, int h, int hk, int dh, int kind, const void* gq, const void* gk, int pdt, float eps, int rot,
                 const int32_t* pos, const float* table, int max_pos) {
  return Shape{T, h, hk, dh, rot, kind, eps, gq, gk, pdt, pos, table, max_pos};
}

// Which shapes the vectorised kernels take, and the lanes of a head
bool vec_covers(int dt, const Shape& s, std::initializer_list<const void*> rows, std::initializer_list<long> lds) {
  const size_t bytes = 4 * dtype_size(dt);
  for (const void* p : rows)
    if ((uintptr_t)p % bytes) return false;
  for (const long ld : lds)
    if (ld % 4) return false;
  return s.dh % 8 == 0 && s.dh <= 256 && s.rot % 8 == 0 && (s.rot == 0 || (uintptr_t)s.table % 16 == 0);
}

int pow2_from(int n) {
  int p = 1;
  while (p < n) p *= 2;
  return p;
}

// f(type tag, layout, lanes of a head) for the shape's instance
template <class F> void vec_instance(int dt, int layout, int dh, F f) {
  auto lanes = [&](auto one, auto lay) {
    switch (pow2_from(dh / 8)) {
      case 32: f(one, lay, std::integral_constant<int, 32>()); break;
      case 16: f(one, lay, std::integral_constant<int, 16>()); break;
      case 8: f(one, lay, std::integral_constant<int, 8>()); break;
      default: f(one, lay, std::integral_constant<int, 4>());   // smaller heads leave lanes over
    }
  };
  auto type = [&](auto lay) {
    if (dt == LS_F32) lanes((float*)nullptr, lay);
    else if (dt == LS_BF16) lanes((bf16_t*)nullptr, lay);
    else lanes((f16_t*)nullptr, lay);
  };
  if (layout == LSK_ROPE_HALF) type(std::integral_constant<int, 0>());
  else type(std::integral_constant<int, 1>());
}

template <int MODE>
ls_status launch_fwd(const void* in, long ld_in, void* out, long ld_out, int dt, Shape s, int layout, const Pages& pg,
                     hipStream_t st) {
  s.norm = s.norm == 1;
  const int heads = s.h + s.hk + (MODE == IN_PLACE ? 0 : s.hk);
  if (vec_covers(dt, s, {in, out, pg.k_pool, pg.v_pool}, {ld_in, ld_out})) {
    vec_instance(dt, layout, s.dh, [&](auto* one, auto lay, auto lph) {
      typedef std::remove_pointer_t<decltype(one)> T;
      constexpr int LPH = decltype(lph)::value, groups = 256 / LPH;
      const int need = pow2_from(heads), per = need < groups ? need : groups, tokens = groups / per;
      const long n = ((long)s.T + tokens - 1) / tokens, x = n < kGridX ? n : kGridX;
      const dim3 grid((unsigned)x, (heads + per * kHeads - 1) / (per * kHeads), (unsigned)((n + x - 1) / x));
      norm_rope_kernel<T, decltype(lay)::value, LPH, MODE><<<grid, 256, 0, st>>>((const T*)in, ld_in, (T*)out, ld_out, s, pg, per);
    });
    LS_CHECK_LAUNCH();
    return LS_OK;
  }
  const long n = ((long)s.T * heads + 3) / 4, x = n < kGridX ? n : kGridX;
  const dim3 grid((unsigned)x, (unsigned)((n + x - 1) / x));
  if (layout == LSK_ROPE_HALF) norm_rope_any_kernel<0, MODE><<<grid, 256, 0, st>>>(in, ld_in, out, ld_out, dt, s, pg);
  else norm_rope_any_kernel<1, MODE><<<grid, 256, 0, st>>>(in, ld_in, out, ld_out, dt, s, pg);
  LS_CHECK_LAUNCH();
  return LS_OK;
}

}  // namespace

extern "C" {

ls_status lsk_rope_table(float* table, int n_pos, int rot_dim, float theta, const lsk_rope_scaling* scaling, void* stream) {
  LS_REQUIRE(table, "rope_table: null table");
  LS_REQUIRE(n_pos > 0, "rope_table: non-positive number of positions");
  LS_REQUIRE(rot_dim >= 2 && rot_dim <= 2 * kMaxHalf && rot_dim % 2 == 0, "rope_table: rot_dim %d is not even or outside 2..%d",
             rot_dim, 2 * kMaxHalf);
  LS_REQUIRE(theta > 0 && isfinite(theta), "rope_table: theta must be positive and finite");
  const lsk_rope_scaling plain = {LSK_ROPE_PLAIN, 1.f, 0, 0.f, 0.f, 1.f};
  const lsk_rope_scaling& sc = scaling ? *scaling : plain;
  LS_REQUIRE(sc.kind >= LSK_ROPE_PLAIN && sc.kind <= LSK_ROPE_PARTS, "rope_table: unknown scaling %d", sc.kind);
  LS_REQUIRE(isfinite(sc.magnitude) && sc.magnitude > 0, "rope_table: magnitude must be positive and finite");
  LS_REQUIRE(sc.kind == LSK_ROPE_PLAIN || (sc.factor >= 1 && isfinite(sc.factor)), "rope_table: factor must be at least 1");
  LS_REQUIRE(sc.kind != LSK_ROPE_BASE || rot_dim > 2, "rope_table: the base of a single pair has no effect");
  LS_REQUIRE(sc.kind != LSK_ROPE_PARTS || (sc.orig_len > 0 && sc.beta_fast > sc.beta_slow && sc.beta_slow >= 0),
             "rope_table: parts need orig_len > 0 and beta_fast > beta_slow >= 0");
  const int half = rot_dim / 2;
  Freqs fr;
  double base = theta;
  if (sc.kind == LSK_ROPE_BASE) base *= pow((double)sc.factor, (double)rot_dim / (rot_dim - 2));
  for (int i = 0; i < half; ++i) {
    double f = pow(base, -2.0 * i / rot_dim);
    if (sc.kind == LSK_ROPE_LINEAR) f /= sc.factor;
    if (sc.kind == LSK_ROPE_PARTS) {
      const double turns = sc.orig_len * f / (2.0 * M_PI);
      double g = (turns - sc.beta_slow) / ((double)sc.beta_fast - sc.beta_slow);
      g = g < 0 ? 0 : g > 1 ? 1 : g;
      f *= g + (1.0 - g) / sc.factor;
    }
    fr.f[i] = f;
  }
  const long threads = ((long)n_pos + kRun - 1) / kRun * half;
  rope_table_kernel<<<(unsigned)((threads + 255) / 256), 256, 0, (hipStream_t)stream>>>(table, n_pos, half, fr,
                                                                                        (double)sc.magnitude);
  LS_CHECK_LAUNCH();
  return LS_OK;
}

ls_status lsk_qk_norm_rope(const void* in, long ld_in, void* out, long ld_out, int dt, int T, int h, int hk, int dh, int kind,
                           const void* gain_q, const void* gain_k, int p_dtype, float eps, int rot_dim, int layout,
                           const int32_t* pos, const float* table, int max_pos, void* stream) {
  const Shape s = make_shape(T, h, hk, dh, kind, gain_q, gain_k, p_dtype, eps, rot_dim, pos, table, max_pos);
  LS_TRY(check_shape("qk_norm_rope", dt, s, layout));
  LS_REQUIRE(in && out, "qk_norm_rope: null argument");
  const long width = (h + 2L * hk) * dh;
  LS_REQUIRE(ld_in >= width && ld_out >= width, "qk_norm_rope: rows of %ld elements are %ld and %ld apart", width, ld_in, ld_out);
  LS_REQUIRE(in != out || ld_in == ld_out, "qk_norm_rope: in place, the rows must be equally far apart");
  const Pages none = {};
  return in == out ? launch_fwd<IN_PLACE>(in, ld_in, out, ld_out, dt, s, layout, none, (hipStream_t)stream)
                   : launch_fwd<OUT_ROWS>(in, ld_in, out, ld_out, dt, s, layout, none, (hipStream_t)stream);
}

ls_status lsk_qk_norm_rope_kv_write(const void* qkv, long ld, void* q_out, long ld_q, int dt, int T, int h, int hk, int dh,
                                    int kind, const void* gain_q, const void* gain_k, int p_dtype, float eps, int rot_dim,
                                    int layout, const int32_t* pos, const float* table, int max_pos, const int32_t* req,
                                    const int32_t* slot, void* k_pool, void* v_pool, const int32_t* block_table,
                                    int max_pages, int page, int n_pages, void* stream) {
  const Shape s = make_shape(T, h, hk, dh, kind, gain_q, gain_k, p_dtype, eps, rot_dim, pos, table, max_pos);
  LS_TRY(check_shape("qk_norm_rope_kv_write", dt, s, layout));
  LS_REQUIRE(qkv && q_out && req && k_pool && v_pool && block_table, "qk_norm_rope_kv_write: null argument");
  LS_REQUIRE(pos || slot, "qk_norm_rope_kv_write: neither slots nor positions");
  LS_REQUIRE(max_pages > 0 && n_pages > 0 && page > 0, "qk_norm_rope_kv_write: non-positive page counts");
  LS_REQUIRE(ld >= (h + 2L * hk) * dh && ld_q >= (long)h * dh, "qk_norm_rope_kv_write: rows overlap (ld %ld, ld_q %ld)", ld, ld_q);
  LS_REQUIRE(qkv != q_out || ld == ld_q, "qk_norm_rope_kv_write: in place, the rows must be equally far apart");
  const Pages pg = {k_pool, v_pool, req, slot ? slot : pos, block_table, max_pages, page, n_pages};
  return launch_fwd<TO_PAGES>(qkv, ld, q_out, ld_q, dt, s, layout, pg, (hipStream_t)stream);
}

size_t lsk_qk_norm_rope_bwd_partial_floats(int T, int h, int hk, int dh) {
  if (T <= 0 || h <= 0 || hk <= 0 || dh <= 0) return 0;
  return (size_t)2 * bwd_blocks((long)T * h) * dh;
}

ls_status lsk_qk_norm_rope_bwd(const void* dout, long ld_dout, const void* in, long ld_in, void* din, long ld_din, int dt, int T,
                               int h, int hk, int dh, int kind, const void* gain_q, const void* gain_k, int p_dtype, float eps,
                               int rot_dim, int layout, const int32_t* pos, const float* table, int max_pos, float* dgain_q,
                               float* dgain_k, int accumulate, const float* alpha_dev, float* partial, void* stream) {
  Shape s = make_shape(T, h, hk, dh, kind, gain_q, gain_k, p_dtype, eps, rot_dim, pos, table, max_pos);
  LS_TRY(check_shape("qk_norm_rope_bwd", dt, s, layout));
  LS_REQUIRE(dout && din && (in || kind == -1), "qk_norm_rope_bwd: null argument");
  const long width = (h + 2L * hk) * dh;
  LS_REQUIRE(ld_dout >= width && ld_din >= width && (kind == -1 || ld_in >= width),
             "qk_norm_rope_bwd: rows of %ld elements are %ld, %ld and %ld apart", width, ld_dout, ld_in, ld_din);
  LS_REQUIRE(din != dout || ld_din == ld_dout, "qk_norm_rope_bwd: in place, the rows must be equally far apart");
  LS_REQUIRE(din != in, "qk_norm_rope_bwd: din must not be the forward's input");
  LS_REQUIRE(!dgain_q == !dgain_k, "qk_norm_rope_bwd: one of the gains' gradients is null");
  LS_REQUIRE(!dgain_q || (gain_q && gain_k), "qk_norm_rope_bwd: gradients of gains that are not there");
  LS_REQUIRE(!dgain_q || partial, "qk_norm_rope_bwd: null partial");
  LS_REQUIRE(!dgain_q || dgain_q != dgain_k, "qk_norm_rope_bwd: the gains' gradients share one place");
  hipStream_t st = (hipStream_t)stream;
  s.norm = s.norm == 1;
  int blocks = bwd_blocks((long)T * h);
  float* sums = dgain_q ? partial : nullptr;
  if (vec_covers(dt, s, {dout, s.norm ? in : nullptr, din}, {ld_dout, s.norm ? ld_in : 0, ld_din})) {
    vec_instance(dt, layout, dh, [&](auto* one, auto lay, auto lph) {
      typedef std::remove_pointer_t<decltype(one)> T_;
      constexpr int LPH = decltype(lph)::value, groups = 256 / LPH;
      const int need = pow2_from(h), per = need < groups ? need : groups, tokens = groups / per;
      const long all = ((long)T + tokens - 1) / tokens;
      if (all < blocks) blocks = (int)all;
      norm_rope_bwd_kernel<T_, decltype(lay)::value, LPH><<<blocks, 256, 0, st>>>(
          (const T_*)dout, ld_dout, (const T_*)in, ld_in, (T_*)din, ld_din, s, per, din != dout, sums);
    });
  } else {
    const dim3 grid(blocks, din == dout ? 2 : 3);
    if (layout == LSK_ROPE_HALF) norm_rope_bwd_any_kernel<0><<<grid, 256, 0, st>>>(dout, ld_dout, in, ld_in, din, ld_din, dt, s, sums);
    else norm_rope_bwd_any_kernel<1><<<grid, 256, 0, st>>>(dout, ld_dout, in, ld_in, din, ld_din, dt, s, sums);
  }
  LS_CHECK_LAUNCH();
  if (sums) {
    gain_sum_kernel<<<dim3((dh + 15) / 16, 2), 1024, 0, st>>>(sums, blocks, dh, dgain_q, dgain_k, accumulate, alpha_dev);
    LS_CHECK_LAUNCH();
  }
  return LS_OK;
}

}  // extern "C"
