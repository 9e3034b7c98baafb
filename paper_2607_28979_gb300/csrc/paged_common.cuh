// Helpers shared by the paged-cache kernels: what a batch's entries are, and the split of an
// attention's work over CTAs.
#pragma once

#include <cuda_bf16.h>

#include "paged_internal.h"
#include "ptx.cuh"

namespace mot {
namespace {

// Sum of v over the CTA's threads before this one; `total` over all of them. `sh`: 33 words.
template <class T>
__device__ __forceinline__ T block_scan(T v, T* sh, T& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, n_warps = blockDim.x >> 5;
  T x = v;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const T y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  __syncthreads();   // sh may still be read by the scan before
  if (lane == 31) sh[warp] = x;
  __syncthreads();
  if (warp == 0) {
    T w = lane < n_warps ? sh[lane] : T(0);
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const T y = __shfl_up_sync(0xffffffffu, w, o);
      if (lane >= o) w += y;
    }
    sh[lane] = w;
  }
  __syncthreads();
  total = sh[n_warps - 1];
  return x - v + (warp ? sh[warp - 1] : T(0));
}

// Entry i of a batch: its slot (-1: outside the table), its rows [r0, r0 + m) and its length,
// clamped into their ranges, so that whatever the arrays hold every index stays in bounds.
struct PagedSeq {
  int32_t slot, r0, m, len;
};
__device__ __forceinline__ PagedSeq paged_seq(const PagedDims& d, const PagedBatch& b, const int32_t* lens,
                                              int32_t* status, int i) {
  PagedSeq s;
  s.slot = b.seqs[i];
  const int a = b.starts[i], e = b.starts[i + 1];
  s.r0 = min(max(a, 0), b.rows);
  s.m = min(max(e, s.r0), b.rows) - s.r0;
  s.len = 0;
  bool bad = a != s.r0 || e - a != s.m;
  if (s.slot < 0 || s.slot >= d.max_seqs) {
    s.slot = -1;
    bad = true;
  } else {
    const int L = lens[s.slot];
    const int64_t cap = min(int64_t(d.max_pages) << d.lp, int64_t(INT32_MAX) / 2);
    s.len = L < 0 ? 0 : (L > cap ? int32_t(cap) : L);
    bad |= s.len != L;
  }
  if (bad) atomicOr(status, kStatusPageUse);
  return s;
}

// ---------------------------------------------------------------- split of an attention's work
//
// An item is (entry i, key/value head, tile of BM rows), a row being (new token t, query head g of
// the group): row r = t G + g of the entry's m G rows. Its units are its tiles of TK keys; causal,
// so an item's units end with the tile that holds its last row's position (one unit at least: rows
// before position 0 are written too). The W units of a call in the order (entry, head, row tile,
// key tile) are dealt to the CTAs in equal runs, CTA c of C taking [W c / C, W (c + 1) / C): every
// CTA has the same work whatever the lengths, at most its first and its last item are shared with
// others, and those items' partial results are joined by the CTA that finishes last, in order.

// sum over i < n of floor((a i + b) / m), for a, b >= 0 and m > 0, by the steps of Euclid's algorithm.
__device__ inline int64_t floor_sum(int64_t n, int64_t m, int64_t a, int64_t b) {
  int64_t s = 0;
  while (n > 0) {
    s += n * (n - 1) / 2 * (a / m) + n * (b / m);
    a %= m;
    b %= m;
    const int64_t y = a * n + b;
    if (y < m) break;
    n = y / m;
    b = y % m;
    const int64_t t = m;
    m = a;
    a = t;
  }
  return s;
}

template <int BM, int TK>
struct PagedSplit {
  // Row tiles of an entry.
  static __device__ __forceinline__ int row_tiles(int m, int G) { return (m * G + BM - 1) / BM; }
  // Units of row tile rt: the position of its last row is len - m + x / G.
  static __device__ __forceinline__ int units(const PagedSeq& s, int G, int rt) {
    const int x = min((rt + 1) * BM, s.m * G) - 1;
    const int p = s.len - s.m + x / G;
    return p < 0 ? 1 : p / TK + 1;
  }
  // Units of the row tiles [0, rt) of one head.
  static __device__ __forceinline__ int64_t before(const PagedSeq& s, int G, int rt) {
    if (rt == 0) return 0;
    if (rt <= 4 || s.len < s.m) {   // few terms, or rows before position 0 (a malformed batch)
      int64_t u = 0;
      for (int r = 0; r < rt; ++r) u += units(s, G, r);
      return u;
    }
    const int R = row_tiles(s.m, G);
    const int whole = rt < R ? rt : R - 1;   // the last tile may be short
    int64_t u = whole + floor_sum(whole, int64_t(G) * TK, BM, int64_t(s.len - s.m) * G + BM - 1);
    if (rt == R) u += units(s, G, R - 1);
    return u;
  }
  static __device__ __forceinline__ int64_t head_units(const PagedSeq& s, int G) {
    return before(s, G, row_tiles(s.m, G));
  }
};

// A run of units: where it stands, and where the call's W units and C CTAs put it.
struct PagedCursor {
  PagedSeq s;
  int64_t u, u_end;      // global units [u, u_end) are left
  int64_t W, head_u;     // all units; units of one head of the entry
  int32_t C;             // CTAs that have work
  int32_t i, hk, rt, kt; // the next unit
  // CTA that unit x belongs to
  __device__ __forceinline__ int owner(int64_t x) const { return int(((x + 1) * C - 1) / W); }
};

// The run of CTA blockIdx.x. Called by all threads; `sh` and `out` are shared. False: no work.
template <int BM, int TK>
__device__ bool paged_begin(const PagedAttnArgs& a, int64_t* sh, PagedCursor* out, PagedCursor& c) {
  using S = PagedSplit<BM, TK>;
  const int G = a.d.Hq / a.d.H, H = a.d.H, T = blockDim.x, tid = threadIdx.x;
  int64_t mine = 0, W = 0, at = 0;
  const int n = a.b.n;
  for (int i0 = 0; i0 < n; i0 += T) {
    mine = 0;
    if (i0 + tid < n) mine = H * S::head_units(paged_seq(a.d, a.b, a.lens, a.status, i0 + tid), G);
    int64_t t;
    at = block_scan(mine, sh, t) + W;
    W += t;
  }
  const int C = W < int64_t(gridDim.x) ? int(W) : int(gridDim.x);
  if (int(blockIdx.x) >= C) return false;
  const int64_t u = W * int(blockIdx.x) / C, u_end = W * (int(blockIdx.x) + 1) / C;
  int64_t carry = 0;
  for (int i0 = 0; i0 < n; i0 += T) {
    if (n > T) {   // more entries than threads: their sums again, a piece at a time
      mine = 0;
      if (i0 + tid < n) mine = H * S::head_units(paged_seq(a.d, a.b, a.lens, a.status, i0 + tid), G);
      int64_t t;
      at = block_scan(mine, sh, t) + carry;
      carry += t;
    }
    if (u >= at && u < at + mine) {
      PagedCursor o;
      o.i = i0 + tid;
      o.s = paged_seq(a.d, a.b, a.lens, a.status, o.i);
      o.W = W;
      o.C = C;
      o.u = u;
      o.u_end = u_end;
      o.head_u = mine / H;
      int64_t r = u - at;
      o.hk = int(r / o.head_u);
      r -= o.hk * o.head_u;
      int lo = 0, hi = S::row_tiles(o.s.m, G) - 1;   // the last rt with before(rt) <= r
      while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (S::before(o.s, G, mid) <= r) lo = mid;
        else hi = mid - 1;
      }
      o.rt = lo;
      o.kt = int(r - S::before(o.s, G, lo));
      *out = o;
    }
    if (n > T && carry > u) break;
  }
  __syncthreads();
  c = *out;
  return true;
}

// One piece of a run: units [kt, kt + n) of the item's `units`.
struct PagedPiece {
  int32_t kt, n, units;
  bool whole;
  int32_t c0, c1;   // the item's CTAs, in order
};
template <int BM, int TK>
__device__ __forceinline__ PagedPiece paged_piece(const PagedCursor& c, int G) {
  PagedPiece p;
  p.units = PagedSplit<BM, TK>::units(c.s, G, c.rt);
  p.kt = c.kt;
  const int64_t left = c.u_end - c.u;
  p.n = left < p.units - c.kt ? int(left) : p.units - c.kt;
  p.whole = p.kt == 0 && p.n == p.units;
  p.c0 = p.c1 = int(blockIdx.x);
  if (!p.whole) {
    p.c0 = c.owner(c.u - c.kt);
    p.c1 = c.owner(c.u - c.kt + p.units - 1);
  }
  return p;
}
// Behind a piece; loads the next entry where the run goes on to it. Uniform over the CTA.
template <int BM, int TK>
__device__ __forceinline__ void paged_next(const PagedAttnArgs& a, PagedCursor& c, const PagedPiece& p) {
  using S = PagedSplit<BM, TK>;
  const int G = a.d.Hq / a.d.H;
  c.u += p.n;
  c.kt = 0;
  if (c.u >= c.u_end) return;
  if (++c.rt < S::row_tiles(c.s.m, G)) return;
  c.rt = 0;
  if (++c.hk < a.d.H) return;
  c.hk = 0;
  do {   // ends: units are left, so an entry with rows follows
    c.s = paged_seq(a.d, a.b, a.lens, a.status, ++c.i);
  } while (c.s.m == 0 && c.i + 1 < a.b.n);
}

// Partial results of a piece: rows [BM][D] of sum_j 2^(s_j - m) v_j, then [BM] m and [BM] l = sum_j
// 2^(s_j - m) (s: scores times log2 e). A CTA has two places: 0 for a piece that does not start its
// item, 1 for one that starts it.
template <int BM, int D>
__device__ __forceinline__ float* paged_part(const PagedAttnArgs& a, int cta, int which) {
  return a.part + (int64_t(cta) * 2 + which) * (BM * (D + 2));
}
// Where row r of the item goes (rows of D elements of q and out).
__device__ __forceinline__ int64_t paged_out_row(const PagedCursor& c, int H, int G, int r) {
  const int t = r / G;
  return (int64_t(c.s.r0 + t) * H + c.hk) * G + (r - t * G);
}
// After the partial results of a piece are written (by all threads that `tid` counts, and a barrier):
// true in one thread that finds itself behind the last of the item's CTAs. The counter is zero again
// for the next call.
__device__ __forceinline__ bool paged_arrive(const PagedAttnArgs& a, const PagedPiece& p) {
  __threadfence();
  const bool last = atomicAdd(&a.count[p.c0], 1) == p.c1 - p.c0;
  if (last) a.count[p.c0] = 0;
  __threadfence();
  return last;
}
// Joins the item's pieces in the order of their CTAs, `rows` rows from row r0 of the entry, and writes
// the output. Four columns a thread.
template <class T>
__device__ __forceinline__ void paged_store4(T* dst, const float (&o)[4], float f) {
  if constexpr (sizeof(T) == 2) {
    __nv_bfloat162 x = __floats2bfloat162_rn(o[0] * f, o[1] * f), y = __floats2bfloat162_rn(o[2] * f, o[3] * f);
    *reinterpret_cast<uint2*>(dst) =
        make_uint2(*reinterpret_cast<uint32_t*>(&x), *reinterpret_cast<uint32_t*>(&y));
  } else {
    *reinterpret_cast<float4*>(dst) = make_float4(o[0] * f, o[1] * f, o[2] * f, o[3] * f);
  }
}
// By all threads of the CTA; `fs`: paged_join_floats<BM>() floats of shared memory that nothing else holds.
constexpr int kJoinPieces = 32;
template <int BM>
__host__ __device__ constexpr int paged_join_floats() {
  return BM * (kJoinPieces + 2);
}
template <class T, int BM, int D>
__device__ __forceinline__ void paged_join(const PagedAttnArgs& a, const PagedCursor& c, const PagedPiece& p, float* fs,
                                           int tid, int n_threads) {
  const int G = a.d.Hq / a.d.H, r0 = c.rt * BM, rows = min(BM, c.s.m * G - r0), n = p.c1 - p.c0 + 1;
  float* sw = fs;                       // [piece][row]: a piece's weight
  float* sms = fs + BM * kJoinPieces;   // the row's maximum
  float* sinv = sms + BM;               // and 1 / its sum
  auto part = [&](int k) { return paged_part<BM, D>(a, p.c0 + k, k == 0); };
  // a warp per row: maximum and sum over the pieces
  const int warp = tid >> 5, lane = tid & 31;
  for (int r = warp; r < rows; r += n_threads >> 5) {
    float m = -INFINITY, l = 0.f;
    for (int k = lane; k < n; k += 32) m = fmaxf(m, __ldcg(part(k) + BM * D + r));
#pragma unroll
    for (int o = 16; o; o >>= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    m = m == -INFINITY ? 0.f : m;
    for (int k = lane; k < n; k += 32)
      l = fmaf(exp2f(__ldcg(part(k) + BM * D + r) - m), __ldcg(part(k) + BM * (D + 1) + r), l);
#pragma unroll
    for (int o = 16; o; o >>= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    if (lane == 0) {
      sms[r] = m;
      sinv[r] = l == 0.f ? 0.f : 1.f / l;
    }
  }
  // then four columns a thread, kJoinPieces pieces at a time
  constexpr int kMine = (BM * D / 4 + 127) / 128;   // at 128 threads
  float o[kMine][4];
#pragma unroll
  for (int y = 0; y < kMine; ++y)
#pragma unroll
    for (int e = 0; e < 4; ++e) o[y][e] = 0.f;
  for (int k0 = 0; k0 < n; k0 += kJoinPieces) {
    const int nk = min(kJoinPieces, n - k0);
    __syncthreads();
    for (int x = tid; x < nk * rows; x += n_threads) {
      const int k = x / rows, r = x - k * rows;
      sw[k * BM + r] = exp2f(__ldcg(part(k0 + k) + BM * D + r) - sms[r]);
    }
    __syncthreads();
#pragma unroll
    for (int y = 0; y < kMine; ++y) {
      const int x = tid + y * n_threads;
      if (x >= rows * (D / 4)) break;
      const int r = x / (D / 4), col = (x - r * (D / 4)) * 4;
#pragma unroll 8
      for (int k = 0; k < nk; ++k) {
        const float f = sw[k * BM + r];
        const float4 v = __ldcg(reinterpret_cast<const float4*>(part(k0 + k) + r * D + col));
        o[y][0] = fmaf(f, v.x, o[y][0]);
        o[y][1] = fmaf(f, v.y, o[y][1]);
        o[y][2] = fmaf(f, v.z, o[y][2]);
        o[y][3] = fmaf(f, v.w, o[y][3]);
      }
    }
  }
#pragma unroll
  for (int y = 0; y < kMine; ++y) {
    const int x = tid + y * n_threads;
    if (x >= rows * (D / 4)) break;
    const int r = x / (D / 4), col = (x - r * (D / 4)) * 4;
    paged_store4(static_cast<T*>(a.out) + paged_out_row(c, a.d.H, G, r0 + r) * D + col, o[y], sinv[r]);
  }
}

// The pool row (in rows of d elements) of position `pos` and head hk of a slot's page entry.
__device__ __forceinline__ int64_t paged_row(const PagedDims& d, int page, int hk, int pos) {
  return (int64_t(page) * d.H + hk) * d.P + (pos & (d.P - 1));
}
// A table entry, held inside the pool.
__device__ __forceinline__ int paged_page(const PagedDims& d, const int32_t* table, int32_t* status,
                                          int slot, int pos) {
  const int p = table[int64_t(slot) * d.max_pages + (pos >> d.lp)];
  if (p >= 0 && p < d.n_pages) return p;
  atomicOr(status, kStatusPageUse);
  return 0;
}

}  // namespace
}  // namespace mot
