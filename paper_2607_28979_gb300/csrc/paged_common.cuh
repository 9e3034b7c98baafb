// Helpers shared by the paged-cache kernels: what a batch's entries are, and the split of an
// attention's work over CTAs.
#pragma once

#include <cuda_bf16.h>

#include "paged_internal.h"
#include "ptx.cuh"

namespace mot {
namespace {

// Whether a change was refused, and none behind it is made.
__device__ __forceinline__ bool refused(const int32_t* status) {
  return (*reinterpret_cast<const volatile int32_t*>(status) & kStatusPages) != 0;
}

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
// before position 0 are written too). Two ways to deal them to the CTAs:
//   runs    the W units of a call in the order (entry, head, row tile, key tile) in equal runs, CTA c of
//           C taking [W c / C, W (c + 1) / C): every CTA has the same work whatever the lengths, and at
//           most its first and its last item are shared with others;
//   pieces  each item in pieces of `coarse` units, one piece per CTA, where that makes no more pieces
//           than CTAs. No CTA then has parts of two items, which cost it some microseconds (a piece's
//           start and end do not overlap with another's): taken while coarse is small, where that
//           outweighs the CTAs that have less than their share.
// The partial results of an item in several pieces are joined by the CTA that finishes last, in order. Where an item
// costs a CTA time of its own beside its units, runs count it as PAD units more, in front of the others.

// sum over i < n of floor((a i + b) / m), for a, b >= 0 and m > 0, by the steps of Euclid's algorithm.
__device__ __noinline__ int64_t floor_sum(int64_t n, int64_t m, int64_t a, int64_t b) {
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

template <int BM, int TK, int PAD = 0>
struct PagedSplit {
  // Row tiles of an entry.
  static __device__ __forceinline__ int row_tiles(int m, int G) { return (m * G + BM - 1) / BM; }
  // Units, or pieces of f units, of row tile rt: the position of its last row is len - m + x / G.
  static __device__ __forceinline__ int units(const PagedSeq& s, int G, int rt, int f = 1) {
    const int x = min((rt + 1) * BM, s.m * G) - 1;
    const int p = s.len - s.m + x / G;
    return p < 0 ? 1 : p / (TK * f) + 1;
  }
  // Those of the row tiles [0, rt) of one head, with the items' own (f = 0: runs; else pieces of f units).
  static __device__ __forceinline__ int64_t before(const PagedSeq& s, int G, int rt, int f) {
    return f ? plain(s, G, rt, f) : plain(s, G, rt, 1) + int64_t(rt) * PAD;
  }
  static __device__ __forceinline__ int64_t plain(const PagedSeq& s, int G, int rt, int f) {
    if (rt == 0) return 0;
    if (rt <= 4 || s.len < s.m) {   // few terms, or rows before position 0 (a malformed batch)
      int64_t u = 0;
      for (int r = 0; r < rt; ++r) u += units(s, G, r, f);
      return u;
    }
    const int R = row_tiles(s.m, G);
    const int whole = rt < R ? rt : R - 1;   // the last tile may be short
    int64_t u = whole + floor_sum(whole, int64_t(G) * TK * f, BM, int64_t(s.len - s.m) * G + BM - 1);
    if (rt == R) u += units(s, G, R - 1, f);
    return u;
  }
  static __device__ __forceinline__ int64_t head_units(const PagedSeq& s, int G, int f) {
    return before(s, G, row_tiles(s.m, G), f);
  }
};

// A CTA's share: where it stands, and where the call's units put the others.
struct PagedCursor {
  PagedSeq s;
  int64_t u, u_end;      // runs: global units [u, u_end) are left; pieces: the piece, and one more
  int64_t W;             // runs: all units
  int32_t C;             // runs: CTAs that have work
  int32_t coarse;        // units of a piece; 0: runs
  int32_t i, hk, rt, kt; // the next unit; runs: kt counts the item's own too
  // runs: the CTA that unit x belongs to
  __device__ __forceinline__ int owner(int64_t x) const;
};

// a / b for a, b >= 0, in 32 bits where they fit (a 64-bit division takes some hundred cycles).
__device__ __forceinline__ int64_t div_fast(int64_t a, int64_t b) {
  return uint64_t(a | b) >> 32 ? a / b : int64_t(uint32_t(a) / uint32_t(b));
}

__device__ __forceinline__ int PagedCursor::owner(int64_t x) const { return int(div_fast((x + 1) * C - 1, W)); }

// One piece of a share: units [kt, kt + n) of the item's `units`.
struct PagedPiece {
  int32_t kt, n, units;
  int32_t run;      // runs: the units that it takes of the run
  bool whole;
  int32_t c0, c1;   // the item's CTAs, in order
};
// A share in shared memory: in registers it would be spilled by the loops that it stands around.
struct PagedShare {
  PagedCursor c;
  PagedPiece p;
  int32_t work;   // whether this CTA has a share, or is not through it
};
template <int BM, int TK, int PAD = 0>
__device__ __forceinline__ PagedPiece paged_piece(const PagedCursor& c, int G) {
  PagedPiece p;
  p.units = PagedSplit<BM, TK>::units(c.s, G, c.rt);
  if (c.coarse) {
    p.kt = c.kt;
    p.n = min(c.coarse, p.units - p.kt);
    p.whole = p.n == p.units;
    p.c0 = int(blockIdx.x) - p.kt / c.coarse;
    p.c1 = p.c0 + (p.units - 1) / c.coarse;
    return p;
  }
  const int64_t left = c.u_end - c.u;
  p.run = left < p.units + PAD - c.kt ? int(left) : p.units + PAD - c.kt;
  p.kt = max(c.kt - PAD, 0);
  p.n = c.kt + p.run - PAD - p.kt;   // above 0: a run that ends in an item's own units has none of it
  p.whole = p.kt == 0 && p.n == p.units;
  p.c0 = p.c1 = int(blockIdx.x);
  if (!p.whole) {
    p.c0 = c.owner(c.u - c.kt + PAD);
    p.c1 = c.owner(c.u - c.kt + PAD + p.units - 1);
  }
  return p;
}
// Behind a piece; loads the next entry where the run goes on to it.
template <int BM, int TK, int PAD = 0>
__device__ __forceinline__ void paged_next(const PagedAttnArgs& a, PagedCursor& c, const PagedPiece& p) {
  using S = PagedSplit<BM, TK>;
  const int G = a.d.Hq / a.d.H;
  c.u = c.coarse ? c.u_end : c.u + p.run;
  c.kt = 0;
  if (c.u >= c.u_end - PAD) {   // nothing is left, or only an item's own units
    c.u = c.u_end;
    return;
  }
  if (++c.rt < S::row_tiles(c.s.m, G)) return;
  c.rt = 0;
  if (++c.hk < a.d.H) return;
  c.hk = 0;
  do {   // ends: units are left, so an entry with rows follows
    c.s = paged_seq(a.d, a.b, a.lens, a.status, ++c.i);
  } while (c.s.m == 0 && c.i + 1 < a.b.n);
}
// The same on a share, in one thread.
template <int BM, int TK, int PAD = 0>
__device__ __forceinline__ void paged_step(const PagedAttnArgs& a, PagedShare& st) {
  paged_next<BM, TK, PAD>(a, st.c, st.p);
  st.work = st.c.u < st.c.u_end;
  if (st.work) st.p = paged_piece<BM, TK, PAD>(st.c, a.d.Hq / a.d.H);
}

// The share of CTA blockIdx.x, with its first piece: a run of `least` units at least where there are as
// many, or a piece of `least` to `most` units (or of more, where `near` is set and that makes no CTA's work more than
// an eighth longer than the runs). Called by all threads, which see st (in shared memory, as
// sh) behind it. Up to 32 entries are one warp's, an entry per lane, without a barrier between.
template <int BM, int TK, int PAD = 0>
__device__ __forceinline__ void paged_begin(const PagedAttnArgs& a, int least, int most, int64_t* sh, PagedShare& st,
                                            bool near = false) {
  using S = PagedSplit<BM, TK, PAD>;
  const int G = a.d.Hq / a.d.H, H = a.d.H, n = a.b.n;
  const bool by_warp = n <= 32;
  const int T = by_warp ? 32 : int(blockDim.x), me = threadIdx.x;
  if (threadIdx.x == 0) st.work = 0;
  // before another thread sets it (shuffles order no memory)
  if (by_warp) __syncwarp();
  else __syncthreads();
  if (!by_warp || threadIdx.x < 32) {
    auto scan = [&](int64_t v, int64_t& t) -> int64_t {
      if (!by_warp) return block_scan(v, sh, t);
      int64_t x = v;
      for (int o = 1; o < n; o <<= 1) {   // the lanes from n on have nothing
        const int64_t y = __shfl_up_sync(0xffffffffu, x, o);
        if (me >= o) x += y;
      }
      t = __shfl_sync(0xffffffffu, x, n - 1);
      return x - v;
    };
    // all entries' units (f = 0), or pieces of f; `at`, `mine`: of this thread's entry among the last T entries
    int64_t mine = 0, at = 0;
    PagedSeq ms{-1, 0, 0, 0};
    if (n <= T && me < n) ms = paged_seq(a.d, a.b, a.lens, a.status, me);
    auto total = [&](int f) -> int64_t {
      int64_t W = 0;
      for (int i0 = 0; i0 < n; i0 += T) {
        if (n > T) {   // more entries than threads: a piece at a time
          ms.m = 0;
          if (i0 + me < n) ms = paged_seq(a.d, a.b, a.lens, a.status, i0 + me);
        }
        mine = ms.m ? H * S::head_units(ms, G, f) : 0;
        int64_t t;
        at = W + scan(mine, t);
        W += t;
      }
      return W;
    };
    int64_t W = total(1);
    const int64_t grid = gridDim.x;
    // the items of the batch: pieces of f units make W / f + items of them at most
    const int64_t items = int64_t(H) * (int64_t(a.max_chunk) * G <= BM ? n : int64_t(a.b.rows) * G / BM + n);
    int f = 0;
    if (items < grid && W > 0) {
      const int64_t need = div_fast(W + grid - items - 1, grid - items);
      if (need <= most || (near && 8 * need * grid <= 9 * W)) {
        f = need < least ? least : int(need);
        if (f > 1) W = total(f);
        if (W > grid) {   // max_chunk was no bound: runs
          f = 0;
          if (!PAD) W = total(1);
        }
      }
    }
    if (PAD && !f) W = total(0);
    const int64_t runs = div_fast(W + least + PAD - 1, least + PAD);
    const int C = f || runs < grid ? int(f ? W : runs) : int(grid);
    if (int(blockIdx.x) < C) {
      const int64_t u = f ? int64_t(blockIdx.x) : div_fast(W * int(blockIdx.x), C);
      int64_t carry = 0;
      for (int i0 = 0; i0 < n; i0 += T) {
        if (n > T) {
          ms.m = 0;
          if (i0 + me < n) ms = paged_seq(a.d, a.b, a.lens, a.status, i0 + me);
          mine = ms.m ? H * S::head_units(ms, G, f) : 0;
          int64_t t;
          at = carry + scan(mine, t);
          carry += t;
        }
        if (u >= at && u < at + mine) {
          PagedCursor o;
          o.i = i0 + me;
          o.s = ms;
          o.W = W;
          o.C = C;
          o.coarse = f;
          o.u = u;
          o.u_end = f ? u + 1 : div_fast(W * (int(blockIdx.x) + 1), C);
          const int64_t head_u = div_fast(mine, H);
          int64_t r = u - at;
          o.hk = int(div_fast(r, head_u));
          r -= o.hk * head_u;
          int lo = 0, hi = S::row_tiles(o.s.m, G) - 1;   // the last rt with before(rt) <= r
          while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (S::before(o.s, G, mid, f) <= r) lo = mid;
            else hi = mid - 1;
          }
          o.rt = lo;
          o.kt = int(r - S::before(o.s, G, lo, f)) * (f ? f : 1);
          if (!f && o.u_end - o.u <= PAD - o.kt) {   // nothing but an item's own units: its first CTA is the next
            st.work = 0;
          } else {
            st.c = o;
            st.p = paged_piece<BM, TK, PAD>(o, G);
            st.work = 1;
          }
        }
        if (n > T && carry > u) break;
      }
    }
  }
  __syncthreads();
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
// Four columns of a result: the weighted sums over the sum of the weights, and 0 where no weight is above 0
// (the sums are 0 or, by values that are not finite, NaN then).
template <class T>
__device__ __forceinline__ void paged_store4(T* dst, const float (&o)[4], float l) {
  const bool none = l == 0.f;
  const float f = 1.f / l;
  const float4 r = none ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(o[0] * f, o[1] * f, o[2] * f, o[3] * f);
  if constexpr (sizeof(T) == 2) {
    __nv_bfloat162 x = __floats2bfloat162_rn(r.x, r.y), y = __floats2bfloat162_rn(r.z, r.w);
    *reinterpret_cast<uint2*>(dst) =
        make_uint2(*reinterpret_cast<uint32_t*>(&x), *reinterpret_cast<uint32_t*>(&y));
  } else {
    *reinterpret_cast<float4*>(dst) = r;
  }
}

// The join of an item's n pieces: up to 8 at once by the CTA that finishes last; more in two levels, in
// groups of 8 (of 32 above 64 pieces), each joined into its first piece's place by its last CTA, and the
// groups by the last of these.
struct PagedGroup {
  int32_t first, n, stride;   // places of the CTAs first, first + stride, ..: n of them
  bool is_item_first;         // `first` is the item's first CTA: its place 1
  bool final;                 // the join gives the item's result
};
template <int BM, int D>
__device__ __forceinline__ float* paged_place(const PagedAttnArgs& a, const PagedGroup& g, int k) {
  return paged_part<BM, D>(a, g.first + k * g.stride, k == 0 && g.is_item_first);
}
__device__ __forceinline__ int paged_group_size(int n) { return n <= 8 ? n : (n <= 64 ? 8 : 32); }
// Counters, zero between calls: [2 cta + place] of a group (its first piece's), then [cta] of an item's groups.
__device__ __forceinline__ bool paged_last(int32_t* counter, int n) {
  // one operation that releases this CTA's writes and acquires the others'
  int before;
  asm volatile("atom.add.acq_rel.gpu.global.s32 %0, [%1], 1;" : "=r"(before) : "l"(counter) : "memory");
  const bool last = before == n - 1;
  if (last) *counter = 0;
  return last;
}
// In one thread, after the partial results of the piece are written (by all threads, and a barrier):
// whether this CTA joins the piece's group, which g becomes.
__device__ __forceinline__ bool paged_arrive(const PagedAttnArgs& a, const PagedPiece& p, PagedGroup& g) {
  const int n = p.c1 - p.c0 + 1, size = paged_group_size(n), k0 = (int(blockIdx.x) - p.c0) / size * size;
  g.first = p.c0 + k0;
  g.n = min(size, n - k0);
  g.stride = 1;
  g.is_item_first = k0 == 0;
  g.final = size == n;
  return paged_last(&a.count[2 * g.first + (k0 == 0)], g.n);
}
// The same after a group that was not final is joined and written: the groups of the item.
__device__ __forceinline__ bool paged_arrive_group(const PagedAttnArgs& a, const PagedPiece& p, PagedGroup& g) {
  const int n = p.c1 - p.c0 + 1, size = paged_group_size(n);
  g.first = p.c0;
  g.n = (n + size - 1) / size;
  g.stride = size;
  g.is_item_first = true;
  g.final = true;
  return paged_last(&a.count[2 * int(gridDim.x) + p.c0], g.n);
}
// An arrival that a CTA owes after a timeout, without a join.
__device__ __forceinline__ void paged_arrive_owed(const PagedAttnArgs& a, const PagedPiece& p) {
  PagedGroup g;
  if (paged_arrive(a, p, g) && !g.final) paged_arrive_group(a, p, g);
}

// Joins a group's places in order, by all threads of the CTA: to the output, or into its first place.
// Four columns a thread; kJoin places at a time with all their loads in flight, under a running maximum. kBar: the
// named barrier of n_threads that join where they are not all of the CTA.
template <class T, int BM, int D, int kBar = 0>
__device__ __forceinline__ void paged_join(const PagedAttnArgs& a, const PagedCursor& c, const PagedGroup& g, int tid,
                                           int n_threads) {
  constexpr int kJoin = 8;
  const int G = a.d.Hq / a.d.H, r0 = c.rt * BM, rows = min(BM, c.s.m * G - r0), items = rows * (D / 4);
  for (int x0 = 0; x0 < items; x0 += n_threads) {
    const int x = min(x0 + tid, items - 1), r = x / (D / 4), col = (x - r * (D / 4)) * 4;
    float m = -INFINITY, l = 0.f, o[4] = {0.f, 0.f, 0.f, 0.f};
    for (int k0 = 0; k0 < g.n; k0 += kJoin) {
      float mk[kJoin], lk[kJoin];
      float4 v[kJoin];
#pragma unroll
      for (int k = 0; k < kJoin; ++k) {
        const float* part = paged_place<BM, D>(a, g, min(k0 + k, g.n - 1));
        mk[k] = __ldcg(part + BM * D + r);
        lk[k] = __ldcg(part + BM * (D + 1) + r);
        v[k] = __ldcg(reinterpret_cast<const float4*>(part + r * D + col));
      }
      float to = m;
#pragma unroll
      for (int k = 0; k < kJoin; ++k) to = fmaxf(to, mk[k]);
      const float ms = to == -INFINITY ? 0.f : to, f0 = exp2f(m - ms);
      m = to;
      l *= f0;
#pragma unroll
      for (int e = 0; e < 4; ++e) o[e] *= f0;
#pragma unroll
      for (int k = 0; k < kJoin; ++k)
        if (k0 + k < g.n) {
          const float f = exp2f(mk[k] - ms);
          l = fmaf(f, lk[k], l);
          o[0] = fmaf(f, v[k].x, o[0]);
          o[1] = fmaf(f, v[k].y, o[1]);
          o[2] = fmaf(f, v[k].z, o[2]);
          o[3] = fmaf(f, v[k].w, o[3]);
        }
    }
    if (g.final) {
      if (x0 + tid < items)
        paged_store4(static_cast<T*>(a.out) + paged_out_row(c, a.d.H, G, r0 + r) * D + col, o, l);
    } else {
      float* part = paged_place<BM, D>(a, g, 0);
      // a row's maximum and sum have been read by the threads of all its columns
      if (kBar) asm volatile("bar.sync %0, %1;" ::"n"(kBar), "r"(n_threads) : "memory");
      else __syncthreads();
      if (x0 + tid < items) {
        __stcg(reinterpret_cast<float4*>(part + r * D + col), make_float4(o[0], o[1], o[2], o[3]));
        if (col == 0) {
          __stcg(part + BM * D + r, m);
          __stcg(part + BM * (D + 1) + r, l);
        }
      }
    }
  }
}
// What follows a piece's partial results in a kernel whose threads all take part; `sh` is shared.
struct PagedJoinShared {
  PagedGroup g;
  int32_t mine;
};
template <class T, int BM, int D>
__device__ __forceinline__ void paged_finish(const PagedAttnArgs& a, const PagedCursor& c, const PagedPiece& p,
                                             PagedJoinShared& sh, int tid, int n_threads) {
  __syncthreads();
  if (tid == 0) sh.mine = paged_arrive(a, p, sh.g);
  __syncthreads();
  if (!sh.mine) return;
  paged_join<T, BM, D>(a, c, sh.g, tid, n_threads);
  if (sh.g.final) return;
  __syncthreads();
  if (tid == 0) sh.mine = paged_arrive_group(a, p, sh.g);
  __syncthreads();
  if (sh.mine) paged_join<T, BM, D>(a, c, sh.g, tid, n_threads);
}

// The pool row (in rows of d elements) of position `pos` and head hk of a slot's page entry.
__device__ __forceinline__ int64_t paged_row(const PagedDims& d, int page, int hk, int pos) {
  return (int64_t(page) * d.H + hk) * d.P + (pos & (d.P - 1));
}
// A table entry; -1, and the status says so, where it is outside the pool.
__device__ __forceinline__ int paged_entry(const PagedDims& d, const int32_t* table, int32_t* status, int slot,
                                           int pos) {
  const int p = table[int64_t(slot) * d.max_pages + (pos >> d.lp)];
  if (p >= 0 && p < d.n_pages) return p;
  atomicOr(status, kStatusPageUse);
  return -1;
}
// The same held inside the pool, for what only reads.
__device__ __forceinline__ int paged_page(const PagedDims& d, const int32_t* table, int32_t* status,
                                          int slot, int pos) {
  return max(paged_entry(d, table, status, slot, pos), 0);
}

}  // namespace
}  // namespace mot
