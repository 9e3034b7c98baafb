// The pages of a paged cache on sm_103a: reserve, fork, free, compact, the copies between pages and
// contiguous caches, and the append of new keys and values.
//
// The bookkeeping (table, lens, refs) lives on the device and is changed there, so that a step of a
// serving loop needs no host round trip. A page is in use while refs > 0; what is taken are always
// the lowest free pages, in the order of the batch and of the positions, so results do not depend on
// the order in which threads run. A change is checked as a whole before anything is written, by one
// CTA (by each for free): a refused one sets kStatusPages and leaves everything as it was, and the
// changes behind it do nothing either until the status is read, since they count on its outcome.
#include "paged_common.cuh"

namespace mot {
namespace {

constexpr int kPlanThreads = 1024;
constexpr int kPerThread = 8;     // pages of a thread in one step of a scan over refs
constexpr int kCopyThreads = 256;

__device__ __forceinline__ bool refused(const int32_t* status) {
  return (*reinterpret_cast<const volatile int32_t*>(status) & kStatusPages) != 0;
}

// Marks slot s of the batch; false where it is outside the table or marked already.
__device__ __forceinline__ bool mark_slot(uint32_t* marks, int s, int max_seqs) {
  if (s < 0 || s >= max_seqs) return false;
  const uint32_t bit = 1u << (s & 31);
  return (atomicOr(&marks[s >> 5], bit) & bit) == 0;
}

__device__ __forceinline__ int pages_of(const PagedDims& d, int len) { return (len + d.P - 1) >> d.lp; }

// take[0 .. total): the lowest pages with refs <= 0, ascending. False where there are fewer.
// All threads of the CTA, which sees take behind it.
__device__ bool take_lowest(const PagedDims& d, const int32_t* refs, int total, int32_t* take, int* sh) {
  int carry = 0;
  for (int64_t base = 0; base < d.n_pages && carry < total; base += int64_t(blockDim.x) * kPerThread) {
    const int64_t p0 = base + int64_t(threadIdx.x) * kPerThread;
    uint32_t mask = 0;
#pragma unroll
    for (int j = 0; j < kPerThread; ++j)
      if (p0 + j < d.n_pages && refs[p0 + j] <= 0) mask |= 1u << j;
    int got;
    int k = carry + block_scan(__popc(mask), sh, got);
    for (; mask; mask &= mask - 1, ++k)
      if (k < total) take[k] = int32_t(p0) + __ffs(mask) - 1;
    carry += got;
  }
  __syncthreads();
  return carry >= total;
}

// Every entry's sequence grows by its rows: the pages that this needs, all or none.
__global__ void __launch_bounds__(kPlanThreads)
    paged_reserve_kernel(const PagedDims d, const PagedCache c, const PagedBatch b, const PagedWork w) {
  __shared__ uint32_t marks[kPagedMaxSeqs / 32];
  __shared__ int sh[33];
  if (refused(w.status)) return;
  const int tid = threadIdx.x, T = blockDim.x;
  for (int i = tid; i < (d.max_seqs + 31) / 32; i += T) marks[i] = 0;
  __syncthreads();
  bool bad = false;
  int64_t total = 0;
  for (int i0 = 0; i0 < b.n; i0 += T) {
    const int i = i0 + tid;
    int need = 0;
    if (i < b.n) {
      const int s = b.seqs[i], m = b.starts[i + 1] - b.starts[i];
      if (!mark_slot(marks, s, d.max_seqs) || m < 0) {
        bad = true;
      } else {
        const int len = c.lens[s];
        if (len < 0 || int64_t(len) + m > (int64_t(d.max_pages) << d.lp) || int64_t(len) + m > INT32_MAX / 2)
          bad = true;
        else
          need = pages_of(d, len + m) - pages_of(d, len);
      }
    }
    int t;
    const int at = block_scan(need, sh, t);
    if (i < b.n && total + at <= d.n_pages) w.first[i] = int(total) + at;
    total += t;   // a piece adds 1024 x 2^26 at most
    if (total > d.n_pages) bad = true;
  }
  if (__syncthreads_or(bad) || !take_lowest(d, c.refs, int(total), w.take, sh)) {
    if (tid == 0) atomicOr(w.status, kStatusPages);
    return;
  }
  // a warp per entry writes its new table entries
  const int lane = tid & 31;
  for (int i = tid >> 5; i < b.n; i += T >> 5) {
    const int s = b.seqs[i], len = c.lens[s], m = b.starts[i + 1] - b.starts[i];
    const int p0 = pages_of(d, len), n = pages_of(d, len + m) - p0, f = w.first[i];
    for (int j = lane; j < n; j += 32) {
      const int p = w.take[f + j];
      c.table[int64_t(s) * d.max_pages + p0 + j] = p;
      c.refs[p] = 1;
    }
    __syncwarp();
    if (lane == 0) c.lens[s] = len + m;
  }
}

// Entries out of the table; each CTA checks the whole batch and frees its share of it.
__global__ void __launch_bounds__(kCopyThreads)
    paged_free_kernel(const PagedDims d, const PagedCache c, const int32_t* seqs, int n, const PagedWork w) {
  __shared__ uint32_t marks[kPagedMaxSeqs / 32];
  if (refused(w.status)) return;
  const int tid = threadIdx.x, T = blockDim.x;
  for (int i = tid; i < (d.max_seqs + 31) / 32; i += T) marks[i] = 0;
  __syncthreads();
  bool bad = false;
  for (int i = tid; i < n; i += T) bad |= !mark_slot(marks, seqs[i], d.max_seqs);
  if (__syncthreads_or(bad)) {
    if (tid == 0) atomicOr(w.status, kStatusPages);
    return;
  }
  for (int i = blockIdx.x; i < n; i += gridDim.x) {
    const int s = seqs[i];
    const int len = c.lens[s];
    const int pages = len <= 0 ? 0 : min(pages_of(d, min(len, INT32_MAX / 2)), d.max_pages);
    int32_t* row = c.table + int64_t(s) * d.max_pages;
    for (int j = tid; j < pages; j += T) {
      const int p = row[j];
      if (p >= 0 && p < d.n_pages)
        atomicSub(&c.refs[p], 1);
      else
        atomicOr(w.status, kStatusPageUse);
      row[j] = -1;
    }
    __syncthreads();   // every thread has read the length
    if (tid == 0) c.lens[s] = 0;
  }
}

// Checks a fork and takes the pages of its partly filled last pages; moves[i]: what is copied.
__global__ void __launch_bounds__(kPlanThreads)
    paged_fork_plan_kernel(const PagedDims d, const PagedCache c, const int32_t* src, const int32_t* dst, int n,
                           const PagedWork w) {
  __shared__ uint32_t marks[kPagedMaxSeqs / 32];
  __shared__ int sh[33];
  if (refused(w.status)) return;
  const int tid = threadIdx.x, T = blockDim.x;
  for (int i = tid; i < (d.max_seqs + 31) / 32; i += T) marks[i] = 0;
  __syncthreads();
  bool bad = false;
  int total = 0;
  for (int i0 = 0; i0 < n; i0 += T) {
    const int i = i0 + tid;
    int need = 0;
    if (i < n) {
      const int a = src[i], b = dst[i];
      if (a < 0 || a >= d.max_seqs || !mark_slot(marks, b, d.max_seqs) || c.lens[b] != 0) {
        bad = true;
      } else {
        const int len = c.lens[a];
        if (len < 0 || len > INT32_MAX / 2 || pages_of(d, len) > d.max_pages)
          bad = true;
        else
          need = (len & (d.P - 1)) != 0;
      }
    }
    int t;
    const int at = block_scan(need, sh, t);
    if (i < n) w.first[i] = need ? total + at : -1;
    total += t;
  }
  __syncthreads();   // a source that is a destination too would change under the copy
  for (int i = tid; i < n; i += T)
    if (src[i] >= 0 && src[i] < d.max_seqs && (marks[src[i] >> 5] >> (src[i] & 31) & 1u)) bad = true;
  if (total > d.n_pages) bad = true;
  if (__syncthreads_or(bad) || !take_lowest(d, c.refs, total, w.take, sh)) {
    if (tid == 0) atomicOr(w.status, kStatusPages);
    return;
  }
  for (int i = tid; i < n; i += T) {
    const int f = w.first[i];
    int2 mv = make_int2(-1, -1);
    if (f >= 0) {
      mv.y = w.take[f];
      c.refs[mv.y] = 1;
      mv.x = paged_page(d, c.table, w.status, src[i], c.lens[src[i]]);
    }
    w.moves[i] = mv;
  }
}

// n 16-byte vectors per thread step from src to dst, contiguous; n_vec in all.
__device__ __forceinline__ void copy_vecs(uint4* __restrict__ dst, const uint4* __restrict__ src, int n_vec) {
  int v = threadIdx.x;
  for (; v + 3 * kCopyThreads < n_vec; v += 4 * kCopyThreads) {
    uint4 x[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) x[j] = src[v + j * kCopyThreads];
#pragma unroll
    for (int j = 0; j < 4; ++j) dst[v + j * kCopyThreads] = x[j];
  }
  for (; v < n_vec; v += kCopyThreads) dst[v] = src[v];
}

__device__ __forceinline__ int elem_bytes(const PagedDims& d) { return d.dtype ? 4 : 2; }

// Block (x, i): fork i's table row (its x-th share) and its copied page, the filled rows of the
// heads and layers x, x + gridDim.x, ..
__global__ void __launch_bounds__(kCopyThreads)
    paged_fork_kernel(const PagedDims d, const PagedCache c, const int32_t* src, const int32_t* dst, int n,
                      const PagedWork w) {
  if (refused(w.status)) return;
  const int i = blockIdx.y, tid = threadIdx.x;
  const int a = src[i], b = dst[i], len = c.lens[a];
  if (len == 0) return;
  const int2 mv = w.moves[i];
  const int pages = pages_of(d, len), full = len >> d.lp, part = len & (d.P - 1);
  for (int j = blockIdx.x * kCopyThreads + tid; j < pages; j += gridDim.x * kCopyThreads) {
    int p = mv.y;
    if (j < full) {
      p = paged_page(d, c.table, w.status, a, j << d.lp);
      atomicAdd(&c.refs[p], 1);
    }
    c.table[int64_t(b) * d.max_pages + j] = p;
  }
  if (blockIdx.x == 0 && tid == 0) c.lens[b] = len;
  if (!part) return;
  const int es = elem_bytes(d), run = d.P * d.d * es / 16, n_vec = part * d.d * es / 16;
  for (int x = blockIdx.x; x < 2 * d.L * d.H; x += gridDim.x) {
    uint4* pool = static_cast<uint4*>(x & 1 ? c.v : c.k);
    const int lh = x >> 1, l = lh / d.H, hk = lh - l * d.H;
    const int64_t row = (int64_t(l) * d.n_pages) * d.H + hk;
    copy_vecs(pool + (row + int64_t(mv.y) * d.H) * run, pool + (row + int64_t(mv.x) * d.H) * run, n_vec);
  }
}

// Which pages move where: the i-th lowest page in use at or above the count of pages in use goes to
// the i-th lowest free page below it.
__global__ void __launch_bounds__(kPlanThreads)
    paged_compact_plan_kernel(const PagedDims d, const PagedCache c, int32_t* live, const PagedWork w) {
  __shared__ int64_t sh[33];
  if (refused(w.status)) {
    if (threadIdx.x == 0) w.count[0] = 0;
    return;
  }
  const int tid = threadIdx.x, T = blockDim.x;
  int64_t mine = 0, used;
  for (int p = tid; p < d.n_pages; p += T) mine += c.refs[p] > 0;
  block_scan(mine, sh, used);
  int64_t carry = 0;   // movers in the upper half, holes in the lower
  for (int64_t base = 0; base < d.n_pages; base += int64_t(T) * kPerThread) {
    const int64_t p0 = base + int64_t(tid) * kPerThread;
    uint32_t hole = 0, mover = 0;
#pragma unroll
    for (int j = 0; j < kPerThread; ++j)
      if (p0 + j < d.n_pages) {
        const bool in = c.refs[p0 + j] > 0;
        if (p0 + j < used) hole |= uint32_t(!in) << j;
        else mover |= uint32_t(in) << j;
      }
    int64_t t;
    const int64_t at = carry + block_scan((int64_t(__popc(mover)) << 32) | __popc(hole), sh, t);
    int k = int(at);
    for (; hole; hole &= hole - 1) w.moves[k++].y = int(p0) + __ffs(hole) - 1;
    k = int(at >> 32);
    for (; mover; mover &= mover - 1) w.moves[k++].x = int(p0) + __ffs(mover) - 1;
    carry += t;
  }
  __syncthreads();
  const int n = int(carry >> 32);   // as many holes
  for (int k = tid; k < n; k += T) {
    const int2 mv = w.moves[k];
    c.refs[mv.y] = c.refs[mv.x];
    c.refs[mv.x] = 0;
    w.map[mv.x] = mv.y;
  }
  if (tid == 0) {
    w.count[0] = n;
    w.count[1] = int(used);
    if (live) *live = int(used);
  }
}

// The moves' pages, all layers; the table's entries at or above the count of pages in use follow.
__global__ void __launch_bounds__(kCopyThreads)
    paged_compact_kernel(const PagedDims d, const PagedCache c, const PagedWork w) {
  const int n = w.count[0], used = w.count[1];
  if (n == 0) return;
  const int vecs = d.H * d.P * d.d * elem_bytes(d) / 16;   // of a page in one layer
  constexpr int kPiece = 4 * kCopyThreads;
  const int pieces = (vecs + kPiece - 1) / kPiece;
  const int64_t items = int64_t(n) * d.L * 2 * pieces;
  for (int64_t x = blockIdx.x; x < items; x += gridDim.x) {
    const int64_t y = x / pieces;
    const int piece = int(x - y * pieces);
    const int64_t z = y >> 1;
    const int l = int(z / n);
    const int2 mv = w.moves[int(z - int64_t(l) * n)];
    uint4* pool = static_cast<uint4*>(y & 1 ? c.v : c.k) + int64_t(l) * d.n_pages * vecs + piece * kPiece;
    copy_vecs(pool + int64_t(mv.y) * vecs, pool + int64_t(mv.x) * vecs, min(kPiece, vecs - piece * kPiece));
  }
  const int lane = threadIdx.x & 31, warps = kCopyThreads / 32;
  for (int s = blockIdx.x * warps + (threadIdx.x >> 5); s < d.max_seqs; s += gridDim.x * warps) {
    const int len = c.lens[s];
    const int pages = len <= 0 ? 0 : min(pages_of(d, min(len, INT32_MAX / 2)), d.max_pages);
    int32_t* row = c.table + int64_t(s) * d.max_pages;
    for (int j = lane; j < pages; j += 32) {
      const int p = row[j];
      if (p >= used && p < d.n_pages) row[j] = w.map[p];
    }
  }
}

// Item (layer, entry, page): its heads' rows between the pool and the contiguous caches.
__global__ void __launch_bounds__(kCopyThreads)
    paged_copy_kernel(const PagedDims d, const PagedCache c, const PagedCopy p, const PagedWork w) {
  if (p.store && refused(w.status)) return;
  const int per_seq = (p.S + d.P - 1) >> d.lp;
  const int64_t items = int64_t(per_seq) * p.n * p.n_layers;
  const int es = elem_bytes(d);
  const int dv = d.d * es / 16;                       // vectors of a row: a power of two
  const int ldv = 31 - __clz(dv), lrun = ldv + d.lp;  // of a head's rows in a page
  for (int64_t x = blockIdx.x; x < items; x += gridDim.x) {
    const int64_t y = x / per_seq;
    const int j = int(x - y * per_seq), l = int(y / p.n), i = int(y - int64_t(l) * p.n);
    const int s = p.seqs[i];
    if (s < 0 || s >= d.max_seqs) {
      if (j == 0 && threadIdx.x == 0) atomicOr(w.status, kStatusPageUse);
      continue;
    }
    const int cap = int(min(int64_t(d.max_pages) << d.lp, int64_t(p.S)));
    const int len = c.lens[s];
    if (j == 0 && threadIdx.x == 0 && (len < 0 || len > cap)) atomicOr(w.status, kStatusPageUse);
    const int rows = min(min(len, cap) - (j << d.lp), d.P);
    if (rows <= 0) continue;
    const int page = paged_page(d, c.table, w.status, s, j << d.lp);
    const int64_t pool = ((int64_t(p.first + l) * d.n_pages + page) * d.H << d.lp) * dv;
    const int64_t flat = ((int64_t(l) * p.B + i) * d.H * p.S + (j << d.lp)) * dv;
    const int n_vec = 2 * d.H << lrun;
    auto spots = [&](int v, uint4*& a, uint4*& b) {   // the vector's places; false: a row behind the last
      const int q = v >> lrun, r = v & ((1 << lrun) - 1);
      const bool is_v = q >= d.H;
      const int hk = is_v ? q - d.H : q;
      a = static_cast<uint4*>(is_v ? c.v : c.k) + pool + (int64_t(hk) << lrun) + r;
      b = static_cast<uint4*>(is_v ? p.v : p.k) + flat + int64_t(hk) * p.S * dv + r;
      return (r >> ldv) < rows;
    };
    for (int v0 = threadIdx.x; v0 < n_vec; v0 += 4 * kCopyThreads) {
      uint4 t[4], *a[4], *b[4];
      bool ok[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int v = v0 + e * kCopyThreads;
        ok[e] = v < n_vec && spots(v, a[e], b[e]);
        if (ok[e]) t[e] = p.store ? *b[e] : *a[e];
      }
#pragma unroll
      for (int e = 0; e < 4; ++e)
        if (ok[e]) *(p.store ? a[e] : b[e]) = t[e];
    }
  }
}

// ---------------------------------------------------------------- append
//
// A row's query, key and value heads, each on d / kV lanes of kV elements (16 bytes): the norm is a
// sum over those lanes, a pair's other half the shuffle from lane +- rot / 2 / kV. Angles: F_i =
// base^(-2 i / rot) / (2 pi) turns per position as a 64-bit fraction, so pos * F_i mod 2^64 is the
// angle in turns, exact to 2^-44 for any position below 2^20; each is evaluated once per row, in
// shared memory, for all heads.
constexpr int kAppendThreads = 256;
constexpr int kAppendRows = 4;

template <class T>
struct Vec16 {
  static constexpr int kV = 16 / sizeof(T);
};
__device__ __forceinline__ void unpack16(uint4 u, float (&x)[8]) {
  const uint32_t w[4] = {u.x, u.y, u.z, u.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    x[2 * i] = __uint_as_float(w[i] << 16);
    x[2 * i + 1] = __uint_as_float(w[i] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ void unpack16(uint4 u, float (&x)[4]) {
  x[0] = __uint_as_float(u.x);
  x[1] = __uint_as_float(u.y);
  x[2] = __uint_as_float(u.z);
  x[3] = __uint_as_float(u.w);
}
__device__ __forceinline__ uint4 pack16(const float (&x)[8]) {
  uint32_t w[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    __nv_bfloat162 v = __floats2bfloat162_rn(x[2 * i], x[2 * i + 1]);
    w[i] = *reinterpret_cast<uint32_t*>(&v);
  }
  return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ uint4 pack16(const float (&x)[4]) {
  return make_uint4(__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3]));
}

// The last entry i with starts[i] <= row, by a 32-way search of one warp.
__device__ __forceinline__ int entry_of(const int32_t* starts, int n, int row) {
  const int lane = threadIdx.x & 31;
  int lo = 0, cnt = n;   // the entry is in [lo, lo + cnt)
  while (cnt > 1) {
    const int step = (cnt + 31) / 32;
    const int i = lo + lane * step;
    const uint32_t le = __ballot_sync(0xffffffffu, lane * step < cnt && (lane == 0 || starts[i] <= row));
    const int k = 31 - __clz(le);   // lane 0 is always set
    lo += k * step;
    cnt = min(step, cnt - k * step);
  }
  return lo;
}

template <class T>
__global__ void __launch_bounds__(kAppendThreads)
    paged_append_kernel(const PagedDims d, const PagedCache c, const PagedAppend p, const PagedWork w) {
  constexpr int kV = Vec16<T>::kV;
  __shared__ float2 cs[kAppendRows][128 / 2];   // cos, sin of a row's angles
  __shared__ int s_pos[kAppendRows];            // position, -1: a row of no entry
  __shared__ int s_page[kAppendRows];           // page of the position, -1: nothing is stored
  const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
  if (refused(w.status)) return;
  const int lph = d.d / kV;                     // lanes per head: 8, 16 or 32
  const int heads = d.Hq + 2 * d.H, per_pass = kAppendThreads / lph;
  const int el = tid & (lph - 1), e0 = el * kV; // this lane's elements of a head
  const int half = d.rot >> 1;
  for (int row0 = blockIdx.x * kAppendRows; row0 < p.b.rows; row0 += gridDim.x * kAppendRows) {
    const int nr = min(kAppendRows, p.b.rows - row0);
    __syncthreads();   // the rows before are done
    if (warp < nr) {
      const int row = row0 + warp;
      const int i = entry_of(p.b.starts, p.b.n, row);
      if (lane == 0) {
        int pos = -1, page = -1;
        if (p.b.n > 0 && row >= p.b.starts[i] && row < p.b.starts[i + 1]) {
          const PagedSeq s = paged_seq(d, p.b, c.lens, w.status, i);
          pos = s.len - s.m + (row - s.r0);
          if (pos < 0)
            atomicOr(w.status, kStatusPageUse);
          else {
            page = c.table[int64_t(s.slot) * d.max_pages + (pos >> d.lp)];
            if (page < 0 || page >= d.n_pages) {
              atomicOr(w.status, kStatusPageUse);
              page = -1;
            }
          }
        }
        s_pos[warp] = pos;
        s_page[warp] = page;
      }
    }
    __syncthreads();
    for (int t = tid; t < nr * half; t += kAppendThreads) {
      const int r = t / half, k = t - r * half;
      if (s_pos[r] >= 0) {
        const int64_t turns = int64_t(uint64_t(s_pos[r]) * p.freq[k]);
        float sn, cn;
        sincospif(__ll2float_rn(turns) * 0x1p-63f, &sn, &cn);
        cs[r][k] = make_float2(cn, sn);
      }
    }
    __syncthreads();
    for (int x0 = 0; x0 < nr * heads; x0 += per_pass) {
      const int x = x0 + tid / lph;
      const bool in = x < nr * heads;
      const int r = in ? x / heads : 0, h = in ? x - r * heads : 0;
      const int pos = s_pos[r], page = s_page[r];
      const int64_t row = row0 + r;
      const bool is_q = h < d.Hq, is_k = !is_q && h < d.Hq + d.H;
      const int hk = is_q ? 0 : (is_k ? h - d.Hq : h - d.Hq - d.H);
      const bool live = in && pos >= 0;
      const T* src = is_q ? static_cast<const T*>(p.q) + row * p.q_stride + h * d.d
                          : (is_k ? static_cast<const T*>(p.k) + row * p.k_stride
                                  : static_cast<const T*>(p.v) + row * p.v_stride) + hk * d.d;
      uint4 u = make_uint4(0, 0, 0, 0);
      if (live) u = *reinterpret_cast<const uint4*>(src + e0);
      if (is_q || is_k) {
        float y[kV];
        unpack16(u, y);
        const T* nw = static_cast<const T*>(is_q ? p.q_norm : p.k_norm);
        if (nw) {
          float ss = 0.f;
#pragma unroll
          for (int e = 0; e < kV; ++e) ss = fmaf(y[e], y[e], ss);
          // the group's lanes are of one kind: a head is a query, a key or a value as a whole
          const uint32_t mask = lph == 32 ? 0xffffffffu : ((1u << lph) - 1) << (lane & ~(lph - 1));
          for (int o = lph >> 1; o; o >>= 1) ss += __shfl_xor_sync(mask, ss, o);
          const float f = rsqrtf(ss / float(d.d) + d.eps);
          float g[kV];
          unpack16(*reinterpret_cast<const uint4*>(nw + e0), g);
#pragma unroll
          for (int e = 0; e < kV; ++e) y[e] = y[e] * f * g[e];
        }
        if (d.rot_pairs) {
          if (e0 < d.rot)
#pragma unroll
            for (int e = 0; e < kV; e += 2) {
              const float2 t = cs[r][(e0 + e) >> 1];
              const float a = y[e], b = y[e + 1];
              y[e] = a * t.x - b * t.y;
              y[e + 1] = b * t.x + a * t.y;
            }
        } else if (d.rot) {
          // element e pairs with e +- rot / 2, rot / 2 / kV lanes away
          const int off = half / kV;
          const bool lo = e0 < half, rotated = e0 < d.rot;
          const int from = rotated ? (lo ? lane + off : lane - off) : lane;
          const uint32_t mask = lph == 32 ? 0xffffffffu : ((1u << lph) - 1) << (lane & ~(lph - 1));
#pragma unroll
          for (int e = 0; e < kV; ++e) {
            const float other = __shfl_sync(mask, y[e], from);
            if (rotated) {
              const float2 t = cs[r][lo ? e0 + e : e0 + e - half];
              y[e] = lo ? y[e] * t.x - other * t.y : y[e] * t.x + other * t.y;
            }
          }
        }
        if (nw || d.rot) u = pack16(y);
      }
      if (!live) continue;
      if (is_q)
        *reinterpret_cast<uint4*>(static_cast<T*>(p.q_out) + (row * d.Hq + h) * d.d + e0) = u;
      else if (page >= 0) {
        T* pool = static_cast<T*>(is_k ? c.k : c.v) + int64_t(p.layer) * d.n_pages * d.H * d.P * d.d;
        *reinterpret_cast<uint4*>(pool + paged_row(d, page, hk, pos) * d.d + e0) = u;
      }
    }
  }
}

int grid_of(int64_t items, int num_sms, int per_sm) {
  const int64_t most = int64_t(num_sms) * per_sm;
  return int(items < 1 ? 1 : (items < most ? items : most));
}

}  // namespace

cudaError_t launch_paged_reserve(const PagedDims& d, const PagedCache& c, const PagedBatch& b,
                                 const PagedWork& w, cudaStream_t st) {
  return launch_kernel(false, paged_reserve_kernel, 1, kPlanThreads, 0, st, d, c, b, w);
}
cudaError_t launch_paged_free(const PagedDims& d, const PagedCache& c, const int32_t* seqs, int32_t n,
                              const PagedWork& w, int num_sms, cudaStream_t st) {
  return launch_kernel(false, paged_free_kernel, grid_of(n, num_sms, 4), kCopyThreads, 0, st, d, c, seqs, n, w);
}
cudaError_t launch_paged_fork_plan(const PagedDims& d, const PagedCache& c, const int32_t* src,
                                   const int32_t* dst, int32_t n, const PagedWork& w, cudaStream_t st) {
  return launch_kernel(false, paged_fork_plan_kernel, 1, kPlanThreads, 0, st, d, c, src, dst, n, w);
}
cudaError_t launch_paged_fork(const PagedDims& d, const PagedCache& c, const int32_t* src, const int32_t* dst,
                              int32_t n, const PagedWork& w, cudaStream_t st) {
  const int x = grid_of(int64_t(2) * d.L * d.H, 64, 1);
  return launch_kernel(false, paged_fork_kernel, dim3(x, n), kCopyThreads, 0, st, d, c, src, dst, n, w);
}
cudaError_t launch_paged_compact_plan(const PagedDims& d, const PagedCache& c, int32_t* live,
                                      const PagedWork& w, cudaStream_t st) {
  return launch_kernel(false, paged_compact_plan_kernel, 1, kPlanThreads, 0, st, d, c, live, w);
}
cudaError_t launch_paged_compact(const PagedDims& d, const PagedCache& c, const PagedWork& w, int num_sms,
                                 cudaStream_t st) {
  return launch_kernel(false, paged_compact_kernel, num_sms * 8, kCopyThreads, 0, st, d, c, w);
}
cudaError_t launch_paged_copy(const PagedDims& d, const PagedCache& c, const PagedCopy& p, const PagedWork& w,
                              int num_sms, cudaStream_t st) {
  const int64_t items = int64_t((p.S + d.P - 1) / d.P) * p.n * p.n_layers;
  return launch_kernel(false, paged_copy_kernel, grid_of(items, num_sms, 8), kCopyThreads, 0, st, d, c, p, w);
}
cudaError_t launch_paged_append(const PagedDims& d, const PagedCache& c, const PagedAppend& p,
                                const PagedWork& w, int num_sms, cudaStream_t st) {
  const int grid = grid_of((int64_t(p.b.rows) + kAppendRows - 1) / kAppendRows, num_sms, 8);
  auto kern = d.dtype ? paged_append_kernel<float> : paged_append_kernel<uint16_t>;
  return launch_kernel(false, kern, grid, kAppendThreads, 0, st, d, c, p, w);
}

}  // namespace mot
