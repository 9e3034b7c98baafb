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

// Whether a stored length, or one that a sequence is to get, is one that the table holds.
__device__ __forceinline__ bool len_fits(const PagedDims& d, int64_t len) {
  return len >= 0 && len <= (int64_t(d.max_pages) << d.lp) && len <= INT32_MAX / 2;
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
      // ascending starts within the rows: the new positions of all entries together are b.rows at most,
      // so that no sum of pages here leaves 32 bits
      const int s = b.seqs[i], from = b.starts[i], to = b.starts[i + 1], m = to - from;
      if (!mark_slot(marks, s, d.max_seqs) || from < 0 || to < from || to > b.rows) {
        bad = true;
      } else {
        const int len = c.lens[s];
        if (len < 0 || !len_fits(d, int64_t(len) + m))
          bad = true;
        else
          need = pages_of(d, len + m) - pages_of(d, len);
      }
    }
    int t;
    const int at = block_scan(need, sh, t);
    if (i < b.n && total + at <= d.n_pages) w.first[i] = int(total) + at;
    total += t;
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
  const int tid = threadIdx.x, T = blockDim.x;
  for (int i = tid; i < (d.max_seqs + 31) / 32; i += T) marks[i] = 0;
  // another CTA of this launch may be setting the bit: one decision for the whole CTA, which then either
  // leaves (the batch is refused) or checks all of it
  if (__syncthreads_or(refused(w.status))) return;
  bool bad = false;
  for (int i = tid; i < n; i += T)   // a length that another CTA has freed by now is 0
    bad |= !mark_slot(marks, seqs[i], d.max_seqs) || !len_fits(d, c.lens[seqs[i]]);
  if (__syncthreads_or(bad)) {
    if (tid == 0) atomicOr(w.status, kStatusPages);
    return;
  }
  for (int i = blockIdx.x; i < n; i += gridDim.x) {
    const int s = seqs[i];
    const int pages = pages_of(d, c.lens[s]);
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

// Checks a fork and takes the pages of its partly filled last pages; moves[i]: what is copied (from < 0:
// nothing).
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
        if (!len_fits(d, len))
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
      mv.x = paged_entry(d, c.table, w.status, src[i], c.lens[src[i]]);
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
// heads and layers x, x + gridDim.x, .. 16 branches of two prefixes, 44 MB of copies, 19 us with the plan
// and the free before it (latency of three launches and of pieces of 16 KB).
__global__ void __launch_bounds__(kCopyThreads)
    paged_fork_kernel(const PagedDims d, const PagedCache c, const int32_t* src, const int32_t* dst, int n,
                      const PagedWork w) {
  pdl_enter();   // behind the plan
  if (refused(w.status)) return;
  const int i = blockIdx.y, tid = threadIdx.x;
  const int a = src[i], b = dst[i], len = c.lens[a];
  if (len == 0) return;
  const int2 mv = w.moves[i];
  const int pages = pages_of(d, len), full = len >> d.lp, part = len & (d.P - 1);
  for (int j = blockIdx.x * kCopyThreads + tid; j < pages; j += gridDim.x * kCopyThreads) {
    int p = mv.y;
    if (j < full) {   // an entry out of range is taken over as it is
      p = c.table[int64_t(a) * d.max_pages + j];
      if (p >= 0 && p < d.n_pages)
        atomicAdd(&c.refs[p], 1);
      else
        atomicOr(w.status, kStatusPageUse);
    }
    c.table[int64_t(b) * d.max_pages + j] = p;
  }
  if (blockIdx.x == 0 && tid == 0) c.lens[b] = len;
  if (!part || mv.x < 0) return;
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

// The moves' pages, all layers; the table's entries at or above the count of pages in use follow (without a
// move the table is not read).
__global__ void __launch_bounds__(kCopyThreads)
    paged_compact_kernel(const PagedDims d, const PagedCache c, const PagedWork w) {
  pdl_enter();   // behind the plan
  const int n = w.count[0], used = w.count[1];
  if (n == 0) return;
  const int vecs = d.H * d.P * (d.d * elem_bytes(d) / 16);   // of a page in one layer; its bytes may pass 2^31
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
    bool bad = !len_fits(d, len);
    int32_t* row = c.table + int64_t(s) * d.max_pages;
    for (int j = lane; j < pages; j += 32) {
      const int p = row[j];
      bad |= p < 0 || p >= d.n_pages;
      if (p >= used && p < d.n_pages) row[j] = w.map[p];
    }
    if (bad) atomicOr(w.status, kStatusPageUse);
  }
}

// Item (layer, entry, page): its heads' rows between the pool and the contiguous caches. 8,192 positions of 28
// layers of 4 heads of 128: 153 us either way (6.1 TB/s read and written).
__global__ void __launch_bounds__(kCopyThreads)
    paged_copy_kernel(const PagedDims d, const PagedCache c, const PagedCopy p, const PagedWork w) {
  if (p.store && refused(w.status)) return;
  const int per_seq = ((p.S - 1) >> d.lp) + 1;
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
    const int page = paged_entry(d, c.table, w.status, s, j << d.lp);
    if (page < 0) continue;   // nothing is copied: whatever page it fell on would be another sequence's
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
// A warp takes some rows, one after another, in steps of 2 or 4 heads (queries, then keys with their
// values): d / 8 lanes per head with 8 elements each, in two groups of four: i .. i + 3 and i + rot / 2
// .. in the half-and-half layout of the rotation, so that a pair's elements are in one lane (no shuffles
// but the norm's sum), 8 in a row otherwise. A lane's angles and norm weights are the same for every
// head; fp32 in packed pairs. Angles: F_i = base^(-2 i / rot) / (2 pi) turns per position as a 64-bit
// fraction, so the upper half of pos * F_i mod 2^64 is the angle in 2^-32 turns (1.5e-9), for any
// position below 2^30. 10,254 rows of 36 heads of 128, normed and rotated, 39.4 us (4.8 TB/s; bound by
// loads that stand still while a warp works), in fp32 73.5 (5.1 TB/s); one row 4.4.
constexpr int kAppendThreads = 128;
constexpr int kAppendDepth = 4;   // steps with their loads in flight

template <class T>
struct Four;   // four elements, as two pairs of fp32
template <>
struct Four<uint16_t> {
  uint2 u;
  __device__ __forceinline__ void unpack(uint64_t (&x)[2]) const {
    x[0] = (uint64_t(u.x & 0xFFFF0000u) << 32) | (u.x << 16);
    x[1] = (uint64_t(u.y & 0xFFFF0000u) << 32) | (u.y << 16);
  }
  __device__ __forceinline__ void pack(const uint64_t (&x)[2]) {
    __nv_bfloat162 a = __floats2bfloat162_rn(lo_f(x[0]), hi_f(x[0])), b = __floats2bfloat162_rn(lo_f(x[1]), hi_f(x[1]));
    u = make_uint2(*reinterpret_cast<uint32_t*>(&a), *reinterpret_cast<uint32_t*>(&b));
  }
  static __device__ __forceinline__ float lo_f(uint64_t x) { return __uint_as_float(uint32_t(x)); }
  static __device__ __forceinline__ float hi_f(uint64_t x) { return __uint_as_float(uint32_t(x >> 32)); }
};
template <>
struct Four<float> {
  uint4 u;
  __device__ __forceinline__ void unpack(uint64_t (&x)[2]) const {
    x[0] = (uint64_t(u.y) << 32) | u.x;
    x[1] = (uint64_t(u.w) << 32) | u.z;
  }
  __device__ __forceinline__ void pack(const uint64_t (&x)[2]) {
    u = make_uint4(uint32_t(x[0]), uint32_t(x[0] >> 32), uint32_t(x[1]), uint32_t(x[1] >> 32));
  }
};

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

enum { kRotNone = 0, kRotHalves = 1, kRotPairs = 2 };

// cos and sin of t / 2^32 turns: the nearest quarter turn off, then their series to x^10 and x^9 (off by
// 2^-29 at most on |x| <= pi / 4).
__device__ __forceinline__ float2 cos_sin_turns(uint32_t t) {
  const uint32_t quarter = (t + 0x20000000u) >> 30;
  const float x = float(int32_t(t - (quarter << 30))) * 1.46291807926715968e-9f;   // 2 pi / 2^32
  const float z = x * x;
  const float sn = fmaf(x * z, fmaf(z, fmaf(z, fmaf(z, 1.f / 362880, -1.f / 5040), 1.f / 120), -1.f / 6), x);
  const float cn =
      fmaf(z, fmaf(z, fmaf(z, fmaf(z, fmaf(z, -1.f / 3628800, 1.f / 40320), -1.f / 720), 1.f / 24), -0.5f), 1.f);
  const float c = quarter & 1u ? sn : cn, s = quarter & 1u ? cn : sn;
  return make_float2((quarter + 1u) & 2u ? -c : c, quarter & 2u ? -s : s);
}

template <class T, int D, int ROT>
__global__ void __launch_bounds__(kAppendThreads, 6)
    paged_append_kernel(const PagedDims d, const PagedCache c, const PagedAppend p, const PagedWork w, int rows_each,
                        int parts) {
  using F = Four<T>;
  constexpr int kLph = D / 8, kAtOnce = 32 / kLph, kStep = kAtOnce * D;   // lanes per head; heads and elements of a step
  __shared__ __align__(16) float2 cs[kAppendThreads / 32][D / 2];        // cos, sin of a row's angles
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  if (refused(w.status)) return;
  const int sub = lane / kLph, el = lane % kLph;           // this lane's head and place in it
  const int half = d.rot >> 1;
  const bool turned = ROT != kRotNone && 8 * el < d.rot;   // the lane's elements are rotated
  const bool halves = ROT == kRotHalves && turned;
  const int eA = halves ? 4 * el : 8 * el, eB = halves ? half + 4 * el : 8 * el + 4;
  uint64_t wq[4], wk[4];
  auto weights = [&](const void* src, uint64_t (&x)[4]) {
    if (!src) return;
    uint64_t a[2], b[2];
    reinterpret_cast<const F*>(static_cast<const T*>(src) + eA)->unpack(a);
    reinterpret_cast<const F*>(static_cast<const T*>(src) + eB)->unpack(b);
    x[0] = a[0];
    x[1] = a[1];
    x[2] = b[0];
    x[3] = b[1];
  };
  weights(p.q_norm, wq);
  weights(p.k_norm, wk);
  // steps 0 .. sq - 1: queries, .. sq + sk - 1: a step of keys and one of values; this warp's: [s0, s1)
  const int sq = (d.Hq + kAtOnce - 1) / kAtOnce, sk = (d.H + kAtOnce - 1) / kAtOnce, steps = sq + sk;
  const int unit = blockIdx.x * (kAppendThreads / 32) + warp, part = unit % parts;
  const int per = (steps + parts - 1) / parts, s0 = part * per, s1 = min(steps, s0 + per);
  const int row_begin = min(int64_t(unit / parts) * rows_each, int64_t(p.b.rows));
  const int row_end = min(row_begin + rows_each, p.b.rows);
  const int off = sub * D + eA, ab = eB - eA;              // the lane's first group in a step, and the second behind it
  const int pool_step = (kAtOnce * D) << d.lp;             // from a step's rows of a page to the next's
  int first = 0, last = 0, pos0 = 0;   // rows [first, last) are of one entry; row r's position is pos0 + r
  int slot = -1, page = -1;
  for (int row = row_begin; row < row_end; ++row) {
    const T* q = static_cast<const T*>(p.q) + row * p.q_stride + off;
    F a[kAppendDepth], b[kAppendDepth];
    auto load_q = [&](int st) {
#pragma unroll
      for (int y = 0; y < kAppendDepth; ++y)
        if (st + y < min(sq, s1) && (st + y) * kAtOnce + sub < d.Hq) {
          a[y] = *reinterpret_cast<const F*>(q + (st + y) * kStep);
          b[y] = *reinterpret_cast<const F*>(q + (st + y) * kStep + ab);
        }
    };
    load_q(s0);   // under way while the row's place is found
    const bool fresh = row < first || row >= last;
    if (fresh) {
      const int i = entry_of(p.b.starts, p.b.n, row);
      const int from = p.b.starts[i], to = p.b.starts[i + 1];
      first = row;
      last = row + 1;
      slot = -1;
      if (row >= from && row < to) {
        const PagedSeq s = paged_seq(d, p.b, c.lens, w.status, i);
        if (row < s.r0 + s.m) last = s.r0 + s.m;   // starts that are out of order: this row alone
        slot = s.slot;
        pos0 = s.len - s.m - s.r0;
      }
    }
    const int pos = slot < 0 ? -1 : pos0 + row;
    if (pos < 0) {   // a row of no entry, or of one that is shorter than its rows
      if (fresh && row >= p.b.starts[0] && row < p.b.starts[p.b.n] && lane == 0) atomicOr(w.status, kStatusPageUse);
      continue;
    }
    if (fresh || (pos & (d.P - 1)) == 0) {
      page = paged_entry(d, c.table, w.status, slot, pos);
    }
    uint64_t tc[2] = {}, ts[2] = {};   // cos and sin of the lane's four angles, in pairs
    if (ROT != kRotNone) {
#pragma unroll
      for (int k = lane; k < D / 2; k += 32)
        if (k < half) cs[warp][k] = cos_sin_turns(uint32_t(uint64_t(pos) * p.freq[k] >> 32));
      __syncwarp();
      if (turned) {
        const float4 x = *reinterpret_cast<const float4*>(&cs[warp][4 * el]);
        const float4 y = *reinterpret_cast<const float4*>(&cs[warp][4 * el + 2]);
        tc[0] = f32x2(x.x, x.z);
        tc[1] = f32x2(y.x, y.z);
        ts[0] = f32x2(x.y, x.w);
        ts[1] = f32x2(y.y, y.w);
      }
      __syncwarp();   // before the next row's
    }
    auto work = [&](F& fa, F& fb, bool norm, const uint64_t (&wt)[4]) {   // by the whole warp
      uint64_t f[2], g[2];
      fa.unpack(f);
      fb.unpack(g);
      if (norm) {
        const uint64_t sq2 = ffma_x2(g[1], g[1], ffma_x2(g[0], g[0], ffma_x2(f[1], f[1], fmul_x2(f[0], f[0]))));
        float ss = __uint_as_float(uint32_t(sq2)) + __uint_as_float(uint32_t(sq2 >> 32));
#pragma unroll
        for (int o = kLph / 2; o; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
        const float rs = rsqrtf(fmaf(ss, 1.f / D, d.eps));
        const uint64_t r2 = f32x2(rs, rs);
        f[0] = fmul_x2(fmul_x2(f[0], r2), wt[0]);
        f[1] = fmul_x2(fmul_x2(f[1], r2), wt[1]);
        g[0] = fmul_x2(fmul_x2(g[0], r2), wt[2]);
        g[1] = fmul_x2(fmul_x2(g[1], r2), wt[3]);
      }
      if (halves) {
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const uint64_t u = f[e], v = g[e], ns = ts[e] ^ 0x8000000080000000ull;
          f[e] = ffma_x2(v, ns, fmul_x2(u, tc[e]));
          g[e] = ffma_x2(u, ts[e], fmul_x2(v, tc[e]));
        }
      } else if (ROT == kRotPairs && turned) {
        // the pairs of angles 0, 1 are f's, those of 2, 3 g's: (x c - y s, y c + x s)
        auto turn = [](uint64_t v, float cn, float sn) {
          const float x = __uint_as_float(uint32_t(v)), y = __uint_as_float(uint32_t(v >> 32));
          return f32x2(x * cn - y * sn, y * cn + x * sn);
        };
        auto lo = [](uint64_t v) { return __uint_as_float(uint32_t(v)); };
        auto hi = [](uint64_t v) { return __uint_as_float(uint32_t(v >> 32)); };
        f[0] = turn(f[0], lo(tc[0]), lo(ts[0]));
        f[1] = turn(f[1], hi(tc[0]), hi(ts[0]));
        g[0] = turn(g[0], lo(tc[1]), lo(ts[1]));
        g[1] = turn(g[1], hi(tc[1]), hi(ts[1]));
      }
      fa.pack(f);
      fb.pack(g);
    };
    T* q_out = static_cast<T*>(p.q_out) + int64_t(row) * d.Hq * D + off;
    for (int sb = s0; sb < min(sq, s1); sb += kAppendDepth) {
      if (sb != s0) load_q(sb);
#pragma unroll
      for (int y = 0; y < kAppendDepth; ++y) {
        const int st = sb + y;
        if (st >= min(sq, s1)) break;
        if (ROT != kRotNone || p.q_norm) work(a[y], b[y], p.q_norm != nullptr, wq);
        if (st * kAtOnce + sub < d.Hq) {
          *reinterpret_cast<F*>(q_out + st * kStep) = a[y];
          *reinterpret_cast<F*>(q_out + st * kStep + ab) = b[y];
        }
      }
    }
    if (s1 <= sq || page < 0) continue;
    const int64_t pool = ((int64_t(p.layer) * d.n_pages + page) * d.H * d.P + (pos & (d.P - 1))) * D +
                         (int64_t(sub * D) << d.lp) + eA;
    const T* k = static_cast<const T*>(p.k) + row * p.k_stride + off;
    const T* v = static_cast<const T*>(p.v) + row * p.v_stride + off;
    T* k_out = static_cast<T*>(c.k) + pool;
    T* v_out = static_cast<T*>(c.v) + pool;
    constexpr int kPairs = kAppendDepth / 2;   // steps of keys and of values at a time
    for (int sb = max(s0, sq) - sq; sb < s1 - sq; sb += kPairs) {
#pragma unroll
      for (int y = 0; y < kPairs; ++y)
        if (sb + y < s1 - sq && (sb + y) * kAtOnce + sub < d.H) {
          a[y] = *reinterpret_cast<const F*>(k + (sb + y) * kStep);
          b[y] = *reinterpret_cast<const F*>(k + (sb + y) * kStep + ab);
          a[kPairs + y] = *reinterpret_cast<const F*>(v + (sb + y) * kStep);
          b[kPairs + y] = *reinterpret_cast<const F*>(v + (sb + y) * kStep + ab);
        }
#pragma unroll
      for (int y = 0; y < kPairs; ++y) {
        const int st = sb + y;
        if (st >= s1 - sq) break;
        if (ROT != kRotNone || p.k_norm) work(a[y], b[y], p.k_norm != nullptr, wk);
        if (st * kAtOnce + sub < d.H) {
          const int64_t at = int64_t(st) * pool_step;
          *reinterpret_cast<F*>(k_out + at) = a[y];
          *reinterpret_cast<F*>(k_out + at + ab) = b[y];
          *reinterpret_cast<F*>(v_out + at) = a[kPairs + y];
          *reinterpret_cast<F*>(v_out + at + ab) = b[kPairs + y];
        }
      }
    }
  }
}

template <class T, int D>
auto append_kernel(const PagedDims& d) {
  return d.rot == 0 ? paged_append_kernel<T, D, kRotNone>
                    : d.rot_pairs ? paged_append_kernel<T, D, kRotPairs> : paged_append_kernel<T, D, kRotHalves>;
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
                              int32_t n, const PagedWork& w, int num_sms, bool overlap, cudaStream_t st) {
  // as many blocks as are resident, a block's pieces of a page evenly
  const int64_t pieces = int64_t(2) * d.L * d.H, most = (int64_t(num_sms) * 8 + n - 1) / n;
  const int x = int(pieces < most ? pieces : most);
  return launch_kernel(overlap, paged_fork_kernel, dim3(x, n), kCopyThreads, 0, st, d, c, src, dst, n, w);
}
cudaError_t launch_paged_compact_plan(const PagedDims& d, const PagedCache& c, int32_t* live,
                                      const PagedWork& w, cudaStream_t st) {
  return launch_kernel(false, paged_compact_plan_kernel, 1, kPlanThreads, 0, st, d, c, live, w);
}
cudaError_t launch_paged_compact(const PagedDims& d, const PagedCache& c, const PagedWork& w, int num_sms,
                                 bool overlap, cudaStream_t st) {
  return launch_kernel(overlap, paged_compact_kernel, num_sms * 8, kCopyThreads, 0, st, d, c, w);
}
cudaError_t launch_paged_copy(const PagedDims& d, const PagedCache& c, const PagedCopy& p, const PagedWork& w,
                              int num_sms, cudaStream_t st) {
  const int64_t items = int64_t((p.S - 1) / d.P + 1) * p.n * p.n_layers;
  return launch_kernel(false, paged_copy_kernel, grid_of(items, num_sms, 8), kCopyThreads, 0, st, d, c, p, w);
}
cudaError_t launch_paged_append(const PagedDims& d, const PagedCache& c, const PagedAppend& p,
                                const PagedWork& w, int num_sms, cudaStream_t st) {
  // few rows: a row's heads over several warps, all of their loads in flight; many: a warp takes a row, or
  // some in a row, which share the search for their entry
  constexpr int kWarps = kAppendThreads / 32;
  const int at_once = 256 / d.d, steps = (d.Hq + at_once - 1) / at_once + (d.H + at_once - 1) / at_once;
  const int64_t fill = int64_t(num_sms) * 24;   // warps that are resident
  const int most = (steps + kAppendDepth - 1) / kAppendDepth;
  const int parts = p.b.rows >= fill ? 1 : int(fill / p.b.rows < most ? fill / p.b.rows : most);
  const int rows_each = int((p.b.rows * int64_t(parts) + fill - 1) / fill);
  const int64_t units = (int64_t(p.b.rows) + rows_each - 1) / rows_each * parts;
  const int grid = int((units + kWarps - 1) / kWarps);
  auto kern = d.dtype == 0 ? (d.d == 64 ? append_kernel<uint16_t, 64>(d) : append_kernel<uint16_t, 128>(d))
                           : (d.d == 64 ? append_kernel<float, 64>(d) : append_kernel<float, 128>(d));
  return launch_kernel(false, kern, grid, kAppendThreads, 0, st, d, c, p, w, rows_each, parts);
}

}  // namespace mot
