// The pages of a paged cache on sm_103a: reserve, fork, free, compact, and the copies between pages and
// contiguous caches.
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
  const int es = paged_elem(d), run = d.P * d.d * es / 16, n_vec = part * d.d * es / 16;
  for (int x = blockIdx.x; x < 2 * d.L * d.H; x += gridDim.x) {
    uint4* pool = static_cast<uint4*>(x & 1 ? c.v : c.k);
    const int lh = x >> 1, l = lh / d.H, hk = lh - l * d.H;
    const int64_t row = (int64_t(l) * d.n_pages) * d.H + hk;
    copy_vecs(pool + (row + int64_t(mv.y) * d.H) * run, pool + (row + int64_t(mv.x) * d.H) * run, n_vec);
    if (d.b8 && tid == 0) {
      float* scale = x & 1 ? c.vs : c.ks;
      scale[row + int64_t(mv.y) * d.H] = scale[row + int64_t(mv.x) * d.H];
    }
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
  const int vecs = d.H * d.P * (d.d * paged_elem(d) / 16);   // of a page in one layer; its bytes may pass 2^31
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
    if (d.b8 && piece == 0) {
      float* scale = (y & 1 ? c.vs : c.ks) + int64_t(l) * d.n_pages * d.H;
      for (int hk = threadIdx.x; hk < d.H; hk += kCopyThreads)
        scale[int64_t(mv.y) * d.H + hk] = scale[int64_t(mv.x) * d.H + hk];
    }
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
  const int es = paged_elem(d);
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
}  // namespace mot
