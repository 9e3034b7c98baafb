// Internal declarations of the paged cache (paged.cu: its pages; paged8.cu: those in 8 bits
// and contiguous caches; paged_append.cu: the append; paged_simt.cu, paged_decode.cu, paged_fmha.cu: attention over
// it), shared with the C-ABI layer.
#pragma once

#include "mot_internal.h"

namespace mot {

// Largest table (sequence slots): a kernel marks the slots of a batch in 4 KB of shared memory.
constexpr int kPagedMaxSeqs = 32768;

// Pools k, v [n_layers][n_pages][H][P][d], table [max_seqs][max_pages], lens [max_seqs], refs
// [n_pages]. A position's page is table[slot][pos >> lp], its row pos & (P - 1).
struct PagedDims {
  int32_t L, Hq, H, d, P, lp;   // P = 1 << lp
  int32_t n_pages, max_seqs, max_pages;
  int32_t rot, rot_pairs;
  float eps;
  int32_t dtype;                // 0 = bf16, 1 = fp32
  int32_t b8;                   // pages in 8 bits
};
// Bytes of an element of the pools.
__host__ __device__ inline int paged_elem(const PagedDims& d) { return d.b8 ? 1 : (d.dtype ? 4 : 2); }

struct PagedCache {
  void* k;
  void* v;
  int32_t* table;
  int32_t* lens;
  int32_t* refs;
  float* ks;   // 8-bit pages: scales [n_layers][n_pages][H]
  float* vs;
};

struct PagedBatch {
  const int32_t* seqs;
  const int32_t* starts;
  int32_t n, rows;
};

// Workspace of the bookkeeping: `first` [max_seqs + 1], `take` and `map` [n_pages], `moves` [n_pages]
// pairs (from, to), `count` [4]: pages moved by the last compaction.
struct PagedWork {
  int32_t* first;
  int32_t* take;
  int32_t* map;
  int2* moves;
  int32_t* count;
  int32_t* status;
};

cudaError_t launch_paged_reserve(const PagedDims& d, const PagedCache& c, const PagedBatch& b,
                                 const PagedWork& w, cudaStream_t st);
cudaError_t launch_paged_free(const PagedDims& d, const PagedCache& c, const int32_t* seqs, int32_t n,
                              const PagedWork& w, int num_sms, cudaStream_t st);
// plan: takes the pages and writes the moves (one per fork, from = -1 without a copy); then the
// copies, with the table rows. overlap: the launch may start before the plan has finished.
cudaError_t launch_paged_fork_plan(const PagedDims& d, const PagedCache& c, const int32_t* src,
                                   const int32_t* dst, int32_t n, const PagedWork& w, cudaStream_t st);
cudaError_t launch_paged_fork(const PagedDims& d, const PagedCache& c, const int32_t* src,
                              const int32_t* dst, int32_t n, const PagedWork& w, int num_sms,
                              bool overlap, cudaStream_t st);
cudaError_t launch_paged_compact_plan(const PagedDims& d, const PagedCache& c, int32_t* live,
                                      const PagedWork& w, cudaStream_t st);
cudaError_t launch_paged_compact(const PagedDims& d, const PagedCache& c, const PagedWork& w, int num_sms,
                                 bool overlap, cudaStream_t st);
// Contiguous [n_layers][B][H][S][d] <-> the pages of layers first ..; store: into the pages.
struct PagedCopy {
  const int32_t* seqs;
  int32_t n, first, n_layers, B, S;
  void* k;
  void* v;
  bool store;
  bool early;   // 8-bit pages: the launch may overlap the kernel before it
};
cudaError_t launch_paged_copy(const PagedDims& d, const PagedCache& c, const PagedCopy& p,
                              const PagedWork& w, int num_sms, cudaStream_t st);

// The same between bf16 and 8-bit pages.
cudaError_t launch_paged8_copy(const PagedDims& d, const PagedCache& c, const PagedCopy& p,
                               const PagedWork& w, int num_sms, cudaStream_t st);

struct PagedAppend {
  PagedBatch b;
  int32_t layer;
  const void *q, *k, *v;            // [rows][heads][d], rows q_stride, k_stride, v_stride elements apart
  int64_t q_stride, k_stride, v_stride;
  const void *q_norm, *k_norm;      // [d] or null
  const uint64_t* freq;             // [rot / 2]: turns per position in units of 2^-64
  void* q_out;                      // [rows][Hq][d]
  bool early;                       // the launch may overlap the kernel before it
};
// Rotation by several positions: pair i of a row turns by at[axis[i]][row] times freq[i] 2^-64 turns. at null: by
// the row's place in its sequence.
constexpr int kPagedMaxAxes = 4;
struct PagedAxes {
  uint64_t freq[64];
  uint8_t axis[64];
  const int32_t* at;   // [axes][rows]
};
cudaError_t launch_paged_append(const PagedDims& d, const PagedCache& c, const PagedAppend& p, const PagedWork& w,
                                const PagedAxes& ax, int num_sms, cudaStream_t st);

// Attention of a batch's rows over one layer's pages. `part` holds the partial results of split
// items, two per CTA; `count` one arrival counter per CTA, zero between calls.
struct PagedAttnArgs {
  PagedDims d;
  PagedBatch b;
  const void* q;
  void* out;
  const void* k;        // the layer's pools
  const void* v;
  const float* ks;      // 8-bit pages: the layer's scales
  const float* vs;
  const int32_t* table;
  const int32_t* lens;
  float* part;
  int32_t* count;
  int32_t* status;
  int32_t max_chunk;      // most rows of an entry: a hint for the split, never relied on
  long long wait_limit;   // bound of every pipeline wait (SM cycles)
  int32_t stall_test;     // test hook: the tensor-core kernel's first CTA loads nothing
  bool early;             // 8-bit pages: the launch may overlap the kernel before it
};
constexpr int kPagedMaxGroup = 16;   // query heads per key/value head
size_t paged_part_floats(const PagedDims& d, int num_sms);
int paged_counters(int num_sms);
// fp32.
cudaError_t launch_paged_simt(const PagedAttnArgs& a, int num_sms, cudaStream_t st);
// bf16, few rows per key/value head (any number is right).
cudaError_t launch_paged_decode(const PagedAttnArgs& a, int num_sms, cudaStream_t st);
// The same over 8-bit pages: maps of bytes, box d x P.
cudaError_t launch_paged8_decode(const PagedAttnArgs& a, const CUtensorMap& tmK, const CUtensorMap& tmV, int num_sms,
                                 cudaStream_t st);
// Chunks in bf16 on the tensor cores: maps over the layer's pools as rows [n_pages * H * P][d], box 64 x P.
bool paged_fmha_takes(const PagedDims& d, int max_chunk);
cudaError_t launch_paged_fmha(const PagedAttnArgs& a, const CUtensorMap& tmK, const CUtensorMap& tmV,
                              int num_sms, cudaStream_t st);
// The same over 8-bit pages: maps of bytes, box d x P.
cudaError_t launch_paged8_fmha(const PagedAttnArgs& a, const CUtensorMap& tmK, const CUtensorMap& tmV,
                               int num_sms, cudaStream_t st);

}  // namespace mot
