// What the tensor-core kernels of chunks share: items of 256 rows over tiles of 128 keys, and the join of their
// partial results.
#pragma once

#include "paged_common.cuh"

namespace mot {
namespace {

constexpr int kChunkRows = 256;

// Tiles of an item that some of its rows see only in part: [first, units).
__device__ __forceinline__ int first_masked(const PagedSeq& s, int G, int row0) {
  const int p = s.len - s.m + row0 / G;
  return p < 0 ? 0 : (p + 1) >> 7;
}

// Joins a group's places in order, a thread per row: to the output, or into its first place. Here the
// partial rows lie by fours of columns, [D / 4][256 rows][4], so that the threads of a warp write and
// read whole lines. 32 columns at a time, two places with all their loads in flight, under a running
// maximum.
template <int D>
__device__ __forceinline__ void join_rows(const PagedAttnArgs& a, const PagedCursor& c, const PagedGroup& g, int r) {
  constexpr int BM = kChunkRows;
  const int G = a.d.Hq / a.d.H, row = c.rt * BM + r;
  if (row >= c.s.m * G) return;
  uint16_t* dst = static_cast<uint16_t*>(a.out) + paged_out_row(c, a.d.H, G, row) * D;
  float* to = paged_place<BM, D>(a, g, 0);
  float m = -INFINITY, l = 0.f;
#pragma unroll 1
  for (int e = 0; e < D / 32; ++e) {
    float o[32];
#pragma unroll
    for (int k = 0; k < 32; ++k) o[k] = 0.f;
    m = -INFINITY;   // the same in every pass
    l = 0.f;
#pragma unroll 1
    for (int k0 = 0; k0 < g.n; k0 += 2) {
      float mk[2], lk[2];
      float4 v[2][8];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const float* pk = paged_place<BM, D>(a, g, min(k0 + k, g.n - 1));
        mk[k] = __ldcg(pk + BM * D + r);
        lk[k] = __ldcg(pk + BM * (D + 1) + r);
        const float4* src = reinterpret_cast<const float4*>(pk) + 8 * e * BM + r;
#pragma unroll
        for (int x = 0; x < 8; ++x) v[k][x] = __ldcg(src + x * BM);
      }
      if (k0 + 1 >= g.n) mk[1] = -INFINITY;
      const float up = fmax3(m, mk[0], mk[1]), ms = up == -INFINITY ? 0.f : up;
      const float f = exp2f(m - ms), f0 = exp2f(mk[0] - ms), f1 = exp2f(mk[1] - ms);
      const bool both = k0 + 1 < g.n;
      m = up;
      l = fmaf(f0, lk[0], l * f);
      if (both) l = fmaf(f1, lk[1], l);
#pragma unroll
      for (int x = 0; x < 8; ++x) {
        const float* u = reinterpret_cast<const float*>(&v[0][x]);
        const float* w = reinterpret_cast<const float*>(&v[1][x]);
#pragma unroll
        for (int y = 0; y < 4; ++y) {
          o[4 * x + y] = fmaf(f0, u[y], o[4 * x + y] * f);
          if (both) o[4 * x + y] = fmaf(f1, w[y], o[4 * x + y]);
        }
      }
    }
    if (!g.final) {
#pragma unroll
      for (int x = 0; x < 8; ++x)
        __stcg(reinterpret_cast<float4*>(to) + (8 * e + x) * BM + r,
               make_float4(o[4 * x], o[4 * x + 1], o[4 * x + 2], o[4 * x + 3]));
      continue;
    }
    const float inv = l == 0.f ? 0.f : 1.f / l;
    if (l == 0.f) {   // no weight is above 0 (values that are not finite make NaN of 0)
#pragma unroll
      for (int k = 0; k < 32; ++k) o[k] = 0.f;
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      uint32_t w[4];
#pragma unroll
      for (int x = 0; x < 4; ++x) {
        __nv_bfloat162 u = __floats2bfloat162_rn(o[8 * k + 2 * x] * inv, o[8 * k + 2 * x + 1] * inv);
        w[x] = *reinterpret_cast<uint32_t*>(&u);
      }
      reinterpret_cast<uint4*>(dst + 32 * e)[k] = make_uint4(w[0], w[1], w[2], w[3]);
    }
  }
  if (!g.final) {   // the row's own thread alone reads these
    __stcg(to + BM * D + r, m);
    __stcg(to + BM * (D + 1) + r, l);
  }
}

}  // namespace
}  // namespace mot
