// Copies between the 8-bit pages of a paged cache and contiguous bf16 caches on sm_103a.
//
//   paged8_store_kernel   a team of 32 to 256 threads takes the rows of one page, head and K or V: their largest
//                         value, the scale, the rows in units of it. Every row stays in registers between the two
//                         (8 loads of 16 bytes a thread), so that it is read once.
//   paged8_load_kernel    the way back, exactly: 16 values a thread.
// Bound by HBM, 2 + 1 bytes a value: 22,432 positions of 28 layers of 4 heads of 128 are stored in 321 us and loaded in
// 322 (6.0 TB/s both ways).
#include "paged_common.cuh"
#include "paged8.cuh"

namespace mot {
namespace {

constexpr int kThreads8 = 256;
constexpr int kVecs = 8;   // 16-byte loads of a thread that stores

// Rows of a call's entry i in its page j (0: none), and their page in the pool (-1: nothing is copied).
struct Span8 {
  int rows, filled, page;   // `filled`: rows that the page holds of the sequence
};
__device__ __forceinline__ Span8 span8(const PagedDims& d, const PagedCache& c, const PagedCopy& p, int32_t* status,
                                       int i, int j, bool tell) {
  Span8 o{0, 0, -1};
  const int s = p.seqs[i];
  if (s < 0 || s >= d.max_seqs) {
    if (tell) atomicOr(status, kStatusPageUse);
    return o;
  }
  const int64_t table = int64_t(d.max_pages) << d.lp;
  const int cap = int(min(table, int64_t(p.S)));
  const int len = c.lens[s];
  if (tell && (len < 0 || len > cap)) atomicOr(status, kStatusPageUse);
  o.rows = min(min(len, cap) - (j << d.lp), d.P);
  if (o.rows <= 0) return o;
  o.filled = int(min(min(int64_t(len), table) - (int64_t(j) << d.lp), int64_t(d.P)));
  o.page = paged_entry(d, c.table, status, s, j << d.lp);
  return o;
}

template <int D>
__global__ void __launch_bounds__(kThreads8, 4)
    paged8_store_kernel(const PagedDims d, const PagedCache c, const PagedCopy p, const PagedWork w) {
  constexpr int kRow = D / 8;   // loads of a row
  __shared__ float top[kThreads8 / 32];
  pdl_wait();
  if (refused(w.status)) return;
  const int n_vec = d.P * kRow, T = max(32, n_vec / kVecs), teams = kThreads8 / T;
  const int team = threadIdx.x / T, t = threadIdx.x % T, lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  auto together = [&] {   // the team's threads, which take the same steps
    if (T == 32) __syncwarp();
    else asm volatile("bar.sync %0, %1;" ::"r"(1 + team), "r"(T) : "memory");
  };
  const int per_seq = ((p.S - 1) >> d.lp) + 1, G = 2 * d.H;
  const int64_t units = int64_t(per_seq) * p.n * p.n_layers * G;
  for (int64_t u = int64_t(blockIdx.x) * teams + team; u < units; u += int64_t(gridDim.x) * teams) {
    const int64_t x = u / G, y = x / per_seq;
    const int g = int(u - x * G), j = int(x - y * per_seq), l = int(y / p.n), i = int(y - int64_t(l) * p.n);
    const bool is_v = g >= d.H;
    const int hk = is_v ? g - d.H : g;
    const Span8 s = span8(d, c, p, w.status, i, j, j == 0 && g == 0 && t == 0);
    if (s.rows <= 0 || s.page < 0) continue;
    const uint4* src = static_cast<const uint4*>(is_v ? p.v : p.k) +
                       (((int64_t(l) * p.B + i) * d.H + hk) * p.S + (j << d.lp)) * kRow;
    const int n = s.rows * kRow;
    uint4 v[kVecs];
#pragma unroll
    for (int e = 0; e < kVecs; ++e) v[e] = e * T + t < n ? src[e * T + t] : make_uint4(0u, 0u, 0u, 0u);
    // the largest magnitude: bf16 without its sign is ordered as an integer
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < kVecs; ++e)
      m = __vmaxu2(m, __vmaxu2(__vmaxu2(v[e].x & 0x7FFF7FFFu, v[e].y & 0x7FFF7FFFu),
                               __vmaxu2(v[e].z & 0x7FFF7FFFu, v[e].w & 0x7FFF7FFFu)));
    float big = fmaxf(__uint_as_float(m << 16), __uint_as_float(m & 0xFFFF0000u));
    if (!(held8(__uint_as_float(m << 16)) && held8(__uint_as_float(m & 0xFFFF0000u)))) {   // without what 8 bits do not hold
      big = 0.f;
#pragma unroll
      for (int e = 0; e < kVecs; ++e) {
        const uint32_t q[4] = {v[e].x, v[e].y, v[e].z, v[e].w};
#pragma unroll
        for (int k = 0; k < 4; ++k) {
          const float a = fabsf(__uint_as_float(q[k] << 16)), b = fabsf(__uint_as_float(q[k] & 0xFFFF0000u));
          if (held8(a)) big = fmaxf(big, a);
          if (held8(b)) big = fmaxf(big, b);
        }
      }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
    float* place = (is_v ? c.vs : c.ks) + (int64_t(p.first + l) * d.n_pages + s.page) * d.H + hk;
    const float was = s.filled > s.rows ? *place : 0.f;   // rows that stay: max_seq cuts the page
    if (T > 32) {
      if (lane == 0) top[warp] = big;
      together();
      for (int k = 0; k < T / 32; ++k) big = fmaxf(big, top[team * (T / 32) + k]);
    }
    float scale = scale8(big);
    uint8_t* dst = static_cast<uint8_t*>(is_v ? c.v : c.k) +
                   ((int64_t(p.first + l) * d.n_pages + s.page) * d.H + hk) * d.P * D;
    if (s.filled > s.rows) {
      const float old = scale_of_page(was, w.status);
      scale = fmaxf(scale, old);
      if (scale != old) rescale8(dst + s.rows * D, (s.filled - s.rows) * D, old / scale, t, T);
    }
    const float inv = 1.f / scale;
#pragma unroll
    for (int e = 0; e < kVecs; ++e) {
      if (e * T + t >= n) continue;
      const uint32_t q[4] = {v[e].x, v[e].y, v[e].z, v[e].w};
      float f[8];
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        f[2 * k] = unit8(__uint_as_float(q[k] << 16), inv);
        f[2 * k + 1] = unit8(__uint_as_float(q[k] & 0xFFFF0000u), inv);
      }
      reinterpret_cast<uint2*>(dst)[e * T + t] = make_uint2(pack8(f[0], f[1], f[2], f[3]), pack8(f[4], f[5], f[6], f[7]));
    }
    together();   // top is read, and the old scale
    if (t == 0) *place = scale;
  }
}

// Item (layer, entry, page), as the copies of other pages have it.
template <int D>
__global__ void __launch_bounds__(kThreads8)
    paged8_load_kernel(const PagedDims d, const PagedCache c, const PagedCopy p, const PagedWork w) {
  constexpr int kRow = D / 16;   // 16-byte loads of a row
  pdl_wait();
  const int per_seq = ((p.S - 1) >> d.lp) + 1;
  const int64_t items = int64_t(per_seq) * p.n * p.n_layers;
  const int n_vec = 2 * d.H * d.P * kRow, run = d.P * kRow;
  for (int64_t x = blockIdx.x; x < items; x += gridDim.x) {
    const int64_t y = x / per_seq;
    const int j = int(x - y * per_seq), l = int(y / p.n), i = int(y - int64_t(l) * p.n);
    const Span8 s = span8(d, c, p, w.status, i, j, j == 0 && threadIdx.x == 0);
    if (s.rows <= 0 || s.page < 0) continue;
    const int64_t at = (int64_t(p.first + l) * d.n_pages + s.page) * d.H;
    for (int v0 = threadIdx.x; v0 < n_vec; v0 += 4 * kThreads8) {
      uint4 q[4], *to[4];
      float f[4];
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int v = v0 + e * kThreads8, g = v / run, r = v - g * run;
        to[e] = nullptr;
        if (v >= n_vec || r / kRow >= s.rows) continue;
        const bool is_v = g >= d.H;
        const int hk = is_v ? g - d.H : g;
        f[e] = (is_v ? c.vs : c.ks)[at + hk];
        q[e] = (static_cast<const uint4*>(is_v ? c.v : c.k) + (at + hk) * run)[r];
        to[e] = static_cast<uint4*>(is_v ? p.v : p.k) +
                ((((int64_t(l) * p.B + i) * d.H + hk) * p.S + (j << d.lp)) * kRow + r) * 2;
      }
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (!to[e]) continue;
        const float by = scale_of_page(f[e], w.status);
        const uint32_t b[4] = {q[e].x, q[e].y, q[e].z, q[e].w};
        uint32_t o[8];
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const float2 z = float2_of8(k & 1 ? b[k >> 1] >> 16 : b[k >> 1]);
          const __nv_bfloat162 r = __floats2bfloat162_rn(z.x * by, z.y * by);
          o[k] = *reinterpret_cast<const uint32_t*>(&r);
        }
        to[e][0] = make_uint4(o[0], o[1], o[2], o[3]);
        to[e][1] = make_uint4(o[4], o[5], o[6], o[7]);
      }
    }
  }
}

}  // namespace

cudaError_t launch_paged8_copy(const PagedDims& d, const PagedCache& c, const PagedCopy& p, const PagedWork& w,
                               int num_sms, cudaStream_t st) {
  const int64_t items = int64_t((p.S - 1) / d.P + 1) * p.n * p.n_layers;
  // some blocks to every place, so that the last of them end together: 22,432 positions of 28 layers of 4 heads of 128,
  // stored in 321 us (339 with as many as are resident) and loaded in 322 (357)
  if (!p.store) {
    const int64_t most = int64_t(num_sms) * 32;
    return launch_kernel(p.early, d.d == 64 ? paged8_load_kernel<64> : paged8_load_kernel<128>,
                         int(items < most ? items : most), kThreads8, 0, st, d, c, p, w);
  }
  const int T = d.P * d.d / 64 > 32 ? d.P * d.d / 64 : 32, teams = kThreads8 / T;
  const int64_t blocks = (items * 2 * d.H + teams - 1) / teams, most = int64_t(num_sms) * 16;
  return launch_kernel(p.early, d.d == 64 ? paged8_store_kernel<64> : paged8_store_kernel<128>,
                       int(blocks < most ? blocks : most), kThreads8, 0, st, d, c, p, w);
}

}  // namespace mot
