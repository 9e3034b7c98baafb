// The append of new queries, keys and values to a paged cache on sm_103a.
#include "paged_common.cuh"
#include "paged8.cuh"

#include <algorithm>

namespace mot {
namespace {

// A warp takes some rows, one after another, in steps of 2 or 4 heads (queries, then keys with their
// values): d / 8 lanes per head with 8 elements each, in two groups of four: i .. i + 3 and i + rot / 2
// .. in the half-and-half layout of the rotation, so that a pair's elements are in one lane (no shuffles
// but the norm's sum), 8 in a row otherwise. A lane's angles and norm weights are the same for every
// head; fp32 in packed pairs. Angles: F_i = base^(-2 i / rot) / (2 pi) turns per position as a 64-bit
// fraction, so the upper half of pos * F_i mod 2^64 is the angle in 2^-32 turns (1.5e-9), for any
// position below 2^30. 10,254 rows of 36 heads of 128, normed and rotated, 37.3 us (5.1 TB/s; bound by
// loads that stand still while a warp works), in fp32 69.8 (5.4 TB/s); one row 3.7. With three positions of a row 39.9.
constexpr int kAppendThreads = 128;
// Steps with their loads in flight, and blocks per SM: in 16 bits 4 and 6 (10,254 rows with three positions: 39.7 us; 4
// and 5 44.0, 6 and 6 42.6, 8 and 5 41.3, 2 and 8 47.1), in fp32 4 and 5 (2,200 rows of 36 heads of 64: 11.8 us; 6 blocks
// 12.7, with spills), where queries go alone beside 8-bit pages 6 and 5 (44.9 us of the example there; 4 46.4, 8 44.3,
// but 34.5 for 33.3 with few heads).
constexpr int kDepth = 4, kDepth8 = 6;
template <class T>
constexpr int kAppendBlocks = sizeof(T) == 4 ? 5 : 6;
constexpr int kAppendBlocks8 = 5;

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

// Rows `unit` of the call; none where a change before it was refused (stop: its load is under way beside the first
// others). AXES: a pair turns by the caller's position of its axis, ax.at[axis][row], else by the
// row's place in its sequence.
template <class T, int D, int ROT, bool AXES, int kAppendDepth>
__device__ __forceinline__ void append_rows(const PagedDims& d, const PagedCache& c, const PagedAppend& p,
                                            const PagedWork& w, const PagedAxes& ax, bool stop, int unit, int rows_each,
                                            int parts) {
  using F = Four<T>;
  constexpr int kLph = D / 8, kAtOnce = 32 / kLph, kStep = kAtOnce * D;   // lanes per head; heads and elements of a step
  __shared__ __align__(16) float2 cs[kAppendThreads / 32][D / 2];        // cos, sin of a row's angles
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
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
  const int part = unit % parts;
  const int per = (steps + parts - 1) / parts, s0 = part * per, s1 = min(steps, s0 + per);
  const int row_begin = min(int64_t(unit / parts) * rows_each, int64_t(p.b.rows));
  const int row_end = min(row_begin + rows_each, p.b.rows);
  const int off = sub * D + eA, ab = eB - eA;              // the lane's first group in a step, and the second behind it
  const int pool_step = (kAtOnce * D) << d.lp;             // from a step's rows of a page to the next's
  uint64_t turn[D / 64];     // AXES: this lane's pairs lane, lane + 32
  const int32_t* at[D / 64];
  if (AXES) {
#pragma unroll
    for (int k = 0; k < D / 64; ++k) {
      turn[k] = ax.freq[lane + 32 * k];
      at[k] = ax.at + int64_t(ax.axis[lane + 32 * k]) * p.b.rows;
    }
  }
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
    if (stop) return;
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
        if (k < half) {
          const uint64_t turns = AXES ? uint64_t(int64_t(at[k / 32][row])) * turn[k / 32] : uint64_t(pos) * p.freq[k];
          cs[warp][k] = cos_sin_turns(uint32_t(turns >> 32));
        }
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
      for (int y0 = 0; y0 < kAppendDepth; y0 += 2) {
        if (sb + y0 >= min(sq, s1)) break;   // two steps in one run of instructions: 37.4 us, 39.0 one by one
#pragma unroll
        for (int y = y0; y < y0 + 2; ++y)
          if (ROT != kRotNone || p.q_norm) work(a[y], b[y], p.q_norm != nullptr, wq);
#pragma unroll
        for (int y = y0; y < y0 + 2; ++y) {
          const int st = sb + y;
          if (st < min(sq, s1) && st * kAtOnce + sub < d.Hq) {
            *reinterpret_cast<F*>(q_out + st * kStep) = a[y];
            *reinterpret_cast<F*>(q_out + st * kStep + ab) = b[y];
          }
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

template <class T, int D, int ROT, bool AXES>
__global__ void __launch_bounds__(kAppendThreads, kAppendBlocks<T>)
    paged_append_kernel(const PagedDims d, const PagedCache c, const PagedAppend p, const PagedWork w,
                        const __grid_constant__ PagedAxes ax, int rows_each, int parts) {
  pdl_wait();
  append_rows<T, D, ROT, AXES, kDepth>(d, c, p, w, ax, refused(w.status),
                                       blockIdx.x * (kAppendThreads / 32) + (threadIdx.x >> 5), rows_each, parts);
}

template <class T, int D, bool AXES>
auto append_kernel(const PagedDims& d) {
  return d.rot == 0 ? paged_append_kernel<T, D, kRotNone, false>
                    : d.rot_pairs ? paged_append_kernel<T, D, kRotPairs, AXES> : paged_append_kernel<T, D, kRotHalves, AXES>;
}
template <class T, int D>
auto append_kernel(const PagedDims& d, const PagedAxes& ax) {
  return ax.at ? append_kernel<T, D, true>(d) : append_kernel<T, D, false>(d);
}

// ---------------------------------------------------------------- 8-bit pages
//
// Queries as above, by some blocks of the grid. The others take units (entry, page, head of keys or of values):
// the new rows of one page, whose scale wants the largest of them before the first is written. A block takes 8 or
// 16 of the rows at a time, d / 8 lanes to a row and the lane's pairs turned by angles of its own (a row of one head
// has each angle once). What comes out waits for the scale in fp32: in registers where that is all, else in shared
// memory, a lane's own (kHeld rows; those behind them, of pages of 128 rows of 128, are worked out a second time).
// Units are dealt out by a scan of the entries in every block, or, with few rows to an entry, by the row. Bound by instructions, and loads that stand still beside them: 10,254 rows of 28 heads on 4
// of 128, normed and turned, pages of 64, 43.3 us (4.1 TB/s; 51.9 with every row worked out twice), of 12 heads on 12
// of 64, pages of 128, 31.6 (52.2). Five blocks per SM 47.9 and 36.6 before the order below, six 49.3 and 39.4, four
// 54.3 and 38.9. One row for each of eight sequences 3.6.
constexpr int kHeld = 8;   // rows of a lane that wait in shared memory for their scale
template <int D, int ROT, bool AXES>
struct Rows8 {
  static constexpr int kLph = D / 8, kAtOnce = kAppendThreads / kLph;   // lanes of a row, rows at a time
  int el, eA, eB;
  bool turned;
  uint64_t turn[4];        // the lane's pairs
  const int32_t* at[4];    // AXES: the positions of their axes
  uint64_t wk[4];

  __device__ __forceinline__ Rows8(const PagedDims& d, const PagedAppend& p, const PagedAxes& ax) {
    using F = Four<uint16_t>;
    el = threadIdx.x % kLph;
    turned = ROT != kRotNone && 8 * el < d.rot;
    const bool halves = ROT == kRotHalves && turned;
    eA = halves ? 4 * el : 8 * el;
    eB = halves ? (d.rot >> 1) + 4 * el : 8 * el + 4;
    if (turned)
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        turn[k] = AXES ? ax.freq[4 * el + k] : p.freq[4 * el + k];
        if (AXES) at[k] = ax.at + int64_t(ax.axis[4 * el + k]) * p.b.rows;
      }
    if (p.k_norm) {
      const uint16_t* src = static_cast<const uint16_t*>(p.k_norm);
      uint64_t a[2], b[2];
      reinterpret_cast<const F*>(src + eA)->unpack(a);
      reinterpret_cast<const F*>(src + eB)->unpack(b);
      wk[0] = a[0];
      wk[1] = a[1];
      wk[2] = b[0];
      wk[3] = b[1];
    }
  }

  // A row's eight values of this lane (two groups of four) in fp32; `key`: normed and rotated. By whole warps.
  __device__ __forceinline__ void values(const PagedDims& d, const PagedAppend& p, const Four<uint16_t> (&raw)[2], bool key,
                                         int row, int pos, float (&x)[8]) const {
    uint64_t f[2], g[2];
    raw[0].unpack(f);
    raw[1].unpack(g);
    if (key && p.k_norm) {
      const uint64_t sq2 = ffma_x2(g[1], g[1], ffma_x2(g[0], g[0], ffma_x2(f[1], f[1], fmul_x2(f[0], f[0]))));
      float ss = Four<uint16_t>::lo_f(sq2) + Four<uint16_t>::hi_f(sq2);
#pragma unroll
      for (int o = kLph / 2; o; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
      const float rs = rsqrtf(fmaf(ss, 1.f / D, d.eps));
      const uint64_t r2 = f32x2(rs, rs);
      f[0] = fmul_x2(fmul_x2(f[0], r2), wk[0]);
      f[1] = fmul_x2(fmul_x2(f[1], r2), wk[1]);
      g[0] = fmul_x2(fmul_x2(g[0], r2), wk[2]);
      g[1] = fmul_x2(fmul_x2(g[1], r2), wk[3]);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      x[2 * k] = Four<uint16_t>::lo_f(f[k]);
      x[2 * k + 1] = Four<uint16_t>::hi_f(f[k]);
      x[4 + 2 * k] = Four<uint16_t>::lo_f(g[k]);
      x[4 + 2 * k + 1] = Four<uint16_t>::hi_f(g[k]);
    }
    if (key && turned) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int64_t by = AXES ? int64_t(at[k][row]) : int64_t(pos);
        const float2 cs = cos_sin_turns(uint32_t(uint64_t(by) * turn[k] >> 32));
        float& a = ROT == kRotHalves ? x[k] : x[2 * k];
        float& b = ROT == kRotHalves ? x[4 + k] : x[2 * k + 1];
        const float u = a, v = b;
        a = fmaf(-v, cs.y, u * cs.x);
        b = fmaf(u, cs.y, v * cs.x);
      }
    }
  }

  // The `rows` new rows from `row` on, at position pos (of one page) and on, of unit g. By the whole block.
  __device__ __forceinline__ void page(const PagedDims& d, const PagedCache& c, const PagedAppend& p, int32_t* status,
                                       float* top, float4 (*held)[kAppendThreads], int slot, int row, int pos, int rows,
                                       int g) const {
    using F = Four<uint16_t>;
    const bool key = g < d.H;
    const int hk = key ? g : g - d.H, old = pos & (d.P - 1), sub = threadIdx.x / kLph;
    const uint16_t* src = static_cast<const uint16_t*>(key ? p.k : p.v) + hk * D;
    const int64_t stride = key ? p.k_stride : p.v_stride;
    constexpr int kAhead = 4;   // rows of a lane with their loads in flight
    F raw[kAhead][2];
    auto load = [&](int r0) {
#pragma unroll
      for (int e = 0; e < kAhead; ++e) {
        const int r = r0 + e * kAtOnce;
        raw[e][0].u = raw[e][1].u = make_uint2(0u, 0u);
        if (r < rows) {
          const uint16_t* s = src + (row + r) * stride;
          raw[e][0] = *reinterpret_cast<const F*>(s + eA);
          raw[e][1] = *reinterpret_cast<const F*>(s + eB);
        }
      }
    };
    load(sub);   // under way while the page is found
    const int page = paged_entry(d, c.table, status, slot, pos);
    if (page < 0) return;
    const int64_t at_head = (int64_t(p.layer) * d.n_pages + page) * d.H + hk;
    float* place = (key ? c.ks : c.vs) + at_head;
    uint8_t* dst = static_cast<uint8_t*>(key ? c.k : c.v) + (at_head << d.lp) * D;
    float was = old ? *place : 0.f;
    float x[8], big = 0.f;
    auto each = [&](int from, auto&& use) {
      for (int r0 = from + sub; r0 < rows + sub; r0 += kAhead * kAtOnce) {   // as often for every lane
        if (r0 != sub) load(r0);
#pragma unroll
        for (int e = 0; e < kAhead; ++e) {
          const int r = r0 + e * kAtOnce;
          if (r - sub >= rows) break;
          values(d, p, raw[e], key, row + min(r, rows - 1), pos + r, x);
          use(r);
        }
      }
    };
    each(0, [&](int r) {
      if (r >= rows) return;
#pragma unroll
      for (int k = 0; k < 8; ++k) big = fmaxf(big, fabsf(x[k]));   // fmaxf passes over NaN, which 8 bits then hold as it is
      if (r < kHeld * kAtOnce && rows > kAtOnce) {   // for this lane, behind the scale
        const int e = r / kAtOnce;
        held[2 * e][threadIdx.x] = make_float4(x[0], x[1], x[2], x[3]);
        held[2 * e + 1][threadIdx.x] = make_float4(x[4], x[5], x[6], x[7]);
      }
    });
    const bool large = __any_sync(0xffffffffu, !held8(big));   // values that have no part in the scale, and become NaN
    if (large) {
      big = 0.f;
      load(sub);
      each(0, [&](int r) {
        if (r >= rows) return;
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (held8(x[k])) big = fmaxf(big, fabsf(x[k]));
      });
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) big = fmaxf(big, __shfl_xor_sync(0xffffffffu, big, o));
    if ((threadIdx.x & 31) == 0) top[threadIdx.x >> 5] = big;
    __syncthreads();   // and the old scale is read
#pragma unroll
    for (int k = 0; k < kAppendThreads / 32; ++k) big = fmaxf(big, top[k]);
    float scale = scale8(big);
    if (old) {
      was = scale_of_page(was, status);
      scale = fmaxf(scale, was);
      if (scale != was) rescale8(dst, old * D, was / scale, threadIdx.x, kAppendThreads);
    }
    if (threadIdx.x == 0) *place = scale;
    const float inv = 1.f / scale;
    auto write = [&](int r) {
      if (r >= rows) return;
      if (large) {
#pragma unroll
        for (int k = 0; k < 8; ++k)
          if (!held8(x[k])) x[k] = __uint_as_float(0x7FC00000u);
      }
      float y[8];
#pragma unroll
      for (int k = 0; k < 8; ++k) y[k] = x[k] * inv;
      uint8_t* to = dst + (old + r) * D;
      *reinterpret_cast<uint32_t*>(to + eA) = pack8(y[0], y[1], y[2], y[3]);
      *reinterpret_cast<uint32_t*>(to + eB) = pack8(y[4], y[5], y[6], y[7]);
    };
    if (rows <= kAtOnce) {   // x is still there
      write(sub);
    } else {
#pragma unroll 4
      for (int e = 0; e < kHeld && e * kAtOnce < rows; ++e) {
        const float4 u = held[2 * e][threadIdx.x], v = held[2 * e + 1][threadIdx.x];
        x[0] = u.x, x[1] = u.y, x[2] = u.z, x[3] = u.w;
        x[4] = v.x, x[5] = v.y, x[6] = v.z, x[7] = v.w;
        write(e * kAtOnce + sub);
      }
      if (rows > kHeld * kAtOnce) each(kHeld * kAtOnce, write);
    }
    __syncthreads();   // top is read
  }
};

// The pages that an entry's new rows touch: first position and count.
struct Touched8 {
  int first, pages;
};
__device__ __forceinline__ Touched8 touched8(const PagedDims& d, const PagedSeq& s) {
  const int first = max(s.len - s.m, 0);
  return {first, s.slot < 0 || s.m == 0 || s.len == 0 ? 0 : ((s.len - 1) >> d.lp) - (first >> d.lp) + 1};
}

template <int D, int ROT, bool AXES>
__global__ void __launch_bounds__(kAppendThreads, kAppendBlocks8)
    paged_append8_kernel(const PagedDims d, const PagedCache c, const PagedAppend p, const PagedWork w,
                         const __grid_constant__ PagedAxes ax, int q_blocks, int rows_each, int parts, int by_row) {
  __shared__ float top[kAppendThreads / 32];
  __shared__ float4 held[2 * kHeld][kAppendThreads];
  __shared__ int64_t sh[33];
  __shared__ int64_t s_at;
  __shared__ int s_i;
  pdl_wait();
  const bool stop = refused(w.status);   // looked at behind the first loads
  const int tid = threadIdx.x;
  // blocks of the pages first, whose shares are the longest; those of the queries behind fill the gaps (46.6 and 33.5 us of
  // the examples above, then; the other way round 47.1 and 36.1)
  const int block = blockIdx.x, blocks = int(gridDim.x) - q_blocks;
  if (block >= blocks) {
    PagedDims dq = d;
    dq.H = 0;   // queries alone
    append_rows<uint16_t, D, ROT, AXES, kDepth8>(dq, c, p, w, ax, stop, (block - blocks) * (kAppendThreads / 32) + (tid >> 5),
                                                 rows_each, parts);
    return;
  }
  const Rows8<D, ROT, AXES> lanes(d, p, ax);
  if (stop) return;
  const int G = 2 * d.H, n = p.b.n;
  if (by_row) {   // a unit for each row that is the first of its entry or of a page
    for (int64_t u = block; u < int64_t(p.b.rows) * G; u += blocks) {
      const int row = int(u / G), g = int(u - int64_t(row) * G);
      const PagedSeq s = paged_seq(d, p.b, c.lens, w.status, entry_of(p.b.starts, n, row));
      const int from = s.len - s.m, pos = from + row - s.r0;
      if (s.slot < 0 || row < s.r0 || row >= s.r0 + s.m || pos < 0) continue;   // the queries' blocks report it
      if (row != s.r0 + max(0, -from) && (pos & (d.P - 1))) continue;
      lanes.page(d, c, p, w.status, top, held, s.slot, row, pos, min(d.P - (pos & (d.P - 1)), s.len - pos), g);
    }
    return;
  }
  int64_t W = 0, mine = 0, at = 0;
  auto scan = [&](int i0) {   // this thread's entry of the next block of them: its units, and those before it
    mine = 0;
    if (i0 + tid < n) mine = int64_t(touched8(d, paged_seq(d, p.b, c.lens, w.status, i0 + tid)).pages) * G;
    int64_t t;
    at = W + block_scan(mine, sh, t);
    W += t;
  };
  for (int i0 = 0; i0 < n; i0 += kAppendThreads) scan(i0);
  const int64_t all = W, u0 = all * block / blocks, u1 = all * (block + 1) / blocks;
  if (u0 >= u1) return;
  if (n > kAppendThreads) W = 0;
  for (int i0 = 0; i0 < n; i0 += kAppendThreads) {
    if (n > kAppendThreads) scan(i0);
    if (u0 >= at && u0 < at + mine) {
      s_i = i0 + tid;
      s_at = u0 - at;
    }
    if (W > u0) break;
  }
  __syncthreads();
  int i = s_i;
  int64_t in = s_at;   // units of entry i before this one
  PagedSeq s = paged_seq(d, p.b, c.lens, w.status, i);
  Touched8 t = touched8(d, s);
  for (int64_t u = u0; u < u1; ++u, ++in) {
    while (in >= int64_t(t.pages) * G) {   // units are left, so an entry with pages follows
      if (++i >= n) return;
      in = 0;
      s = paged_seq(d, p.b, c.lens, w.status, i);
      t = touched8(d, s);
    }
    const int j = int(in / G), g = int(in - int64_t(j) * G);
    const int pos = j ? ((t.first >> d.lp) + j) << d.lp : t.first;
    const int rows = min(d.P - (pos & (d.P - 1)), s.len - pos);
    lanes.page(d, c, p, w.status, top, held, s.slot, s.r0 + pos - (s.len - s.m), pos, rows, g);
  }
}

template <int D, bool AXES>
auto append8_kernel(const PagedDims& d) {
  return d.rot == 0 ? paged_append8_kernel<D, kRotNone, false>
                    : d.rot_pairs ? paged_append8_kernel<D, kRotPairs, AXES> : paged_append8_kernel<D, kRotHalves, AXES>;
}

}  // namespace

cudaError_t launch_paged_append(const PagedDims& d, const PagedCache& c, const PagedAppend& p, const PagedWork& w,
                                const PagedAxes& ax, int num_sms, cudaStream_t st) {
  // few rows: a row's heads over several warps, all of their loads in flight; many: a warp takes a row, or
  // some in a row, which share the search for their entry
  constexpr int kWarps = kAppendThreads / 32;
  const int at_once = 256 / d.d, kv = d.b8 ? 0 : d.H;
  const int steps = (d.Hq + at_once - 1) / at_once + (kv + at_once - 1) / at_once;
  // warps that are resident; in 8 bits smaller shares, behind those of the pages
  const int64_t fill = int64_t(num_sms) * (d.b8 ? 48 : kWarps * (d.dtype ? kAppendBlocks<float> : kAppendBlocks<uint16_t>));
  const int depth = d.b8 ? kDepth8 : kDepth, most = (steps + depth - 1) / depth;
  const int parts = p.b.rows >= fill ? 1 : int(fill / p.b.rows < most ? fill / p.b.rows : most);
  const int rows_each = int((p.b.rows * int64_t(parts) + fill - 1) / fill);
  const int64_t units = (int64_t(p.b.rows) + rows_each - 1) / rows_each * parts;
  const int grid = int((units + kWarps - 1) / kWarps);
  if (d.b8) {
    // Units by the row where entries have two rows at most on the average, whatever the longest has: rows that are no
    // page's first cost a look each, a scan has every block read all entries. 2,000 single rows of 4 key/value heads of
    // 128 57 us (98 by a scan), with a prompt of 500 beside them 63 (110), with one of 4,000 103 (118); of 12 of 64 on
    // pages of 16 167 (159), 181 (160) and 293 (194); four rows each 142 (111) and 384 (208), sixteen 582 (156) and
    // 1,275 (322). 64 single rows 4.3 (4.9), with a prompt of 500 11.7 (9.0).
    const bool by_row = p.b.rows <= 2 * int64_t(p.b.n);
    // pages that the rows touch: an entry of m rows at most (m - 2) / P + 2
    const int64_t pages = std::min(int64_t(p.b.rows), int64_t(p.b.rows) / d.P + 2 * int64_t(p.b.n));
    const int64_t blocks = std::min((by_row ? int64_t(p.b.rows) : pages) * 2 * d.H, int64_t(num_sms) * 16);
    auto kern = d.d == 64 ? (ax.at ? append8_kernel<64, true>(d) : append8_kernel<64, false>(d))
                          : (ax.at ? append8_kernel<128, true>(d) : append8_kernel<128, false>(d));
    return launch_kernel(p.early, kern, int(grid + blocks), kAppendThreads, 0, st, d, c, p, w, ax, grid, rows_each, parts,
                         int(by_row));
  }
  auto kern = d.dtype == 0 ? (d.d == 64 ? append_kernel<uint16_t, 64>(d, ax) : append_kernel<uint16_t, 128>(d, ax))
                           : (d.d == 64 ? append_kernel<float, 64>(d, ax) : append_kernel<float, 128>(d, ax));
  return launch_kernel(p.early, kern, grid, kAppendThreads, 0, st, d, c, p, w, ax, rows_each, parts);
}

}  // namespace mot
