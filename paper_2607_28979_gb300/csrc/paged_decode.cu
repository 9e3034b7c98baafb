// Attention of few rows per key/value head over a paged cache on sm_103a (bf16): decoding steps.
//
//   paged_decode_kernel   up to 8 NT rows (new token, query head of the group) of one key/value head
//                         over a run of keys (paged_common.cuh), four warps with 16 keys of each 64.
//                         Bound by the bytes of the keys and values: they go from global memory
//                         straight into the registers of mma.sync m16n8k16 as they lie, a block ahead,
//                         so no shared memory and no barrier stands between a load and its use:
//                           S^T [16 keys][8 rows] = K Q^T: thread (g, t) of a warp loads 16 bytes of
//                             keys g and g + 8, the dimensions 32 i + 8 t ..; a product's order of
//                             dimensions is free as long as Q has the same;
//                           O^T [d][8 rows] += V^T P^T: it loads 16 bytes of keys 2 t, 2 t + 1,
//                             2 t + 8, 2 t + 9, dimensions 64 h + 8 g ..; two keys' values of a
//                             dimension are paired by byte permutes, and the rows of a fragment are
//                             whatever dimensions a thread holds.
//                         tcgen05 would need 128 rows where there are 1 to 16. The weights enter the
//                         second product as two bf16 parts (2^-17): it has the tensor pipe to itself,
//                         and the result is that of 32-bit weights. Per warp a running maximum and
//                         sum; the four warps meet at the end of a piece. Measured, 28 heads on 4:
//                         64 sequences of 16,384 positions 321 us (6.7 TB/s), of 100 to 16,384 5.2 TB/s;
//                         two blocks ahead instead of one, in as many warps as hold them: 72.5 us for
//                         74.5 with two contexts of 131,072 and 70,001, but 85 for 79 with the 64. One
//                         token on 517 positions: the work dealt out after 3.6 us, the pieces done after
//                         7.9, joined after 11.0.
#include "paged_common.cuh"

namespace mot {
namespace {

constexpr int kWarps = 4;
constexpr int kDecThreads = 32 * kWarps;
constexpr int kDecTK = 16 * kWarps;
// Units of a share. A join costs about as much as four tiles: one token on 517 positions, 12 heads of 128 on 2,
// takes 10.3 us in a graph with two tiles at least, 12.0 with one and 11.9 with four; on 8,000 14.4, 18.2 and
// 15.4 (on 64 positions one tile is better, 6.1 for 6.7). Pieces against runs (kMost = 0): 10.3 for 12.4 on 517
// positions, 14.4 for 16.4 on 8,000, 12.3 for 13.8 for 16 tokens of 12 heads of 64 on 500 each. Longer pieces
// leave CTAs without work: with 16, those 16 on 2,000 positions take 25.5 for 23.7.
constexpr int kLeast = 2, kMost = 8;

// 16 bytes that are read once
__device__ __forceinline__ uint4 ld_stream(const void* p) {
  uint4 v;
  asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
               : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
               : "l"(p));
  return v;
}
__device__ __forceinline__ uint32_t movmatrix(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack2(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *reinterpret_cast<uint32_t*>(&v);
}
__device__ __forceinline__ uint32_t word(const uint4& u, int i) { return i == 0 ? u.x : i == 1 ? u.y : i == 2 ? u.z : u.w; }

// CTAs per SM: as many as have their registers without spilling (16 warps of D = 128 that spill: 84 us
// for two contexts of 131,072 and 70,001, 12 that do not: 76).
template <int D, int NT>
constexpr int kResident = (D == 64 ? 5 : 4) - NT;

template <int D, int NT>
__global__ void __launch_bounds__(kDecThreads, kResident<D, NT>) paged_decode_kernel(const __grid_constant__ PagedAttnArgs a) {
  constexpr int BM = 8 * NT, TK = kDecTK, kI = D / 32, kH = D / 64;
  constexpr int kLd = D + 4;
  __shared__ int64_t scan[33];
  __shared__ PagedShare st;
  __shared__ PagedJoinShared s_join;
  __shared__ __align__(16) float so[kWarps][BM][kLd];   // read and written 16 bytes at a time
  __shared__ float sm[kWarps][BM], sl[kWarps][BM];
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int H = a.d.H, G = a.d.Hq / H;
  paged_begin<BM, TK>(a, kLeast, kMost, scan, st);
  const PagedCursor& c = st.c;
  const PagedPiece& p = st.p;
  const float sl2 = rsqrtf(float(D)) * 1.4426950408889634f;   // log2(e) / sqrt(d)
  const uint16_t* kp = static_cast<const uint16_t*>(a.k);
  const uint16_t* vp = static_cast<const uint16_t*>(a.v);

  while (st.work) {
    const int r0 = c.rt * BM, n_rows = min(BM, c.s.m * G - r0), len = c.s.len, hk = c.hk, slot = c.s.slot;
    uint4 q[NT][kI];
    int pos[NT][2];   // rows 8 nt + 2 t, + 1 see the keys 0 .. pos
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int r = 8 * n + g;
      const uint16_t* src = static_cast<const uint16_t*>(a.q) + (r < n_rows ? paged_out_row(c, H, G, r0 + r) : 0) * D + 8 * t;
#pragma unroll
      for (int i = 0; i < kI; ++i)
        q[n][i] = r < n_rows ? *reinterpret_cast<const uint4*>(src + 32 * i) : make_uint4(0u, 0u, 0u, 0u);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const int rr = 8 * n + 2 * t + e;
        pos[n][e] = rr < n_rows ? len - c.s.m + (r0 + rr) / G : -1;
      }
    }
    const int all_pos = len - c.s.m + r0 / G;   // every row sees the keys up to here
    float m[NT][2], l[NT][2], o[NT][kH][4][4];
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        m[n][e] = -INFINITY;
        l[n][e] = 0.f;
      }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int h = 0; h < kH; ++h)
#pragma unroll
        for (int e = 0; e < 16; ++e) o[n][h][e >> 2][e & 3] = 0.f;

    // lane l holds the page of this warp's block in tile `base` + l
    const int kt_begin = p.kt, kt_end = kt_begin + p.n;
    int base = kt_begin, held = 0;
    auto hold = [&](int kt) {
      base = kt;
      const int k = (kt + lane) * TK + 16 * warp;
      held = kt + lane < kt_end && k < len ? paged_page(a.d, a.table, a.status, slot, k) : 0;
    };
    hold(kt_begin);
    auto row_of = [&](int kt) -> int64_t {   // pool row of the block's first key
      if (kt - base >= 32) hold(kt);
      return paged_row(a.d, __shfl_sync(0xffffffffu, held, kt - base), hk, kt * TK + 16 * warp);
    };
    uint4 kr[2][kI], vr[4][kH];
    auto load_k = [&](int kt, int64_t row) {
      const int k0 = kt * TK + 16 * warp;
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        const bool in = k0 + g + 8 * e < len;
        const uint16_t* src = kp + (row + g + 8 * e) * D + 8 * t;
#pragma unroll
        for (int i = 0; i < kI; ++i) kr[e][i] = in ? ld_stream(src + 32 * i) : make_uint4(0u, 0u, 0u, 0u);
      }
    };
    auto load_v = [&](int kt, int64_t row) {
      const int k0 = kt * TK + 16 * warp;
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        const int j = 2 * t + (e & 1) + 8 * (e >> 1);
        const bool in = k0 + j < len;
        const uint16_t* src = vp + (row + j) * D + 8 * g;
#pragma unroll
        for (int h = 0; h < kH; ++h) vr[e][h] = in ? ld_stream(src + 64 * h) : make_uint4(0u, 0u, 0u, 0u);
      }
    };
    int64_t row = row_of(kt_begin);
    load_k(kt_begin, row);
    load_v(kt_begin, row);
    for (int kt = kt_begin; kt < kt_end; ++kt) {
      const int k0 = kt * TK + 16 * warp;
      float s[NT][4];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int e = 0; e < 4; ++e) s[n][e] = 0.f;
#pragma unroll
        for (int i = 0; i < kI; ++i) {
          mma_bf16(s[n], kr[0][i].x, kr[1][i].x, kr[0][i].y, kr[1][i].y, q[n][i].x, q[n][i].y);
          mma_bf16(s[n], kr[0][i].z, kr[1][i].z, kr[0][i].w, kr[1][i].w, q[n][i].z, q[n][i].w);
        }
      }
      const bool more = kt + 1 < kt_end;
      if (more) {
        row = row_of(kt + 1);
        load_k(kt + 1, row);
      }
      const bool part_seen = k0 + 15 > all_pos;   // some rows do not see all of the block
      bool up = false;
      float mx[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {   // key g + 8 (e / 2), row 2 t + e % 2
          s[n][e] *= sl2;
          if (part_seen && k0 + g + 8 * (e >> 1) > pos[n][e & 1]) s[n][e] = -INFINITY;
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float x = fmaxf(s[n][e], s[n][e + 2]);
#pragma unroll
          for (int w = 4; w < 32; w <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, w));
          mx[n][e] = x;
          up |= x > m[n][e];
        }
      }
      if (__any_sync(0xffffffffu, up)) {
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            const float to = fmaxf(m[n][e], mx[n][e]);
            const float f = exp2f(m[n][e] - (to == -INFINITY ? 0.f : to));
            m[n][e] = to;
            l[n][e] *= f;
#pragma unroll
            for (int h = 0; h < kH; ++h)
#pragma unroll
              for (int x = 0; x < 4; ++x) {
                o[n][h][x][e] *= f;
                o[n][h][x][e + 2] *= f;
              }
          }
      }
      uint32_t hi[NT][2], lo[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float pr[4];
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const float mu = m[n][e & 1];
          pr[e] = exp2f(s[n][e] - (mu == -INFINITY ? 0.f : mu));
          l[n][e & 1] += pr[e];
        }
#pragma unroll
        for (int e = 0; e < 2; ++e) {   // keys g, then keys g + 8
          const uint32_t u = pack2(pr[2 * e], pr[2 * e + 1]);
          hi[n][e] = movmatrix(u);
          lo[n][e] = movmatrix(pack2(pr[2 * e] - __uint_as_float(u << 16), pr[2 * e + 1] - __uint_as_float(u & 0xFFFF0000u)));
        }
      }
      bool odd = false;   // an infinite or NaN value that some rows must not meet
      if (part_seen && all_pos < min(k0 + 15, len - 1)) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int h = 0; h < kH; ++h)
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              const uint32_t u = word(vr[e][h], w);
              odd |= (u & 0x7F80u) == 0x7F80u || (u & 0x7F800000u) == 0x7F800000u;
            }
        odd = __any_sync(0xffffffffu, odd);
      }
      if (odd) {   // taken out of the product, and added below where they are seen
#pragma unroll
        for (int e = 0; e < 4; ++e)
#pragma unroll
          for (int h = 0; h < kH; ++h) {
            uint32_t u[4] = {vr[e][h].x, vr[e][h].y, vr[e][h].z, vr[e][h].w};
#pragma unroll
            for (int w = 0; w < 4; ++w) {
              if ((u[w] & 0x7F80u) == 0x7F80u) u[w] &= 0xFFFF0000u;
              if ((u[w] & 0x7F800000u) == 0x7F800000u) u[w] &= 0xFFFFu;
            }
            vr[e][h] = make_uint4(u[0], u[1], u[2], u[3]);
          }
      }
#pragma unroll
      for (int h = 0; h < kH; ++h)
#pragma unroll
        for (int x = 0; x < 4; ++x) {   // dimensions 64 h + 8 g + 2 x, + 1
          const uint32_t w0 = word(vr[0][h], x), w1 = word(vr[1][h], x), w2 = word(vr[2][h], x), w3 = word(vr[3][h], x);
          const uint32_t a0 = __byte_perm(w0, w1, 0x5410), a1 = __byte_perm(w0, w1, 0x7632);
          const uint32_t a2 = __byte_perm(w2, w3, 0x5410), a3 = __byte_perm(w2, w3, 0x7632);
#pragma unroll
          for (int n = 0; n < NT; ++n) {
            mma_bf16(o[n][h][x], a0, a1, a2, a3, hi[n][0], hi[n][1]);
            mma_bf16(o[n][h][x], a0, a1, a2, a3, lo[n][0], lo[n][1]);
          }
        }
      if (odd) {
        const int64_t at = paged_row(a.d, paged_page(a.d, a.table, a.status, slot, k0), hk, k0);
        for (int j = 0; j < 16 && k0 + j < len; ++j)
#pragma unroll
          for (int h = 0; h < kH; ++h)
#pragma unroll
            for (int e = 0; e < 8; ++e) {
              const float x = __uint_as_float(uint32_t(vp[(at + j) * D + 64 * h + 8 * g + e]) << 16);
              if (isfinite(x)) continue;
#pragma unroll
              for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int b = 0; b < 2; ++b)
                  if (k0 + j <= pos[n][b]) o[n][h][e >> 1][b + 2 * (e & 1)] += x;
            }
      }
      if (more) load_v(kt + 1, row);
    }
    // An infinite value that is seen: its weight's second part may be 0 or negative, which makes NaN of
    // the sum. Where a sum is not finite the piece's values are gone through again, and those that are
    // not finite and seen are the sum (an infinity, or NaN). Looked for once a piece, not in the loop.
    bool spoilt = false;
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int h = 0; h < kH; ++h)
#pragma unroll
        for (int e = 0; e < 16; ++e) spoilt |= !isfinite(o[n][h][e >> 2][e & 3]);
    if (__any_sync(0xffffffffu, spoilt)) {
#pragma unroll
      for (int h = 0; h < kH; ++h)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          float add[NT][2];
#pragma unroll
          for (int n = 0; n < NT; ++n) add[n][0] = add[n][1] = 0.f;
#pragma unroll 1
          for (int kt = kt_begin; kt < kt_end; ++kt) {
            const int k0 = kt * TK + 16 * warp;
            if (k0 >= len) break;
            const int64_t at = paged_row(a.d, paged_page(a.d, a.table, a.status, slot, k0), hk, k0);
#pragma unroll 1
            for (int j = 0; j < 16 && k0 + j < len; ++j) {
              const float x = __uint_as_float(uint32_t(vp[(at + j) * D + 64 * h + 8 * g + e]) << 16);
              if (isfinite(x)) continue;
#pragma unroll
              for (int n = 0; n < NT; ++n)
#pragma unroll
                for (int b = 0; b < 2; ++b)
                  if (k0 + j <= pos[n][b]) add[n][b] += x;
            }
          }
#pragma unroll
          for (int n = 0; n < NT; ++n)
#pragma unroll
            for (int b = 0; b < 2; ++b)
              if (add[n][b] != 0.f) o[n][h][e >> 1][b + 2 * (e & 1)] = add[n][b];   // NaN too
        }
    }
#pragma unroll
    for (int n = 0; n < NT; ++n)
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        float x = l[n][e];
#pragma unroll
        for (int w = 4; w < 32; w <<= 1) x += __shfl_xor_sync(0xffffffffu, x, w);
        const int r = 8 * n + 2 * t + e;
        if (g == 0) {
          sm[warp][r] = m[n][e];
          sl[warp][r] = x;
        }
#pragma unroll
        for (int h = 0; h < kH; ++h)
#pragma unroll
          for (int y = 0; y < 2; ++y)
            *reinterpret_cast<float4*>(&so[warp][r][64 * h + 8 * g + 4 * y]) =
                make_float4(o[n][h][2 * y][e], o[n][h][2 * y][e + 2], o[n][h][2 * y + 1][e], o[n][h][2 * y + 1][e + 2]);
      }
    __syncthreads();
    // the four warps' results: to the output, or to the piece's place
    float* part = p.whole ? nullptr : paged_part<BM, D>(a, blockIdx.x, p.kt == 0);
    for (int x = tid; x < n_rows * (D / 4); x += kDecThreads) {
      const int r = x / (D / 4), col = (x - r * (D / 4)) * 4;
      float mm = sm[0][r];
#pragma unroll
      for (int w = 1; w < kWarps; ++w) mm = fmaxf(mm, sm[w][r]);
      const float ms = mm == -INFINITY ? 0.f : mm;
      float ll = 0.f, y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int w = 0; w < kWarps; ++w) {
        const float f = exp2f(sm[w][r] - ms);
        const float4 v = *reinterpret_cast<const float4*>(&so[w][r][col]);
        ll = fmaf(f, sl[w][r], ll);
        y[0] = fmaf(f, v.x, y[0]);
        y[1] = fmaf(f, v.y, y[1]);
        y[2] = fmaf(f, v.z, y[2]);
        y[3] = fmaf(f, v.w, y[3]);
      }
      if (part) {
        *reinterpret_cast<float4*>(part + r * D + col) = make_float4(y[0], y[1], y[2], y[3]);
        if (col == 0) {
          part[BM * D + r] = mm;
          part[BM * (D + 1) + r] = ll;
        }
      } else {
        paged_store4(static_cast<uint16_t*>(a.out) + paged_out_row(c, H, G, r0 + r) * D + col, y, ll);
      }
    }
    if (part) paged_finish<uint16_t, BM, D>(a, c, p, s_join, tid, kDecThreads);
    __syncthreads();   // st, so and s_join are read
    if (tid == 0) paged_step<BM, TK>(a, st);
    __syncthreads();
  }
}

template <int D, int NT>
cudaError_t launch_decode(const PagedAttnArgs& a, int num_sms, cudaStream_t st) {
  return launch_kernel(false, paged_decode_kernel<D, NT>, num_sms * kResident<D, NT>, kDecThreads, 0, st, a);
}

}  // namespace

cudaError_t launch_paged_decode(const PagedAttnArgs& a, int num_sms, cudaStream_t st) {
  const bool one = int64_t(a.max_chunk) * (a.d.Hq / a.d.H) <= 8;
  if (a.d.d == 64) return one ? launch_decode<64, 1>(a, num_sms, st) : launch_decode<64, 2>(a, num_sms, st);
  return one ? launch_decode<128, 1>(a, num_sms, st) : launch_decode<128, 2>(a, num_sms, st);
}

}  // namespace mot
