// Attention of few rows per key/value head over 8-bit pages on sm_103a: decoding steps (any number of rows is right).
//
//   paged8_decode_kernel  up to 8 NT rows (new token, query head of the group) of one key/value head over a run of
//                         keys (paged_common.cuh), four warps with 32 keys of each 128, as two blocks of 16 that lie
//                         in one page each. Bound by the bytes of the keys and values: they go from global memory
//                         straight into registers, a step ahead, and through cvt to fp16, which holds 8-bit floats
//                         exactly, into mma.sync m16n8k16:
//                           S^T [16 keys][8 rows] = K Q^T: thread (g, t) of a warp loads 16 bytes of keys g and
//                             g + 8, the dimensions 64 i + 16 t ..; a product's order of dimensions is free as long
//                             as Q has the same. Q's rows are put in fp16 by a power of two each, so that their
//                             largest value is at 2^12: a bf16 keeps its bits down to 2^-26 of that;
//                           O^T [d][8 rows] += V^T P^T: it loads the dimensions d / 8 g .. of keys 2 t, 2 t + 1,
//                             2 t + 8, 2 t + 9; bytes of two keys are paired by permutes before they are converted.
//                         The scales: a block's key scale multiplies its scores. Its value scale 2^e goes into the
//                         weights, w = 2^(s + e - R) with R the running maximum of s + e, so that all of them are
//                         at most 1 and in fp16 (2^-11 of each, 2^-25 of the largest at the least); the sum
//                         of the weights in fp32 takes 2^e out again, exactly.
#include "paged_common.cuh"
#include "paged8.cuh"

namespace mot {
namespace {

constexpr int kWarps = 4;
constexpr int kDecThreads = 32 * kWarps;
constexpr int kDecTK = 32 * kWarps;
constexpr int kLeast = 1, kMost = 4;   // units of a share

template <int N>
struct Bytes;   // N bytes of a row that are read once
template <>
struct Bytes<16> {
  uint32_t w[4];
  __device__ __forceinline__ void load(const void* p) {
    asm volatile("ld.global.nc.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                 : "l"(p));
  }
};
template <>
struct Bytes<8> {
  uint32_t w[2];
  __device__ __forceinline__ void load(const void* p) {
    asm volatile("ld.global.nc.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(w[0]), "=r"(w[1]) : "l"(p));
  }
};

__device__ __forceinline__ uint32_t movmatrix(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// c[16 x 8] += A[16 x 16] B[16 x 8], fp16 operands, fp32 accumulators.
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

// CTAs per SM: as many as have their registers without spilling.
template <int D, int NT>
constexpr int kResident = (D == 64 ? 5 : 4) - NT;

template <int D, int NT>
__global__ void __launch_bounds__(kDecThreads, kResident<D, NT>) paged8_decode_kernel(const __grid_constant__ PagedAttnArgs a) {
  constexpr int BM = 8 * NT, TK = kDecTK, kI = D / 64;   // loads of a key's row
  constexpr int kV = D / 8, kX = kV / 2;                 // dimensions of a thread in V; products of a block
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
  const uint8_t* kp = static_cast<const uint8_t*>(a.k);
  const uint8_t* vp = static_cast<const uint8_t*>(a.v);

  while (st.work) {
    const int r0 = c.rt * BM, n_rows = min(BM, c.s.m * G - r0), len = c.s.len, hk = c.hk, slot = c.s.slot;
    uint32_t q[NT][kI][8];   // 16 dimensions of row 8 n + g, fp16
    float rf[NT][2];         // what takes the scores of rows 8 n + 2 t, + 1 to base-2 exponents, but for the key scale
    int pos[NT][2];          // these rows see the keys 0 .. pos
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      const int r = 8 * n + g;
      const uint16_t* src = static_cast<const uint16_t*>(a.q) + (r < n_rows ? paged_out_row(c, H, G, r0 + r) : 0) * D + 16 * t;
      uint4 u[kI][2];
      uint32_t top = 0;
#pragma unroll
      for (int i = 0; i < kI; ++i)
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          u[i][e] = r < n_rows ? *reinterpret_cast<const uint4*>(src + 64 * i + 8 * e) : make_uint4(0u, 0u, 0u, 0u);
          top = __vmaxu2(top, __vmaxu2(__vmaxu2(u[i][e].x & 0x7FFF7FFFu, u[i][e].y & 0x7FFF7FFFu),
                                       __vmaxu2(u[i][e].z & 0x7FFF7FFFu, u[i][e].w & 0x7FFF7FFFu)));
        }
      top = max(top & 0xFFFFu, top >> 16);   // magnitudes of bf16 are ordered as integers
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
      top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
      const int up = min(12 + 127 - int(top >> 7), 126);
      const float by = __uint_as_float(uint32_t(up + 127) << 23);
#pragma unroll
      for (int i = 0; i < kI; ++i)
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const uint4& x = u[i][e >> 2];
          const uint32_t w = (e & 3) == 0 ? x.x : (e & 3) == 1 ? x.y : (e & 3) == 2 ? x.z : x.w;
          q[n][i][e] = pack_half2(__uint_as_float(w << 16) * by, __uint_as_float(w & 0xFFFF0000u) * by);
        }
      // a row that holds an infinity or NaN: its scores are NaN
      const float f = top >= 0x7F80u ? __uint_as_float(0x7FC00000u) : sl2 * __uint_as_float(uint32_t(127 - up) << 23);
#pragma unroll
      for (int e = 0; e < 2; ++e) {
        rf[n][e] = __shfl_sync(0xffffffffu, f, 4 * (2 * t + e));
        const int rr = 8 * n + 2 * t + e;
        pos[n][e] = rr < n_rows ? len - c.s.m + (r0 + rr) / G : -1;
      }
    }
    const int all_pos = len - c.s.m + r0 / G;   // every row sees the keys up to here
    float m[NT][2], l[NT][2], o[NT][kX][4];     // m: of scores with the value scale's exponent
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
      for (int x = 0; x < kX; ++x)
#pragma unroll
        for (int e = 0; e < 4; ++e) o[n][x][e] = 0.f;

    // lane l holds the page and the scales of block l % 2 of this warp's keys in tile `base` + l / 2
    const int kt_begin = p.kt, kt_end = kt_begin + p.n;
    int base = kt_begin, held = 0;
    float held_k = 0.f, held_v = 0.f;
    auto hold = [&](int kt) {
      base = kt;
      const int k = (kt + (lane >> 1)) * TK + 32 * warp + 16 * (lane & 1);
      const bool in = kt + (lane >> 1) < kt_end && k < len;
      held = in ? paged_page(a.d, a.table, a.status, slot, k) : 0;
      held_k = in ? a.ks[int64_t(held) * H + hk] : 1.f;
      held_v = in ? a.vs[int64_t(held) * H + hk] : 1.f;
    };
    hold(kt_begin);
    int64_t row[2];    // pool rows of the blocks' first keys
    float sk[2], sv[2];
    auto find = [&](int kt) {
      if (kt - base >= 16) hold(kt);
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int from = 2 * (kt - base) + b;
        row[b] = paged_row(a.d, __shfl_sync(0xffffffffu, held, from), hk, kt * TK + 32 * warp + 16 * b);
        sk[b] = __shfl_sync(0xffffffffu, held_k, from);
        sv[b] = __shfl_sync(0xffffffffu, held_v, from);
      }
    };
    Bytes<16> kr[2][2][kI];
    Bytes<kV> vr[2][4];
    auto load_k = [&](int kt) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int k0 = kt * TK + 32 * warp + 16 * b;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          const bool in = k0 + g + 8 * e < len;
          const uint8_t* src = kp + (row[b] + g + 8 * e) * D + 16 * t;
#pragma unroll
          for (int i = 0; i < kI; ++i) {
            if (in) kr[b][e][i].load(src + 64 * i);
            else
#pragma unroll
              for (int w = 0; w < 4; ++w) kr[b][e][i].w[w] = 0u;
          }
        }
      }
    };
    auto load_v = [&](int kt) {
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        const int k0 = kt * TK + 32 * warp + 16 * b;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          const int j = 2 * t + (e & 1) + 8 * (e >> 1);
          if (k0 + j < len) vr[b][e].load(vp + (row[b] + j) * D + kV * g);
          else
#pragma unroll
            for (int w = 0; w < kV / 4; ++w) vr[b][e].w[w] = 0u;
        }
      }
    };
    find(kt_begin);
    load_k(kt_begin);
    load_v(kt_begin);
    for (int kt = kt_begin; kt < kt_end; ++kt) {
      const int k0 = kt * TK + 32 * warp;
      float s[NT][2][4];
#pragma unroll
      for (int n = 0; n < NT; ++n)
#pragma unroll
        for (int e = 0; e < 8; ++e) s[n][e >> 2][e & 3] = 0.f;
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int i = 0; i < kI; ++i)
#pragma unroll
          for (int w = 0; w < 4; ++w) {
            const uint32_t u0 = kr[b][0][i].w[w], u1 = kr[b][1][i].w[w];
            const uint32_t a0 = half2_of8(u0), a1 = half2_of8(u1), a2 = half2_of8(u0 >> 16), a3 = half2_of8(u1 >> 16);
#pragma unroll
            for (int n = 0; n < NT; ++n) mma_f16(s[n][b], a0, a1, a2, a3, q[n][i][2 * w], q[n][i][2 * w + 1]);
          }
      float key_scale[2], ev[2], inv[2];   // a value scale 2^e: e and 2^-e
#pragma unroll
      for (int b = 0; b < 2; ++b) {
        key_scale[b] = sk[b];
        const int e = int(__float_as_uint(sv[b]) >> 23 & 255u) - 127;
        ev[b] = float(e);
        inv[b] = __uint_as_float(uint32_t(127 - e) << 23);
      }
      const bool more = kt + 1 < kt_end;
      if (more) {
        find(kt + 1);
        load_k(kt + 1);
      }
      const bool part_seen = k0 + 31 > all_pos;   // some rows do not see all of the keys
      bool up = false;
      float mx[NT][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e) {   // key 16 b + g + 8 (e / 2), row 2 t + e % 2
            s[n][b][e] = fmaf(s[n][b][e], rf[n][e & 1] * key_scale[b], ev[b]);
            if (part_seen && k0 + 16 * b + g + 8 * (e >> 1) > pos[n][e & 1]) s[n][b][e] = -INFINITY;
          }
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float x = fmaxf(fmaxf(s[n][0][e], s[n][0][e + 2]), fmaxf(s[n][1][e], s[n][1][e + 2]));
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
            for (int x = 0; x < kX; ++x) {
              o[n][x][e] *= f;
              o[n][x][e + 2] *= f;
            }
          }
      }
      uint32_t pr[NT][2][2];
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        float mu[2];
#pragma unroll
        for (int e = 0; e < 2; ++e) mu[e] = m[n][e] == -INFINITY ? 0.f : m[n][e];
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          float x[4];
#pragma unroll
          for (int e = 0; e < 4; ++e) x[e] = exp2f(s[n][b][e] - mu[e & 1]);
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            l[n][e] = fmaf(x[e] + x[e + 2], inv[b], l[n][e]);
            pr[n][b][e] = movmatrix(pack_half2(x[2 * e], x[2 * e + 1]));   // keys g, then keys g + 8
          }
        }
      }
      bool odd = false;   // a NaN value that some rows must not meet
      if (part_seen && all_pos < min(k0 + 31, len - 1)) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int w = 0; w < kV / 4; ++w) odd |= nan8(vr[e >> 2][e & 3].w[w]) != 0;
        odd = __any_sync(0xffffffffu, odd);
      }
      if (odd) {   // taken out of the product, and added below where it is seen
#pragma unroll
        for (int e = 0; e < 8; ++e)
#pragma unroll
          for (int w = 0; w < kV / 4; ++w) {
            uint32_t& u = vr[e >> 2][e & 3].w[w];
            u &= ~((nan8(u) >> 7) * 255u);
          }
      }
#pragma unroll
      for (int b = 0; b < 2; ++b)
#pragma unroll
        for (int w = 0; w < kV / 4; ++w) {
          const uint32_t w0 = vr[b][0].w[w], w1 = vr[b][1].w[w], w2 = vr[b][2].w[w], w3 = vr[b][3].w[w];
#pragma unroll
          for (int h = 0; h < 2; ++h) {   // dimensions kV g + 4 w + 2 h, + 1
            const uint32_t u = __byte_perm(w0, w1, h ? 0x7362 : 0x5140), v = __byte_perm(w2, w3, h ? 0x7362 : 0x5140);
            const uint32_t a0 = half2_of8(u), a1 = half2_of8(u >> 16), a2 = half2_of8(v), a3 = half2_of8(v >> 16);
#pragma unroll
            for (int n = 0; n < NT; ++n) mma_f16(o[n][2 * w + h], a0, a1, a2, a3, pr[n][b][0], pr[n][b][1]);
          }
        }
      if (odd) {
#pragma unroll 1
        for (int j = 0; j < 32 && k0 + j < len; ++j) {
          const int page = paged_page(a.d, a.table, a.status, slot, k0 + j);
          const uint8_t* src = vp + paged_row(a.d, page, hk, k0 + j) * D + kV * g;
#pragma unroll
          for (int e = 0; e < kV; ++e) {
            if ((src[e] & 0x7Fu) != kNaN8) continue;
#pragma unroll
            for (int n = 0; n < NT; ++n)
#pragma unroll
              for (int b = 0; b < 2; ++b)
                if (k0 + j <= pos[n][b]) o[n][e >> 1][b + 2 * (e & 1)] = __uint_as_float(0x7FC00000u);
          }
        }
      }
      if (more) load_v(kt + 1);
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
        for (int y = 0; y < kX / 2; ++y)
          *reinterpret_cast<float4*>(&so[warp][r][kV * g + 4 * y]) =
              make_float4(o[n][2 * y][e], o[n][2 * y][e + 2], o[n][2 * y + 1][e], o[n][2 * y + 1][e + 2]);
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
  return launch_kernel(false, paged8_decode_kernel<D, NT>, num_sms * kResident<D, NT>, kDecThreads, 0, st, a);
}

}  // namespace

cudaError_t launch_paged8_decode(const PagedAttnArgs& a, int num_sms, cudaStream_t st) {
  const bool one = int64_t(a.max_chunk) * (a.d.Hq / a.d.H) <= 8;
  if (a.d.d == 64) return one ? launch_decode<64, 1>(a, num_sms, st) : launch_decode<64, 2>(a, num_sms, st);
  return one ? launch_decode<128, 1>(a, num_sms, st) : launch_decode<128, 2>(a, num_sms, st);
}

}  // namespace mot
