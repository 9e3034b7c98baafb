// Attention of new tokens over a paged cache on sm_103a, in fp32 on the FMA units.
//
//   paged_simt_kernel   o_r = sum_{j <= p_r} softmax_j(q_r . k_j / sqrt(d)) v_j for BM rows (new token,
//                       query head of the group) of one key/value head at a time, in tiles of 64
//                       keys: scores, running maximum and sum (base 2), and the output rows in
//                       registers, 16 x 16 threads; keys, values and probabilities of the tile in
//                       shared memory, the next tile's copies under way. Both products run on pairs of
//                       fp32: a score sums the even and the odd dimensions apart, an output pair takes
//                       its probability doubled from shared memory. 4 x 4 results a thread: 1,024 tokens
//                       on 4,096 positions, 28 heads of 128, 1,525 us (34.5 TFLOP/s), shared-memory
//                       reads at 68% of their rate before the FMA units, 8 warps an SM. The work is
//                       dealt to the CTAs as paged_common.cuh says.
#include "paged_common.cuh"

namespace mot {
namespace {

constexpr int kTK = 64;
constexpr int kSimtThreads = 256;
// Units of a share. Pieces against runs (kMost = 0), us in a graph: a prompt of 64 on 1,024 positions beside a
// step, 12 heads of 64, 23 for 35; one token on 8,000, 12 heads of 128 on 2, 21 for 24. Longer pieces leave
// CTAs without work where the items are many: with 8, 256 new tokens on 1,024 positions take 56 for 43, six
// prompts of 60 on 500 positions 50 for 36. kLeast = 2 makes one token on 300 positions 13.3 for 9.5.
constexpr int kLeast = 1, kMost = 4;

template <int D, int BM>
struct Simt {
  static constexpr int kLd = D + 4;    // floats from a query or key row to the next: 16-byte rows, spread over banks
  static constexpr int kLp = 2 * kTK + 4;          // of a row of doubled probabilities
  static constexpr int kTile = kTK * (kLd + D);    // keys and values
  static constexpr int kSmem = 4 * (BM * kLd + 2 * kTile + BM * kLp);
};

// 16 bytes from global to shared memory, or zeros.
__device__ __forceinline__ void cp_async_16_or_0(uint32_t dst, const void* src, bool in) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(in ? 16 : 0) : "memory");
}
__device__ __forceinline__ bool finite4(const float4& v) {
  return isfinite(v.x) && isfinite(v.y) && isfinite(v.z) && isfinite(v.w);
}
__device__ __forceinline__ float lo_f(uint64_t x) { return __uint_as_float(uint32_t(x)); }
__device__ __forceinline__ float hi_f(uint64_t x) { return __uint_as_float(uint32_t(x >> 32)); }
// Four floats of shared memory as two pairs.
__device__ __forceinline__ ulonglong2 pairs(const float* p) { return *reinterpret_cast<const ulonglong2*>(p); }

template <int D, int BM>
__global__ void __launch_bounds__(kSimtThreads) paged_simt_kernel(const __grid_constant__ PagedAttnArgs a) {
  using P = Simt<D, BM>;
  constexpr int kR = BM / 16;     // rows of a thread
  constexpr int kC = D / 64;      // float4 columns of a thread
  extern __shared__ float4 smem4[];
  float* sq = reinterpret_cast<float*>(smem4);
  float* stage = sq + BM * P::kLd;      // two tiles: keys [kTK][kLd], values [kTK][D]
  float* sp = stage + 2 * P::kTile;
  __shared__ int64_t sh[33];
  __shared__ PagedShare st;
  __shared__ PagedJoinShared s_join;
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  const int H = a.d.H, G = a.d.Hq / H;
  paged_begin<BM, kTK>(a, kLeast, kMost, sh, st);
  const PagedCursor& c = st.c;
  const PagedPiece& p = st.p;
  const float sl2 = rsqrtf(float(D)) * 1.4426950408889634f;   // log2(e) / sqrt(d)

  while (st.work) {
    const int r0 = c.rt * BM, n_rows = min(BM, c.s.m * G - r0);
    // the rows' queries
    for (int x = tid; x < BM * (D / 4); x += kSimtThreads) {
      const int r = x / (D / 4), col = (x - r * (D / 4)) * 4;
      float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r < n_rows)
        v = *reinterpret_cast<const float4*>(static_cast<const float*>(a.q) + paged_out_row(c, H, G, r0 + r) * D + col);
      *reinterpret_cast<float4*>(sq + r * P::kLd + col) = v;
    }
    int pos[kR];   // a row sees the keys 0 .. pos
#pragma unroll
    for (int i = 0; i < kR; ++i) {
      const int r = ty * kR + i;
      pos[i] = r < n_rows ? c.s.len - c.s.m + (r0 + r) / G : -1;
    }
    const int first_pos = c.s.len - c.s.m + r0 / G;
    float m[kR], l[kR];
    uint64_t o[kR][2 * kC];   // columns 64 h + 4 tx + 2 e, + 1 in o[i][2 h + e]
#pragma unroll
    for (int i = 0; i < kR; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
#pragma unroll
      for (int e = 0; e < 2 * kC; ++e) o[i][e] = 0ull;
    }
    const int len = c.s.len, kt_end = p.kt + p.n, slot = c.s.slot, hk = c.hk;
    constexpr int kVecs = kTK * (D / 4) / kSimtThreads;   // of a thread, in keys and in values
    auto fetch = [&](int kt) {
      float* sk = stage + (kt & 1) * P::kTile;
      float* sv = sk + kTK * P::kLd;
#pragma unroll
      for (int y = 0; y < kVecs; ++y) {
        const int x = tid + y * kSimtThreads, j = x / (D / 4), col = (x - j * (D / 4)) * 4, pos_j = kt * kTK + j;
        const bool in = pos_j < len;
        const int64_t row =
            in ? paged_row(a.d, paged_page(a.d, a.table, a.status, slot, pos_j), hk, pos_j) * D + col : 0;
        cp_async_16_or_0(smem_u32(sk + j * P::kLd + col), static_cast<const float*>(a.k) + row, in);
        cp_async_16_or_0(smem_u32(sv + j * D + col), static_cast<const float*>(a.v) + row, in);
      }
      cp_async_commit();
    };
    fetch(p.kt);
    for (int kt = p.kt; kt < kt_end; ++kt) {
      const int k0 = kt * kTK, n_keys = min(kTK, len - k0);
      const float* sk = stage + (kt & 1) * P::kTile;
      const float* sv = sk + kTK * P::kLd;
      if (kt + 1 < kt_end) {
        fetch(kt + 1);
        cp_async_wait_group<1>();
      } else {
        cp_async_wait_group<0>();
      }
      bool odd = false;   // an infinite or NaN value in a tile that is masked for some rows
      if (first_pos < k0 + n_keys - 1) {
#pragma unroll
        for (int y = 0; y < kVecs; ++y) {   // what this thread has copied
          const int x = tid + y * kSimtThreads, j = x / (D / 4), col = (x - j * (D / 4)) * 4;
          odd |= !finite4(*reinterpret_cast<const float4*>(sv + j * D + col));
        }
      }
      odd = __syncthreads_or(odd);
      uint64_t s2[kR][4];
#pragma unroll
      for (int i = 0; i < kR; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) s2[i][j] = 0ull;
#pragma unroll 4
      for (int e = 0; e < D; e += 4) {
        ulonglong2 q4[kR], k4[4];
#pragma unroll
        for (int i = 0; i < kR; ++i) q4[i] = pairs(sq + (ty * kR + i) * P::kLd + e);
#pragma unroll
        for (int j = 0; j < 4; ++j) k4[j] = pairs(sk + (tx + 16 * j) * P::kLd + e);
#pragma unroll
        for (int i = 0; i < kR; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) s2[i][j] = ffma_x2(q4[i].y, k4[j].y, ffma_x2(q4[i].x, k4[j].x, s2[i][j]));
      }
#pragma unroll
      for (int i = 0; i < kR; ++i) {
        float mx = m[i], s[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          s[j] = (lo_f(s2[i][j]) + hi_f(s2[i][j])) * sl2;
          if (k0 + tx + 16 * j <= pos[i]) mx = fmaxf(mx, s[j]);
        }
#pragma unroll
        for (int w = 8; w; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
        const float ms = mx == -INFINITY ? 0.f : mx;   // a row without keys so far: every 2^(-inf) is 0
        const float f = exp2f(m[i] - ms);
        m[i] = mx;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float pr = k0 + tx + 16 * j <= pos[i] ? exp2f(s[j] - ms) : 0.f;
          sum += pr;
          *reinterpret_cast<float2*>(sp + (ty * kR + i) * P::kLp + 2 * (tx + 16 * j)) = make_float2(pr, pr);
        }
#pragma unroll
        for (int w = 8; w; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
        l[i] = fmaf(l[i], f, sum);
        const uint64_t f2 = f32x2(f, f);
#pragma unroll
        for (int e = 0; e < 2 * kC; ++e) o[i][e] = fmul_x2(o[i][e], f2);
      }
      __syncwarp();   // a row's probabilities are written and read by one half-warp
      if (!odd) {
#pragma unroll 4
        for (int j = 0; j < kTK; j += 2) {
          ulonglong2 p2[kR];
#pragma unroll
          for (int i = 0; i < kR; ++i) p2[i] = pairs(sp + (ty * kR + i) * P::kLp + 2 * j);
#pragma unroll
          for (int h = 0; h < kC; ++h) {
            const ulonglong2 v0 = pairs(sv + j * D + 64 * h + 4 * tx), v1 = pairs(sv + (j + 1) * D + 64 * h + 4 * tx);
#pragma unroll
            for (int i = 0; i < kR; ++i) {
              o[i][2 * h] = ffma_x2(p2[i].y, v1.x, ffma_x2(p2[i].x, v0.x, o[i][2 * h]));
              o[i][2 * h + 1] = ffma_x2(p2[i].y, v1.y, ffma_x2(p2[i].x, v0.y, o[i][2 * h + 1]));
            }
          }
        }
      } else {   // a masked key adds nothing, where 0 times its value would be NaN
        for (int j = 0; j < n_keys; ++j)
#pragma unroll
          for (int i = 0; i < kR; ++i)
            if (k0 + j <= pos[i]) {
              const uint64_t pr = *reinterpret_cast<const uint64_t*>(sp + (ty * kR + i) * P::kLp + 2 * j);
#pragma unroll
              for (int h = 0; h < kC; ++h) {
                const ulonglong2 v = pairs(sv + j * D + 64 * h + 4 * tx);
                o[i][2 * h] = ffma_x2(pr, v.x, o[i][2 * h]);
                o[i][2 * h + 1] = ffma_x2(pr, v.y, o[i][2 * h + 1]);
              }
            }
      }
      __syncthreads();   // the tile is read; the copies after the next may come
    }
    if (p.whole) {
#pragma unroll
      for (int i = 0; i < kR; ++i) {
        const int r = ty * kR + i;
        if (r >= n_rows) continue;
        float* dst = static_cast<float*>(a.out) + paged_out_row(c, H, G, r0 + r) * D;
#pragma unroll
        for (int h = 0; h < kC; ++h) {
          const float t[4] = {lo_f(o[i][2 * h]), hi_f(o[i][2 * h]), lo_f(o[i][2 * h + 1]), hi_f(o[i][2 * h + 1])};
          paged_store4(dst + 64 * h + 4 * tx, t, l[i]);
        }
      }
    } else {
      float* part = paged_part<BM, D>(a, blockIdx.x, p.kt == 0);
#pragma unroll
      for (int i = 0; i < kR; ++i) {
        const int r = ty * kR + i;
        if (r >= n_rows) continue;
#pragma unroll
        for (int h = 0; h < kC; ++h)
          *reinterpret_cast<float4*>(part + r * D + 64 * h + 4 * tx) =
              make_float4(lo_f(o[i][2 * h]), hi_f(o[i][2 * h]), lo_f(o[i][2 * h + 1]), hi_f(o[i][2 * h + 1]));
        if (tx == 0) {
          part[BM * D + r] = m[i];
          part[BM * (D + 1) + r] = l[i];
        }
      }
      paged_finish<float, BM, D>(a, c, p, s_join, tid, kSimtThreads);
    }
    __syncthreads();   // st, s_join and the queries are read
    if (tid == 0) paged_step<BM, kTK>(a, st);
    __syncthreads();
  }
}

template <int D, int BM>
cudaError_t launch_simt(const PagedAttnArgs& a, int num_sms, cudaStream_t st) {
  static SmemOptIn opt_in;
  auto kern = paged_simt_kernel<D, BM>;
  if (cudaError_t e = opt_in(kern, Simt<D, BM>::kSmem)) return e;
  const int per_sm = BM == 16 && D == 64 ? 2 : 1;   // by shared memory
  return launch_kernel(false, kern, num_sms * per_sm, kSimtThreads, Simt<D, BM>::kSmem, st, a);
}

}  // namespace

// Two places per CTA: 256 rows with one CTA per SM, fewer rows with more. Three counters per CTA.
size_t paged_part_floats(const PagedDims& d, int num_sms) { return size_t(num_sms) * 2 * 256 * (d.d + 2); }
int paged_counters(int num_sms) { return num_sms * 4 * 3; }
bool paged_fmha_takes(const PagedDims& d, int max_chunk) {
  return d.dtype == 0 && int64_t(max_chunk) * (d.Hq / d.H) > 16;
}

cudaError_t launch_paged_simt(const PagedAttnArgs& a, int num_sms, cudaStream_t st) {
  const bool few = int64_t(a.max_chunk) * (a.d.Hq / a.d.H) <= 16;
  if (a.d.d == 64) return few ? launch_simt<64, 16>(a, num_sms, st) : launch_simt<64, 64>(a, num_sms, st);
  return few ? launch_simt<128, 16>(a, num_sms, st) : launch_simt<128, 64>(a, num_sms, st);
}

}  // namespace mot
