// Attention of new tokens over a paged cache on sm_103a, in fp32 on the FMA units.
//
//   paged_simt_kernel   o_r = sum_{j <= p_r} softmax_j(q_r . k_j / sqrt(d)) v_j for BM rows (new token,
//                       query head of the group) of one key/value head at a time, in tiles of 64
//                       keys: scores, running maximum and sum (base 2), and the output rows in
//                       registers, 16 x 16 threads; keys, values and probabilities of the tile in
//                       shared memory. The work is dealt to the CTAs as paged_common.cuh says.
#include "paged_common.cuh"

namespace mot {
namespace {

constexpr int kTK = 64;
constexpr int kSimtThreads = 256;
constexpr int kLeast = 1, kMost = 8;   // units of a share

template <int D, int BM>
struct Simt {
  static constexpr int kLd = D + 4;    // floats from a query or key row to the next: 16-byte rows, spread over banks
  static constexpr int kLp = kTK + 4;  // of a probability row
  static constexpr int kSmem = 4 * (BM * kLd + kTK * kLd + kTK * D + BM * kLp);
};

__device__ __forceinline__ float4 load4(const float* p) { return *reinterpret_cast<const float4*>(p); }
__device__ __forceinline__ bool finite4(const float4& v) {
  return isfinite(v.x) && isfinite(v.y) && isfinite(v.z) && isfinite(v.w);
}

template <int D, int BM>
__global__ void __launch_bounds__(kSimtThreads) paged_simt_kernel(const __grid_constant__ PagedAttnArgs a) {
  using P = Simt<D, BM>;
  constexpr int kR = BM / 16;     // rows of a thread
  constexpr int kC = D / 64;      // float4 columns of a thread
  extern __shared__ float4 smem4[];
  float* sq = reinterpret_cast<float*>(smem4);
  float* sk = sq + BM * P::kLd;
  float* sv = sk + kTK * P::kLd;
  float* sp = sv + kTK * D;
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
      if (r < n_rows) v = load4(static_cast<const float*>(a.q) + paged_out_row(c, H, G, r0 + r) * D + col);
      *reinterpret_cast<float4*>(sq + r * P::kLd + col) = v;
    }
    int pos[kR];   // a row sees the keys 0 .. pos
#pragma unroll
    for (int i = 0; i < kR; ++i) {
      const int r = ty * kR + i;
      pos[i] = r < n_rows ? c.s.len - c.s.m + (r0 + r) / G : -1;
    }
    const int first_pos = c.s.len - c.s.m + r0 / G;
    float m[kR], l[kR], o[kR][4 * kC];
#pragma unroll
    for (int i = 0; i < kR; ++i) {
      m[i] = -INFINITY;
      l[i] = 0.f;
#pragma unroll
      for (int e = 0; e < 4 * kC; ++e) o[i][e] = 0.f;
    }
    const int len = c.s.len, kt_end = p.kt + p.n;
    for (int kt = p.kt; kt < kt_end; ++kt) {
      const int k0 = kt * kTK, n_keys = min(kTK, len - k0);
      bool odd = false;   // an infinite or NaN value in a tile that is masked for some rows
      for (int x = tid; x < kTK * (D / 4); x += kSimtThreads) {
        const int j = x / (D / 4), col = (x - j * (D / 4)) * 4;
        float4 kv = make_float4(0.f, 0.f, 0.f, 0.f), vv = kv;
        if (j < n_keys) {
          const int page = paged_page(a.d, a.table, a.status, c.s.slot, k0 + j);
          const int64_t row = paged_row(a.d, page, c.hk, k0 + j) * D + col;
          kv = load4(static_cast<const float*>(a.k) + row);
          vv = load4(static_cast<const float*>(a.v) + row);
          odd |= !finite4(vv);
        }
        *reinterpret_cast<float4*>(sk + j * P::kLd + col) = kv;
        *reinterpret_cast<float4*>(sv + j * D + col) = vv;
      }
      odd = __syncthreads_or(odd && first_pos < k0 + n_keys - 1);
      float s[kR][4];
#pragma unroll
      for (int i = 0; i < kR; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) s[i][j] = 0.f;
#pragma unroll 4
      for (int e = 0; e < D; e += 4) {
        float4 q4[kR], k4[4];
#pragma unroll
        for (int i = 0; i < kR; ++i) q4[i] = *reinterpret_cast<const float4*>(sq + (ty * kR + i) * P::kLd + e);
#pragma unroll
        for (int j = 0; j < 4; ++j) k4[j] = *reinterpret_cast<const float4*>(sk + (tx + 16 * j) * P::kLd + e);
#pragma unroll
        for (int i = 0; i < kR; ++i)
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            s[i][j] = fmaf(q4[i].x, k4[j].x, s[i][j]);
            s[i][j] = fmaf(q4[i].y, k4[j].y, s[i][j]);
            s[i][j] = fmaf(q4[i].z, k4[j].z, s[i][j]);
            s[i][j] = fmaf(q4[i].w, k4[j].w, s[i][j]);
          }
      }
#pragma unroll
      for (int i = 0; i < kR; ++i) {
        float mx = m[i];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          s[i][j] *= sl2;
          if (k0 + tx + 16 * j <= pos[i]) mx = fmaxf(mx, s[i][j]);
        }
#pragma unroll
        for (int w = 8; w; w >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, w));
        const float ms = mx == -INFINITY ? 0.f : mx;   // a row without keys so far: every 2^(-inf) is 0
        const float f = exp2f(m[i] - ms);
        m[i] = mx;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float pr = k0 + tx + 16 * j <= pos[i] ? exp2f(s[i][j] - ms) : 0.f;
          sum += pr;
          sp[(ty * kR + i) * P::kLp + tx + 16 * j] = pr;
        }
#pragma unroll
        for (int w = 8; w; w >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, w);
        l[i] = fmaf(l[i], f, sum);
#pragma unroll
        for (int e = 0; e < 4 * kC; ++e) o[i][e] *= f;
      }
      __syncwarp();   // a row's probabilities are written and read by one half-warp
      if (!odd) {
#pragma unroll 2
        for (int j = 0; j < kTK; j += 4) {
          float4 p4[kR];
#pragma unroll
          for (int i = 0; i < kR; ++i) p4[i] = *reinterpret_cast<const float4*>(sp + (ty * kR + i) * P::kLp + j);
#pragma unroll
          for (int jj = 0; jj < 4; ++jj)
#pragma unroll
            for (int h = 0; h < kC; ++h) {
              const float4 v = *reinterpret_cast<const float4*>(sv + (j + jj) * D + 64 * h + 4 * tx);
#pragma unroll
              for (int i = 0; i < kR; ++i) {
                const float pr = jj == 0 ? p4[i].x : jj == 1 ? p4[i].y : jj == 2 ? p4[i].z : p4[i].w;
                o[i][4 * h] = fmaf(pr, v.x, o[i][4 * h]);
                o[i][4 * h + 1] = fmaf(pr, v.y, o[i][4 * h + 1]);
                o[i][4 * h + 2] = fmaf(pr, v.z, o[i][4 * h + 2]);
                o[i][4 * h + 3] = fmaf(pr, v.w, o[i][4 * h + 3]);
              }
            }
        }
      } else {   // a masked key adds nothing, where 0 times its value would be NaN
        for (int j = 0; j < n_keys; ++j)
#pragma unroll
          for (int i = 0; i < kR; ++i)
            if (k0 + j <= pos[i]) {
              const float pr = sp[(ty * kR + i) * P::kLp + j];
#pragma unroll
              for (int h = 0; h < kC; ++h) {
                const float4 v = *reinterpret_cast<const float4*>(sv + j * D + 64 * h + 4 * tx);
                o[i][4 * h] = fmaf(pr, v.x, o[i][4 * h]);
                o[i][4 * h + 1] = fmaf(pr, v.y, o[i][4 * h + 1]);
                o[i][4 * h + 2] = fmaf(pr, v.z, o[i][4 * h + 2]);
                o[i][4 * h + 3] = fmaf(pr, v.w, o[i][4 * h + 3]);
              }
            }
      }
      __syncthreads();   // the tile is read; the next one may come
    }
    if (p.whole) {
#pragma unroll
      for (int i = 0; i < kR; ++i) {
        const int r = ty * kR + i;
        if (r >= n_rows) continue;
        const float f = l[i] == 0.f ? 0.f : 1.f / l[i];
        float* dst = static_cast<float*>(a.out) + paged_out_row(c, H, G, r0 + r) * D;
#pragma unroll
        for (int h = 0; h < kC; ++h) {
          const float t[4] = {o[i][4 * h], o[i][4 * h + 1], o[i][4 * h + 2], o[i][4 * h + 3]};
          paged_store4(dst + 64 * h + 4 * tx, t, f);
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
              make_float4(o[i][4 * h], o[i][4 * h + 1], o[i][4 * h + 2], o[i][4 * h + 3]);
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
  const int per_sm = BM == 16 ? 2 : 1;   // 64 rows at D = 64 fit twice, but make twice the pieces: 24.8 -> 28.6 us
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
