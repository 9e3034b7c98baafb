// Attention of few rows per key/value head over 8-bit pages on sm_103a: decoding steps (any number of rows is right).
//
//   paged8_decode_kernel  up to 8 NT rows (new token, query head of the group) of one key/value head over a run of
//                         keys (paged_common.cuh), tiles of 128, four warps with 32 keys of each, as two blocks of 16
//                         that lie in one page each. Bound by the bytes of the keys and values: a fifth warp brings
//                         them into a ring in shared memory by TMA, pages as they lie, with their scales, and goes on
//                         to the next piece while the others finish one. From there into mma.sync:
//                           S^T [16 keys][8 rows] = K Q^T, 8-bit, m16n8k32, with Q in two parts (Split8): thread
//                             (g, t) of a warp takes 16 bytes of two keys, the dimensions 64 i + 16 t ..; a
//                             product's order of dimensions is free as long as Q has the same;
//                           O^T [d][8 rows] += V^T P^T, fp16, m16n8k16: it takes d / 8 dimensions of four keys;
//                             bytes of two keys are paired by permutes and go through cvt to fp16, which holds 8-bit
//                             floats exactly.
//                         Which key is row g of a block, and which dimensions are a thread's, is free too, and such
//                         that no quarter of a warp meets a bank of the swizzled rows twice (row_of, part_of).
//                         The scales: a block's key scale multiplies its scores. Its value scale 2^e goes into the
//                         weights, w = 2^(s + e - R) with R the running maximum of s + e less 15, so that all of them
//                         are at most 2^15 and in fp16 (2^-11 of each, 2^-40 of the largest at the least); the sum
//                         of the weights in fp32 takes 2^e out again, exactly.
//                         One token of 28 heads on 4 of 128 on 131,072 positions and on 70,001: 46.2 us (4.4 TB/s), 64 of 100
//                         to 16,384 48.3 (4.5 TB/s), 32 heads on 32 on the two contexts 248 (6.6 TB/s); 57.8 and 64.1 with
//                         keys and values from global memory straight into registers.
#include "paged_common.cuh"
#include "paged8.cuh"

namespace mot {
namespace {

constexpr int kWarps = 4;
constexpr int kDecThreads = 2 * 32 * kWarps;   // warp 4 loads; 5 to 7 make up the group whose registers are given away
constexpr int kRowThreads = 32 * kWarps;       // those that compute
constexpr int kDecTK = 32 * kWarps;
// Units of a share, and what an item costs a CTA beside its units (its queries, the results' end: some microseconds). A
// CTA whose run is many short items would finish last: one token of 28 heads on 4 for 64 sequences of 100 to 16,384
// positions takes 48.3 us with three units for each, 65.8 with none, 49.0 with six; 64 of 4,096 take 55.5 for 55.0.
// Pieces where they make no CTA's work much longer: contexts of 131,072 and 70,001 positions 46.2 us, 53.9 in runs. Of one
// tile at least: 517 positions of 12 heads on 2 take 10.0 us, with two 11.2, with four 12.7, 8,000 14.4, 15.0 and 16.5;
// between them two are better, at 200 (8.4 us for 9.7) and at 2,000 (11.6 for 12.9).
constexpr int kLeast = 1, kMost = 4, kPad = 3;
constexpr float kTop = 15.f;   // weights are 2^15 at most: fp16 holds them down to 2^-40 of that, and many small ones count

// Key of a block of 16 that is row g of its first 8: of the swizzled rows of 128 bytes a quarter of a warp takes
// those that differ in the upper half of the 16-byte pieces, of the rows of 64 bytes both halves of 128.
template <int D>
__device__ __forceinline__ int row_of(int g) {
  return D == 128 ? (g & 1) << 2 | g >> 1 : g ^ (g >> 1 & 1);
}
// A thread's dimensions of V are D / 8 part_of(g) ..
template <int D>
__device__ __forceinline__ int part_of(int g) {
  return D == 128 ? (g & 1) << 2 | g >> 1 : g;
}
// 16-byte piece c of row r of a block, as TMA swizzles rows of D bytes.
template <int D>
__device__ __forceinline__ uint32_t piece_at(int r, int c) {
  return r * D + ((D == 128 ? c ^ (r & 7) : c ^ (r >> 1 & 3)) << 4);
}

__device__ __forceinline__ void ld_shared_v2(uint32_t addr, uint32_t& x, uint32_t& y) {
  asm volatile("ld.shared.v2.u32 {%0, %1}, [%2];" : "=r"(x), "=r"(y) : "r"(addr) : "memory");
}
__device__ __forceinline__ uint32_t movmatrix(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ uint32_t pack_half2(float lo, float hi) {
  const __half2 v = __floats2half2_rn(lo, hi);
  return *reinterpret_cast<const uint32_t*>(&v);
}
// c[16 x 8] += A[16 x 32] B[32 x 8], 8-bit operands, fp32 accumulators.
__device__ __forceinline__ void mma_f8(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                       uint32_t b1) {
  asm("mma.sync.aligned.m16n8k32.row.col.f32.e4m3.e4m3.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// c[16 x 8] += A[16 x 16] B[16 x 8], fp16 operands, fp32 accumulators.
__device__ __forceinline__ void mma_f16(float (&c)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0,
                                        uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
      : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
      : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}

template <int D, int NT>
struct Dec8 {
  static constexpr int kTile = kDecTK * D;               // bytes of a tile of keys, or of values
  static constexpr int kStages = D == 128 ? 2 : 3;
  static constexpr int kResident = D == 128 ? 2 : 3;     // CTAs per SM
  // registers at launch are 65,536 over the threads that are resident (128, or 80); dealt to the two groups of warps
  static constexpr int kLoadRegs = D == 128 ? 48 : 40, kRowRegs = D == 128 ? 208 : 120;
  static constexpr int kLd = D + 4;
  static constexpr int kSmem = 2 * kStages * kTile + kWarps * 8 * NT * kLd * 4 + 1024;   // ring, results; alignment
};

template <int D, int NT>
__global__ void __launch_bounds__(kDecThreads, Dec8<D, NT>::kResident)
    paged8_decode_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                         const __grid_constant__ PagedAttnArgs a) {
  using F = Dec8<D, NT>;
  constexpr int BM = 8 * NT, TK = kDecTK, kI = D / 64;   // 16-byte pieces of a thread in a key's row
  constexpr int kV = D / 8, kX = kV / 2;                 // dimensions of a thread in V; products of a block
  constexpr int kLd = F::kLd, kS = F::kStages;
  extern __shared__ uint8_t smem_raw[];
  __shared__ int64_t scan[33];
  __shared__ PagedShare shares[3];   // of piece k: k % 3; the one behind it is known
  __shared__ PagedJoinShared s_join;
  __shared__ float sm[kWarps][BM], sl[kWarps][BM];
  __shared__ uint64_t full[kS], empty[kS];
  __shared__ float2 scales[kS][8];   // of a tile's blocks: keys, values
  __shared__ int32_t s_abort;
  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31, g = lane >> 2, t = lane & 3;
  const int H = a.d.H, G = a.d.Hq / H;
  uint8_t* ring =
      reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  float* results = reinterpret_cast<float*>(ring + 2 * kS * F::kTile);   // [kWarps][BM][kLd]
  volatile int* abort_flag = reinterpret_cast<volatile int*>(&s_abort);
  if (tid == kRowThreads) {   // while warp 0 deals out the work
#pragma unroll
    for (int s = 0; s < kS; ++s) {
      mbar_init(&full[s], 1);
      mbar_init(&empty[s], kWarps);
    }
    s_abort = 0;
    fence_barrier_init();
    tma_prefetch_desc(&tmK);
    tma_prefetch_desc(&tmV);
  }
  pdl_wait();
  paged_begin<BM, TK, kPad>(a, kLeast, kMost, scan, shares[0], true);
  if (!shares[0].work) return;
  uint32_t tile = 0;   // of this CTA so far
  bool ok = true;
  int piece = 0;

  if (warp >= kWarps) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(F::kLoadRegs));
    if (warp == kWarps) {
      // ------------------------------------------------ TMA producer
      PagedCursor c = shares[0].c;
      ok = a.stall_test == 0 || blockIdx.x != 0;   // test hook: CTA 0 loads nothing
      while (ok && c.u < c.u_end) {
        const PagedPiece p = paged_piece<BM, TK, kPad>(c, G);
        const int kt_end = p.kt + p.n;
        // lanes 0 .. 7: a tile's blocks; their table entries are read two tiles ahead, their scales one
        auto mine = [&](int kt) { return lane < 8 && kt < kt_end && kt * TK + 16 * lane < c.s.len; };
        auto entry = [&](int kt) {
          return mine(kt) ? paged_page(a.d, a.table, a.status, c.s.slot, kt * TK + 16 * lane) : 0;
        };
        auto scale = [&](int kt, int page) {
          const int64_t x = int64_t(page) * H + c.hk;
          return mine(kt) ? make_float2(a.ks[x], a.vs[x]) : make_float2(1.f, 1.f);
        };
        int page = entry(p.kt), next = entry(p.kt + 1);
        float2 sc = scale(p.kt, page);
        for (int kt = p.kt; kt < kt_end; ++kt, ++tile) {
          if (!is_scale8(sc.x) || !is_scale8(sc.y))
            sc = make_float2(scale_of_page(sc.x, a.status), scale_of_page(sc.y, a.status));
          // behind the look at sc, which waits for every load before it: 16 sequences of 4,000, heads of 64, 34.7 us (38.5)
          const int next2 = entry(kt + 2);
          const float2 sc2 = scale(kt + 1, next);
          const uint32_t s = tile % kS;
          ok = __all_sync(0xffffffffu, mbar_wait(&empty[s], ((tile / kS) & 1u) ^ 1u, abort_flag, a.wait_limit));
          if (!ok) break;
          const int n_keys = min(TK, c.s.len - kt * TK), n_pages = n_keys <= 0 ? 0 : (n_keys + a.d.P - 1) >> a.d.lp;
          if (lane < 8) scales[s][lane] = sc;
          __syncwarp();
          if (lane == 0) mbar_arrive_expect_tx(&full[s], n_pages * a.d.P * 2 * D);
          __syncwarp();
          if (mine(kt) && (16 * lane & (a.d.P - 1)) == 0) {
            const int row = (page * H + c.hk) << a.d.lp;
            uint8_t* to = ring + s * 2 * F::kTile + 16 * lane * D;
            tma_load_2d(to, &tmK, &full[s], 0, row);
            tma_load_2d(to + F::kTile, &tmV, &full[s], 0, row);
          }
          page = next;
          next = next2;
          sc = sc2;
        }
        paged_next<BM, TK, kPad>(a, c, p);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(F::kRowRegs));
    const float sl2 = rsqrtf(float(D)) * 1.4426950408889634f;   // log2(e) / sqrt(d)
    const uint8_t* vp = static_cast<const uint8_t*>(a.v);
    float (*so)[kLd] = reinterpret_cast<float (*)[kLd]>(results) + warp * BM;
    const uint32_t ring_at = smem_u32(ring) + 32 * warp * D;
    if (tid == 0) {   // seen by the others behind the first piece's barriers
      shares[1] = shares[0];
      paged_step<BM, TK, kPad>(a, shares[1]);
    }
    for (; shares[piece % 3].work; ++piece) {
      const PagedCursor& c = shares[piece % 3].c;
      const PagedPiece& p = shares[piece % 3].p;
      const int r0 = c.rt * BM, n_rows = min(BM, c.s.m * G - r0), len = c.s.len, hk = c.hk, slot = c.s.slot;
      const int kt_begin = p.kt, kt_end = kt_begin + p.n;
      uint32_t q[NT][kI][2][4];   // 16 dimensions of row 8 n + g, in two parts
      float rf[NT][2];     // what takes the scores of rows 8 n + 2 t, + 1 to base-2 exponents, but for the key scale
      int pos[NT][2];          // these rows see the keys 0 .. pos
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        const int r = 8 * n + g;
        const int64_t at = r < n_rows ? paged_out_row(c, H, G, r0 + r) : 0;
        const uint16_t* src = static_cast<const uint16_t*>(a.q) + at * D + 16 * t;
        uint4 u[kI][2];
        uint32_t top = 0;
#pragma unroll
        for (int i = 0; i < kI; ++i)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            u[i][e] = r < n_rows ? *reinterpret_cast<const uint4*>(src + 64 * i + 8 * e) : make_uint4(0u, 0u, 0u, 0u);
            top = top_bf16x2(top, u[i][e]);
          }
        top = max(top & 0xFFFFu, top >> 16);
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 1));
        top = max(top, __shfl_xor_sync(0xffffffffu, top, 2));
        const Split8 split(top);
#pragma unroll
        for (int i = 0; i < kI; ++i)
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            split(u[i][e].x, u[i][e].y, q[n][i][0][2 * e], q[n][i][1][2 * e]);
            split(u[i][e].z, u[i][e].w, q[n][i][0][2 * e + 1], q[n][i][1][2 * e + 1]);
          }
        const float f = sl2 * split.factor;
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          rf[n][e] = __shfl_sync(0xffffffffu, f, 4 * (2 * t + e));
          const int rr = 8 * n + 2 * t + e;
          pos[n][e] = rr < n_rows ? len - c.s.m + (r0 + rr) / G : -1;
        }
      }
      const int all_pos = len - c.s.m + r0 / G;   // every row sees the keys up to here
      float m[NT][2], l[NT][2], o[NT][kX][4];     // m: largest score with the value scale's exponent, less kTop
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

      for (int kt = kt_begin; kt < kt_end; ++kt) {
        const int k0 = kt * TK + 32 * warp;
        const uint32_t stage = tile % kS, at = ring_at + stage * 2 * F::kTile;
        ok = __all_sync(0xffffffffu, mbar_wait(&full[stage], (tile / kS) & 1u, abort_flag, a.wait_limit));
        if (!ok) break;
        ++tile;
        const bool tail = k0 + 31 >= len;   // rows behind the sequence are whatever lies in the page, or in the ring
        float s[NT][2][4], s2[NT][2][4];   // of the queries' two parts
#pragma unroll
        for (int n = 0; n < NT; ++n)
#pragma unroll
          for (int e = 0; e < 8; ++e) s[n][e >> 2][e & 3] = s2[n][e >> 2][e & 3] = 0.f;
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int i = 0; i < kI; ++i) {
            const uint4 lo = ld_shared_v4(at + b * 16 * D + piece_at<D>(row_of<D>(g), 4 * i + t));
            const uint4 hi = ld_shared_v4(at + b * 16 * D + piece_at<D>(row_of<D>(g) + 8, 4 * i + t));
#pragma unroll
            for (int n = 0; n < NT; ++n) {
              mma_f8(s[n][b], lo.x, hi.x, lo.y, hi.y, q[n][i][0][0], q[n][i][0][1]);
              mma_f8(s2[n][b], lo.x, hi.x, lo.y, hi.y, q[n][i][1][0], q[n][i][1][1]);
              mma_f8(s[n][b], lo.z, hi.z, lo.w, hi.w, q[n][i][0][2], q[n][i][0][3]);
              mma_f8(s2[n][b], lo.z, hi.z, lo.w, hi.w, q[n][i][1][2], q[n][i][1][3]);
            }
          }
        uint32_t vr[2][4][kV / 4];   // of keys row_of(2 t), row_of(2 t + 1) and the same of the block's second half
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const int j = row_of<D>(2 * t + (e & 1)) + 8 * (e >> 1);
            const uint32_t from = at + F::kTile + 16 * b * D;
            if (D == 128) {
              const uint4 x = ld_shared_v4(from + piece_at<D>(j, part_of<D>(g)));
              vr[b][e][0] = x.x;
              vr[b][e][1] = x.y;
              vr[b][e][kV / 4 - 2] = x.z;
              vr[b][e][kV / 4 - 1] = x.w;
            } else {
              ld_shared_v2(from + piece_at<D>(j, g >> 1) + 8 * (g & 1), vr[b][e][0], vr[b][e][1]);
            }
          }
        if (tail) {
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e)
              if (k0 + 16 * b + row_of<D>(2 * t + (e & 1)) + 8 * (e >> 1) >= len)
#pragma unroll
                for (int w = 0; w < kV / 4; ++w) vr[b][e][w] = 0u;
        }
        float key_scale[2], ev[2], inv[2];   // a value scale 2^e: e and 2^-e
#pragma unroll
        for (int b = 0; b < 2; ++b) {
          const float2 sc = scales[stage][2 * warp + b];
          key_scale[b] = sc.x;
          const int e = int(__float_as_uint(sc.y) >> 23 & 255u) - 127;
          ev[b] = float(e);
          inv[b] = __uint_as_float(uint32_t(127 - e) << 23);
        }
        __syncwarp();
        if (lane == 0) mbar_arrive(&empty[stage]);   // the warp is through the tile's place
        const bool part_seen = k0 + 31 > all_pos;   // some rows do not see all of the keys
        bool up = false;
        float mx[NT][2];
#pragma unroll
        for (int n = 0; n < NT; ++n) {
#pragma unroll
          for (int b = 0; b < 2; ++b)
#pragma unroll
            for (int e = 0; e < 4; ++e) {   // key 16 b + row_of(g) + 8 (e / 2), row 2 t + e % 2
              s[n][b][e] = fmaf(s[n][b][e] + s2[n][b][e], factor8(rf[n][e & 1], key_scale[b]), ev[b]);
              if (part_seen && k0 + 16 * b + row_of<D>(g) + 8 * (e >> 1) > pos[n][e & 1]) s[n][b][e] = -INFINITY;
            }
#pragma unroll
          for (int e = 0; e < 2; ++e) {
            float x = fmaxf(fmaxf(s[n][0][e], s[n][0][e + 2]), fmaxf(s[n][1][e], s[n][1][e + 2]));
#pragma unroll
            for (int w = 4; w < 32; w <<= 1) x = fmaxf(x, __shfl_xor_sync(0xffffffffu, x, w));
            mx[n][e] = __fadd_ru(x, -kTop);
            up |= mx[n][e] > m[n][e];
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
            for (int w = 0; w < kV / 4; ++w) odd |= nan8(vr[e >> 2][e & 3][w]) != 0;
          odd = __any_sync(0xffffffffu, odd);
        }
        if (odd) {   // taken out of the product, and added below where it is seen
#pragma unroll
          for (int e = 0; e < 8; ++e)
#pragma unroll
            for (int w = 0; w < kV / 4; ++w) {
              uint32_t& u = vr[e >> 2][e & 3][w];
              u &= ~((nan8(u) >> 7) * 255u);
            }
        }
#pragma unroll
        for (int b = 0; b < 2; ++b)
#pragma unroll
          for (int w = 0; w < kV / 4; ++w) {
            const uint32_t w0 = vr[b][0][w], w1 = vr[b][1][w], w2 = vr[b][2][w], w3 = vr[b][3][w];
#pragma unroll
            for (int h = 0; h < 2; ++h) {   // dimensions kV part_of(g) + 4 w + 2 h, + 1
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
            const uint8_t* src = vp + paged_row(a.d, page, hk, k0 + j) * D + kV * part_of<D>(g);
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
            *reinterpret_cast<float4*>(&so[r][kV * part_of<D>(g) + 4 * y]) =
                make_float4(o[n][2 * y][e], o[n][2 * y][e + 2], o[n][2 * y + 1][e], o[n][2 * y + 1][e + 2]);
        }
      if (!bar_and(1, kRowThreads, ok)) break;   // a wait that ran out
      if (tid == 0) {   // by the barrier at this piece's end
        PagedShare& s = shares[(piece + 2) % 3];
        s = shares[(piece + 1) % 3];
        if (s.work) paged_step<BM, TK, kPad>(a, s);
      }
      // the four warps' results: to the output, or to the piece's place
      float* part = p.whole ? nullptr : paged_part<BM, D>(a, blockIdx.x, p.kt == 0);
      for (int x = tid; x < n_rows * (D / 4); x += kRowThreads) {
        const int r = x / (D / 4), col = (x - r * (D / 4)) * 4;
        float mm = sm[0][r];
#pragma unroll
        for (int w = 1; w < kWarps; ++w) mm = fmaxf(mm, sm[w][r]);
        const float ms = mm == -INFINITY ? 0.f : mm;
        float ll = 0.f, y[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kWarps; ++w) {
          const float f = exp2f(sm[w][r] - ms);
          const float4 v = *reinterpret_cast<const float4*>(results + (w * BM + r) * kLd + col);
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
      if (part) {
        asm volatile("bar.sync 1, %0;" ::"n"(kRowThreads) : "memory");
        if (tid == 0) s_join.mine = paged_arrive(a, p, s_join.g);
        asm volatile("bar.sync 1, %0;" ::"n"(kRowThreads) : "memory");
        if (s_join.mine) {
          paged_join<uint16_t, BM, D, 1>(a, c, s_join.g, tid, kRowThreads);
          if (!s_join.g.final) {
            asm volatile("bar.sync 1, %0;" ::"n"(kRowThreads) : "memory");
            if (tid == 0) s_join.mine = paged_arrive_group(a, p, s_join.g);
            asm volatile("bar.sync 1, %0;" ::"n"(kRowThreads) : "memory");
            if (s_join.mine) paged_join<uint16_t, BM, D, 1>(a, c, s_join.g, tid, kRowThreads);
          }
        }
      }
      asm volatile("bar.sync 1, %0;" ::"n"(kRowThreads) : "memory");   // results and s_join are read
    }
  }
  __syncthreads();
  if (*abort_flag) {
    if (tid == kRowThreads && (a.stall_test == 0 || blockIdx.x != 0)) {   // copies in flight: the last tiles'
      for (uint32_t k = tile < kS ? 0 : tile - kS; k != tile; ++k) {
        const long long t0 = clock64();
        while (!mbar_try_wait(smem_u32(&full[k % kS]), (k / kS) & 1u) && clock64() - t0 < a.wait_limit) {
        }
      }
    }
    if (tid == 0) {   // the arrivals that are still owed, so that the counters are zero for the next call
      for (PagedShare& s = shares[piece % 3]; s.work; paged_step<BM, TK, kPad>(a, s))
        if (!s.p.whole) paged_arrive_owed(a, s.p);
      atomicOr(a.status, kStatusTimeout);
    }
    __syncthreads();
  }
}

template <int D, int NT>
cudaError_t launch_decode(const PagedAttnArgs& a, const CUtensorMap& tmK, const CUtensorMap& tmV, int num_sms,
                          cudaStream_t st) {
  using F = Dec8<D, NT>;
  static SmemOptIn opt_in;
  auto kern = paged8_decode_kernel<D, NT>;
  if (cudaError_t e = opt_in(kern, F::kSmem)) return e;
  return launch_kernel(a.early, kern, num_sms * F::kResident, kDecThreads, F::kSmem, st, tmK, tmV, a);
}

}  // namespace

cudaError_t launch_paged8_decode(const PagedAttnArgs& a, const CUtensorMap& tmK, const CUtensorMap& tmV, int num_sms,
                                 cudaStream_t st) {
  const bool one = int64_t(a.max_chunk) * (a.d.Hq / a.d.H) <= 8;
  if (a.d.d == 64)
    return one ? launch_decode<64, 1>(a, tmK, tmV, num_sms, st) : launch_decode<64, 2>(a, tmK, tmV, num_sms, st);
  return one ? launch_decode<128, 1>(a, tmK, tmV, num_sms, st) : launch_decode<128, 2>(a, tmK, tmV, num_sms, st);
}

}  // namespace mot
