// Attention of chunks of new tokens over 8-bit pages on the tensor cores of sm_103a.
//
//   paged8_fmha_kernel  persistent, one CTA per SM over its run of key tiles (paged_common.cuh), an item being 256
//                       rows of one key/value head as two streams of 128, over tiles of 128 keys, as in the kernel of
//                       16-bit pages. What is different:
//                         keys       go as they lie into an 8-bit product (kind::f8f6f4), with Q in two parts (Split8);
//                         values     are turned to fp16, which holds them exactly, by warps 2 and 3, between two
//                                    rings of shared memory (16 values a thread and step: one 16-byte load, two
//                                    stores, without bank conflicts); P in two 8-bit parts would leave them as they
//                                    are, but cost the softmax, which paces the kernel, three conversions for one;
//                         scales     of 16 keys (a page has 16 at least) each, by way of a ring: that of the keys
//                                    multiplies the scores, that of the values, 2^e, goes into the weights, w =
//                                    2^(s + e - R) with R the running maximum of s + e less 7 (raised only where a
//                                    tile passes that maximum by 8, so that w is 2^15 at most, and in fp16 off by 2^-11
//                                    of itself or 2^-25 at the least, 2^-32 of the row's largest); the sum takes 2^e
//                                    out again, exactly. Where the scales of a
//                                    tile and of those before it span more than 2^60, weights below 2^-126 count in
//                                    the sum (w 2^-e beside 2^-e' of the row's largest), and are not flushed to 0.
//                       Bound by the chain of products and softmax, with shared memory near its limit beside it (both parts
//                       of Q and the keys are read from it twice, the values three times): 4,096 tokens of 28 heads on 4
//                       of 128 on 32,768 positions 1,287 us (1,402 TFLOP/s; a tenth less were the values in fp16 already).
//                       Every wait is bounded; on a timeout the roles unwind, copies and MMAs in flight are drained,
//                       TMEM is freed and kStatusTimeout is raised.
#include "paged_chunk.cuh"
#include "paged8.cuh"

namespace mot {
namespace {

// Units of a share, as with 16-bit pages, and what an item costs beside its units: its queries and its end, about as
// much as eight tiles, which a CTA with a run of short items has many times. 28 heads on 4, prompts of 2,111, 700 and 3,000
// tokens from nothing: 174 us with eight, 176 with six, 178 with ten, 295 with none (now 182); a mixture with long contexts (500
// of 9,000, 2,111 of 2,500, 1,999 of 4,097, 48 of 700) 229, 249, 238 and 363.
constexpr int kLeast = 1, kMost = 16, kPad = 8;

template <int D>
struct Pf8 {
  static constexpr int kBM = kChunkRows, kTK = 128;
  static constexpr int kTile = 128 * D;                // bytes of 128 rows in 8 bits
  static constexpr int kBlk = 128 * 128;               // 128 rows of 64 fp16
  static constexpr int kTile16 = D / 64 * kBlk;
  static constexpr int kNK = 2, kNV = 3, kNH = 2;      // tiles in flight: keys, values, values in fp16
  static constexpr int kThreads = 32 * 12;
  static constexpr int kBytes = (4 + kNK + kNV) * kTile + kNH * kTile16;
  static constexpr int kSmem = kBytes + 4096 + 1024;   // barriers, scales and notes; alignment
  static constexpr int kO = 256;                       // TMEM: S at 0 and 128, O at 256 and 256 + D
  // 16-byte piece c of row r, swizzled as TMA writes rows of D bytes
  static __device__ __forceinline__ uint32_t at(int r, int c) {
    return r * D + ((D == 128 ? c ^ (r & 7) : c ^ (r >> 1 & 3)) << 4);
  }
};
static_assert(Pf8<128>::kSmem <= 232448, "shared memory budget");
static_assert(Pf8<128>::kO + 2 * 128 <= 512, "TMEM columns");

constexpr int kScaleRing = 8;
struct alignas(16) Scales8 {   // of a tile's groups of 16 keys
  float k[8], e[8], inv[8];   // of keys; a value scale's exponent and 2^-e
  int32_t wide;               // value scales so far apart that a weight in the sum may lie below 2^-126
};

// Barriers and what the roles leave for one another.
struct Pf8Shared {
  uint64_t q_ready[2], s_full[2], p_half[2][2], pv_done[2];
  uint64_t k_full[3], k_empty[3], v_full[3], v_empty[3], h_full[3], h_empty[3], drain;
  uint32_t tmem;
  int32_t abort;
  PagedJoinShared join;
  uint32_t notes[4][4][4];   // [piece & 3][tile of the masked ones][128 keys]: values that are NaN
  Scales8 scales[kScaleRing];
  Scales8 done[8];   // a softmax warp's, of a tile whose scores are worked out already
  float rf[256];     // what takes a row's scores to base-2 exponents, but for the key scales: a thread's own
};
static_assert(sizeof(Pf8Shared) <= 4096, "barrier block");

// K-major operand of 64-byte rows with 64-byte swizzling: 8-row groups 512 B apart.
__device__ __forceinline__ uint64_t sdesc_k_sw64(uint32_t saddr) {
  uint64_t d = 0;
  d |= static_cast<uint64_t>((saddr & 0x3FFFFu) >> 4);
  d |= static_cast<uint64_t>(1u) << 16;
  d |= static_cast<uint64_t>(512u >> 4) << 32;
  d |= static_cast<uint64_t>(1u) << 46;
  d |= static_cast<uint64_t>(4u) << 61;
  return d;
}
// D[tmem] (+)= A[smem] * B[smem]^T of 8-bit floats, 32 of K, issued by a single thread.
__device__ __forceinline__ void umma_f8(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc,
                                        uint32_t accumulate) {
  asm volatile(
      "{\n\t.reg .pred p;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "tcgen05.mma.cta_group::1.kind::f8f6f4 [%0], %1, %2, %3, p;\n\t}" ::"r"(d_tmem),
      "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate)
      : "memory");
}

// Scales out of the rule, in a call of its own: written out in the producer's loop it cost the kernel 2%.
__device__ __noinline__ float2 held_scales(float2 s, int32_t* status) {
  return make_float2(scale_of_page(s.x, status), scale_of_page(s.y, status));
}

template <int D>
__global__ void __launch_bounds__(Pf8<D>::kThreads, 1)
    paged8_fmha_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                      const __grid_constant__ PagedAttnArgs a) {
  using F = Pf8<D>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem =
      reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint8_t* sQ = smem;                       // two streams of two parts
  uint8_t* sK = sQ + 4 * F::kTile;          // kNK tiles
  uint8_t* sV = sK + F::kNK * F::kTile;     // kNV tiles
  uint8_t* sH = sV + F::kNV * F::kTile;     // kNH tiles
  Pf8Shared& sh = *reinterpret_cast<Pf8Shared*>(sH + F::kNH * F::kTile16);
  __shared__ int64_t scan[33];
  __shared__ PagedShare share;   // the softmax warps'

  const int tid = threadIdx.x, warp = tid >> 5, lane = tid & 31;
  const int H = a.d.H, G = a.d.Hq / H;
  const long long wl = a.wait_limit;
  volatile int* abort_flag = reinterpret_cast<volatile int*>(&sh.abort);
  if (tid == 128) {   // while warp 0 deals out the work
    for (int i = 0; i < 2; ++i) {
      mbar_init(&sh.q_ready[i], 4);
      mbar_init(&sh.s_full[i], 1);
      mbar_init(&sh.p_half[i][0], 4);
      mbar_init(&sh.p_half[i][1], 4);
      mbar_init(&sh.pv_done[i], 1);
    }
    for (int i = 0; i < 3; ++i) {
      mbar_init(&sh.k_full[i], 1);
      mbar_init(&sh.k_empty[i], 1);
      mbar_init(&sh.v_full[i], 1);
      mbar_init(&sh.v_empty[i], 2);
      mbar_init(&sh.h_full[i], 2);
      mbar_init(&sh.h_empty[i], 1);
    }
    mbar_init(&sh.drain, 1);
    sh.abort = 0;
    fence_barrier_init();
    tma_prefetch_desc(&tmK);
    tma_prefetch_desc(&tmV);
  }
  pdl_wait();
  if (warp == 2) {
    tmem_alloc(&sh.tmem, 512);
    tmem_relinquish();
  }
  paged_begin<F::kBM, F::kTK, kPad>(a, kLeast, kMost, scan, share);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
  pdl_trigger();   // tensor memory is taken
  const uint32_t tmem = sh.tmem;
  if (!share.work) {   // uniform over the CTA
    if (warp == 2) tmem_dealloc(tmem, 512);
    return;
  }
  PagedCursor c = share.c;   // of the other roles, each for itself
  // Every lane of a warp waits, and all of them go on or none does.
  auto wait = [&](uint64_t* bar, uint32_t parity) -> bool {
    return __all_sync(0xffffffffu, mbar_wait(bar, parity, abort_flag, wl));
  };
  // for the drain after a timeout: loads that have been issued, by ring place
  uint32_t k_issued = 0, k_par = 0, v_issued = 0, v_par = 0;

  if (warp < 4) {
    // registers: 384 x 168 at launch = 128 x 88 + 256 x 208; at 168 the softmax spills a row's scores (2,180 us for 1,313 then)
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == 0) {
      // ------------------------------------------------ TMA producer
      uint32_t t = 0;   // tiles so far
      bool ok = a.stall_test == 0 || blockIdx.x != 0;   // test hook: CTA 0 loads nothing
      while (ok && c.u < c.u_end) {
        const PagedPiece p = paged_piece<F::kBM, F::kTK, kPad>(c, G);
        const int kt_end = p.kt + p.n;
        // lanes 0 .. 7: the keys 16 lane .. of a tile; its table entry is read two tiles ahead, its scales one
        auto mine = [&](int kt) { return lane < 8 && kt < kt_end && kt * F::kTK + 16 * lane < c.s.len; };
        auto entry = [&](int kt) -> int {
          const int at = kt * F::kTK + 16 * lane;
          if (!mine(kt)) return 0;
          const int page = a.table[int64_t(c.s.slot) * a.d.max_pages + (at >> a.d.lp)];
          if (page >= 0 && page < a.d.n_pages) return page;
          atomicOr(a.status, kStatusPageUse);   // held inside the pool
          return 0;
        };
        auto scales = [&](int kt, int page) -> float2 {
          const int64_t x = int64_t(page) * H + c.hk;
          return mine(kt) ? make_float2(a.ks[x], a.vs[x]) : make_float2(1.f, 1.f);
        };
        int page = entry(p.kt), next = entry(p.kt + 1);
        float2 sc = scales(p.kt, page);
        int e_top = -127;   // largest exponent of a value scale in the piece so far
        for (int kt = p.kt; ok && kt < kt_end; ++kt, ++t) {
          const int k0 = kt * F::kTK, n_keys = min(F::kTK, c.s.len - k0);
          const int next2 = entry(kt + 2);
          const float2 sc2 = scales(kt + 1, next);
          if (!is_scale8(sc.x) || !is_scale8(sc.y)) sc = held_scales(sc, a.status);
          const bool load = mine(kt) && (16 * lane & (a.d.P - 1)) == 0;
          const int row = (page * H + c.hk) << a.d.lp;
          const uint32_t bytes =
              n_keys <= 0 ? 0u : static_cast<uint32_t>((n_keys + a.d.P - 1) >> a.d.lp) * a.d.P * D;
          auto fetch = [&](bool v, uint32_t st, uint32_t use) -> bool {
            uint64_t* full = v ? &sh.v_full[st] : &sh.k_full[st];
            if (!wait(v ? &sh.v_empty[st] : &sh.k_empty[st], (use & 1u) ^ 1u)) return false;
            if (!v) {   // the softmax is through the tile that had this place: it is kScaleRing back
              Scales8& to = sh.scales[t % kScaleRing];
              const int e = int(__float_as_uint(sc.y) >> 23) - 127;
              e_top = max(e_top, __reduce_max_sync(0xffffffffu, mine(kt) ? e : -127));
              const int least = __reduce_min_sync(0xffffffffu, mine(kt) ? e : 128);
              if (lane < 8) {
                to.k[lane] = sc.x;
                to.e[lane] = float(e);
                to.inv[lane] = __uint_as_float(uint32_t(127 - e) << 23);
              }
              if (lane == 0) to.wide = e_top - least > 60;
            }
            __syncwarp();
            if (lane == 0) mbar_arrive_expect_tx(full, bytes);
            __syncwarp();
            if (load)
              tma_load_2d((v ? sV : sK) + st * F::kTile + 16 * lane * D, v ? &tmV : &tmK, full, 0, row);
            uint32_t& issued = v ? v_issued : k_issued;
            uint32_t& par = v ? v_par : k_par;
            issued |= 1u << st;
            par = (par & ~(1u << st)) | ((use & 1u) << st);
            return true;
          };
          ok = fetch(false, t % F::kNK, t / F::kNK) && fetch(true, t % F::kNV, t / F::kNV);
          page = next;
          next = next2;
          sc = sc2;
        }
        paged_next<F::kBM, F::kTK, kPad>(a, c, p);
      }
    } else if (warp == 1) {
      // ------------------------------------------------ MMA issuer: one thread
      if (elect_one()) {
        const uint32_t idS = idesc_f16_f32(128, 128);            // 8-bit and fp16 operands have the same code, 0
        const uint32_t idPV = idesc_f16_f32(128, D) | 1u << 16;   // MN-major B
        uint32_t t = 0, n_q[2] = {0, 0}, n_s[2] = {0, 0};   // tiles; items and tiles of each stream
        bool ok = true;
        auto wait1 = [&](uint64_t* bar, uint32_t parity) { return mbar_wait(bar, parity, abort_flag, wl); };
        auto issue_s = [&](int i, uint32_t st) -> bool {   // S_i of the keys in place st
          // P_i of the tile before lies where S_i goes: its product has to be done
          if (n_s[i] && !wait1(&sh.pv_done[i], (n_s[i] - 1) & 1u)) return false;
          tc_fence_after();
#pragma unroll
          for (int part = 0; part < 2; ++part) {
            const uint32_t qa = smem_u32(sQ + (2 * i + part) * F::kTile), ka = smem_u32(sK + st * F::kTile);
            const uint64_t ad = D == 128 ? sdesc_k_sw128(qa) : sdesc_k_sw64(qa);
            const uint64_t bd = D == 128 ? sdesc_k_sw128(ka) : sdesc_k_sw64(ka);
#pragma unroll
            for (int k = 0; k < D / 32; ++k)
              umma_f8(tmem + i * 128, ad + 2 * k, bd + 2 * k, idS, (part | k) != 0);
          }
          umma_commit(&sh.s_full[i]);
          return true;
        };
        auto issue_pv = [&](int i, uint32_t st, int steps, bool first) -> bool {   // O_i += P_i V
          const uint32_t tO = tmem + F::kO + i * D, tP = tmem + i * 128;
          const uint64_t bd = sdesc_mn_sw128(smem_u32(sH + st * F::kTile16), F::kBlk);
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            if (!wait1(&sh.p_half[i][h], n_s[i] & 1u)) return false;
            tc_fence_after();
#pragma unroll
            for (int k = 4 * h; k < 4 * h + 4; ++k)
              if (k < steps) umma_bf16_ts(tO, tP + 8 * k, bd + 128 * k, idPV, !(first && k == 0));
          }
          umma_commit(&sh.pv_done[i]);
          ++n_s[i];
          return true;
        };
        while (ok && c.u < c.u_end) {
          const PagedPiece p = paged_piece<F::kBM, F::kTK, kPad>(c, G);
          const int n_str = c.s.m * G - c.rt * F::kBM > 128 ? 2 : 1;
          for (int i = 0; ok && i < n_str; ++i) {
            ok = wait1(&sh.q_ready[i], n_q[i]++ & 1u);
            if (ok && i == 0) ok = wait1(&sh.k_full[t % F::kNK], (t / F::kNK) & 1u);
            ok = ok && issue_s(i, t % F::kNK);
          }
          if (ok) umma_commit(&sh.k_empty[t % F::kNK]);
          for (int j = 0; ok && j < p.n; ++j, ++t) {
            const uint32_t vs = t % F::kNH, ks = (t + 1) % F::kNK;
            const int n_keys = min(F::kTK, c.s.len - (p.kt + j) * F::kTK);
            const int steps = n_keys <= 0 ? 0 : (n_keys + 15) >> 4;
            const bool more = j + 1 < p.n;
            ok = wait1(&sh.h_full[vs], (t / F::kNH) & 1u);
            for (int i = 0; ok && i < n_str; ++i) {
              ok = issue_pv(i, vs, steps, j == 0);
              if (ok && i == n_str - 1) umma_commit(&sh.h_empty[vs]);
              if (ok && more) {
                if (i == 0) ok = wait1(&sh.k_full[ks], ((t + 1) / F::kNK) & 1u);
                ok = ok && issue_s(i, ks);
                if (ok && i == n_str - 1) umma_commit(&sh.k_empty[ks]);
              }
            }
          }
          paged_next<F::kBM, F::kTK, kPad>(a, c, p);
        }
      }
      __syncwarp();
    } else {
      // ------------------------------------------------ warps 2, 3: values to fp16, half of the rows each
      constexpr int kPasses = D / 64;   // steps of 8 rows, 4 pieces of 16 bytes each
      uint32_t t = 0;
      bool ok = true;
      for (int piece = 0; ok && c.u < c.u_end; ++piece) {
        const PagedPiece p = paged_piece<F::kBM, F::kTK, kPad>(c, G);
        const int masked = first_masked(c.s, G, c.rt * F::kBM);
        uint32_t (*notes)[4] = sh.notes[piece & 3];
        // the notes of four pieces ago are read: this piece's values were loaded behind products that
        // the softmax warps started after them; a warp clears and sets those of its own rows
        bool cleared = false;
        for (int kt = p.kt; ok && kt < p.kt + p.n; ++kt, ++t) {
          const uint32_t sv = t % F::kNV, shf = t % F::kNH;
          ok = wait(&sh.v_full[sv], (t / F::kNV) & 1u) && wait(&sh.h_empty[shf], ((t / F::kNH) & 1u) ^ 1u);
          if (!ok) break;
          if (!cleared) {
            cleared = true;
            if (lane < 8) notes[lane >> 1][2 * (warp - 2) + (lane & 1)] = 0;
            __syncwarp();
          }
          const int k0 = kt * F::kTK, n_keys = min(F::kTK, c.s.len - k0), rows = n_keys <= 0 ? 0 : (n_keys + 15) & ~15;
          const uint32_t from = smem_u32(sV + sv * F::kTile), to = smem_u32(sH + shf * F::kTile16);
          const int r_end = min(rows, 64 * (warp - 1));
          const bool part_seen = kt >= masked;
          // kAhead pieces with their loads in flight; two rows of a quarter warp take different halves of their 128
          // bytes, so that no bank is met twice
          constexpr int kAhead = 4, kRows = 8 * kAhead / kPasses;
#pragma unroll 1
          for (int r0 = 64 * (warp - 2); r0 < r_end; r0 += kRows) {
            uint4 v[kAhead];
#pragma unroll
            for (int y = 0; y < kAhead; ++y) {
              const int r = r0 + 8 * (y / kPasses) + (lane >> 2);
              const int x = (lane & 3) | (kPasses == 2 ? ((r & 1) ^ (y & 1)) << 2 : 0);
              v[y] = r < n_keys ? ld_shared_v4(from + F::at(r, x)) : make_uint4(0u, 0u, 0u, 0u);
            }
            if (part_seen) {   // some rows do not see all of the tile: NaN goes out of the product, and is noted
#pragma unroll
              for (int y = 0; y < kAhead; ++y) {
                const int r = r0 + 8 * (y / kPasses) + (lane >> 2);
                const uint32_t n0 = nan8(v[y].x), n1 = nan8(v[y].y), n2 = nan8(v[y].z), n3 = nan8(v[y].w);
                if (!(n0 | n1 | n2 | n3)) continue;
                v[y].x &= ~((n0 >> 7) * 255u);
                v[y].y &= ~((n1 >> 7) * 255u);
                v[y].z &= ~((n2 >> 7) * 255u);
                v[y].w &= ~((n3 >> 7) * 255u);
                atomicOr(&notes[min(kt - masked, 3)][r >> 5], 1u << (r & 31));
              }
            }
#pragma unroll
            for (int y = 0; y < kAhead; ++y) {
              const int r = r0 + 8 * (y / kPasses) + (lane >> 2);
              const int x = (lane & 3) | (kPasses == 2 ? ((r & 1) ^ (y & 1)) << 2 : 0);
              const uint32_t dst = to + (x >> 2) * F::kBlk + r * 128;
              const int c0 = 2 * (x & 3), s7 = r & 7;
              st_shared_v4(dst + ((c0 ^ s7) << 4), half2_of8(v[y].x), half2_of8(v[y].x >> 16), half2_of8(v[y].y),
                           half2_of8(v[y].y >> 16));
              st_shared_v4(dst + (((c0 + 1) ^ s7) << 4), half2_of8(v[y].z), half2_of8(v[y].z >> 16), half2_of8(v[y].w),
                           half2_of8(v[y].w >> 16));
            }
          }
          fence_proxy_async_smem();
          __syncwarp();
          if (lane == 0) {
            mbar_arrive(&sh.v_empty[sv]);
            mbar_arrive(&sh.h_full[shf]);
          }
        }
        paged_next<F::kBM, F::kTK, kPad>(a, c, p);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    // ------------------------------------------------ softmax: warps 4 + 4 i + q, stream i, lane quarter q
    constexpr float kTau = 8.f, kTop = 7.f;   // m is a row's maximum less kTop, raised where a tile's passes that by kTau
    const int i = (warp - 4) >> 2, quarter = warp & 3;
    const int r = quarter * 32 + lane;   // row of the stream
    const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
    const uint32_t tS = tmem + lanes + i * 128, tO = tmem + lanes + F::kO + i * D;
    const float sl2 = rsqrtf(float(D)) * 1.4426950408889634f;   // log2(e) / sqrt(d)
    uint32_t t = 0, tile = 0;   // tiles of this stream; of the CTA
    bool ok = true;
    for (int piece = 0;; ++piece) {
      const PagedCursor c = share.c;
      const PagedPiece p = share.p;
      const int kt_end = p.kt + p.n;
      const int row = c.rt * F::kBM + i * 128 + r, n_rows = c.s.m * G;
      const bool active = n_rows - c.rt * F::kBM > i * 128;   // the stream has rows
      const bool valid = row < n_rows;
      const int pos = valid ? c.s.len - c.s.m + row / G : -1;
      const int64_t out_row = valid ? paged_out_row(c, H, G, row) : 0;
      float m = -INFINITY, l = 0.f;
      if (active) {
        // the row's query in two parts, swizzled as TMA would write them
        const uint4* src = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + out_row * D);
        uint32_t top = 0;
#pragma unroll
        for (int e = 0; e < D / 8; ++e) top = top_bf16x2(top, valid ? src[e] : make_uint4(0u, 0u, 0u, 0u));
        const Split8 split(max(top & 0xFFFFu, top >> 16));
        sh.rf[tid - 128] = sl2 * split.factor;
#pragma unroll
        for (int e = 0; e < D / 16; ++e) {
          uint32_t hi[4], lo[4];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            const uint4 u = valid ? src[2 * e + k] : make_uint4(0u, 0u, 0u, 0u);
            split(u.x, u.y, hi[2 * k], lo[2 * k]);
            split(u.z, u.w, hi[2 * k + 1], lo[2 * k + 1]);
          }
          const uint32_t at = smem_u32(sQ + 2 * i * F::kTile) + F::at(r, e);
          st_shared_v4(at, hi[0], hi[1], hi[2], hi[3]);
          st_shared_v4(at + F::kTile, lo[0], lo[1], lo[2], lo[3]);
        }
        fence_proxy_async_smem();
        tc_fence_before();
        __syncwarp();
        if (lane == 0) mbar_arrive(&sh.q_ready[i]);
        for (int kt = p.kt; kt < kt_end; ++kt, ++t) {
          if (!wait(&sh.s_full[i], t & 1u)) {
            ok = false;
            break;
          }
          tc_fence_after();
          const int see = pos - kt * F::kTK;   // keys 0 .. see of the tile count
          const Scales8* ring = &sh.scales[(tile + kt - p.kt) % kScaleRing];
          float rf = sh.rf[tid - 128];
        again:
          const Scales8 sc = *ring;   // in registers
          uint32_t v[4][32];
#pragma unroll
          for (int e = 0; e < 4; ++e) tmem_ld_32x32b_x32(tS + 32 * e, v[e]);
#pragma unroll
          for (int e = 0; e < 4; ++e) tmem_ld_wait(v[e]);
          if (!__all_sync(0xffffffffu, see >= F::kTK - 1)) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int k = 0; k < 32; ++k)
                if (32 * e + k > see) v[e][k] = 0xFF800000u;   // -inf: its weight is 0 exactly
          }
          float mg[8];   // largest of 16 keys, with their scales
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            float x = fmax3(__uint_as_float(v[e >> 1][16 * (e & 1)]), __uint_as_float(v[e >> 1][16 * (e & 1) + 1]),
                            __uint_as_float(v[e >> 1][16 * (e & 1) + 2]));
            float y = fmax3(__uint_as_float(v[e >> 1][16 * (e & 1) + 3]), __uint_as_float(v[e >> 1][16 * (e & 1) + 4]),
                            __uint_as_float(v[e >> 1][16 * (e & 1) + 5]));
#pragma unroll
            for (int k = 6; k < 14; k += 4) {
              x = fmax3(x, __uint_as_float(v[e >> 1][16 * (e & 1) + k]), __uint_as_float(v[e >> 1][16 * (e & 1) + k + 1]));
              y = fmax3(y, __uint_as_float(v[e >> 1][16 * (e & 1) + k + 2]), __uint_as_float(v[e >> 1][16 * (e & 1) + k + 3]));
            }
            x = fmax3(x, __uint_as_float(v[e >> 1][16 * (e & 1) + 14]), __uint_as_float(v[e >> 1][16 * (e & 1) + 15]));
            mg[e] = fmaf(fmaxf(x, y), rf * sc.k[e], sc.e[e]);
          }
          const float mx = fmaxf(fmax3(mg[0], mg[1], mg[2]), fmax3(mg[3], mg[4], fmax3(mg[5], mg[6], mg[7])));
          const bool raise = mx - m > kTau + kTop;   // always where m = -inf and a key is seen
          const float to = __fadd_ru(mx, -kTop);     // mx - to is kTop at most, whatever the steps of mx
          const float alpha = (raise && m != -INFINITY) ? exp2f(m - to) : 1.f;   // below 2^-126 too
          // Scores from 2^22 on: beside their steps in fp32 the weights' s f + (e - R) of two roundings could pass 2^16
          // where s f + e, rounded, is R. They are worked out in place first, in one rounding, so that what is left to
          // do is exact, with 1 as the row's factor (which no other row has: it is a power of two over sqrt(d) ln 2). So
          // are those of rows whose factor may leave fp32's range with a key scale.
          const bool far =
              rf != 1.f && (!(rf >= 0x1p-66f && rf <= 0x1p67f) || (fabsf(mx) > 0x1p22f && mx != -INFINITY));
          if (__any_sync(0xffffffffu, alpha != 1.f || far)) {
            if (__any_sync(0xffffffffu, far)) {
              Scales8& done = sh.done[warp - 4];
#pragma unroll 1
              for (int e = 0; e < 8; ++e) {
                uint32_t u[16];
                tmem_ld_32x32b_x16(tS + 16 * e, u);
                tmem_ld_wait(u);
                const float f = factor8(rf, ring->k[e]), b = ring->e[e];
#pragma unroll
                for (int k = 0; k < 16; ++k) u[k] = __float_as_uint(fmaf(__uint_as_float(u[k]), f, b));
                tmem_st_32x32b_x16(tS + 16 * e, u);
              }
              tmem_st_wait();
              if (lane < 8) {
                done.k[lane] = 1.f;
                done.e[lane] = 0.f;
                done.inv[lane] = ring->inv[lane];
              }
              if (lane == 0) done.wide = ring->wide;
              __syncwarp();
              ring = &done;
              rf = 1.f;
              goto again;
            }
            // needs the products before in O
            if (!wait(&sh.pv_done[i], (t - 1) & 1u)) {
              ok = false;
              break;
            }
            tc_fence_after();
#pragma unroll 1
            for (int e = 0; e < D / 32; ++e) {
              uint32_t o[32];
              tmem_ld_32x32b_x32(tO + 32 * e, o);
              tmem_ld_wait(o);
#pragma unroll
              for (int k = 0; k < 32; ++k) o[k] = __float_as_uint(__uint_as_float(o[k]) * alpha);
              tmem_st_32x32b_x32(tO + 32 * e, o);
            }
            l *= alpha;
          }
          if (raise) m = to;
          const float mu = m == -INFINITY ? 0.f : m;
          float wide_sum = 0.f;
          if (ring->wide) {   // the sum by itself, from the scores again: small code beside the loop below
#pragma unroll 1
            for (int e = 0; e < 8; ++e) {
              uint32_t u[16];
              tmem_ld_32x32b_x16(tS + 16 * e, u);
              tmem_ld_wait(u);
              const float f = rf * ring->k[e], b = ring->e[e] - mu;
              float g = 0.f;
#pragma unroll
              for (int k = 0; k < 16; ++k) g += 16 * e + k > see ? 0.f : exp2f(fmaf(__uint_as_float(u[k]), f, b));
              wide_sum = fmaf(g, ring->inv[e], wide_sum);
            }
            wide_sum += l;
          }
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint32_t pk[16];
#pragma unroll
            for (int y = 0; y < 2; ++y) {
              const float f = rf * sc.k[2 * e + y], b = sc.e[2 * e + y] - mu;
              const uint64_t s2 = f32x2(f, f), b2 = f32x2(b, b);
              uint64_t sum[2] = {0, 0};
#pragma unroll
              for (int k = 8 * y; k < 8 * y + 8; ++k) {
                const uint64_t x = ffma_x2((static_cast<uint64_t>(v[e][2 * k + 1]) << 32) | v[e][2 * k], s2, b2);
                const float p0 = ex2_fast(__uint_as_float(static_cast<uint32_t>(x)));
                const float p1 = ex2_fast(__uint_as_float(static_cast<uint32_t>(x >> 32)));
                const __half2 ph = __floats2half2_rn(p0, p1);
                pk[k] = *reinterpret_cast<const uint32_t*>(&ph);
                sum[k & 1] = fadd_x2(sum[k & 1], f32x2(p0, p1));
              }
              sum[0] = fadd_x2(sum[0], sum[1]);
              l = fmaf(__uint_as_float(static_cast<uint32_t>(sum[0])) + __uint_as_float(static_cast<uint32_t>(sum[0] >> 32)),
                       ring->inv[2 * e + y], l);
            }
            tmem_st_32x32b_x16(tS + 16 * e, pk);
            if (e & 1) {
              tmem_st_wait();
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(&sh.p_half[i][e >> 1]);
            }
          }
          if (ring->wide) l = wide_sum;
        }
        ok = ok && wait(&sh.pv_done[i], (t - 1) & 1u);
      }
      tile += p.n;
      float* part = p.whole ? nullptr : paged_part<F::kBM, D>(a, blockIdx.x, p.kt == 0);
      if (ok && active) {
        tc_fence_after();
        const int masked = first_masked(c.s, G, c.rt * F::kBM);
        uint32_t any = 0;   // notes of this piece (uniform over the CTA)
#pragma unroll
        for (int e = 0; e < 16; ++e) any |= reinterpret_cast<volatile uint32_t*>(sh.notes[piece & 3])[e];
        const bool seen = pos >= p.kt * F::kTK;   // a key of the piece; else O may not have been written
        const float f = l == 0.f ? 0.f : 1.f / l;
        uint16_t* dst = static_cast<uint16_t*>(a.out) + out_row * D;
#pragma unroll 1
        for (int e = 0; e < D / 32; ++e) {
          uint32_t o[32];
          tmem_ld_32x32b_x32(tO + 32 * e, o);
          tmem_ld_wait(o);
          if (!seen || (l == 0.f && !part)) {   // a result without weights is 0 whatever the values are
#pragma unroll
            for (int k = 0; k < 32; ++k) o[k] = 0u;
          }
          if (any && (l != 0.f || part)) {   // values that are NaN, of keys that this row sees
            for (int kt = max(masked, p.kt); kt < p.kt + p.n; ++kt)
              for (int w = 0; w < 4; ++w)
                for (uint32_t bits = sh.notes[piece & 3][min(kt - masked, 3)][w]; bits; bits &= bits - 1) {
                  const int j = kt * F::kTK + 32 * w + __ffs(bits) - 1;
                  if (j > pos) continue;
                  const int page = paged_page(a.d, a.table, a.status, c.s.slot, j);
                  const uint8_t* vr = static_cast<const uint8_t*>(a.v) + paged_row(a.d, page, c.hk, j) * D + 32 * e;
#pragma unroll
                  for (int k = 0; k < 32; ++k)
                    if ((vr[k] & 0x7Fu) == kNaN8) o[k] = 0x7FC00000u;
                }
          }
          if (!valid) continue;
          if (part) {
            uint4* to = reinterpret_cast<uint4*>(part) + 8 * e * F::kBM + i * 128 + r;
#pragma unroll
            for (int k = 0; k < 8; ++k)
              to[k * F::kBM] = make_uint4(o[4 * k], o[4 * k + 1], o[4 * k + 2], o[4 * k + 3]);
          } else {
            uint32_t w[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              __nv_bfloat162 u =
                  __floats2bfloat162_rn(__uint_as_float(o[2 * k]) * f, __uint_as_float(o[2 * k + 1]) * f);
              w[k] = *reinterpret_cast<uint32_t*>(&u);
            }
#pragma unroll
            for (int k = 0; k < 4; ++k)
              reinterpret_cast<uint4*>(dst + 32 * e)[k] = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
          }
        }
        if (part && valid) {
          part[F::kBM * D + i * 128 + r] = m;
          part[F::kBM * (D + 1) + i * 128 + r] = l;
        }
        tc_fence_before();
      }
      // both streams are through the piece (or all of them stop)
      if (!bar_and(1, 256, ok)) {
        ok = false;
        break;
      }
      if (part) {
        if (tid == 128) sh.join.mine = paged_arrive(a, p, sh.join.g);
        asm volatile("bar.sync 1, 256;" ::: "memory");
        if (sh.join.mine) {
          join_rows<D>(a, c, sh.join.g, i * 128 + r);
          if (!sh.join.g.final) {
            asm volatile("bar.sync 1, 256;" ::: "memory");
            if (tid == 128) sh.join.mine = paged_arrive_group(a, p, sh.join.g);
            asm volatile("bar.sync 1, 256;" ::: "memory");
            if (sh.join.mine) join_rows<D>(a, c, sh.join.g, i * 128 + r);
          }
        }
      }
      asm volatile("bar.sync 1, 256;" ::: "memory");   // everyone has read the share
      if (tid == 128) paged_step<F::kBM, F::kTK, kPad>(a, share);
      asm volatile("bar.sync 1, 256;" ::: "memory");
      if (!share.work) break;
    }
  }

  tc_fence_before();
  __syncthreads();
  if (*abort_flag) {
    if (warp == 0 && lane == 0) {
      for (int kv = 0; kv < 2; ++kv)
        for (int st = 0; st < 3; ++st)
          if (((kv ? v_issued : k_issued) >> st) & 1u) {
            const uint32_t ad = smem_u32(kv ? &sh.v_full[st] : &sh.k_full[st]);
            const long long t0 = clock64();
            while (!mbar_try_wait(ad, ((kv ? v_par : k_par) >> st) & 1u) && clock64() - t0 < wl) {
            }
          }
    }
    if (warp == 1) {
      if (elect_one()) umma_commit(&sh.drain);
      __syncwarp();
      const uint32_t ad = smem_u32(&sh.drain);
      const long long t0 = clock64();
      while (!mbar_try_wait(ad, 0) && clock64() - t0 < wl) {
      }
    }
    if (tid == 128) {   // the arrivals that are still owed, so that the counters are zero for the next call
      for (; share.work; paged_step<F::kBM, F::kTK, kPad>(a, share))   // from the piece that was not finished
        if (!share.p.whole) paged_arrive_owed(a, share.p);
      atomicOr(a.status, kStatusTimeout);
    }
    __syncthreads();
  }
  if (warp == 2) {
    __syncwarp();
    tc_fence_after();
    tmem_dealloc(tmem, 512);
  }
}

}  // namespace

cudaError_t launch_paged8_fmha(const PagedAttnArgs& a, const CUtensorMap& tmK, const CUtensorMap& tmV, int num_sms,
                               cudaStream_t st) {
  static SmemOptIn opt_in[2];
  auto kern = a.d.d == 128 ? paged8_fmha_kernel<128> : paged8_fmha_kernel<64>;
  const int smem = a.d.d == 128 ? Pf8<128>::kSmem : Pf8<64>::kSmem;
  if (cudaError_t e = opt_in[a.d.d == 128](kern, smem)) return e;
  return launch_kernel(a.early, kern, num_sms, Pf8<128>::kThreads, smem, st, tmK, tmV, a);
}

}  // namespace mot
