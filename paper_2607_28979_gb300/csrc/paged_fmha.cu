// Attention of chunks of new tokens over a paged cache on the tensor cores of sm_103a (bf16).
//
//   paged_fmha_kernel   persistent, one CTA per SM over its run of key tiles (paged_common.cuh). An
//                       item is 256 rows (new token, query head of the group) of one key/value head, as
//                       two streams of 128 rows whose softmax and products alternate, over tiles of
//                       128 keys:
//                         warp 0     TMA: a tile's pages, keys and values as they lie in the pool, a
//                                    lane per (page, 64 dimensions), into rings of 2 and 3 tiles;
//                         warp 1     S_i = Q_i K^T (Q_i and K from shared memory) and O_i += P_i V (P_i
//                                    from TMEM, over S_i; V's rows are keys, so it is an MN-major
//                                    operand and needs no transpose), i = 0, 1 in turn, by one thread
//                                    without an election at each step;
//                         warp 2     values before the second product: rows behind the sequence's
//                                    end become zeros, and in tiles that some rows see only in part
//                                    infinite and NaN values do too (a masked key's weight is 0, and 0
//                                    times them would not be); their keys are noted, and the rows
//                                    that do see them add them at the end;
//                         warps 4-11 one thread per row: queries into shared memory, scores from TMEM,
//                                    running maximum (base 2; raised, and O and the sum rescaled, only
//                                    when a tile exceeds it by 2^8) and sum, P as bf16 pairs into TMEM
//                                    in two halves, so that the second product starts on the first
//                                    while the other is made (a second part of each weight, as the
//                                    few-row kernel has it, would double the second product); the sum
//                                    is of the rounded weights, 2% of the time more than of the
//                                    unrounded ones, else one heavy weight's rounding (2^-8) stays in
//                                    the result; at the end O from TMEM to the output or
//                                    to the piece's partial results.
//                       What bounds it: S_i cannot be made again before P_i V is done (P_i lies over it),
//                       so a stream is a chain of two products, the softmax and the commits and wake-ups
//                       between them; two streams in turn keep the tensor cores 54% busy (4,096 tokens of
//                       28 heads on 4 on 32,768 positions: 1,191 to 1,218 us, 1,500 TFLOP/s). Slower there:
//                       two buffers of 64 keys per stream instead of one of 128 (1,385 us: twice the
//                       steps), P as a whole (1,223); P in three quarters and one, or one and three, the
//                       same. The waits poll without a sleep.
//                       Every wait is bounded; on a timeout the roles unwind, copies and MMAs in flight
//                       are drained, TMEM is freed and kStatusTimeout is raised.
#include "paged_chunk.cuh"

namespace mot {
namespace {

// Units of a share. A piece's start, end and join cost about as much as eight tiles, and a run often has two of
// them. Pieces against runs (kMost = 0), us in a graph: 256 new tokens of 12 heads of 128 on 2, on 4,096 and
// 16,384 positions, 41 for 59 and 55 for 67; 1,024 from nothing, 12 heads of 64, 22 for 29. Longer pieces leave
// CTAs without work: with 32, 200 tokens of each of six on 3,584 positions take 56 for 42 (with 16, on 2,048, 39
// for 33: the price of 39 for 51 where 30 chunks of 40 have 60 items). kLeast = 4 gains where an item has few
// tiles (64 tokens on 2,000 positions, 29 for 35) and loses where it has many rows (1,024 from nothing, 23 for 22).
constexpr int kLeast = 1, kMost = 16;

template <int D>
struct Pf {
  static constexpr int kBM = kChunkRows, kTK = 128;
  static constexpr int kBlk = 128 * 128;               // 128 rows of 64 elements
  static constexpr int kTile = D / 64 * kBlk;          // a tile of keys, of values or of queries
  static constexpr int kNK = 2, kNV = 3;               // tiles in flight
  static constexpr int kThreads = 32 * 12;
  static constexpr int kBytes = (2 + kNK + kNV) * kTile;
  static constexpr int kSmem = kBytes + 1024 + 1024;   // barriers and notes; alignment
  static constexpr int kO = 256;                       // TMEM: S at 0 and 128, O at 256 and 256 + D
};
static_assert(Pf<128>::kSmem <= 232448, "shared memory budget");
static_assert(Pf<128>::kO + 2 * 128 <= 512, "TMEM columns");

// Barriers and what the roles leave for one another.
struct PfShared {
  uint64_t q_ready[2], s_full[2], p_half[2][2], pv_done[2];
  uint64_t k_full[2], k_empty[2], v_full[3], v_ready[3], v_empty[3], drain;
  uint32_t tmem;
  int32_t abort;
  PagedJoinShared join;
  uint32_t notes[4][4][4];   // [piece & 3][tile of the masked ones][128 keys]: values that are not finite
};
static_assert(sizeof(PfShared) <= 1024, "barrier block");

template <int D>
__global__ void __launch_bounds__(Pf<D>::kThreads, 1)
    paged_fmha_kernel(const __grid_constant__ CUtensorMap tmK, const __grid_constant__ CUtensorMap tmV,
                      const __grid_constant__ PagedAttnArgs a) {
  using F = Pf<D>;
  constexpr int kHalves = D / 64;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* smem =
      reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~static_cast<uintptr_t>(1023));
  uint8_t* sQ = smem;                       // two tiles
  uint8_t* sK = sQ + 2 * F::kTile;          // kNK tiles
  uint8_t* sV = sK + F::kNK * F::kTile;     // kNV tiles
  PfShared& sh = *reinterpret_cast<PfShared*>(sV + F::kNV * F::kTile);
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
      mbar_init(&sh.k_full[i], 1);
      mbar_init(&sh.k_empty[i], 1);
    }
    for (int i = 0; i < 3; ++i) {
      mbar_init(&sh.v_full[i], 1);
      mbar_init(&sh.v_ready[i], 1);
      mbar_init(&sh.v_empty[i], 1);
    }
    mbar_init(&sh.drain, 1);
    sh.abort = 0;
    fence_barrier_init();
    tma_prefetch_desc(&tmK);
    tma_prefetch_desc(&tmV);
  }
  if (warp == 2) {
    tmem_alloc(&sh.tmem, 512);
    tmem_relinquish();
  }
  paged_begin<F::kBM, F::kTK>(a, kLeast, kMost, scan, share);
  tc_fence_before();
  __syncthreads();
  tc_fence_after();
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
    // registers: 384 x 168 at launch = 128 x 88 + 256 x 208; at 168 the softmax spills (1,258 us for 1,205 for
    // 4,096 tokens on 32,768 positions)
    asm volatile("setmaxnreg.dec.sync.aligned.u32 88;");
    if (warp == 0) {
      // ------------------------------------------------ TMA producer
      uint32_t t = 0;   // tiles so far
      bool ok = a.stall_test == 0 || blockIdx.x != 0;   // test hook: CTA 0 loads nothing
      const int pages = F::kTK >> a.d.lp;                       // of a tile
      const int x = lane / kHalves, half = lane % kHalves;      // this lane's page and half
      while (ok && c.u < c.u_end) {
        const PagedPiece p = paged_piece<F::kBM, F::kTK>(c, G);
        // this lane's table entry of a tile, read a tile ahead
        auto entry = [&](int kt) -> int {
          const int at = kt * F::kTK + (x << a.d.lp);
          return lane < pages * kHalves && kt < p.kt + p.n && at < c.s.len
                     ? a.table[int64_t(c.s.slot) * a.d.max_pages + (at >> a.d.lp)]
                     : 0;
        };
        int next = entry(p.kt);
        for (int kt = p.kt; ok && kt < p.kt + p.n; ++kt, ++t) {
          const int k0 = kt * F::kTK, n_keys = min(F::kTK, c.s.len - k0);
          const bool mine = lane < pages * kHalves && k0 + (x << a.d.lp) < c.s.len;
          int page = next;
          next = entry(kt + 1);
          if (mine && (page < 0 || page >= a.d.n_pages)) {   // held inside the pool
            page = 0;
            atomicOr(a.status, kStatusPageUse);
          }
          const int row = (page * H + c.hk) << a.d.lp;
          const uint32_t bytes =
              n_keys <= 0 ? 0u : static_cast<uint32_t>((n_keys + a.d.P - 1) >> a.d.lp) * a.d.P * 128 * kHalves;
          auto fetch = [&](bool v, uint32_t st, uint32_t use) -> bool {
            uint64_t* full = v ? &sh.v_full[st] : &sh.k_full[st];
            if (!wait(v ? &sh.v_empty[st] : &sh.k_empty[st], (use & 1u) ^ 1u)) return false;
            if (lane == 0) mbar_arrive_expect_tx(full, bytes);
            __syncwarp();
            if (mine)
              tma_load_2d((v ? sV : sK) + st * F::kTile + half * F::kBlk + (x << a.d.lp) * 128, v ? &tmV : &tmK, full,
                          half * 64, row);
            uint32_t& issued = v ? v_issued : k_issued;
            uint32_t& par = v ? v_par : k_par;
            issued |= 1u << st;
            par = (par & ~(1u << st)) | ((use & 1u) << st);
            return true;
          };
          ok = fetch(false, t % F::kNK, t / F::kNK) && fetch(true, t % F::kNV, t / F::kNV);
        }
        paged_next<F::kBM, F::kTK>(a, c, p);
      }
    } else if (warp == 1) {
      // ------------------------------------------------ MMA issuer: one thread
      if (elect_one()) {
        const uint32_t idS = idesc_bf16_f32(128, 128), idPV = idesc_bf16_f32_bmn(128, D);
        uint32_t t = 0, n_q[2] = {0, 0}, n_s[2] = {0, 0};   // tiles; items and tiles of each stream
        bool ok = true;
        auto wait1 = [&](uint64_t* bar, uint32_t parity) { return mbar_wait(bar, parity, abort_flag, wl); };
        auto issue_s = [&](int i, uint32_t st) -> bool {   // S_i of the keys in place st
          // P_i of the tile before lies where S_i goes: its product has to be done
          if (n_s[i] && !wait1(&sh.pv_done[i], (n_s[i] - 1) & 1u)) return false;
          tc_fence_after();
#pragma unroll
          for (int kb = 0; kb < kHalves; ++kb) {
            const uint64_t ad = sdesc_k_sw128(smem_u32(sQ + i * F::kTile + kb * F::kBlk));
            const uint64_t bd = sdesc_k_sw128(smem_u32(sK + st * F::kTile + kb * F::kBlk));
#pragma unroll
            for (int k = 0; k < 4; ++k)
              umma_bf16(tmem + i * 128, ad + 2 * k, bd + 2 * k, idS, (kb | k) != 0);
          }
          umma_commit(&sh.s_full[i]);
          return true;
        };
        auto issue_pv = [&](int i, uint32_t st, int steps, bool first) -> bool {   // O_i += P_i V
          const uint32_t tO = tmem + F::kO + i * D, tP = tmem + i * 128;
          const uint64_t bd = sdesc_mn_sw128(smem_u32(sV + st * F::kTile), F::kBlk);
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
          const PagedPiece p = paged_piece<F::kBM, F::kTK>(c, G);
          const int n_str = c.s.m * G - c.rt * F::kBM > 128 ? 2 : 1;
          for (int i = 0; ok && i < n_str; ++i) {
            ok = wait1(&sh.q_ready[i], n_q[i]++ & 1u);
            if (ok && i == 0) ok = wait1(&sh.k_full[t % F::kNK], (t / F::kNK) & 1u);
            ok = ok && issue_s(i, t % F::kNK);
          }
          if (ok) umma_commit(&sh.k_empty[t % F::kNK]);
          for (int j = 0; ok && j < p.n; ++j, ++t) {
            const uint32_t vs = t % F::kNV, ks = (t + 1) % F::kNK;
            const int n_keys = min(F::kTK, c.s.len - (p.kt + j) * F::kTK);
            const int steps = n_keys <= 0 ? 0 : (n_keys + 15) >> 4;
            const bool more = j + 1 < p.n;
            ok = wait1(&sh.v_ready[vs], (t / F::kNV) & 1u);
            for (int i = 0; ok && i < n_str; ++i) {
              ok = issue_pv(i, vs, steps, j == 0);
              if (ok && i == n_str - 1) umma_commit(&sh.v_empty[vs]);
              if (ok && more) {
                if (i == 0) ok = wait1(&sh.k_full[ks], ((t + 1) / F::kNK) & 1u);
                ok = ok && issue_s(i, ks);
                if (ok && i == n_str - 1) umma_commit(&sh.k_empty[ks]);
              }
            }
          }
          paged_next<F::kBM, F::kTK>(a, c, p);
        }
      }
      __syncwarp();
    } else if (warp == 2) {
      // ------------------------------------------------ values before the second product
      uint32_t t = 0;
      bool ok = true;
      for (int piece = 0; ok && c.u < c.u_end; ++piece) {
        const PagedPiece p = paged_piece<F::kBM, F::kTK>(c, G);
        const int masked = first_masked(c.s, G, c.rt * F::kBM);
        uint32_t (*notes)[4] = sh.notes[piece & 3];
        // the notes of four pieces ago are read: this piece's values were loaded behind products that
        // the softmax warps started after them
        bool cleared = false;
        for (int kt = p.kt; ok && kt < p.kt + p.n; ++kt, ++t) {
          const uint32_t st = t % F::kNV;
          ok = wait(&sh.v_full[st], (t / F::kNV) & 1u);
          if (!ok) break;
          if (!cleared) {
            cleared = true;
            if (lane < 16) notes[lane >> 2][lane & 3] = 0;
            __syncwarp();
          }
          if (kt >= masked) {
            const int k0 = kt * F::kTK, n_keys = min(F::kTK, c.s.len - k0), rows = n_keys <= 0 ? 0 : (n_keys + 15) & ~15;
            uint8_t* tile = sV + st * F::kTile;
            // lane: 16 bytes of a row, 4 rows at a time
            const __nv_bfloat162 zero = __floats2bfloat162_rn(0.f, 0.f);
            for (int b = 0; b < kHalves; ++b)
#pragma unroll 4
              for (int r = lane >> 3; r < rows; r += 4) {
                const uint32_t at = smem_u32(tile + b * F::kBlk + r * 128 + (lane & 7) * 16);
                if (r >= n_keys) {
                  st_shared_v4(at, 0u, 0u, 0u, 0u);
                  continue;
                }
                uint4 v = ld_shared_v4(at);
                __nv_bfloat162 x = zero;   // NaN where a value is not finite: 0 times it
                x = __hfma2(*reinterpret_cast<__nv_bfloat162*>(&v.x), zero, x);
                x = __hfma2(*reinterpret_cast<__nv_bfloat162*>(&v.y), zero, x);
                x = __hfma2(*reinterpret_cast<__nv_bfloat162*>(&v.z), zero, x);
                x = __hfma2(*reinterpret_cast<__nv_bfloat162*>(&v.w), zero, x);
                const uint32_t bits = *reinterpret_cast<uint32_t*>(&x);
                if ((bits & 0x7FFF7FFFu) == 0) continue;
                uint32_t u[4] = {v.x, v.y, v.z, v.w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                  if ((u[e] & 0x7F80u) == 0x7F80u) u[e] &= 0xFFFF0000u;
                  if ((u[e] & 0x7F800000u) == 0x7F800000u) u[e] &= 0xFFFFu;
                }
                st_shared_v4(at, u[0], u[1], u[2], u[3]);
                atomicOr(&notes[min(kt - masked, 3)][r >> 5], 1u << (r & 31));
              }
            fence_proxy_async_smem();
          }
          __syncwarp();
          if (lane == 0) mbar_arrive(&sh.v_ready[st]);
        }
        paged_next<F::kBM, F::kTK>(a, c, p);
      }
    }
  } else {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 208;");
    // ------------------------------------------------ softmax: warps 4 + 4 i + q, stream i, lane quarter q
    constexpr float kTau = 8.f;
    const int i = (warp - 4) >> 2, quarter = warp & 3;
    const int r = quarter * 32 + lane;   // row of the stream
    const uint32_t lanes = static_cast<uint32_t>(quarter * 32) << 16;
    const uint32_t tS = tmem + lanes + i * 128, tO = tmem + lanes + F::kO + i * D;
    const float sl2 = rsqrtf(float(D)) * 1.4426950408889634f;   // log2(e) / sqrt(d)
    uint32_t t = 0;   // tiles of this stream
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
        // the row's query, swizzled as TMA would write it
        const uint4* src = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q) + out_row * D);
#pragma unroll
        for (int e = 0; e < D / 8; ++e) {
          const uint4 u = valid ? src[e] : make_uint4(0u, 0u, 0u, 0u);
          st_shared_v4(smem_u32(sQ + i * F::kTile + (e >> 3) * F::kBlk + r * 128 + (((e & 7) ^ (r & 7)) << 4)), u.x,
                       u.y, u.z, u.w);
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
          float by = sl2;   // what takes the scores in tensor memory to base-2 exponents
        again:
          uint32_t v[4][32];
#pragma unroll
          for (int e = 0; e < 4; ++e) tmem_ld_32x32b_x32(tS + 32 * e, v[e]);
#pragma unroll
          for (int e = 0; e < 4; ++e) tmem_ld_wait(v[e]);
          const int see = pos - kt * F::kTK;   // keys 0 .. see of the tile count
          if (!__all_sync(0xffffffffu, see >= F::kTK - 1)) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
#pragma unroll
              for (int k = 0; k < 32; ++k)
                if (32 * e + k > see) v[e][k] = 0xFF800000u;   // -inf: its weight is 0 exactly
          }
          float mk[8];
#pragma unroll
          for (int e = 0; e < 8; ++e) mk[e] = -INFINITY;
#pragma unroll
          for (int e = 0; e < 4; ++e)
#pragma unroll
            for (int k = 0; k < 16; ++k)
              mk[k & 7] = fmax3(mk[k & 7], __uint_as_float(v[e][2 * k]), __uint_as_float(v[e][2 * k + 1]));
          const float mx =
              fmaxf(fmax3(mk[0], mk[1], mk[2]), fmax3(mk[3], mk[4], fmax3(mk[5], mk[6], mk[7]))) * by;
          const bool raise = mx > m + kTau;   // always where m = -inf and a key is seen
          const float alpha = (raise && m != -INFINITY) ? ex2_fast(m - mx) : 1.f;
          // From 2^28 on s sl2 - R may be far from 0 where s sl2, rounded, is R, and the weight of a row's best key 0 or
          // infinite: such scores are worked out in place first, so that what is left to do is exact.
          const bool far = by != 1.f && fabsf(mx) > 0x1p28f && mx != -INFINITY;
          if (__any_sync(0xffffffffu, alpha != 1.f || far)) {
            if (__any_sync(0xffffffffu, far)) {
#pragma unroll 1
              for (int e = 0; e < 8; ++e) {
                uint32_t u[16];
                tmem_ld_32x32b_x16(tS + 16 * e, u);
                tmem_ld_wait(u);
#pragma unroll
                for (int k = 0; k < 16; ++k) u[k] = __float_as_uint(__uint_as_float(u[k]) * sl2);
                tmem_st_32x32b_x16(tS + 16 * e, u);
              }
              tmem_st_wait();
              by = 1.f;
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
          if (raise) m = mx;
          const float mu = m == -INFINITY ? 0.f : m;
          const uint64_t s2 = f32x2(by, by), nm2 = f32x2(-mu, -mu);
          // the sum of the weights as the product takes them: where one of them is most of it, its rounding cancels
          float sum[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            uint32_t pk[16];
#pragma unroll
            for (int k = 0; k < 16; ++k) {
              const uint64_t x = ffma_x2((static_cast<uint64_t>(v[e][2 * k + 1]) << 32) | v[e][2 * k], s2, nm2);
              const float p0 = ex2_fast(__uint_as_float(static_cast<uint32_t>(x)));
              const float p1 = ex2_fast(__uint_as_float(static_cast<uint32_t>(x >> 32)));
              __nv_bfloat162 pb = __floats2bfloat162_rn(p0, p1);
              pk[k] = *reinterpret_cast<uint32_t*>(&pb);
              add_bf16x2(sum[2 * (k & 1)], sum[2 * (k & 1) + 1], pk[k]);
            }
            tmem_st_32x32b_x16(tS + 16 * e, pk);
            if (e & 1) {
              tmem_st_wait();
              tc_fence_before();
              __syncwarp();
              if (lane == 0) mbar_arrive(&sh.p_half[i][e >> 1]);
            }
          }
          l += (sum[0] + sum[1]) + (sum[2] + sum[3]);
        }
        ok = ok && wait(&sh.pv_done[i], (t - 1) & 1u);
      }
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
          if (any && (l != 0.f || part)) {   // values that are not finite, of keys that this row sees
            for (int kt = max(masked, p.kt); kt < p.kt + p.n; ++kt)
              for (int w = 0; w < 4; ++w)
                for (uint32_t bits = sh.notes[piece & 3][min(kt - masked, 3)][w]; bits; bits &= bits - 1) {
                  const int j = kt * F::kTK + 32 * w + __ffs(bits) - 1;
                  if (j > pos) continue;
                  const int page = paged_page(a.d, a.table, a.status, c.s.slot, j);
                  const uint16_t* vr = static_cast<const uint16_t*>(a.v) + paged_row(a.d, page, c.hk, j) * D + 32 * e;
#pragma unroll
                  for (int k = 0; k < 32; ++k) {
                    const float x = __uint_as_float(static_cast<uint32_t>(vr[k]) << 16);
                    if (!isfinite(x)) o[k] = __float_as_uint(__uint_as_float(o[k]) + x);
                  }
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
      if (tid == 128) paged_step<F::kBM, F::kTK>(a, share);
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
      for (; share.work; paged_step<F::kBM, F::kTK>(a, share))   // from the piece that was not finished
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

cudaError_t launch_paged_fmha(const PagedAttnArgs& a, const CUtensorMap& tmK, const CUtensorMap& tmV, int num_sms,
                              cudaStream_t st) {
  static SmemOptIn opt_in[2];
  auto kern = a.d.d == 128 ? paged_fmha_kernel<128> : paged_fmha_kernel<64>;
  const int smem = a.d.d == 128 ? Pf<128>::kSmem : Pf<64>::kSmem;
  if (cudaError_t e = opt_in[a.d.d == 128](kern, smem)) return e;
  return launch_kernel(false, kern, num_sms, Pf<128>::kThreads, smem, st, tmK, tmV, a);
}

}  // namespace mot
