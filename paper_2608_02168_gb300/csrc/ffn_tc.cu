// Gated feed-forward block on the tensor cores (bf16 storage, fp32 accumulation), forward.
//
//   [G | U] = X [W_gate | W_up],  H = act(G) * U (rounded to bf16: the operand of the next product),
//   Y = H W_down (+ X)
//
// One persistent CTA an SM, or at d = 256 a pair of CTAs on two.  A group of two 128-row tiles (one at d = 256 and for
// few rows) stays in shared memory while the hidden features pass by in chunks of 64: the weights' pieces arrive by TMA
// in two rings, in the stored layout (MN-major operands), [G | U] of a chunk goes to one of two tensor-memory slots,
// two warpgroups turn it into H (half of a row a thread) in shared memory, and the product with W_down adds into Y,
// which starts at X for a residual.  The hidden rows never leave the chip.  The slots take turns (the two tiles, or
// even and odd chunks): one's gates are computed while the other's products run.  Each of the two products has an
// issuing warp of its own.  Rows leave through H's place by TMA.
//
// Bound by the tensor pipe (6 d f flops a row against 4 d bytes).  Measured: 300003 rows, f = 704 at d = 256 223 us
// (1.45 PFLOP/s, 0.76 of the measured bf16 rate; one issuing warp and one CTA 313 us), f = 384 at d = 128 88.5 us (1.0
// PFLOP/s: the gates' e^x and 1/x of every hidden feature take the special-function unit 49 us, the products the tensor
// pipe 46 us, and the two do not run wholly side by side), f = 200 at d = 64 62 us (0.37 PFLOP/s).  Few row tiles: a
// tile's chunks follow one another in one CTA, so the time does not fall with the rows (300, 3000 and 10000 rows at
// d = 128, f = 384: 14 us from a cold cache, 9 us in a replayed graph of such calls; at d = 256, f = 704: 22.5 us).
#include <algorithm>

#include "ffn_kernels.cuh"
#include "ffn_tc.cuh"
#include "layer_kernels.cuh"
#include "tc_util.cuh"

namespace hg {

using namespace tc;

namespace {

constexpr int kRows = 128;
constexpr int kHc = 64;              // hidden features of a chunk
constexpr int kBlk = kRows * 128;    // a 64-column block of a 128-row tile
// warps 0..3: TMA, [G | U], tensor memory, H W_down; then two warpgroups for the gates of each slot: with one, a
// scheduler's single warp of a slot waits out every latency of its own (300003 rows, d = 256, one issuing warp: 405
// against 313 us)
constexpr int kThreads = 640;
constexpr int kSms = 152;

// Row tiles of a CTA's group.  Up to a tile an SM one, whose even and odd chunks take turns in the slots (kernel with
// its timing, d = 128, f = 384: 300 rows 17 | 13.5 us with two | one, 19400 rows 17.9 | 14.6, 30000 rows 18.4 | 21.2);
// at d = 256, where Y fills half of the tensor memory, always one.
int tiles_of(int d, int64_t n) { return d == 256 || n <= (int64_t)kSms * kRows ? 1 : 2; }

template <int D, int NT>
struct FCfg {
  static constexpr int NB = D / 64;
  // CTAs that share the weights: at d = 256 a lone CTA's operands, read at 8 KB a 64-cycle product and written at 96 KB
  // a chunk, ask more of shared memory than it gives (300003 rows: 284 us; a pair, whose products read half of the
  // weights from each, 223 us); at d = 128 two tiles share them already (a pair 93 us, one CTA 88.5 us)
  static constexpr int CL = D == 256 ? 2 : 1;
  // a CTA's part of a chunk's weights: of a pair W_gate's or W_up's columns, and half of W_down's
  static constexpr int kPiece = D * 128 * 2 / CL, kDown = kHc * D * 2 / CL;
  static constexpr int NG = D == 64 ? 4 : 3, ND = D == 64 ? 4 : 2;  // ring slots
  static constexpr int kX = NT * NB * kBlk;
  static constexpr int kH = kRows * 128;
  static constexpr int kSmem = kX + NG * kPiece + ND * kDown + 2 * kH + 512 + 1024;
  static constexpr uint32_t kYCol = 0, kGuCol = 256;         // tensor memory: Y (tile x at x D), slots of 128
};

struct FwdP {
  int64_t n;
  int nch;
  int64_t groups;
  int residual;
  int* status;
};

template <int D, int NT, int kAct>
__cluster_dims__(FCfg<D, NT>::CL, 1, 1) __global__ void __launch_bounds__(kThreads, 1)
    ffn_fwd_tc_kernel(const __grid_constant__ CUtensorMap tm_X, const __grid_constant__ CUtensorMap tm_G,
                      const __grid_constant__ CUtensorMap tm_U, const __grid_constant__ CUtensorMap tm_W,
                      const __grid_constant__ CUtensorMap tm_Y, FwdP p) {
  pdl_begin();
  using C = FCfg<D, NT>;
  constexpr int NB = C::NB, NG = C::NG, ND = C::ND, CL = C::CL;
  using I = Issuer<CL>;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* Xs = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* Ws = Xs + C::kX;
  uint8_t* Ds = Ws + NG * C::kPiece;
  uint8_t* Hs = Ds + ND * C::kDown;
  uint64_t* bars = reinterpret_cast<uint64_t*>(Hs + 2 * C::kH);
  uint64_t *wfull = bars, *wfree = wfull + NG, *dfull = wfree + NG, *dfree = dfull + ND, *xfull = dfree + ND,
           *xfree = xfull + 1, *xpeer = xfree + 1, *gfull = xpeer + 1, *hfull = gfull + 2, *hfree = hfull + 2,
           *yfull = hfree + 2, *yready = yfull + 2, *sfull = yready + 2, *sdone = sfull + 2, *gfree = sdone + 2,
           *quit = gfree + 2;
  uint32_t* tslot = reinterpret_cast<uint32_t*>(quit + 2);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < NG; ++i) {
      mbar_init(&wfull[i], 1);
      mbar_init(&wfree[i], 1);
    }
    for (int i = 0; i < ND; ++i) {
      mbar_init(&dfull[i], 1);
      mbar_init(&dfree[i], 1);
    }
    mbar_init(xfull, 1);
    mbar_init(xfree, p.residual ? 17 : 1);
    mbar_init(xpeer, 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&gfull[i], 1);
      mbar_init(&gfree[i], 8 * CL);
      mbar_init(&hfull[i], 8 * CL);
      mbar_init(&hfree[i], 1);
      mbar_init(&yfull[i], 1);
      mbar_init(&yready[i], (NT == 2 ? 8 : 16) * CL);
      mbar_init(&sfull[i], 8);
      mbar_init(&sdone[i], 1);
    }
    mbar_init(&quit[0], 1);
    mbar_init(&quit[1], 1);
    fence_mbar_init();
  }
  if (warp == 2) I::alloc(tslot, 512);
  fence_before_sync();
  I::sync_all();
  fence_after_sync();
  const uint32_t tmem = *tslot;
  const int nch = p.nch;
  // A pair's CTAs take neighbouring groups at the same pace (one past the last is rows past n).  The first one issues
  // the products of both; its barriers gather both CTAs' arrivals, its commits arrive in both.
  const uint32_t rank = I::rank();
  const int64_t gr0 = blockIdx.x, gend = (p.groups + CL - 1) / CL * CL;

  if (warp == 0 && lane == 0) {
    // ---------------------------------------------------------------- loads
    Waiter wait{p.status};
    uint32_t q = 0, qd = 0, xn = 0;  // pieces of the two rings and row groups asked for
    auto load_gu = [&](int c) {
      const uint32_t s = q % NG;
      if (!wait.ok || (q >= NG && !wait(&wfree[s], (q / NG - 1) & 1))) return;
      if (rank == 0) mbar_expect_tx(&wfull[s], C::kPiece * CL);
      ++q;
      uint8_t* dst = Ws + s * C::kPiece;
      if (CL == 2) {
        I::load(dst, rank ? &tm_U : &tm_G, c * kHc, 0, &wfull[s]);
      } else {
        I::load(dst, &tm_G, c * kHc, 0, &wfull[s]);
        I::load(dst + D * 128, &tm_U, c * kHc, 0, &wfull[s]);
      }
    };
    auto load_down = [&](int c) {
      const uint32_t s = qd % ND;
      if (!wait.ok || (qd >= ND && !wait(&dfree[s], (qd / ND - 1) & 1))) return;
      if (rank == 0) mbar_expect_tx(&dfull[s], C::kDown * CL);
      ++qd;
      for (int b = 0; b < NB / CL; ++b)
        I::load(Ds + s * C::kDown + b * kHc * 128, &tm_W, (rank * (NB / CL) + b) * 64, c * kHc, &dfull[s]);
    };
    for (int64_t gr = gr0; wait.ok && gr < gend; gr += gridDim.x) {
      if (xn >= 1 && !wait(xfree, (xn - 1) & 1)) break;
      mbar_expect_tx(xfull, C::kX);
      for (int t = 0; t < NT; ++t)
        for (int b = 0; b < NB; ++b)
          tma_load_2d(Xs + (t * NB + b) * kBlk, &tm_X, b * 64, (int)((gr * NT + t) * kRows), xfull);
      ++xn;
      load_gu(0);
      for (int c = 0; wait.ok && c < nch; ++c) {
        if (c + 1 < nch) load_gu(c + 1);
        load_down(c);
      }
    }
    // The last arrivals from the other CTA land before this one is gone; so do, after a give-up, the loads asked for.
    drain_rounds(wfree, NG, q);
    drain_rounds(dfree, ND, qd);
    if (xn) mbar_wait(xfree, (xn - 1) & 1);
    if (!wait.ok) {
      if (xn) mbar_wait(xfull, (xn - 1) & 1);
      if (rank == 0) {
        drain_rounds(wfull, NG, q);
        drain_rounds(dfull, ND, qd);
      }
    }
  } else if (warp == 1 && rank != 0) {
    // ---------------------------------------------------------------- X is there, for the issuing CTA
    WarpWaiter wait{p.status};
    uint32_t gi = 0;
    for (int64_t gr = gr0; gr < gend && wait(xfull, gi & 1); gr += gridDim.x, ++gi) I::arrive(xpeer);
  } else if (warp == 1) {
    // ---------------------------------------------------------------- [G | U]
    const I issue;
    WarpWaiter wait{p.status};
    uint32_t q = 0, gi = 0;
    uint32_t gk[2] = {0, 0};  // [G | U] of each slot so far
    const uint64_t xd = desc_sw128(smem_u32(Xs), 16, 1024), gd = desc_sw128(smem_u32(Ws), D * 128, 1024);
    constexpr uint32_t id_gu = idesc_bf16(128 * CL, 128, false, true);
    for (int64_t gr = gr0; wait.ok && gr < gend; gr += gridDim.x, ++gi) {
      if (!wait(xfull, gi & 1) || (CL == 2 && !wait(xpeer, gi & 1))) break;
      for (int c = 0; wait.ok && c < nch; ++c, ++q) {
        if (!wait(&wfull[q % NG], (q / NG) & 1)) break;
        const uint64_t w = desc_at(gd, q % NG * C::kPiece);
        for (int t = 0; wait.ok && t < NT; ++t) {
          const int s = NT == 2 ? t : c & 1;
          // once the gates have read what the slot held
          if (gk[s] >= 1 && !wait(&gfree[s], (gk[s] - 1) & 1)) break;
          const uint64_t x = desc_at(xd, t * NB * kBlk);
#pragma unroll
          for (int j = 0; j < D / 16; ++j)
            issue.mma(tmem + C::kGuCol + s * 128, desc_at(x, (j >> 2) * kBlk + (j & 3) * 32), desc_at(w, j * 2048), id_gu,
                      j > 0 ? 1u : 0u);
          ++gk[s];
          issue.commit(&gfull[s]);
        }
        if (!wait.ok) break;
        issue.commit(&wfree[q % NG]);
        if (c == nch - 1) issue.commit(xfree);
      }
    }
    if (!wait.ok) issue.drain(&quit[0]);
  } else if (warp == 3 && rank == 0) {
    // ---------------------------------------------------------------- H W_down
    // by a warp of its own: a wait or a commit takes this role some hundred cycles beside the gates' warps, and neither
    // product should stand behind the other's
    const I issue;
    WarpWaiter wait{p.status};
    uint32_t q = 0, gi = 0;
    uint32_t hk[2] = {0, 0};  // chunks of each slot so far
    const uint64_t hd = desc_sw128(smem_u32(Hs), 16, 1024), wd = desc_sw128(smem_u32(Ds), kHc * 128, 1024);
    constexpr uint32_t id_y = idesc_bf16(128 * CL, D, false, true);
    for (int64_t gr = gr0; wait.ok && gr < gend; gr += gridDim.x, ++gi) {
      for (int c = 0; wait.ok && c < nch; ++c, ++q) {
        if (!wait(&dfull[q % ND], (q / ND) & 1)) break;
        const uint64_t w = desc_at(wd, q % ND * C::kDown);
        for (int t = 0; wait.ok && t < NT; ++t) {
          const int s = NT == 2 ? t : c & 1;
          if ((c == 0 && !wait(&yready[t], gi & 1)) || !wait(&hfull[s], hk[s] & 1)) break;
          ++hk[s];
          const uint64_t h = desc_at(hd, s * C::kH);
#pragma unroll
          for (int j = 0; j < 4; ++j)
            issue.mma(tmem + C::kYCol + t * D, desc_at(h, j * 32), desc_at(w, j * 2048), id_y,
                      (c > 0 || j > 0 || p.residual) ? 1u : 0u);
          issue.commit(&hfree[s]);
          if (c == nch - 1) issue.commit(&yfull[t]);
        }
        if (wait.ok) issue.commit(&dfree[q % ND]);
      }
    }
    if (!wait.ok) issue.drain(&quit[1]);
  } else if (warp >= 4) {
    // ---------------------------------------------------------------- gates and rows out
    // half of the slot's hidden features (and of its tile's columns) for each warpgroup
    const int s = (warp - 4) >> 3, half = ((warp - 4) >> 2) & 1, row = (warp & 3) * 32 + lane;
    const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
    const uint32_t gcol = tmem + C::kGuCol + s * 128 + half * 32 + lane_off;
    uint8_t* H = Hs + s * C::kH;
    WarpWaiter wait{p.status};
    uint32_t k = 0, gi = 0;
    // the slot's columns of Y: NT == 2 all of its tile's, else half of the tile's; 64 of them a round
    const int t = NT == 2 ? s : 0;
    constexpr int RN = NT == 2 ? D / 64 : D >= 128 ? D / 128 : 1;
    const bool leaves = NT == 2 || D >= 128 || s == 0;  // one tile of 64 columns: the first slot's
    const int blk0 = NT == 2 ? 0 : s * RN;
    const uint32_t ycol = tmem + C::kYCol + t * D + lane_off + blk0 * 64 + half * 32;
    uint32_t rounds = 0;
    for (int64_t gr = gr0; wait.ok && gr < gend; gr += gridDim.x, ++gi) {
      if (p.residual) {  // Y starts at X, so that X's place can take the next group while this one is finished
        if (!wait(xfull, gi & 1)) break;
#pragma unroll
        for (int b = 0; b < (leaves ? RN : 0); ++b) {
          const uint8_t* xb = Xs + (t * NB + blk0 + b) * kBlk;
#pragma unroll
          for (int x = 0; x < 32; x += 16) {
            float v[16];
            unpack(ld16(xb + sw128_offset(row, half * 64 + x * 2)), v, __nv_bfloat16());
            unpack(ld16(xb + sw128_offset(row, half * 64 + x * 2 + 16)), v + 8, __nv_bfloat16());
            st16_issue(ycol + b * 64 + x, v);
          }
        }
        st_wait();
        warp_arrive(xfree);
      }
      fence_before_sync();
      I::arrive(&yready[t]);
      bool first = rounds > 0;  // the rows of the group before leave through H's place
      for (int c = NT == 2 ? 0 : s; wait.ok && c < nch; c += 3 - NT, ++k) {
        if (!wait(&gfull[s], k & 1)) break;
        uint32_t g[32], u[32], h[16];
        ld16_issue(gcol, reinterpret_cast<uint32_t(&)[16]>(g[0]));
        ld16_issue(gcol + 64, reinterpret_cast<uint32_t(&)[16]>(u[0]));
        ld16_issue(gcol + 16, reinterpret_cast<uint32_t(&)[16]>(g[16]));
        ld16_issue(gcol + 80, reinterpret_cast<uint32_t(&)[16]>(u[16]));
        ld_wait();
        fence_before_sync();
        I::arrive(&gfree[s]);  // the next [G | U] runs while these gates are computed
#pragma unroll
        for (int e = 0; e < 32; e += 2)
          h[e / 2] = pack2_bf16(gate<kAct>(__uint_as_float(g[e])) * __uint_as_float(u[e]),
                                gate<kAct>(__uint_as_float(g[e + 1])) * __uint_as_float(u[e + 1]));
        if (k >= 1 && !wait(&hfree[s], (k - 1) & 1)) break;
        if (first && !wait(&sdone[s], (rounds - 1) & 1)) break;
        first = false;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          st16(H + sw128_offset(row, half * 64 + e * 16), make_uint4(h[4 * e], h[4 * e + 1], h[4 * e + 2], h[4 * e + 3]));
        fence_async_smem();
        fence_before_sync();
        I::arrive(&hfull[s]);
      }
      if (!wait.ok) break;
      // rows out, 64 columns a round: through H's place, and by a TMA store (it leaves out the rows past n)
      const int64_t r0 = (gr * NT + t) * kRows;
      if (!wait(&yfull[t], gi & 1)) break;
#pragma unroll 1
      for (int b = 0; b < (leaves ? RN : 0); ++b, ++rounds) {
        uint32_t y[32];
        ld16_issue(ycol + b * 64, reinterpret_cast<uint32_t(&)[16]>(y[0]));
        ld16_issue(ycol + b * 64 + 16, reinterpret_cast<uint32_t(&)[16]>(y[16]));
        ld_wait();
        // a slot without a chunk (one chunk, odd slot) has not waited for its last rows to leave yet
        if ((b > 0 || first) && !wait(&sdone[s], (rounds - 1) & 1)) break;
#pragma unroll
        for (int e = 0; e < 4; ++e)
          st16(H + sw128_offset(row, half * 64 + e * 16), pack(reinterpret_cast<float*>(y) + 8 * e, __nv_bfloat16()));
        fence_async_smem();
        warp_arrive(&sfull[s]);
        if ((threadIdx.x - 128) % 256 == 0) {
          if (mbar_wait(&sfull[s], rounds & 1)) {
            if (r0 < p.n) tma_store_2d(&tm_Y, H, (blk0 + b) * 64, (int)r0);
            bulk_commit();
            bulk_wait_read();
          } else {
            record_device_error(p.status, kErrTimeout);
          }
          mbar_arrive(&sdone[s]);
        }
        __syncwarp();
      }
    }
    if (k >= 1) wait(&hfree[s], (k - 1) & 1);
    bulk_wait();
  }
  fence_before_sync();
  I::sync_all();
  if (warp == 2) I::dealloc(tmem, 512);
}

template <int D, int NT, int kAct>
hg_status fwd_t(const hg_ffn_params* w, const void* X, int64_t n, void* Y, cudaStream_t s) {
  using C = FCfg<D, NT>;
  static bool done = false;
  if (!done) {
    HG_CUDA(cudaFuncSetAttribute(ffn_fwd_tc_kernel<D, NT, kAct>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                                 C::kSmem));
    done = true;
  }
  CUtensorMap tm_X, tm_G, tm_U, tm_W, tm_Y;
  HG_TRY(make_tmap_bf16(&tm_X, X, (uint64_t)n, D, kRows));
  HG_TRY(make_tmap_bf16(&tm_G, w->W_gate, D, (uint64_t)w->f, D));
  HG_TRY(make_tmap_bf16(&tm_U, w->W_up, D, (uint64_t)w->f, D));
  HG_TRY(make_tmap_bf16(&tm_W, w->W_down, (uint64_t)w->f, D, kHc));
  HG_TRY(make_tmap_bf16(&tm_Y, Y, (uint64_t)n, D, kRows));
  FwdP p{n, (int)ceil_div(w->f, kHc), ceil_div(n, (int64_t)kRows * NT), w->residual != 0, device_status_ptr()};
  const int grid = (int)std::min<int64_t>(ceil_div(p.groups, C::CL) * C::CL, kSms / C::CL * C::CL);
  return launch("ffn_fwd_tc", ffn_fwd_tc_kernel<D, NT, kAct>, dim3(grid), dim3(kThreads), C::kSmem, s, tm_X, tm_G, tm_U,
                tm_W, tm_Y, p);
}

template <int D, int NT>
hg_status fwd_a(const hg_ffn_params* w, const void* X, int64_t n, void* Y, cudaStream_t s) {
  if (w->act == HG_ACT_RELU) return fwd_t<D, NT, HG_ACT_RELU>(w, X, n, Y, s);
  if (w->act == HG_ACT_GELU_TANH) return fwd_t<D, NT, HG_ACT_GELU_TANH>(w, X, n, Y, s);
  if (w->act == HG_ACT_SILU) return fwd_t<D, NT, HG_ACT_SILU>(w, X, n, Y, s);
  return fwd_t<D, NT, HG_ACT_NONE>(w, X, n, Y, s);
}

template <int D>
hg_status fwd_d(const hg_ffn_params* w, const void* X, int64_t n, void* Y, cudaStream_t s) {
  if constexpr (D != 256)
    if (tiles_of(D, n) == 2) return fwd_a<D, 2>(w, X, n, Y, s);
  return fwd_a<D, 1>(w, X, n, Y, s);
}

}  // namespace

hg_status ffn_fwd_tc(const hg_ffn_params* w, const void* X, int64_t n, void* Y, cudaStream_t s) {
  if (w->d == 64) return fwd_d<64>(w, X, n, Y, s);
  if (w->d == 128) return fwd_d<128>(w, X, n, Y, s);
  return fwd_d<256>(w, X, n, Y, s);
}

}  // namespace hg
