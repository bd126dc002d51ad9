// Gated feed-forward block on the tensor cores (bf16 storage, fp32 accumulation), forward.
//
//   [G | U] = X [W_gate | W_up],  H = act(G) * U (rounded to bf16: the operand of the next product),
//   Y = H W_down (+ X)
//
// One persistent CTA an SM.  A group of two 128-row tiles (d <= 128; one at d = 256, whose Y fills half of the
// tensor memory) stays in shared memory while the hidden features pass by in chunks of 64: the weights'
// pieces arrive by TMA in a ring, in the stored layout (MN-major operands), [G | U] of a chunk goes to
// one of two tensor-memory slots, a warpgroup turns it into H (one row a thread) in shared memory, and the
// product with W_down adds into Y.  The hidden rows never leave the chip.  The slots take turns (the two
// tiles, or even and odd chunks): one's gates are computed while the other's products run, so the tensor pipe
// waits only for the slower of the two.  The gate's reciprocals are taken for two features at once, since the
// special-function rate (e^x and 1/x of every hidden feature) is as scarce as the tensor rate at d = 128.
// Bound by the tensor pipe (6 d f flops a row against 4 d bytes).
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
// warps 0..3: TMA, MMA issue, tensor memory, idle; then two warpgroups for the gates of each slot: with one, a
// scheduler's single warp of a slot waits out every latency of its own (1M rows, d = 256: 1370 us)
constexpr int kThreads = 640;
constexpr int kSms = 152;

template <int D>
struct FCfg {
  static constexpr int NB = D / 64;
  static constexpr int NT = D == 256 ? 1 : 2;                // row tiles of a group
  static constexpr int KP = D == 256 ? 2 : 1;                // pieces of [W_gate | W_up] (by rows)
  static constexpr int PR = D / KP;                          // their rows
  static constexpr int kPiece = PR * 128 * 2;                // bytes; W_down's piece is 64 D 2 <= kPiece
  static constexpr int kDown = kHc * D * 2;
  static constexpr int NS = D == 64 ? 6 : 4;                 // ring slots
  static constexpr int kX = NT * NB * kBlk;
  static constexpr int kH = kRows * 128;
  static constexpr int kSmem = kX + NS * kPiece + 2 * kH + 512 + 1024;
  static constexpr uint32_t kYCol = 0, kGuCol = 256;         // tensor memory: Y (tile x at x D), slots of 128
};

struct FwdP {
  int64_t n;
  int nch;
  int64_t groups;
  int residual;
  int* status;
};

template <int D, int kAct>
__global__ void __launch_bounds__(kThreads, 1)
    ffn_fwd_tc_kernel(const __grid_constant__ CUtensorMap tm_X, const __grid_constant__ CUtensorMap tm_G,
                      const __grid_constant__ CUtensorMap tm_U, const __grid_constant__ CUtensorMap tm_W,
                      const __grid_constant__ CUtensorMap tm_Y, FwdP p) {
  pdl_begin();
  using C = FCfg<D>;
  constexpr int NB = C::NB, NT = C::NT, NS = C::NS, KP = C::KP;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* Xs = reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(smem_raw) + 1023) & ~uintptr_t(1023));
  uint8_t* Ws = Xs + C::kX;
  uint8_t* Hs = Ws + NS * C::kPiece;
  uint64_t* bars = reinterpret_cast<uint64_t*>(Hs + 2 * C::kH);
  uint64_t *wfull = bars, *wfree = bars + NS, *xfull = bars + 2 * NS, *xfree = xfull + 1, *gfull = xfull + 2,
           *hfull = gfull + 2, *hfree = hfull + 2, *yfull = hfree + 2, *yready = yfull + 2, *sfull = yready + 2,
           *sdone = sfull + 2, *gfree = sdone + 2, *quit = gfree + 2;
  uint32_t* tslot = reinterpret_cast<uint32_t*>(quit + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    for (int i = 0; i < NS; ++i) {
      mbar_init(&wfull[i], 1);
      mbar_init(&wfree[i], 1);
    }
    mbar_init(xfull, 1);
    mbar_init(xfree, p.residual ? 513 : 1);
    for (int i = 0; i < 2; ++i) {
      mbar_init(&gfull[i], 1);
      mbar_init(&gfree[i], 256);
      mbar_init(&hfull[i], 256);
      mbar_init(&hfree[i], 1);
      mbar_init(&yfull[i], 1);
      mbar_init(&yready[i], NT == 2 ? 256 : 512);
      mbar_init(&sfull[i], 256);
      mbar_init(&sdone[i], 1);
    }
    mbar_init(quit, 1);
    fence_mbar_init();
  }
  if (warp == 2) tmem_alloc(tslot, 512);
  fence_before_sync();
  __syncthreads();
  fence_after_sync();
  const uint32_t tmem = *tslot;
  const int nch = p.nch;

  if (warp == 0 && lane == 0) {
    // ---------------------------------------------------------------- loads
    bool ok = true;
    uint32_t q = 0, xn = 0;  // pieces and row groups asked for
    auto wait = [&](uint64_t* b, uint32_t parity) {
      if (ok && !mbar_wait(b, parity)) {
        ok = false;
        record_device_error(p.status, kErrTimeout);
      }
      return ok;
    };
    auto slot = [&](uint32_t bytes) -> uint8_t* {
      const uint32_t s = q % NS;
      if (q >= NS && !wait(&wfree[s], (q / NS - 1) & 1)) return nullptr;
      mbar_expect_tx(&wfull[s], bytes);
      ++q;
      return Ws + s * C::kPiece;
    };
    auto load_gu = [&](int c) {
      for (int k = 0; ok && k < KP; ++k) {
        uint8_t* dst = slot(C::kPiece);
        if (!dst) return;
        uint64_t* b = &wfull[(q - 1) % NS];
        tma_load_2d(dst, &tm_G, c * kHc, k * C::PR, b);
        tma_load_2d(dst + C::PR * 128, &tm_U, c * kHc, k * C::PR, b);
      }
    };
    auto load_down = [&](int c) {
      uint8_t* dst = ok ? slot(C::kDown) : nullptr;
      if (!dst) return;
      for (int b = 0; b < NB; ++b) tma_load_2d(dst + b * kHc * 128, &tm_W, b * 64, c * kHc, &wfull[(q - 1) % NS]);
    };
    for (int64_t gr = blockIdx.x; ok && gr < p.groups; gr += gridDim.x) {
      if (xn >= 1 && !wait(xfree, (xn - 1) & 1)) break;
      mbar_expect_tx(xfull, C::kX);
      for (int t = 0; t < NT; ++t)
        for (int b = 0; b < NB; ++b)
          tma_load_2d(Xs + (t * NB + b) * kBlk, &tm_X, b * 64, (int)((gr * NT + t) * kRows), xfull);
      ++xn;
      load_gu(0);
      if (NT == 1 && nch > 1) load_gu(1);
      for (int c = 0; ok && c < nch; ++c) {
        if (NT == 2 && c + 1 < nch) load_gu(c + 1);
        load_down(c);
        if (NT == 1 && c + 2 < nch) load_gu(c + 2);
      }
    }
    if (!ok) {  // what was asked for lands before the CTA ends
      if (xn) mbar_wait(xfull, (xn - 1) & 1);
      drain_rounds(wfull, NS, q);
    }
  } else if (warp == 1) {
    // ---------------------------------------------------------------- products
    const Issuer issue;
    WarpWaiter wait{p.status};
    uint32_t q = 0, gi = 0;
    uint32_t hk[2] = {0, 0};  // chunks of each slot so far
    const uint64_t xd = desc_sw128(smem_u32(Xs), 16, 1024), hd = desc_sw128(smem_u32(Hs), 16, 1024);
    const uint64_t gd = desc_sw128(smem_u32(Ws), C::PR * 128, 1024), wd = desc_sw128(smem_u32(Ws), kHc * 128, 1024);
    constexpr uint32_t id_gu = idesc_bf16(128, 128, false, true), id_y = idesc_bf16(128, D, false, true);
    uint32_t gk[2] = {0, 0};  // [G | U] of each slot so far
    // tile t times the chunk's pieces q .. q + KP - 1 into slot s, once the gates have read what it held
    auto gu = [&](int t, int s) {
      if (NT == 2 && gk[s] >= 1 && !wait(&gfree[s], (gk[s] - 1) & 1)) return;
#pragma unroll
      for (int k = 0; k < KP; ++k) {
        if (!wait(&wfull[(q + k) % NS], ((q + k) / NS) & 1)) return;
        const uint64_t w = desc_at(gd, (q + k) % NS * C::kPiece), x = desc_at(xd, t * NB * kBlk);
#pragma unroll
        for (int j = 0; j < C::PR / 16; ++j) {
          const int jj = k * (C::PR / 16) + j;
          issue.mma(tmem + C::kGuCol + s * 128, desc_at(x, (jj >> 2) * kBlk + (jj & 3) * 32), desc_at(w, j * 2048),
                    id_gu, jj > 0 ? 1u : 0u);
        }
      }
      ++gk[s];
      issue.commit(&gfull[s]);
    };
    // the hidden rows of slot s times W_down's piece q into its tile's Y
    auto down = [&](int c, int s) {
      const int t = NT == 2 ? s : 0;
      if (!wait(&wfull[q % NS], (q / NS) & 1) || !wait(&hfull[s], hk[s] & 1)) return;
      if (c == 0 && !wait(&yready[t], gi & 1)) return;
      ++hk[s];
      const uint64_t w = desc_at(wd, q % NS * C::kPiece), h = desc_at(hd, s * C::kH);
#pragma unroll
      for (int j = 0; j < 4; ++j)
        issue.mma(tmem + C::kYCol + t * D, desc_at(h, j * 32), desc_at(w, j * 2048), id_y,
                  (c > 0 || j > 0 || p.residual) ? 1u : 0u);
      issue.commit(&hfree[s]);
      if (c == nch - 1) issue.commit(&yfull[t]);
    };
    auto release = [&](int count) {
      for (int i = 0; i < count; ++i, ++q) issue.commit(&wfree[q % NS]);
    };
    // chunk c's [G | U] of every tile of the group
    auto hidden = [&](int c) {
      for (int t = 0; wait.ok && t < NT; ++t) gu(t, NT == 2 ? t : c & 1);
      if (!wait.ok) return;
      release(KP);
      if (c == nch - 1) issue.commit(xfree);
    };
    for (int64_t gr = blockIdx.x; wait.ok && gr < p.groups; gr += gridDim.x, ++gi) {
      if (!wait(xfull, gi & 1)) break;
      for (int c = 0; wait.ok && c < 3 - NT && c < nch; ++c) hidden(c);
      for (int c = 0; wait.ok && c < nch; ++c) {
        // two tiles: the next [G | U] of both goes ahead, it is wanted first; one tile: the other slot's [G | U]
        // is under way, and the next one would only stand before this product (300k rows, d = 256: 275 -> 317 us)
        if (NT == 2 && c + 1 < nch) hidden(c + 1);
        for (int t = 0; wait.ok && t < NT; ++t) down(c, NT == 2 ? t : c & 1);
        if (!wait.ok) break;
        release(1);
        if (NT == 1 && c + 2 < nch) hidden(c + 2);
      }
    }
    if (!wait.ok) issue.drain(quit);
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
    constexpr int RN = (NT == 2 ? D : D / 2) / 64;
    const int blk0 = NT == 2 ? 0 : s * RN;
    const uint32_t ycol = tmem + C::kYCol + t * D + lane_off + blk0 * 64 + half * 32;
    uint32_t rounds = 0;
    for (int64_t gr = blockIdx.x; wait.ok && gr < p.groups; gr += gridDim.x, ++gi) {
      if (p.residual) {  // Y starts at X, so that X's place can take the next group while this one is finished
        if (!wait(xfull, gi & 1)) break;
#pragma unroll
        for (int b = 0; b < RN; ++b) {
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
        mbar_arrive(xfree);
      }
      fence_before_sync();
      mbar_arrive(&yready[t]);
      bool first = rounds > 0;  // the rows of the group before leave through H's place
      for (int c = NT == 2 ? 0 : s; wait.ok && c < nch; c += 3 - NT, ++k) {
        if (!wait(&gfull[s], k & 1)) break;
        uint32_t g[32], u[32], h[16];
        ld16_issue(gcol, reinterpret_cast<uint32_t(&)[16]>(g[0]));
        ld16_issue(gcol + 64, reinterpret_cast<uint32_t(&)[16]>(u[0]));
        ld16_issue(gcol + 16, reinterpret_cast<uint32_t(&)[16]>(g[16]));
        ld16_issue(gcol + 80, reinterpret_cast<uint32_t(&)[16]>(u[16]));
        ld_wait();
        if (NT == 2) {  // the next [G | U] runs while these gates are computed
          fence_before_sync();
          mbar_arrive(&gfree[s]);
        }
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
        mbar_arrive(&hfull[s]);
      }
      if (!wait.ok) break;
      // rows out, 64 columns a round: through H's place, and by a TMA store (it leaves out the rows past n)
      const int64_t r0 = (gr * NT + t) * kRows;
      if (!wait(&yfull[t], gi & 1)) break;
#pragma unroll 1
      for (int b = 0; b < RN; ++b, ++rounds) {
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
        mbar_arrive(&sfull[s]);
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
    bulk_wait();
  }
  fence_before_sync();
  __syncthreads();
  if (warp == 2) tmem_dealloc(tmem, 512);
}

template <int D, int kAct>
hg_status fwd_t(const hg_ffn_params* w, const void* X, int64_t n, void* Y, cudaStream_t s) {
  using C = FCfg<D>;
  static bool done = false;
  if (!done) {
    HG_CUDA(cudaFuncSetAttribute(ffn_fwd_tc_kernel<D, kAct>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem));
    done = true;
  }
  CUtensorMap tm_X, tm_G, tm_U, tm_W, tm_Y;
  HG_TRY(make_tmap_bf16(&tm_X, X, (uint64_t)n, D, kRows));
  HG_TRY(make_tmap_bf16(&tm_G, w->W_gate, D, (uint64_t)w->f, C::PR));
  HG_TRY(make_tmap_bf16(&tm_U, w->W_up, D, (uint64_t)w->f, C::PR));
  HG_TRY(make_tmap_bf16(&tm_W, w->W_down, (uint64_t)w->f, D, kHc));
  HG_TRY(make_tmap_bf16(&tm_Y, Y, (uint64_t)n, D, kRows));
  FwdP p{n, (int)ceil_div(w->f, kHc), ceil_div(n, (int64_t)kRows * C::NT),
         w->residual != 0, device_status_ptr()};
  const int grid = (int)std::min<int64_t>(p.groups, kSms);
  return launch("ffn_fwd_tc", ffn_fwd_tc_kernel<D, kAct>, dim3(grid), dim3(kThreads), C::kSmem, s, tm_X, tm_G, tm_U,
                tm_W, tm_Y, p);
}

template <int D>
hg_status fwd_d(const hg_ffn_params* w, const void* X, int64_t n, void* Y, cudaStream_t s) {
  if (w->act == HG_ACT_RELU) return fwd_t<D, HG_ACT_RELU>(w, X, n, Y, s);
  if (w->act == HG_ACT_GELU_TANH) return fwd_t<D, HG_ACT_GELU_TANH>(w, X, n, Y, s);
  if (w->act == HG_ACT_SILU) return fwd_t<D, HG_ACT_SILU>(w, X, n, Y, s);
  return fwd_t<D, HG_ACT_NONE>(w, X, n, Y, s);
}

}  // namespace

hg_status ffn_fwd_tc(const hg_ffn_params* w, const void* X, int64_t n, void* Y, cudaStream_t s) {
  if (w->d == 64) return fwd_d<64>(w, X, n, Y, s);
  if (w->d == 128) return fwd_d<128>(w, X, n, Y, s);
  return fwd_d<256>(w, X, n, Y, s);
}

}  // namespace hg
