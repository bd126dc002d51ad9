// Gated feed-forward block on the tensor cores (bf16 storage, fp32 accumulation), backward.
//
//   [G | U] = X [W_gate | W_up] and dH = dY W_down^T again, chunk by chunk of the hidden features
//   dG = dH * U * act'(G), dU = dH * act(G), H = act(G) * U
//   dX = dG W_gate^T + dU W_up^T (+ dY)                               (ffn_dx_tc)
//   dW_gate = X^T dG, dW_up = X^T dU, dW_down^T = dY^T H              (ffn_wgrad_tc)
//
// The hidden rows are formed twice, once in each kernel, instead of being stored: three of the five and of the
// nine products are theirs, but n x f values written and read would take an order of magnitude longer.
//
// ffn_dx_tc: as the forward (ffn_tc.cu) with one CTA and one 128-row tile at a time, two slots of chunks (one at
// d = 256).  The weights' pieces serve twice, as MN-major operands of [G | U] and as K-major operands of dX.  dG and
// dU are rounded to bf16.  At d = 256 X, dY and a chunk's weights fill the shared memory, so dG and dU go back to
// tensor memory, as the products' first operand.
//
// ffn_wgrad_tc: a CTA owns a chunk of hidden features, keeps its weights in shared memory and takes a share of the row
// tiles.  The gradients are fp32 results, so dG, dU and H enter as sums of two bf16 numbers (16 bits; 2.5e-6 of a
// gradient is lost, where one number would leave three digits; a third one's place is not there at d = 128).  The
// tensor pipe's own additions cut their results short, which shrinks a long sum (3.8e-5 of it over 16000 rows): each
// tile's products are therefore drained into registers and added there.  The shares' sums are added in order.  With
// d = 64 the rows of X and dY stand side by side as one 128-wide operand (half of the products is not used: a 64-wide
// one would run at half the rate).
//
// Bound by the chain of a tile: products, gates and products (or a drain) follow one another, with the tensor pipe
// active 40 % (dX) and 33 % (weight gradients) of the time, and 28 d f flops a row are run where 16 are needed.  In dX
// the two slots share one place for dG and dU; a second row tile's operands have no place for the weight gradients.
// Measured: dX 116 us at 200003 rows, d = 128, f = 384 and 243 us at 100003 rows, d = 256, f = 704 (0.85 and 0.74
// PFLOP/s of its ten units); weight gradients 234 us (32-feature chunks with two tiles in shared memory 294 us) and 468
// us (0.76 and 0.69 PFLOP/s of their eighteen units).  At 96 registers up to 56 bytes of a lane (dX) and 72 (weight
// gradients, d = 256) lie in local memory.
#include <algorithm>

#include "ffn_kernels.cuh"
#include "ffn_tc.cuh"
#include "layer_kernels.cuh"
#include "tc_util.cuh"

namespace hg {

using namespace tc;

namespace {

constexpr int kRows = 128;
constexpr int kBlk = kRows * 128;  // a 64-column block of a 128-row tile
constexpr int kThreads = 640;      // warps 0..3: TMA, first products, tensor memory, dX; four warpgroups for the gates
constexpr int kSms = 152;

// eight 32-bit columns of this thread's lane
__device__ __forceinline__ void st8(uint32_t taddr, const uint32_t* r) {
  asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};" ::"r"(taddr), "r"(r[0]),
               "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7])
               : "memory");
}
__device__ __forceinline__ uint8_t* align1024(uint8_t* p) {
  return reinterpret_cast<uint8_t*>((reinterpret_cast<uintptr_t>(p) + 1023) & ~uintptr_t(1023));
}

// ---------------------------------------------------------------------------------------------
// dX
// ---------------------------------------------------------------------------------------------
template <int D>
struct DxCfg {
  static constexpr int HC = 64;
  static constexpr int NB = D / 64;
  static constexpr bool kTs = D == 256;              // dG, dU in tensor memory
  static constexpr int SLOTS = kTs ? 1 : 2;
  static constexpr int NG = D == 256 ? 1 : 3;        // ring of [W_gate | W_up]
  static constexpr int ND = D == 256 ? 1 : 2;        // ring of W_down
  static constexpr int kGu = D * 128 * 2, kDown = HC * D * 2;
  static constexpr int kX = NB * kBlk;
  static constexpr int kOps = kTs ? 0 : 2 * kBlk;    // dG, dU: 64 columns each
  static constexpr int kSmem = 2 * kX + NG * kGu + ND * kDown + kOps + 512 + 1024;
  static constexpr int kStoreThreads = D == 64 ? 512 : D == 128 ? 256 : 128;  // that fill a 64-column block of dX
  static constexpr int PR = D < 128 ? D : 128;       // rows of a TMA box of [W_gate | W_up]
  // tensor memory: dX, the slots ([G | U | dH], 192 columns), dG and dU (kTs)
  static constexpr uint32_t kSlot = D, kSlotCols = 192, kOpsCol = 448;
};

struct DxP {
  int64_t n;
  int nch;
  int64_t tiles;
  int residual;
  int* status;
};

template <int D, int kAct>
__global__ void __launch_bounds__(kThreads, 1)
    ffn_dx_tc_kernel(const __grid_constant__ CUtensorMap tm_X, const __grid_constant__ CUtensorMap tm_dY,
                     const __grid_constant__ CUtensorMap tm_G, const __grid_constant__ CUtensorMap tm_U,
                     const __grid_constant__ CUtensorMap tm_W, const __grid_constant__ CUtensorMap tm_dX, DxP p) {
  pdl_begin();
  using C = DxCfg<D>;
  constexpr int NB = C::NB, HC = C::HC, NG = C::NG, ND = C::ND, SLOTS = C::SLOTS;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* Xs = align1024(smem_raw);
  uint8_t* Ys = Xs + C::kX;
  uint8_t* Gs = Ys + C::kX;
  uint8_t* Ds = Gs + NG * C::kGu;
  uint8_t* Os = Ds + ND * C::kDown;
  uint64_t* bars = reinterpret_cast<uint64_t*>(Os + C::kOps);
  uint64_t *wfull = bars, *wfree = wfull + NG, *dfull = wfree + NG, *dfree = dfull + ND, *xfull = dfree + ND,
           *xfree = xfull + 1, *gfull = xfree + 1, *ofull = gfull + 2, *ofree = ofull + 1, *yfull = ofree + 2,
           *yfree = yfull + 1, *sfull = yfree + 1,
           *sdone = sfull + 4, *gfree = sdone + 1, *quit = gfree + 2;
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
    mbar_init(xfree, C::kTs ? 512 / C::kStoreThreads : p.residual ? 17 : 1);
    mbar_init(sdone, 512 / C::kStoreThreads);
    for (int i = 0; i < 512 / C::kStoreThreads; ++i) mbar_init(&sfull[i], C::kStoreThreads / 32);
    mbar_init(&gfull[0], 1);
    mbar_init(&gfull[1], 1);
    mbar_init(ofull, SLOTS == 2 ? 8 : 16);
    mbar_init(&ofree[0], 1);
    mbar_init(&ofree[1], 1);
    mbar_init(yfull, 1);
    mbar_init(yfree, 16);
    mbar_init(&gfree[0], SLOTS == 2 ? 8 : 16);
    mbar_init(&gfree[1], 8);
    mbar_init(&quit[0], 1);
    mbar_init(&quit[1], 1);
    fence_mbar_init();
  }
  if (warp == 2) tmem_alloc(tslot, 512);
  fence_before_sync();
  __syncthreads();
  fence_after_sync();
  const uint32_t tmem = *tslot;
  const int nch = p.nch;

  if (warp == 0 && lane == 0) {
    Waiter wait{p.status};
    uint32_t q = 0, xn = 0;  // chunks and tiles asked for
    for (int64_t tile = blockIdx.x; wait.ok && tile < p.tiles; tile += gridDim.x) {
      if (xn >= 1 && !wait(xfree, (xn - 1) & 1)) break;
      mbar_expect_tx(xfull, 2 * C::kX);
      for (int b = 0; b < NB; ++b) {
        tma_load_2d(Xs + b * kBlk, &tm_X, b * 64, (int)(tile * kRows), xfull);
        tma_load_2d(Ys + b * kBlk, &tm_dY, b * 64, (int)(tile * kRows), xfull);
      }
      ++xn;
      for (int c = 0; c < nch; ++c, ++q) {
        const uint32_t sg = q % NG, sd = q % ND;
        if (q >= ND && !wait(&dfree[sd], (q / ND - 1) & 1)) break;
        mbar_expect_tx(&dfull[sd], C::kDown);
        for (int b = 0; b < NB; ++b)
          tma_load_2d(Ds + sd * C::kDown + b * HC * 128, &tm_W, b * 64, c * HC, &dfull[sd]);
        if (q >= NG && !wait(&wfree[sg], (q / NG - 1) & 1)) {
          mbar_wait(&dfull[sd], (q / ND) & 1);
          break;
        }
        mbar_expect_tx(&wfull[sg], C::kGu);
        uint8_t* dst = Gs + sg * C::kGu;
        for (int r = 0; r < D; r += C::PR) {
          tma_load_2d(dst + r * 128, &tm_G, c * HC, r, &wfull[sg]);
          tma_load_2d(dst + D * 128 + r * 128, &tm_U, c * HC, r, &wfull[sg]);
        }
      }
    }
    if (!wait.ok) {  // what was asked for lands before the CTA ends
      if (xn) mbar_wait(xfull, (xn - 1) & 1);
      drain_rounds(dfull, ND, q);
      drain_rounds(wfull, NG, q);
    }
  } else if (warp == 1) {
    // [G | U | dH]
    const Issuer<1> issue;
    WarpWaiter wait{p.status};
    uint32_t q = 0, ti = 0;
    uint32_t gk[2] = {0, 0};  // chunks of each slot so far
    const uint64_t xd = desc_sw128(smem_u32(Xs), 16, 1024), yd = desc_sw128(smem_u32(Ys), 16, 1024);
    const uint64_t gd = desc_sw128(smem_u32(Gs), D * 128, 1024), dd = desc_sw128(smem_u32(Ds), 16, 1024);
    constexpr uint32_t id_gu = idesc_bf16(128, 128, false, true), id_h = idesc_bf16(128, 64, false, false);
    for (int64_t tile = blockIdx.x; wait.ok && tile < p.tiles; tile += gridDim.x, ++ti) {
      if (!wait(xfull, ti & 1)) break;
      for (int c = 0; c < nch; ++c, ++q) {
        const uint32_t sg = q % NG, sd = q % ND;
        const int s = c % SLOTS;
        // once the gates have read what the slot held
        if (gk[s] >= 1 && !wait(&gfree[s], (gk[s] - 1) & 1)) break;
        if (!wait(&wfull[sg], (q / NG) & 1) || !wait(&dfull[sd], (q / ND) & 1)) break;
        ++gk[s];
        const uint64_t w = desc_at(gd, sg * C::kGu), w2 = desc_at(dd, sd * C::kDown);
        const uint32_t t = tmem + C::kSlot + s * C::kSlotCols;
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
          issue.mma(t, desc_at(xd, (j >> 2) * kBlk + (j & 3) * 32), desc_at(w, j * 2048), id_gu, j > 0 ? 1u : 0u);
#pragma unroll
        for (int j = 0; j < D / 16; ++j)
          issue.mma(t + 128, desc_at(yd, (j >> 2) * kBlk + (j & 3) * 32),
                    desc_at(w2, (j >> 2) * (HC * 128) + (j & 3) * 32), id_h, j > 0 ? 1u : 0u);
        issue.commit(&gfull[s]);
        issue.commit(&dfree[sd]);
        if (!C::kTs && c == nch - 1) issue.commit(xfree);
      }
    }
    if (!wait.ok) issue.drain(&quit[0]);
  } else if (warp == 3) {
    // dX, by a warp of its own (see the forward)
    const Issuer<1> issue;
    WarpWaiter wait{p.status};
    uint32_t done = 0, ti = 0;
    const uint64_t gkd = desc_sw128(smem_u32(Gs), 16, 1024), od = desc_sw128(smem_u32(Os), 16, 1024);
    constexpr uint32_t id_dx = idesc_bf16(128, D, false, false);
    for (int64_t tile = blockIdx.x; wait.ok && tile < p.tiles; tile += gridDim.x, ++ti) {
      // kTs: the sums of the tile before were read; else dX is ready to be added to
      if (C::kTs ? ti >= 1 && !wait(yfree, (ti - 1) & 1) : !wait(yfree, ti & 1)) break;
      for (int c = 0; c < nch; ++c, ++done) {
        const uint32_t sg = done % NG;
        if (!wait(&wfull[sg], (done / NG) & 1) || !wait(ofull, done & 1)) break;
        const uint64_t w = desc_at(gkd, sg * C::kGu);
#pragma unroll
        for (int half = 0; half < 2; ++half)
#pragma unroll
          for (int j = 0; j < HC / 16; ++j) {
            const uint64_t b = desc_at(w, half * D * 128 + j * 32);
            const uint32_t acc = (c > 0 || half > 0 || j > 0 || (!C::kTs && p.residual)) ? 1u : 0u;
            if constexpr (C::kTs)
              issue.mma_ts(tmem, tmem + C::kOpsCol + half * 32 + j * 8, b, id_dx, acc);
            else
              issue.mma(tmem, desc_at(od, half * kBlk + j * 32), b, id_dx, acc);
          }
        issue.commit(&ofree[done & 1]);
        issue.commit(&wfree[sg]);
        if (c == nch - 1) issue.commit(yfull);
      }
    }
    if (!wait.ok) issue.drain(&quit[1]);
  } else if (warp >= 4) {
    const int wg = (warp - 4) >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
    const int s = SLOTS == 2 ? wg >> 1 : 0;
    const uint32_t t0 = tmem + C::kSlot + s * C::kSlotCols + lane_off;
    constexpr int HW = HC * SLOTS / 4;  // hidden features of a warpgroup
    const int h0 = (SLOTS == 2 ? wg & 1 : wg) * HW;
    WarpWaiter wait{p.status};
    uint32_t k = 0, done = 0, ti = 0;  // chunks of this slot, of all slots; tiles
    constexpr int CW = D / 4;  // columns of dX of a warpgroup
    const int col0 = wg * CW;
    for (int64_t tile = blockIdx.x; wait.ok && tile < p.tiles; tile += gridDim.x, ++ti) {
      if (!C::kTs) {
        // dX starts at dY, so that X's and dY's places can take the next tile while this one is finished
        if (p.residual) {
          if (!wait(xfull, ti & 1)) break;
#pragma unroll
          for (int c = 0; c < CW; c += 16) {
            const uint8_t* yb = Ys + col0 / 64 * kBlk;
            float v[16];
            unpack(ld16(yb + sw128_offset(row, (col0 % 64 + c) * 2)), v, __nv_bfloat16());
            unpack(ld16(yb + sw128_offset(row, (col0 % 64 + c) * 2 + 16)), v + 8, __nv_bfloat16());
            st16_issue(tmem + lane_off + col0 + c, v);
          }
          st_wait();
          warp_arrive(xfree);
        }
        fence_before_sync();
        warp_arrive(yfree);
      }
      bool first = ti > 0;  // the rows of the tile before leave through the operands' place
      for (int c = 0; wait.ok && c < nch; ++c, ++done) {
        if (SLOTS == 2 && (c & 1) != s) continue;
        if (!wait(&gfull[s], k & 1)) break;
        ++k;
        uint32_t dg[HW / 2], du[HW / 2];
#pragma unroll
        for (int x = 0; x < HW; x += 16) {
          uint32_t g[16], u[16], h[16];
          ld16_issue(t0 + h0 + x, g);
          ld16_issue(t0 + 64 + h0 + x, u);
          ld16_issue(t0 + 128 + h0 + x, h);
          ld_wait();
          if (x + 16 == HW) {  // the slot's next products run while these gates are computed
            fence_before_sync();
            warp_arrive(&gfree[s]);
          }
#pragma unroll
          for (int e = 0; e < 16; e += 2) {
            float d0, d1;
            const float a0 = gate_grad<kAct>(__uint_as_float(g[e]), &d0);
            const float a1 = gate_grad<kAct>(__uint_as_float(g[e + 1]), &d1);
            const float y0 = __uint_as_float(h[e]), y1 = __uint_as_float(h[e + 1]);
            dg[(x + e) / 2] = pack2_bf16(y0 * __uint_as_float(u[e]) * d0, y1 * __uint_as_float(u[e + 1]) * d1);
            du[(x + e) / 2] = pack2_bf16(y0 * a0, y1 * a1);
          }
        }
        // The product before has read the operands.  A slot looks at every other product, so even and odd ones have
        // barriers of their own: no phase of one passes unseen.
        if (done >= 1 && !wait(&ofree[(done - 1) & 1], ((done - 1) >> 1) & 1)) break;
        if (C::kTs) {
#pragma unroll
          for (int x = 0; x < HW / 2; x += 8) {
            st8(tmem + C::kOpsCol + lane_off + h0 / 2 + x, dg + x);
            st8(tmem + C::kOpsCol + 32 + lane_off + h0 / 2 + x, du + x);
          }
          st_wait();
        } else {
          if (first && !wait(sdone, (ti - 1) & 1)) break;
          first = false;
#pragma unroll
          for (int e = 0; e < HW / 8; ++e) {
            st16(Os + sw128_offset(row, h0 * 2 + e * 16), make_uint4(dg[4 * e], dg[4 * e + 1], dg[4 * e + 2], dg[4 * e + 3]));
            st16(Os + kBlk + sw128_offset(row, h0 * 2 + e * 16),
                 make_uint4(du[4 * e], du[4 * e + 1], du[4 * e + 2], du[4 * e + 3]));
          }
          fence_async_smem();
        }
        fence_before_sync();
        warp_arrive(ofull);
      }
      if (!wait.ok) break;
      // Rows out, a TMA store each 64 columns (it leaves out the rows past n): through the operands' place, which the
      // last product has read; kTs: dY's place takes dX (+ dY).
      uint8_t* ob = (C::kTs ? Ys : Os) + col0 / 64 * kBlk;
      if ((C::kTs && !wait(xfull, ti & 1)) || !wait(yfull, ti & 1)) break;
      if (!C::kTs && first && !wait(sdone, (ti - 1) & 1)) break;
#pragma unroll
      for (int c = 0; c < CW; c += 16) {
        uint32_t y[16];
        ld16_issue(tmem + lane_off + col0 + c, y);
        uint4* x0 = reinterpret_cast<uint4*>(ob + sw128_offset(row, (col0 % 64 + c) * 2));
        uint4* x1 = reinterpret_cast<uint4*>(ob + sw128_offset(row, (col0 % 64 + c) * 2 + 16));
        const bool add = C::kTs && p.residual;
        float v[16];
        unpack(add ? *x0 : make_uint4(0u, 0u, 0u, 0u), v, __nv_bfloat16());
        unpack(add ? *x1 : make_uint4(0u, 0u, 0u, 0u), v + 8, __nv_bfloat16());
        ld_wait();
#pragma unroll
        for (int i = 0; i < 16; ++i) v[i] += __uint_as_float(y[i]);
        *x0 = pack(v, __nv_bfloat16());
        *x1 = pack(v + 8, __nv_bfloat16());
      }
      fence_async_smem();
      fence_before_sync();
      if (C::kTs) warp_arrive(yfree);
      uint64_t* sb = &sfull[(threadIdx.x - 128) / C::kStoreThreads];
      warp_arrive(sb);
      if ((threadIdx.x - 128) % C::kStoreThreads == 0) {
        if (mbar_wait(sb, ti & 1)) {
          tma_store_2d(&tm_dX, ob, col0 / 64 * 64, (int)(tile * kRows));
          bulk_commit();
          bulk_wait_read();
        } else {
          record_device_error(p.status, kErrTimeout);
        }
        mbar_arrive(C::kTs ? xfree : sdone);
      }
      __syncwarp();
    }
    bulk_wait();
  }
  fence_before_sync();
  __syncthreads();
  if (warp == 2) tmem_dealloc(tmem, 512);
}

// ---------------------------------------------------------------------------------------------
// weight gradients
// ---------------------------------------------------------------------------------------------
template <int D>
struct WgCfg {
  static constexpr int HC = D == 256 ? 32 : 64;       // hidden features of a CTA
  static constexpr int NB = D / 64;
  static constexpr int MB = D == 256 ? 2 : 1;         // 128-row blocks of the gradients
  static constexpr int XS = D == 64 ? 2 : 1;          // row tiles in shared memory
  static constexpr int kX = NB * kBlk;
  static constexpr int N2 = 2 * HC;                   // columns of [G | U], of [dG | dU] and of [H hi | H lo]
  static constexpr int kW = N2 * D * 2, kDown = HC * D * 2;
  static constexpr int kOps = N2 / 64 * kBlk;
  static constexpr int kSmem = XS * 2 * kX + kW + kDown + 3 * kOps + 512 + 1024;
  // tensor memory: gradients ([dG | dU] of each block, then [H hi | H lo]), then [G | U | dH]
  static constexpr uint32_t kAcc2 = MB * N2, kHid = 2 * MB * N2;
  static constexpr int PC = 6;                        // pieces of 8 columns whose sums a warpgroup keeps
};

struct WgP {
  int64_t n, tiles;
  int f, splits, chunks;
  float* part;  // [splits][3 d f]
  int* status;
};

template <int D, int kAct>
__global__ void __launch_bounds__(kThreads, 1)
    ffn_wgrad_tc_kernel(const __grid_constant__ CUtensorMap tm_X, const __grid_constant__ CUtensorMap tm_dY,
                        const __grid_constant__ CUtensorMap tm_Wt, const __grid_constant__ CUtensorMap tm_W, WgP p) {
  pdl_begin();
  using C = WgCfg<D>;
  constexpr int NB = C::NB, HC = C::HC, XS = C::XS, MB = C::MB, N2 = C::N2;
  extern __shared__ uint8_t smem_raw[];
  uint8_t* Xs = align1024(smem_raw);               // [XS] (X tile, dY tile)
  uint8_t* Ws = Xs + XS * 2 * C::kX;
  uint8_t* Ds = Ws + C::kW;
  uint8_t* Os = Ds + C::kDown;                     // [dG | dU] hi, lo, [H hi | H lo]
  uint64_t* bars = reinterpret_cast<uint64_t*>(Os + 3 * C::kOps);
  uint64_t *wfull = bars, *xfull = bars + 1, *xfree = xfull + XS, *yfull = xfree + XS, *yfree = yfull + XS,
           *gfull = yfree + XS, *ofull = gfull + 1, *ofree = ofull + 1, *quit = ofree + 1;
  uint32_t* tslot = reinterpret_cast<uint32_t*>(quit + 1);
  const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
  if (threadIdx.x == 0) {
    mbar_init(wfull, 1);
    for (int i = 0; i < XS; ++i) {
      mbar_init(&xfull[i], 1);
      mbar_init(&xfree[i], 1);
      mbar_init(&yfull[i], 1);
      mbar_init(&yfree[i], 1);
    }
    mbar_init(gfull, 1);
    mbar_init(ofull, 16);
    mbar_init(ofree, 1);
    mbar_init(quit, 1);
    fence_mbar_init();
  }
  if (warp == 2) tmem_alloc(tslot, 512);
  fence_before_sync();
  __syncthreads();
  fence_after_sync();
  const uint32_t tmem = *tslot;
  const int chunk = blockIdx.x % p.chunks, split = blockIdx.x / p.chunks;
  const int64_t tile0 = p.tiles * split / p.splits, tile1 = p.tiles * (split + 1) / p.splits;
  const int count = (int)(tile1 - tile0);  // at least one

  if (warp == 0 && lane == 0) {
    Waiter wait{p.status};
    mbar_expect_tx(wfull, C::kW + C::kDown);
    for (int b = 0; b < NB; ++b) {
      tma_load_2d(Ws + b * N2 * 128, &tm_Wt, b * 64, chunk * N2, wfull);
      tma_load_2d(Ds + b * HC * 128, &tm_W, b * 64, chunk * HC, wfull);
    }
    uint32_t q = 0, qy = 0;  // X and dY tiles asked for
    for (; q < (uint32_t)count; ++q) {
      const uint32_t s = q % XS;
      const int r = (int)((tile0 + q) * kRows);
      uint8_t* dst = Xs + s * 2 * C::kX;
      if (q >= XS && !wait(&xfree[s], (q / XS - 1) & 1)) break;
      mbar_expect_tx(&xfull[s], C::kX);
      for (int b = 0; b < NB; ++b) tma_load_2d(dst + b * kBlk, &tm_X, b * 64, r, &xfull[s]);
      if (q >= XS && !wait(&yfree[s], (q / XS - 1) & 1)) {
        ++q;
        break;
      }
      mbar_expect_tx(&yfull[s], C::kX);
      for (int b = 0; b < NB; ++b) tma_load_2d(dst + C::kX + b * kBlk, &tm_dY, b * 64, r, &yfull[s]);
      ++qy;
    }
    if (!wait.ok) {
      mbar_wait(wfull, 0);
      drain_rounds(xfull, XS, q);
      drain_rounds(yfull, XS, qy);
    }
  } else if (warp == 1) {
    const Issuer<1> issue;
    WarpWaiter wait{p.status};
    const uint64_t xd = desc_sw128(smem_u32(Xs), 16, 1024), xmd = desc_sw128(smem_u32(Xs), kBlk, 1024);
    const uint64_t wd = desc_sw128(smem_u32(Ws), 16, 1024), dd = desc_sw128(smem_u32(Ds), 16, 1024);
    const uint64_t od = desc_sw128(smem_u32(Os), kBlk, 1024);
    constexpr uint32_t id_gu = idesc_bf16(128, N2, false, false), id_h = idesc_bf16(128, HC, false, false),
                       id_w = idesc_bf16(128, N2, true, true);
    wait(wfull, 0);
    for (int i = 0; wait.ok && i < count; ++i) {
      const int s = i % XS;
      if (!wait(&xfull[s], (i / XS) & 1)) break;
      const uint64_t x = desc_at(xd, s * 2 * C::kX), xm = desc_at(xmd, s * 2 * C::kX);
      const uint32_t hid = tmem + C::kHid;
#pragma unroll
      for (int j = 0; j < D / 16; ++j)
        issue.mma(hid, desc_at(x, (j >> 2) * kBlk + (j & 3) * 32), desc_at(wd, (j >> 2) * (N2 * 128) + (j & 3) * 32),
                  id_gu, j > 0 ? 1u : 0u);
      if (!wait(&yfull[s], (i / XS) & 1)) break;
#pragma unroll
      for (int j = 0; j < D / 16; ++j)
        issue.mma(hid + N2, desc_at(x, C::kX + (j >> 2) * kBlk + (j & 3) * 32),
                  desc_at(dd, (j >> 2) * (HC * 128) + (j & 3) * 32), id_h, j > 0 ? 1u : 0u);
      issue.commit(gfull);
      if (!wait(ofull, i & 1)) break;
      // X's products first: its place takes the next tile while dY's run
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int part = 0; part < 2; ++part)
#pragma unroll
          for (int j = 0; j < 8; ++j)
            issue.mma(tmem + m * N2, desc_at(xm, m * 2 * kBlk + j * 2048), desc_at(od, part * C::kOps + j * 2048), id_w,
                      (part > 0 || j > 0) ? 1u : 0u);
      if (D != 64) issue.commit(&xfree[s]);
#pragma unroll
      for (int m = 0; m < MB; ++m)
#pragma unroll
        for (int j = 0; j < 8; ++j)  // d = 64: X and dY side by side are the 128 rows of both gradients
          issue.mma(tmem + C::kAcc2 + m * N2, desc_at(xm, (D == 64 ? 0 : C::kX) + m * 2 * kBlk + j * 2048),
                    desc_at(od, 2 * C::kOps + j * 2048), id_w, j > 0 ? 1u : 0u);
      if (D == 64) issue.commit(&xfree[s]);
      issue.commit(&yfree[s]);
      issue.commit(ofree);
    }
    if (!wait.ok) issue.drain(quit);
  } else if (warp >= 4) {
    const int wg = (warp - 4) >> 2, row = (warp & 3) * 32 + lane;
    const uint32_t lane_off = (uint32_t)((warp & 3) * 32) << 16;
    constexpr int HW = HC / 4, PC = C::PC;  // hidden features of a warpgroup
    const int h0 = wg * HW;
    const uint32_t hid = tmem + C::kHid + lane_off + h0;
    WarpWaiter wait{p.status};
    // This thread's sums: six pieces of 8 columns of its row.  The pieces of a row of a block (24; 12 at d = 256, where
    // two warpgroups share a block) are first those of [dG | dU], then H's, whose two halves are added.
    float sum[PC * 8];
#pragma unroll
    for (int e = 0; e < PC * 8; ++e) sum[e] = 0.f;
    const int m = MB == 2 ? wg >> 1 : 0;
    auto place = [&](int b, bool* pair) -> uint32_t {  // columns of piece b, from the block's first
      const int gb = (MB == 2 ? wg & 1 : wg) * PC + b, first = N2 / 8;
      *pair = gb >= first;
      return gb < first ? gb * 8 : C::kAcc2 + (gb - first) * 8;
    };
    auto drain = [&]() {
#pragma unroll
      for (int b = 0; b < PC; ++b) {
        bool pair;
        const uint32_t col = tmem + lane_off + m * N2 + place(b, &pair);
        uint32_t v[8], w[8];
        ld8_issue(col, v);
        ld8_issue(pair ? col + HC : col, w);
        ld_wait();
#pragma unroll
        for (int e = 0; e < 8; ++e) sum[b * 8 + e] += __uint_as_float(v[e]) + (pair ? __uint_as_float(w[e]) : 0.f);
      }
    };
    for (int i = 0; i < count; ++i) {
      if (i >= 1) {  // while the next tile is loaded and its hidden rows are formed
        if (!wait(ofree, (i - 1) & 1)) break;
        drain();
      }
      if (!wait(gfull, i & 1)) break;
#pragma unroll
      for (int x = 0; x < HW; x += 8) {
        uint32_t g[8], u[8], h[8];
        ld8_issue(hid + x, g);
        ld8_issue(hid + HC + x, u);
        ld8_issue(hid + N2 + x, h);
        ld_wait();
        uint32_t hi[3][4], lo[3][4];
#pragma unroll
        for (int e = 0; e < 8; e += 2) {
          float d0, d1;
          const float a0 = gate_grad<kAct>(__uint_as_float(g[e]), &d0);
          const float a1 = gate_grad<kAct>(__uint_as_float(g[e + 1]), &d1);
          const float u0 = __uint_as_float(u[e]), u1 = __uint_as_float(u[e + 1]);
          const float y0 = __uint_as_float(h[e]), y1 = __uint_as_float(h[e + 1]);
          const float v[3][2] = {{y0 * u0 * d0, y1 * u1 * d1}, {y0 * a0, y1 * a1}, {a0 * u0, a1 * u1}};
#pragma unroll
          for (int k = 0; k < 3; ++k) {
            const uint32_t w = pack2_bf16(v[k][0], v[k][1]);
            hi[k][e / 2] = w;
            lo[k][e / 2] = pack2_bf16(v[k][0] - __uint_as_float(w << 16), v[k][1] - __uint_as_float(w & 0xffff0000u));
          }
        }
        // 16 bytes of this row: feature h0 + x on, of the first or the second half of the columns
        auto put = [&](uint8_t* o, int c, const uint32_t* v) {
          c += h0 + x;
          st16(o + (c >> 6) * kBlk + sw128_offset(row, (c & 63) * 2), make_uint4(v[0], v[1], v[2], v[3]));
        };
        put(Os, 0, hi[0]);
        put(Os, HC, hi[1]);
        put(Os + C::kOps, 0, lo[0]);
        put(Os + C::kOps, HC, lo[1]);
        put(Os + 2 * C::kOps, 0, hi[2]);
        put(Os + 2 * C::kOps, HC, lo[2]);
      }
      fence_async_smem();
      fence_before_sync();
      warp_arrive(ofull);
    }
    // the sums of this share: part[split] = [dW_gate d x f | dW_up d x f | dW_down f x d]
    if (wait.ok && wait(ofree, (count - 1) & 1)) {
      drain();
      float* out = p.part + (int64_t)split * 3 * D * p.f;
      const int64_t df = (int64_t)D * p.f;
      const int dr = m * 128 + row;
#pragma unroll
      for (int b = 0; b < PC; ++b) {
        bool pair;
        const int col = (int)place(b, &pair);
        if (!pair) {
          const int hcol = chunk * HC + col % HC;
          if (dr < D && hcol < p.f) {
            float* o = out + (col / HC) * df + (int64_t)dr * p.f + hcol;
            st16(o, pack(sum + b * 8, 0.f));
            st16(o + 4, pack(sum + b * 8 + 4, 0.f));
          }
        } else {
          const int r = D == 64 ? row - 64 : dr;  // d = 64: the lower half is dY's
          const int hcol = chunk * HC + col - (int)C::kAcc2;
          if (r >= 0 && hcol < p.f) {
            float* o = out + 2 * df + (int64_t)hcol * D + r;
#pragma unroll
            for (int e = 0; e < 8; ++e) o[(int64_t)e * D] = sum[b * 8 + e];
          }
        }
      }
    }
  }
  fence_before_sync();
  __syncthreads();
  if (warp == 2) tmem_dealloc(tmem, 512);
}

// out[((c * 2 + w) * hc + j) * d + k] = W_w[k][c * hc + j] (W_0 = W_gate, W_1 = W_up; zero from f on): the
// weights of a chunk of hidden features as rows along d.  32 x 32 tiles through shared memory.
__global__ void __launch_bounds__(256) ffn_pack_weights(const __nv_bfloat16* __restrict__ Wg,
                                                        const __nv_bfloat16* __restrict__ Wu, int d, int f, int hc,
                                                        __nv_bfloat16* __restrict__ out) {
  pdl_begin();
  __shared__ __nv_bfloat16 t[32][34];
  const __nv_bfloat16* W = blockIdx.z ? Wu : Wg;
  const int x = threadIdx.x & 31, y = threadIdx.x >> 5;
  const int h0 = blockIdx.x * 32, k0 = blockIdx.y * 32;
#pragma unroll
  for (int r = y; r < 32; r += 8) t[r][x] = h0 + x < f ? W[(int64_t)(k0 + r) * f + h0 + x] : __float2bfloat16(0.f);
  __syncthreads();
#pragma unroll
  for (int r = y; r < 32; r += 8) {
    const int h = h0 + r, c = h / hc, j = h % hc;
    out[((int64_t)(c * 2 + blockIdx.z) * hc + j) * d + k0 + x] = t[x][r];
  }
}

// out = the shares' sums in order: 32 float4 columns x 8 runs of shares a block, then the runs in order.
__global__ void __launch_bounds__(256) ffn_sum_shares_kernel(const float* __restrict__ part, int splits, int64_t df,
                                                      float* __restrict__ o0, float* __restrict__ o1,
                                                      float* __restrict__ o2) {
  pdl_begin();
  __shared__ float4 red[8][32];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int64_t total = 3 * df, c = ((int64_t)blockIdx.x * 32 + lane) * 4;
  float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
  if (c < total) {
#pragma unroll 4
    for (int k = splits * w / 8; k < splits * (w + 1) / 8; ++k) {
      const float4 v = *reinterpret_cast<const float4*>(part + k * total + c);
      s.x += v.x;
      s.y += v.y;
      s.z += v.z;
      s.w += v.w;
    }
  }
  red[w][lane] = s;
  __syncthreads();
  if (w > 0 || c >= total) return;
  for (int k = 1; k < 8; ++k) {
    const float4 v = red[k][lane];
    s.x += v.x;
    s.y += v.y;
    s.z += v.z;
    s.w += v.w;
  }
  float* o = c < df ? o0 : c < 2 * df ? o1 : o2;
  *reinterpret_cast<float4*>(o + c % df) = s;
}

// ---------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------
template <int D, int kAct>
hg_status dx_t(const hg_ffn_params* w, const void* X, int64_t n, const void* dY, void* dX, cudaStream_t s) {
  using C = DxCfg<D>;
  static bool done = false;
  if (!done) {
    HG_CUDA(cudaFuncSetAttribute(ffn_dx_tc_kernel<D, kAct>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem));
    done = true;
  }
  CUtensorMap tm_X, tm_dY, tm_G, tm_U, tm_W, tm_dX;
  HG_TRY(make_tmap_bf16(&tm_X, X, (uint64_t)n, D, kRows));
  HG_TRY(make_tmap_bf16(&tm_dY, dY, (uint64_t)n, D, kRows));
  HG_TRY(make_tmap_bf16(&tm_G, w->W_gate, D, (uint64_t)w->f, C::PR));
  HG_TRY(make_tmap_bf16(&tm_U, w->W_up, D, (uint64_t)w->f, C::PR));
  HG_TRY(make_tmap_bf16(&tm_W, w->W_down, (uint64_t)w->f, D, C::HC));
  HG_TRY(make_tmap_bf16(&tm_dX, dX, (uint64_t)n, D, kRows));
  DxP p{n, (int)ceil_div(w->f, C::HC), ceil_div(n, kRows), w->residual != 0, device_status_ptr()};
  return launch("ffn_dx_tc", ffn_dx_tc_kernel<D, kAct>, dim3((unsigned)std::min<int64_t>(p.tiles, kSms)),
                dim3(kThreads), C::kSmem, s, tm_X, tm_dY, tm_G, tm_U, tm_W, tm_dX, p);
}

int wg_chunk(int d) { return d == 256 ? WgCfg<256>::HC : WgCfg<128>::HC; }

// Shares of the row tiles: the count that makes the longest SM's work shortest (whole waves of chunks x shares).
int wg_splits(int64_t n, int d, int f) {
  const int64_t tiles = ceil_div(n, kRows), chunks = ceil_div(f, wg_chunk(d));
  int64_t best = 1, best_cost = INT64_MAX;
  for (int64_t sp = 1; sp <= std::min<int64_t>(tiles, kSms); ++sp) {
    // a CTA's fixed cost (weights in, gradients out) is about four tiles' time
    const int64_t cost = ceil_div(chunks * sp, kSms) * (ceil_div(tiles, sp) + 4);
    if (cost < best_cost) {
      best = sp;
      best_cost = cost;
    }
  }
  return (int)best;
}

struct WgLayout {
  void* Wt;
  float* part;
};
void carve_wg(void* scratch, const hg_ffn_params* w, int64_t n, WgLayout* L, size_t* bytes) {
  Carve k(scratch);
  const int hc = wg_chunk(w->d);
  L->Wt = k.take<__nv_bfloat16>((size_t)ceil_div(w->f, hc) * 2 * hc * w->d);
  L->part = k.take<float>((size_t)wg_splits(std::max<int64_t>(n, 1), w->d, w->f) * 3 * w->d * w->f);
  if (bytes) *bytes = k.used;
}

template <int D, int kAct>
hg_status wg_t(const hg_ffn_params* w, const void* X, int64_t n, const void* dY, const hg_ffn_grads* g,
               const WgLayout& L, cudaStream_t s) {
  using C = WgCfg<D>;
  static bool done = false;
  if (!done) {
    HG_CUDA(cudaFuncSetAttribute(ffn_wgrad_tc_kernel<D, kAct>, cudaFuncAttributeMaxDynamicSharedMemorySize, C::kSmem));
    done = true;
  }
  const int chunks = (int)ceil_div(w->f, C::HC), splits = wg_splits(n, D, w->f);
  HG_TRY(launch("ffn_pack_weights", ffn_pack_weights, dim3(chunks * C::HC / 32, D / 32, 2), dim3(256), 0, s,
                (const __nv_bfloat16*)w->W_gate, (const __nv_bfloat16*)w->W_up, D, w->f, C::HC, (__nv_bfloat16*)L.Wt));
  CUtensorMap tm_X, tm_dY, tm_Wt, tm_W;
  HG_TRY(make_tmap_bf16(&tm_X, X, (uint64_t)n, D, kRows));
  HG_TRY(make_tmap_bf16(&tm_dY, dY, (uint64_t)n, D, kRows));
  HG_TRY(make_tmap_bf16(&tm_Wt, L.Wt, (uint64_t)chunks * C::N2, D, C::N2));
  HG_TRY(make_tmap_bf16(&tm_W, w->W_down, (uint64_t)w->f, D, C::HC));
  WgP p{n, ceil_div(n, kRows), w->f, splits, chunks, L.part, device_status_ptr()};
  HG_TRY(launch("ffn_wgrad_tc", ffn_wgrad_tc_kernel<D, kAct>, dim3((unsigned)(chunks * splits)), dim3(kThreads),
                C::kSmem, s, tm_X, tm_dY, tm_Wt, tm_W, p));
  const int64_t df = (int64_t)D * w->f;
  return ffn_sum_shares(L.part, splits, df, g, s);
}

template <int D, int kAct>
hg_status bwd_t(const hg_ffn_params* w, const void* X, int64_t n, const void* dY, void* dX, const hg_ffn_grads* g,
                void* scratch, cudaStream_t s) {
  if (dX) HG_TRY((dx_t<D, kAct>(w, X, n, dY, dX, s)));
  if (!g) return HG_OK;
  WgLayout L;
  carve_wg(scratch, w, n, &L, nullptr);
  return wg_t<D, kAct>(w, X, n, dY, g, L, s);
}

template <int D>
hg_status bwd_d(const hg_ffn_params* w, const void* X, int64_t n, const void* dY, void* dX, const hg_ffn_grads* g,
                void* scratch, cudaStream_t s) {
  if (w->act == HG_ACT_RELU) return bwd_t<D, HG_ACT_RELU>(w, X, n, dY, dX, g, scratch, s);
  if (w->act == HG_ACT_GELU_TANH) return bwd_t<D, HG_ACT_GELU_TANH>(w, X, n, dY, dX, g, scratch, s);
  if (w->act == HG_ACT_SILU) return bwd_t<D, HG_ACT_SILU>(w, X, n, dY, dX, g, scratch, s);
  return bwd_t<D, HG_ACT_NONE>(w, X, n, dY, dX, g, scratch, s);
}

}  // namespace

hg_status ffn_sum_shares(const float* part, int splits, int64_t df, const hg_ffn_grads* g, cudaStream_t s) {
  return launch("ffn_sum_shares", ffn_sum_shares_kernel, dim3((unsigned)ceil_div(3 * df, 128)), dim3(256), 0, s, part,
                splits, df, g->dW_gate, g->dW_up, g->dW_down);
}

size_t ffn_bwd_tc_scratch(const hg_ffn_params* w, int64_t n) {
  WgLayout L;
  size_t bytes = 0;
  carve_wg(nullptr, w, n, &L, &bytes);
  return bytes;
}

hg_status ffn_bwd_tc(const hg_ffn_params* w, const void* X, int64_t n, const void* dY, void* dX, const hg_ffn_grads* g,
                     void* scratch, cudaStream_t s) {
  if (w->d == 64) return bwd_d<64>(w, X, n, dY, dX, g, scratch, s);
  if (w->d == 128) return bwd_d<128>(w, X, n, dY, dX, g, scratch, s);
  return bwd_d<256>(w, X, n, dY, dX, g, scratch, s);
}

}  // namespace hg
