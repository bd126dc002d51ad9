// Gated feed-forward block: entry points and the CUDA-core path (fp32 storage).
//
//   G = X W_gate, U = X W_up, H = act(G) * U, Y = H W_down (+ X)
//   dH = dY W_down^T, dG = dH * U * act'(G), dU = dH * act(G)
//   dX = dG W_gate^T + dU W_up^T (+ dY), dW_gate = X^T dG, dW_up = X^T dU, dW_down = H^T dY
//
// CUDA-core path: 128 x 64 tiles, 8 x 4 results a thread, operands in shared memory by k; the two
// projections (and dH) share a pass over k, their gate is applied to the sums in registers, and H, dG and dU
// go to scratch.  The weights' gradients split the rows; the splits are added in order.  Bound by the FMA rate:
// 100003 rows, d = 128, f = 384: forward 575 us (51 TFLOP/s), backward 1765 us (45 TFLOP/s), where loads that wait
// for the products took 652 and 2251 us.
#include <algorithm>

#include "ffn_kernels.cuh"
#include "ffn_tc.cuh"
#include "row_sets.cuh"

namespace hg {

namespace {

constexpr int kBm = 128, kBn = 64, kBk = 16, kThr = 256;
constexpr int kSms = 152;
constexpr int kMaxF = 16384;

// One operand as the tile loaders see it: element (r, c) at p[r * ld + c], rows r < nr, columns c < nc.
struct Mat {
  const float* p;
  int64_t ld, nr, nc;
};

// A tile dst[k][x], kBk of k and X of x (row stride X + 4), of an operand whose rows are x and columns k (kByRow) or
// whose rows are k and columns x.  Zero outside.  nr, nc and the starts are such that four neighbouring columns are
// all inside or all outside.  fetch loads a thread's pieces, put lays them in shared memory: the loads of the next
// tile run while this one is multiplied.
template <int X, bool kByRow>
struct Piece {
  static constexpr int PER = X * kBk / 4 / kThr;
  float4 v[PER];
  __device__ __forceinline__ void fetch(const Mat& a, int64_t x0, int64_t k0) {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int e = threadIdx.x + i * kThr;
      const int r = kByRow ? e / (kBk / 4) : e / (X / 4);
      const int c = (kByRow ? e % (kBk / 4) : e % (X / 4)) * 4;
      const int64_t row = (kByRow ? x0 : k0) + r, col = (kByRow ? k0 : x0) + c;
      v[i] = make_float4(0.f, 0.f, 0.f, 0.f);
      if (row < a.nr && col < a.nc) v[i] = *reinterpret_cast<const float4*>(a.p + row * a.ld + col);
    }
  }
  __device__ __forceinline__ void put(float* dst) const {
#pragma unroll
    for (int i = 0; i < PER; ++i) {
      const int e = threadIdx.x + i * kThr;
      const int r = kByRow ? e / (kBk / 4) : e / (X / 4);
      const int c = (kByRow ? e % (kBk / 4) : e % (X / 4)) * 4;
      if (kByRow) {
        dst[(c + 0) * (X + 4) + r] = v[i].x;
        dst[(c + 1) * (X + 4) + r] = v[i].y;
        dst[(c + 2) * (X + 4) + r] = v[i].z;
        dst[(c + 3) * (X + 4) + r] = v[i].w;
      } else {
        *reinterpret_cast<float4*>(dst + r * (X + 4) + c) = v[i];
      }
    }
  }
};

// A thread's 8 x 4 sums; rows 2 i and 2 i + 1 lie in one register pair, for the FMA of two.
struct Acc {
  float2 v[4][4];
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
      for (int j = 0; j < 4; ++j) v[i][j] = make_float2(0.f, 0.f);
  }
  __device__ __forceinline__ float at(int i, int j) const { return i & 1 ? v[i >> 1][j].y : v[i >> 1][j].x; }
};

// thread (ty, tx) holds rows ty * 4 + {0..3}, 64 + ty * 4 + {0..3} and columns tx * 4 + {0..3}
__device__ __forceinline__ int acc_row(int i) { return (i < 4 ? 0 : 64) + (threadIdx.x / 16) * 4 + (i & 3); }

__device__ __forceinline__ void fma2(float2& c, float2 a, float b) {
  asm("{\n\t.reg .b64 x, y, z;\n\t"
      "mov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %4};\n\tmov.b64 z, {%0, %1};\n\t"
      "fma.rn.f32x2 z, x, y, z;\n\tmov.b64 {%0, %1}, z;\n\t}"
      : "+f"(c.x), "+f"(c.y)
      : "f"(a.x), "f"(a.y), "f"(b));
}

// acc += A B, and acc2 += A B2: an operand of both is read once
__device__ __forceinline__ void mul(const float* A, const float* B, Acc& acc, const float* B2 = nullptr,
                                    Acc* acc2 = nullptr) {
  const int ty = threadIdx.x / 16, tx = threadIdx.x % 16;
#pragma unroll
  for (int k = 0; k < kBk; ++k) {
    const float4 a0 = *reinterpret_cast<const float4*>(A + k * (kBm + 4) + ty * 4);
    const float4 a1 = *reinterpret_cast<const float4*>(A + k * (kBm + 4) + 64 + ty * 4);
    const float2 av[4] = {{a0.x, a0.y}, {a0.z, a0.w}, {a1.x, a1.y}, {a1.z, a1.w}};
#pragma unroll
    for (int t = 0; t < 2; ++t) {
      if (t && !B2) break;
      const float4 b = *reinterpret_cast<const float4*>((t ? B2 : B) + k * (kBn + 4) + tx * 4);
      const float bv[4] = {b.x, b.y, b.z, b.w};
      Acc& c = t ? *acc2 : acc;
#pragma unroll
      for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) fma2(c.v[i][j], av[i], bv[j]);
    }
  }
}

// H = act(X W_gate) * (X W_up), a tile a block, the column tiles of a row tile one after another; with kBwd also
// dH = dY W_down^T, and dG, dU.
template <int kAct, bool kBwd>
__global__ void __launch_bounds__(kThr, kBwd ? 1 : 2)
    ffn_hidden_simt(Mat X, Mat Wg, Mat Wu, Mat dY, Mat Wd, float* __restrict__ H, float* __restrict__ dG,
                    float* __restrict__ dU) {
  pdl_begin();
  __shared__ __align__(16) float As[kBk * (kBm + 4)], Bs[kBk * (kBn + 4)], Cs[kBk * (kBn + 4)];
  __shared__ __align__(16) float Ds[kBwd ? kBk * (kBm + 4) : 4], Es[kBwd ? kBk * (kBn + 4) : 4];
  const int ctiles = (int)((Wg.nc + kBn - 1) / kBn);
  const int64_t r0 = (int64_t)(blockIdx.x / ctiles) * kBm, c0 = (int64_t)(blockIdx.x % ctiles) * kBn;
  Acc g, u, h;
  g.zero();
  u.zero();
  h.zero();
  Piece<kBm, true> pa, pd;
  Piece<kBn, false> pb, pc;
  Piece<kBn, true> pe;
  auto fetch = [&](int64_t k0) {
    pa.fetch(X, r0, k0);
    pb.fetch(Wg, c0, k0);
    pc.fetch(Wu, c0, k0);
    if (kBwd) {
      pd.fetch(dY, r0, k0);
      pe.fetch(Wd, c0, k0);
    }
  };
  fetch(0);
  for (int64_t k0 = 0; k0 < X.nc; k0 += kBk) {
    __syncthreads();
    pa.put(As);
    pb.put(Bs);
    pc.put(Cs);
    if (kBwd) {
      pd.put(Ds);
      pe.put(Es);
    }
    __syncthreads();
    if (k0 + kBk < X.nc) fetch(k0 + kBk);
    mul(As, Bs, g, Cs, &u);
    if (kBwd) mul(Ds, Es, h);
  }
  const int64_t col = c0 + threadIdx.x % 16 * 4;
  if (col >= Wg.nc) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t row = r0 + acc_row(i);
    if (row >= X.nr) continue;
    float hv[4], gv[4], uv[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      if (kBwd) {
        float d;
        const float a = gate_grad<kAct>(g.at(i, j), &d);
        hv[j] = a * u.at(i, j);
        gv[j] = h.at(i, j) * u.at(i, j) * d;
        uv[j] = h.at(i, j) * a;
      } else {
        hv[j] = gate<kAct>(g.at(i, j)) * u.at(i, j);
      }
    }
    const int64_t at = row * Wg.nc + col;
    *reinterpret_cast<float4*>(H + at) = make_float4(hv[0], hv[1], hv[2], hv[3]);
    if (kBwd) {
      *reinterpret_cast<float4*>(dG + at) = make_float4(gv[0], gv[1], gv[2], gv[3]);
      *reinterpret_cast<float4*>(dU + at) = make_float4(uv[0], uv[1], uv[2], uv[3]);
    }
  }
}

// out = A B (+ A2 B2) (+ add): the second product when A2.p is set; kTransB: B given by its transpose.
template <bool kTransB>
__global__ void __launch_bounds__(kThr, 3) ffn_out_simt(Mat A, Mat B, Mat A2, Mat B2, const float* add,
                                                     float* __restrict__ out, int64_t nc) {
  pdl_begin();
  __shared__ __align__(16) float As[kBk * (kBm + 4)], Bs[kBk * (kBn + 4)];
  const int ctiles = (int)((nc + kBn - 1) / kBn);
  const int64_t r0 = (int64_t)(blockIdx.x / ctiles) * kBm, c0 = (int64_t)(blockIdx.x % ctiles) * kBn;
  Acc acc;
  acc.zero();
  Piece<kBm, true> pa;
  Piece<kBn, kTransB> pb;
  const int64_t steps = (A.nc + kBk - 1) / kBk, all = A2.p ? 2 * steps : steps;
  auto fetch = [&](int64_t i) {
    const bool second = i >= steps;
    const int64_t k0 = (second ? i - steps : i) * kBk;
    pa.fetch(second ? A2 : A, r0, k0);
    pb.fetch(second ? B2 : B, c0, k0);
  };
  fetch(0);
  for (int64_t i = 0; i < all; ++i) {
    __syncthreads();
    pa.put(As);
    pb.put(Bs);
    __syncthreads();
    if (i + 1 < all) fetch(i + 1);
    mul(As, Bs, acc);
  }
  const int64_t col = c0 + threadIdx.x % 16 * 4;
  if (col >= nc) return;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t row = r0 + acc_row(i);
    if (row >= A.nr) continue;
    const int64_t at = row * nc + col;
    const float4 x = add ? *reinterpret_cast<const float4*>(add + at) : make_float4(0.f, 0.f, 0.f, 0.f);
    *reinterpret_cast<float4*>(out + at) =
        make_float4(acc.at(i, 0) + x.x, acc.at(i, 1) + x.y, acc.at(i, 2) + x.z, acc.at(i, 3) + x.w);
  }
}

// part[blockIdx.y] = [X^T dG | X^T dU | H^T dY] over the split's rows, a tile a block.
__global__ void __launch_bounds__(kThr, 3) ffn_wgrad_simt(Mat X, Mat dG, Mat dU, Mat H, Mat dY, int64_t rows,
                                                       float* __restrict__ part) {
  pdl_begin();
  __shared__ __align__(16) float As[kBk * (kBm + 4)], Bs[kBk * (kBn + 4)];
  const int64_t d = X.nc, f = H.nc;
  const int tiles = (int)((d + kBm - 1) / kBm * ((f + kBn - 1) / kBn));  // of each of the first two
  const int which = min((int)blockIdx.x / tiles, 2), x = blockIdx.x - which * tiles;
  Mat A = which < 2 ? X : H, B = which == 0 ? dG : which == 1 ? dU : dY;
  const int ct = (int)((B.nc + kBn - 1) / kBn);
  const int64_t m0 = (int64_t)(x / ct) * kBm, c0 = (int64_t)(x % ct) * kBn;
  const int64_t k1 = min(X.nr, (int64_t)(blockIdx.y + 1) * rows);
  A.nr = B.nr = k1;
  Acc acc;
  acc.zero();
  Piece<kBm, false> pa;
  Piece<kBn, false> pb;
  int64_t k0 = (int64_t)blockIdx.y * rows;
  pa.fetch(A, m0, k0);
  pb.fetch(B, c0, k0);
  for (; k0 < k1; k0 += kBk) {
    __syncthreads();
    pa.put(As);
    pb.put(Bs);
    __syncthreads();
    if (k0 + kBk < k1) {
      pa.fetch(A, m0, k0 + kBk);
      pb.fetch(B, c0, k0 + kBk);
    }
    mul(As, Bs, acc);
  }
  const int64_t col = c0 + threadIdx.x % 16 * 4;
  if (col >= B.nc) return;
  float* out = part + (blockIdx.y * 3 + which) * d * f;
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const int64_t m = m0 + acc_row(i);
    if (m < A.nc)
      *reinterpret_cast<float4*>(out + m * B.nc + col) =
          make_float4(acc.at(i, 0), acc.at(i, 1), acc.at(i, 2), acc.at(i, 3));
  }
}

// ---------------------------------------------------------------------------------------------
// host
// ---------------------------------------------------------------------------------------------
// Splits of the rows: tiles enough for two rounds of three blocks an SM, none shorter than 128 rows.
int wg_tiles(int d, int f) {
  return (int)(2 * ceil_div(d, kBm) * ceil_div(f, kBn) + ceil_div(f, kBm) * ceil_div(d, kBn));
}
int wg_splits(int64_t n, int d, int f) {
  return (int)std::max<int64_t>(1, std::min<int64_t>(ceil_div(6 * kSms, wg_tiles(d, f)), n / 128));
}

struct FfnLayout {
  float* H;
  float* dG;
  float* dU;
  float* part;
};

void carve_simt(void* scratch, const hg_ffn_params* p, int64_t n, bool bwd, FfnLayout* L, size_t* bytes) {
  Carve k(scratch);
  const size_t nf = (size_t)std::max<int64_t>(n, 1) * p->f;
  *L = FfnLayout{};
  L->H = k.take<float>(nf);
  if (bwd) {
    L->dG = k.take<float>(nf);
    L->dU = k.take<float>(nf);
    const int sp = wg_splits(n, p->d, p->f);
    L->part = k.take<float>((size_t)sp * 3 * p->d * p->f);
  }
  if (bytes) *bytes = k.used;
}

template <int kAct, bool kBwd>
hg_status hidden(const hg_ffn_params* p, const void* X, int64_t n, const void* dY, const FfnLayout& L, cudaStream_t s) {
  const int64_t d = p->d, f = p->f;
  const Mat x{(const float*)X, d, n, d}, g{(const float*)p->W_gate, f, d, f}, u{(const float*)p->W_up, f, d, f},
      dy{(const float*)dY, d, n, d}, w{(const float*)p->W_down, d, f, d};
  return launch(kBwd ? "ffn_hidden_bwd_simt" : "ffn_hidden_simt", ffn_hidden_simt<kAct, kBwd>,
                dim3((unsigned)(ceil_div(f, kBn) * ceil_div(n, kBm))), dim3(kThr), 0, s, x, g, u, dy, w, L.H,
                L.dG, L.dU);
}

template <bool kBwd>
hg_status hidden_act(const hg_ffn_params* p, const void* X, int64_t n, const void* dY, const FfnLayout& L,
                     cudaStream_t s) {
  if (p->act == HG_ACT_RELU) return hidden<HG_ACT_RELU, kBwd>(p, X, n, dY, L, s);
  if (p->act == HG_ACT_GELU_TANH) return hidden<HG_ACT_GELU_TANH, kBwd>(p, X, n, dY, L, s);
  if (p->act == HG_ACT_SILU) return hidden<HG_ACT_SILU, kBwd>(p, X, n, dY, L, s);
  return hidden<HG_ACT_NONE, kBwd>(p, X, n, dY, L, s);
}

hg_status fwd_simt(const hg_ffn_params* p, const void* X, int64_t n, void* Y, const FfnLayout& L, cudaStream_t s) {
  const int64_t d = p->d, f = p->f;
  HG_TRY((hidden_act<false>(p, X, n, nullptr, L, s)));
  const Mat h{L.H, f, n, f}, w{(const float*)p->W_down, d, f, d}, none{};
  return launch("ffn_out_simt", ffn_out_simt<false>, dim3((unsigned)(ceil_div(d, kBn) * ceil_div(n, kBm))), dim3(kThr),
                0, s, h, w, none, w, (const float*)(p->residual ? X : nullptr), (float*)Y, d);
}

hg_status bwd_simt(const hg_ffn_params* p, const void* X, int64_t n, const void* dY, void* dX, const hg_ffn_grads* g,
                   const FfnLayout& L, cudaStream_t s) {
  const int64_t d = p->d, f = p->f;
  HG_TRY((hidden_act<true>(p, X, n, dY, L, s)));
  if (dX) {
    const Mat a{L.dG, f, n, f}, a2{L.dU, f, n, f}, b{(const float*)p->W_gate, f, d, f},
        b2{(const float*)p->W_up, f, d, f};
    HG_TRY(launch("ffn_dx_simt", ffn_out_simt<true>, dim3((unsigned)(ceil_div(d, kBn) * ceil_div(n, kBm))), dim3(kThr),
                  0, s, a, b, a2, b2, (const float*)(p->residual ? dY : nullptr), (float*)dX, d));
  }
  if (!g) return HG_OK;
  const int sp = wg_splits(n, p->d, p->f);
  const Mat x{(const float*)X, d, n, d}, dg{L.dG, f, n, f}, du{L.dU, f, n, f}, h{L.H, f, n, f},
      dy{(const float*)dY, d, n, d};
  HG_TRY(launch("ffn_wgrad_simt", ffn_wgrad_simt, dim3((unsigned)wg_tiles(p->d, p->f), (unsigned)sp), dim3(kThr), 0, s,
                x, dg, du, h, dy, (int64_t)align_up((size_t)ceil_div(n, sp), kBk), L.part));
  return ffn_sum_shares(L.part, sp, d * f, g, s);
}

size_t scratch_bytes(const hg_ffn_params* p, int64_t n, bool bwd) {
  if (p->dtype == HG_BF16) return bwd ? ffn_bwd_tc_scratch(p, n) : 0;
  FfnLayout L;
  size_t bytes = 0;
  carve_simt(nullptr, p, n, bwd, &L, &bytes);
  return bytes;
}

hg_status check_params(const hg_ffn_params* p, int64_t n) {
  HG_REQUIRE(p != nullptr, "params must be non-null");
  if (!(p->d == 64 || p->d == 128 || p->d == 256) || !(p->dtype == HG_F32 || p->dtype == HG_BF16)) {
    set_error("unsupported d=%d / dtype=%d", p->d, (int)p->dtype);
    return HG_ERR_UNSUPPORTED;
  }
  HG_REQUIRE(p->f >= 8 && p->f <= kMaxF && p->f % 8 == 0, "f must be a multiple of 8 in [8, %d]", kMaxF);
  HG_REQUIRE(p->act == HG_ACT_RELU || p->act == HG_ACT_GELU_TANH || p->act == HG_ACT_NONE || p->act == HG_ACT_SILU,
             "unknown activation %d", (int)p->act);
  HG_REQUIRE(n >= 0 && n < (int64_t(1) << 31) && ceil_div(n, kBm) * ceil_div(p->f, kBn) < (int64_t(1) << 31),
             "n must be in [0, 2^31), n * f below 2^44");
  return HG_OK;
}

// Two arrays of n x d values share no byte.
hg_status check_apart(const hg_ffn_params* p, int64_t n, const void* out, const void* in, const char* names) {
  HG_REQUIRE(!shared(out, in, (size_t)n * p->d * (p->dtype == HG_BF16 ? 2 : 4)), "%s must not overlap", names);
  return HG_OK;
}

hg_status check_weights(const hg_ffn_params* p) {
  HG_REQUIRE(p->W_gate && p->W_up && p->W_down, "every weight pointer must be non-null");
  HG_REQUIRE((((uintptr_t)p->W_gate | (uintptr_t)p->W_up | (uintptr_t)p->W_down) & 15) == 0,
             "weights must be 16-byte aligned");
  return HG_OK;
}

}  // namespace
}  // namespace hg

using namespace hg;

extern "C" hg_status hg_ffn_workspace_size(const hg_ffn_params* params, int64_t n, size_t* fwd_bytes,
                                           size_t* bwd_bytes) {
  clear_error();
  HG_REQUIRE(fwd_bytes && bwd_bytes, "fwd_bytes and bwd_bytes must be non-null");
  HG_TRY(check_params(params, n));
  *fwd_bytes = scratch_bytes(params, n, false);
  *bwd_bytes = scratch_bytes(params, n, true);
  return HG_OK;
}

extern "C" hg_status hg_ffn_fwd(const hg_ffn_params* params, const void* X, int64_t n, void* Y, void* scratch,
                                hg_stream stream) {
  clear_error();
  HG_TRY(device_guard());
  HG_TRY(check_params(params, n));
  HG_TRY(check_weights(params));
  if (n == 0) return HG_OK;
  HG_REQUIRE(X && Y && (scratch || params->dtype == HG_BF16), "X, Y and scratch must be non-null");
  HG_REQUIRE((((uintptr_t)X | (uintptr_t)Y) & 15) == 0, "X and Y must be 16-byte aligned");
  HG_TRY(check_apart(params, n, Y, X, "Y and X"));
  HG_REQUIRE(((uintptr_t)scratch & 255) == 0, "scratch must be 256-byte aligned");
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (params->dtype == HG_BF16) return ffn_fwd_tc(params, X, n, Y, s);
  FfnLayout L;
  carve_simt(scratch, params, n, false, &L, nullptr);
  return fwd_simt(params, X, n, Y, L, s);
}

extern "C" hg_status hg_ffn_bwd(const hg_ffn_params* params, const void* X, int64_t n, const void* dY, void* dX,
                                const hg_ffn_grads* grads, void* scratch, hg_stream stream) {
  clear_error();
  HG_TRY(device_guard());
  HG_TRY(check_params(params, n));
  HG_TRY(check_weights(params));
  HG_REQUIRE(!grads || (grads->dW_gate && grads->dW_up && grads->dW_down), "every gradient pointer must be non-null");
  HG_REQUIRE(!grads || (((uintptr_t)grads->dW_gate | (uintptr_t)grads->dW_up | (uintptr_t)grads->dW_down) & 15) == 0,
             "gradients must be 16-byte aligned");
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const size_t wbytes = sizeof(float) * (size_t)params->d * params->f;
  HG_REQUIRE(!grads || !(shared(grads->dW_gate, grads->dW_up, wbytes) ||
                         shared(grads->dW_gate, grads->dW_down, wbytes) ||
                         shared(grads->dW_up, grads->dW_down, wbytes)),
             "the gradients must not overlap one another");
  if (n == 0) {
    if (grads) {
      HG_CUDA(cudaMemsetAsync(grads->dW_gate, 0, wbytes, s));
      HG_CUDA(cudaMemsetAsync(grads->dW_up, 0, wbytes, s));
      HG_CUDA(cudaMemsetAsync(grads->dW_down, 0, wbytes, s));
    }
    return HG_OK;
  }
  HG_REQUIRE(X && dY, "X and dY must be non-null");
  HG_REQUIRE(scratch || (params->dtype == HG_BF16 && !grads), "scratch must be non-null");
  HG_REQUIRE((((uintptr_t)X | (uintptr_t)dY | (uintptr_t)dX) & 15) == 0, "X, dY and dX must be 16-byte aligned");
  if (dX) {
    HG_TRY(check_apart(params, n, dX, X, "dX and X"));
    HG_TRY(check_apart(params, n, dX, dY, "dX and dY"));
  }
  HG_REQUIRE(((uintptr_t)scratch & 255) == 0, "scratch must be 256-byte aligned");
  if (!dX && !grads) return HG_OK;
  if (params->dtype == HG_BF16) return ffn_bwd_tc(params, X, n, dY, dX, grads, scratch, s);
  FfnLayout L;
  carve_simt(scratch, params, n, true, &L, nullptr);
  return bwd_simt(params, X, n, dY, dX, grads, L, s);
}
