// Norm and rotation of query and key heads in one pass, forward and backward.
//
//   r = 1 / sqrt(mean(x^2) + eps), u = x r, y = u * gamma, then each pair (a, b) of y is turned by the
//   angle w = pos base^(-2 i / rot):  (a cos w - b sin w, b cos w + a sin w)
//   backward: g = dy turned by -w;  dgamma = sum over rows of g u;  with c = g gamma:
//             dx = r (c - u mean(c u))
//
// The angle is taken in turns as a 64-bit fraction: pos times the frequency in units of 2^-64 turns,
// modulo 2^64, leaves out the whole turns exactly.  The frequency itself is rounded to such a unit (3 of them off at
// most with 80-bit host arithmetic), so the angle is off by up to |pos| 2^-59 rad: nothing for days or seconds, all of
// it for nanoseconds since 1970.  The upper 32 bits as a signed number are the angle in (-1/2, 1/2] turns.
//
// A group of d_h / (2 V) lanes holds one head (V = values in 16 bytes): each lane two 16-byte pieces that
// contain both features of V pairs, so a turn needs no exchange and the norm is a shuffle over the group.
// A group keeps its head for the whole run (the grid's stride is a multiple of the row's heads), so the
// gain, its gradient's sum and the frequencies stay in registers.  The sines and cosines of a row are those of all its
// heads: neighbouring heads share them out and exchange them by shuffles (8 + 2 heads of 64, 300001 rows: 169 us by
// each for itself, 134 us).  Bound by HBM: a head is read once and written once (forward above 0.78 of the measured
// rate, 1000003 rows backward 0.86; fp32, 200001 rows of 4 + 2 heads of 64, exact sines: 0.88).
#include <algorithm>
#include <cmath>
#include <initializer_list>

#include "hg_internal.cuh"
#include "row_sets.cuh"

namespace hg {

namespace {

constexpr int kThreads = 256;
constexpr int kMaxHeads = 64;
constexpr int kSms = 152;

// CTAs of an SM (registers against rows in flight; bf16, 500003 rows of 4 + 4 heads of 32 forward: 2 104, 3 97, 4 101
// us; 1000003 rows backward: 1 355, 2 262, 3 532 us).  A run has no more of them, since a second wave would find a part
// of the SMs' room empty.  In bf16 up to 64 bytes of a lane then lie in local memory.
constexpr int resident(bool bwd) { return bwd ? 2 : 3; }

struct RotRows {
  const void* x;
  const void* dy;
  void* out;
  int64_t sx, sdy, sout;
};

struct RotArgs {
  RotRows q, k;
  const int64_t* pos;
  const void* gamma_q;
  const void* gamma_k;
  float* part;  // [grid][2][d_h] sums of the gains' gradients (backward)
  int64_t n;
  int hq, heads, rot;
  float eps;
  uint64_t freq[64];  // 2^64 base^(-2 i / rot) / (2 pi)
};

template <bool kExact>
__device__ __forceinline__ void turn_sincos(uint64_t phase, float* s, float* c) {
  const float t = (float)(int32_t)(phase >> 32) * 0x1p-32f;  // turns
  if (kExact) {
    sincospif(2.f * t, s, c);
  } else {
    // Below 2^-20 in all, far below half a bf16 step of a product with it: the functions 2^-21.2 on [-pi, pi], t
    // rounded to 24 bits 9.4e-8 rad, the constant 8.7e-8, the product 1.2e-7.
    const float w = 6.283185307f * t;
    *s = __sinf(w);
    *c = __cosf(w);
  }
}

template <typename T, int DH, bool kInter, bool kBwd, int K>
__global__ void __launch_bounds__(kThreads, resident(kBwd)) qkrot_kernel(const __grid_constant__ RotArgs a) {
  pdl_begin();
  constexpr int V = VecTraits<T>::kElems;
  constexpr int L = DH / (2 * V);
  constexpr int G = kThreads / L;
  constexpr bool kExact = sizeof(T) == 4;
  const int l = threadIdx.x % L, g = threadIdx.x / L;
  const int64_t groups = (int64_t)gridDim.x * G / a.heads * a.heads;
  const int64_t gid = (int64_t)blockIdx.x * G + g;
  const int r = (int)(gid % a.heads);
  const bool is_q = r < a.hq;
  const int h = is_q ? r : r - a.hq;
  const RotRows rows = is_q ? a.q : a.k;
  // this lane's two pieces, and its V pairs' frequencies
  int o0, o1, f0;
  bool turned;
  if (kInter) {
    o0 = l * 2 * V;
    o1 = o0 + V;
    f0 = l * V;
    turned = o0 < a.rot;
  } else {
    const int nr = a.rot / (2 * V);
    turned = l < nr;
    o0 = turned ? l * V : a.rot + (l - nr) * 2 * V;
    o1 = turned ? a.rot / 2 + l * V : o0 + V;
    f0 = l * V;
  }
  // This lane's share of its V pairs: those e with e % K == j.  The K lanes that follow each other by L have the same
  // row and the same pairs.
  const int lane = threadIdx.x & 31, j = lane / L % K, first = lane - j * L;
  uint64_t fr[V / K];
  float gm[2 * V], acc[2 * V];
  const T* gamma = static_cast<const T*>(is_q ? a.gamma_q : a.gamma_k);
#pragma unroll
  for (int e = 0; e < V; ++e) {
    if (e % K == 0) {
      fr[e / K] = 0;
      if (turned) fr[e / K] = a.freq[f0 + e + j];
    }
    gm[e] = gamma ? to_f32(gamma[o0 + e]) : 1.f;
    gm[V + e] = gamma ? to_f32(gamma[o1 + e]) : 1.f;
    acc[e] = acc[V + e] = 0.f;
  }
  const int64_t step = groups / a.heads;
  const int64_t iters = (a.n + step - 1) / step;
  int64_t i = gid < groups ? gid / a.heads : a.n;
  // the next row's loads run ahead of this row's arithmetic
  uint4 v0, v1, w0, w1;
  int64_t p;
  auto fetch = [&]() {
    v0 = v1 = w0 = w1 = make_uint4(0, 0, 0, 0);
    p = 0;
    if (i < a.n) {
      const T* src = static_cast<const T*>(rows.x) + i * rows.sx + h * DH;
      v0 = ld16(src + o0);
      v1 = ld16(src + o1);
      if (kBwd) {
        const T* dsrc = static_cast<const T*>(rows.dy) + i * rows.sdy + h * DH;
        w0 = ld16(dsrc + o0);
        w1 = ld16(dsrc + o1);
      }
      p = a.pos ? a.pos[i] : i;
    }
  };
  fetch();
  for (int64_t it = 0; it < iters; ++it) {
    const int64_t row = i;
    const uint64_t at = (uint64_t)p;
    float x[2 * V], y[2 * V];
    unpack(v0, x, T());
    unpack(v1, x + V, T());
    if (kBwd) {
      unpack(w0, y, T());
      unpack(w1, y + V, T());
    }
    i += step;
    fetch();
    float ss = 0.f;
#pragma unroll
    for (int e = 0; e < 2 * V; ++e) ss = fmaf(x[e], x[e], ss);
#pragma unroll
    for (int o = L / 2; o > 0; o >>= 1) ss += __shfl_xor_sync(0xffffffffu, ss, o);
    const float rn = rsqrtf(ss * (1.f / DH) + a.eps);
    if (!kBwd) {
#pragma unroll
      for (int e = 0; e < 2 * V; ++e) y[e] = x[e] * rn * gm[e];
    }
    if (a.rot) {
      float sn[V / K], cs[V / K];
#pragma unroll
      for (int e = 0; e < V / K; ++e) turn_sincos<kExact>(at * fr[e], &sn[e], &cs[e]);
#pragma unroll
      for (int e = 0; e < V; ++e) {
        float s = sn[e / K], c = cs[e / K];
        if (K > 1) {
          s = __shfl_sync(0xffffffffu, s, first + e % K * L);
          c = __shfl_sync(0xffffffffu, c, first + e % K * L);
        }
        if (kBwd) s = -s;
        if (turned) {
          const int ia = kInter ? 2 * e : e, ib = kInter ? 2 * e + 1 : V + e;
          const float ya = y[ia], yb = y[ib];
          y[ia] = ya * c - yb * s;
          y[ib] = yb * c + ya * s;
        }
      }
    }
    if (kBwd) {
      float m = 0.f;
#pragma unroll
      for (int e = 0; e < 2 * V; ++e) {
        const float u = x[e] * rn;
        acc[e] = fmaf(y[e], u, acc[e]);
        y[e] *= gm[e];
        m = fmaf(y[e], u, m);
        x[e] = u;
      }
#pragma unroll
      for (int o = L / 2; o > 0; o >>= 1) m += __shfl_xor_sync(0xffffffffu, m, o);
      m *= 1.f / DH;
#pragma unroll
      for (int e = 0; e < 2 * V; ++e) y[e] = rn * (y[e] - x[e] * m);
    }
    if (row < a.n) {
      T* dst = static_cast<T*>(rows.out) + row * rows.sout + h * DH;
      st16(dst + o0, pack(y, T()));
      st16(dst + o1, pack(y + V, T()));
    }
  }
  if (kBwd) {
    __shared__ float red[G][DH + 1];
    __shared__ int8_t kind[G];
#pragma unroll
    for (int e = 0; e < V; ++e) {
      red[g][o0 + e] = acc[e];
      red[g][o1 + e] = acc[V + e];
    }
    if (l == 0) kind[g] = gid >= groups ? 2 : is_q ? 0 : 1;
    __syncthreads();
    for (int c = threadIdx.x; c < 2 * DH; c += kThreads) {
      const int want = c / DH, col = c % DH;
      float s = 0.f;
      for (int j = 0; j < G; ++j)
        if (kind[j] == want) s += red[j][col];
      a.part[(int64_t)blockIdx.x * 2 * DH + c] = s;
    }
  }
}

// out_q[c], out_k[c] = the blocks' partial sums in order: eight threads a column, then their sums in order.
__global__ void __launch_bounds__(256) qkrot_gains(const float* __restrict__ part, int blocks, int dh,
                                                   float* __restrict__ out_q, float* __restrict__ out_k) {
  pdl_begin();
  __shared__ float red[8][33];
  const int lane = threadIdx.x & 31, w = threadIdx.x >> 5;
  const int c = blockIdx.x * 32 + lane;
  float s = 0.f;
#pragma unroll 8
  for (int b = w; b < blocks; b += 8) s += part[(int64_t)b * 2 * dh + c];
  red[w][lane] = s;
  __syncthreads();
  if (w == 0) {
    float t = 0.f;
    for (int j = 0; j < 8; ++j) t += red[j][lane];
    if (c < dh) {
      if (out_q) out_q[c] = t;
    } else if (out_k) {
      out_k[c - dh] = t;
    }
  }
}

// Blocks of a run: enough for every head of every row, at least one block per row's heads, at most a
// resident set.
int rot_grid(int64_t n, int heads, int dh, hg_dtype dt, bool bwd) {
  const int bytes = dt == HG_BF16 ? 2 : 4;
  const int64_t groups = kThreads / (dh * bytes / 32);
  const int64_t want = ceil_div(n * heads, groups);
  return (int)std::max(ceil_div(heads, groups), std::min<int64_t>(want, kSms * resident(bwd)));
}

template <typename T, int DH, bool kBwd, int K>
hg_status rot_pairs(const RotArgs& a, int grid, bool inter, cudaStream_t s) {
  const char* name = kBwd ? "qkrot_bwd" : "qkrot_fwd";
  if (inter) return launch(name, qkrot_kernel<T, DH, true, kBwd, K>, dim3(grid), dim3(kThreads), 0, s, a);
  return launch(name, qkrot_kernel<T, DH, false, kBwd, K>, dim3(grid), dim3(kThreads), 0, s, a);
}

// Lanes that share their sines and cosines: those of neighbouring heads of a row, as far as every warp holds whole sets
// of them (a power of two that divides the heads, and at most a warp).
template <typename T, int DH, bool kBwd>
hg_status rot_launch(const RotArgs& a, int grid, bool inter, cudaStream_t s) {
  constexpr int L = DH / (2 * VecTraits<T>::kElems);
  if constexpr (4 * L <= 32)
    if (a.heads % 4 == 0) return rot_pairs<T, DH, kBwd, 4>(a, grid, inter, s);
  if constexpr (2 * L <= 32)
    if (a.heads % 2 == 0) return rot_pairs<T, DH, kBwd, 2>(a, grid, inter, s);
  return rot_pairs<T, DH, kBwd, 1>(a, grid, inter, s);
}

template <typename T, bool kBwd>
hg_status rot_width(const RotArgs& a, int dh, int grid, bool inter, cudaStream_t s) {
  if (dh == 16) return rot_launch<T, 16, kBwd>(a, grid, inter, s);
  if (dh == 32) return rot_launch<T, 32, kBwd>(a, grid, inter, s);
  if (dh == 64) return rot_launch<T, 64, kBwd>(a, grid, inter, s);
  return rot_launch<T, 128, kBwd>(a, grid, inter, s);
}

hg_status check_params(const hg_qkrot_params* p, int64_t n) {
  HG_REQUIRE(p != nullptr, "params must be non-null");
  if (!(p->d_h == 16 || p->d_h == 32 || p->d_h == 64 || p->d_h == 128) ||
      !(p->dtype == HG_F32 || p->dtype == HG_BF16)) {
    set_error("unsupported d_h=%d / dtype=%d", p->d_h, (int)p->dtype);
    return HG_ERR_UNSUPPORTED;
  }
  HG_REQUIRE(p->heads_q >= 1 && p->heads_q <= kMaxHeads && p->heads_k >= 0 && p->heads_k <= kMaxHeads,
             "heads_q must be in [1, %d], heads_k in [0, %d]", kMaxHeads, kMaxHeads);
  HG_REQUIRE(p->rot >= 0 && p->rot <= p->d_h && p->rot % 16 == 0, "rot must be a multiple of 16 in [0, d_h]");
  HG_REQUIRE(std::isfinite(p->eps) && p->eps > 0.f, "eps must be positive and finite");
  HG_REQUIRE(std::isfinite(p->base) && p->base >= 1.0, "base must be finite and at least 1");
  HG_REQUIRE(n >= 0 && n < (int64_t(1) << 40), "n must be in [0, 2^40)");
  return HG_OK;
}

hg_status check_rows(const hg_rows* r, const char* name, int64_t n, int64_t width, size_t esz, bool written) {
  HG_REQUIRE(r != nullptr && r->p != nullptr, "%s must be non-null", name);
  HG_REQUIRE(((uintptr_t)r->p & 15) == 0, "%s must be 16-byte aligned", name);
  if (n < 2) return HG_OK;
  HG_REQUIRE(r->stride >= 0 && r->stride < (int64_t(1) << 40) && (r->stride * (int64_t)esz) % 16 == 0,
             "%s: the row stride must be a non-negative multiple of 16 bytes", name);
  HG_REQUIRE(!written || r->stride >= width, "%s: rows that are written must not overlap", name);
  return HG_OK;
}

// A call's rows with their width.
struct Rows {
  const hg_rows* r;
  int64_t width;
};

// An output may be its own input, rows at the same places; it meets no other array's rows.
hg_status check_apart(Rows out, Rows own, const char* name, int64_t n, size_t esz, std::initializer_list<Rows> others) {
  auto set = [&](Rows x) { return row_set(x.r->p, n, 1, x.r->stride, 0, x.width, esz); };
  const bool same = out.r->p == own.r->p;
  HG_REQUIRE(!same || n < 2 || out.r->stride == own.r->stride, "%s: in place, the strides must agree", name);
  HG_REQUIRE(same || !rows_meet(set(out), set(own)), "%s must not overlap an input but in place", name);
  for (Rows x : others) HG_REQUIRE(!rows_meet(set(out), set(x)), "%s must not overlap another array", name);
  return HG_OK;
}

size_t rot_scratch(const hg_qkrot_params* p, int64_t n) {
  return align_up(sizeof(float) * 2 * p->d_h *
                  (size_t)rot_grid(std::max<int64_t>(n, 1), p->heads_q + p->heads_k, p->d_h, p->dtype, true));
}

void fill_args(RotArgs* a, const hg_qkrot_params* p, const int64_t* pos, int64_t n) {
  *a = RotArgs{};
  a->pos = pos;
  a->gamma_q = p->gamma_q;
  a->gamma_k = p->gamma_k;
  a->n = n;
  a->hq = p->heads_q;
  a->heads = p->heads_q + p->heads_k;
  a->rot = p->rot;
  a->eps = p->eps;
  if (p->rot == 0) return;
  // The ratio is the m-th root of 1 / base: a double's, and one Newton step on it (powl takes 1.5 us of a call where
  // long doubles are emulated); the powers are products, 64 of which stay within 2^-57 of their value.
  const int m = p->rot / 2;
  long double ratio = std::pow(p->base, -1.0 / m), power = 1.0L;
  for (int i = 0; i < m; ++i) power *= ratio;
  ratio += ratio * (1.0L - (long double)p->base * power) / m;
  long double turns = 18446744073709551616.0L / 6.28318530717958647692528676655900577L;
  for (int i = 0; i < m; ++i, turns *= ratio) a->freq[i] = (uint64_t)(turns + 0.5L);
}

}  // namespace
}  // namespace hg

using namespace hg;

extern "C" hg_status hg_qkrot_workspace_size(const hg_qkrot_params* params, int64_t n, size_t* scratch_bytes) {
  clear_error();
  HG_REQUIRE(scratch_bytes, "scratch_bytes must be non-null");
  HG_TRY(check_params(params, n));
  *scratch_bytes = rot_scratch(params, n);
  return HG_OK;
}

extern "C" hg_status hg_qkrot_fwd(const hg_qkrot_params* params, const hg_rows* q, const hg_rows* k, const int64_t* pos,
                                  int64_t n, const hg_rows* q_out, const hg_rows* k_out, hg_stream stream) {
  clear_error();
  HG_TRY(device_guard());
  HG_TRY(check_params(params, n));
  if (n == 0) return HG_OK;
  const size_t esz = params->dtype == HG_BF16 ? 2 : 4;
  const int64_t wq = (int64_t)params->heads_q * params->d_h, wk = (int64_t)params->heads_k * params->d_h;
  HG_TRY(check_rows(q, "q", n, wq, esz, false));
  HG_TRY(check_rows(q_out, "q_out", n, wq, esz, true));
  if (wk) {
    HG_TRY(check_rows(k, "k", n, wk, esz, false));
    HG_TRY(check_rows(k_out, "k_out", n, wk, esz, true));
    HG_TRY(check_apart({q_out, wq}, {q, wq}, "q_out", n, esz, {{k, wk}, {k_out, wk}}));
    HG_TRY(check_apart({k_out, wk}, {k, wk}, "k_out", n, esz, {{q, wq}}));
  } else {
    HG_TRY(check_apart({q_out, wq}, {q, wq}, "q_out", n, esz, {}));
  }
  RotArgs a;
  fill_args(&a, params, pos, n);
  a.q = {q->p, nullptr, q_out->p, q->stride, 0, q_out->stride};
  if (wk) a.k = {k->p, nullptr, k_out->p, k->stride, 0, k_out->stride};
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const bool inter = params->interleaved != 0;
  const int grid = rot_grid(n, a.heads, params->d_h, params->dtype, false);
  if (params->dtype == HG_F32) return rot_width<float, false>(a, params->d_h, grid, inter, s);
  return rot_width<__nv_bfloat16, false>(a, params->d_h, grid, inter, s);
}

extern "C" hg_status hg_qkrot_bwd(const hg_qkrot_params* params, const hg_rows* q, const hg_rows* k, const int64_t* pos,
                                  int64_t n, const hg_rows* dq_out, const hg_rows* dk_out, const hg_rows* dq,
                                  const hg_rows* dk, float* dgamma_q, float* dgamma_k, void* scratch,
                                  hg_stream stream) {
  clear_error();
  HG_TRY(device_guard());
  HG_TRY(check_params(params, n));
  HG_REQUIRE(!shared(dgamma_q, dgamma_k, sizeof(float) * params->d_h), "dgamma_q and dgamma_k must not overlap");
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (n == 0) {
    if (dgamma_q) HG_CUDA(cudaMemsetAsync(dgamma_q, 0, sizeof(float) * params->d_h, s));
    if (dgamma_k) HG_CUDA(cudaMemsetAsync(dgamma_k, 0, sizeof(float) * params->d_h, s));
    return HG_OK;
  }
  const size_t esz = params->dtype == HG_BF16 ? 2 : 4;
  const int64_t wq = (int64_t)params->heads_q * params->d_h, wk = (int64_t)params->heads_k * params->d_h;
  HG_TRY(check_rows(q, "q", n, wq, esz, false));
  HG_TRY(check_rows(dq_out, "dq_out", n, wq, esz, false));
  HG_TRY(check_rows(dq, "dq", n, wq, esz, true));
  if (wk) {
    HG_TRY(check_rows(k, "k", n, wk, esz, false));
    HG_TRY(check_rows(dk_out, "dk_out", n, wk, esz, false));
    HG_TRY(check_rows(dk, "dk", n, wk, esz, true));
    HG_TRY(check_apart({dq, wq}, {dq_out, wq}, "dq", n, esz, {{q, wq}, {k, wk}, {dk_out, wk}, {dk, wk}}));
    HG_TRY(check_apart({dk, wk}, {dk_out, wk}, "dk", n, esz, {{q, wq}, {k, wk}, {dq_out, wq}}));
  } else {
    HG_TRY(check_apart({dq, wq}, {dq_out, wq}, "dq", n, esz, {{q, wq}}));
  }
  HG_REQUIRE(scratch != nullptr && ((uintptr_t)scratch & 255) == 0, "scratch must be non-null and 256-byte aligned");
  RotArgs a;
  fill_args(&a, params, pos, n);
  a.q = {q->p, dq_out->p, dq->p, q->stride, dq_out->stride, dq->stride};
  if (wk) a.k = {k->p, dk_out->p, dk->p, k->stride, dk_out->stride, dk->stride};
  a.part = static_cast<float*>(scratch);
  const bool inter = params->interleaved != 0;
  const int grid = rot_grid(n, a.heads, params->d_h, params->dtype, true);
  if (params->dtype == HG_F32)
    HG_TRY((rot_width<float, true>(a, params->d_h, grid, inter, s)));
  else
    HG_TRY((rot_width<__nv_bfloat16, true>(a, params->d_h, grid, inter, s)));
  if (!dgamma_q && !dgamma_k) return HG_OK;
  return launch("qkrot_gains", qkrot_gains, dim3(params->d_h / 16), dim3(256), 0, s, (const float*)a.part, grid,
                params->d_h, dgamma_q, dgamma_k);
}
