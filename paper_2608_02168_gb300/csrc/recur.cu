// Gated linear recurrence over whole histories (hg_recur_fwd, hg_recur_bwd) and for one new snapshot
// (hg_recur_step).  A channel's chain:
//   z_t = sigmoid(g_t + b),  h_t = h_(t-1) + z_t (x_t - h_(t-1)),
// and, from the end, with R_t = dy_t + (1 - z_(t+1)) R_(t+1):
//   dx_t = z_t R_t,  dg_t = R_t (x_t - h_(t-1)) z_t (1 - z_t),  db = sum of dg.
// An update is the nearer end plus a share of the difference, h + z (x - h) or x + (1 - z) (h - x), whichever share is
// below a half: no 1 - z is rounded (at z = 1e-5 that alone would change the mean's weight by 0.3 %), and a state that
// an open gate has just left does not leave its rounding behind.
//
// Each value is read and written once and costs two special functions and some ten other instructions: all forms are
// bound by HBM, or by latency where there are few chains.  A thread owns the chain of one 4-byte piece of a row (two
// bf16 channels or one fp32 channel), walks its positions 16 at a time and holds the next 16 rows' loads in flight.
// Few chains of many positions are split over time instead: see recur_fwd_split.
#include <algorithm>

#include "ffn_kernels.cuh"
#include "row_sets.cuh"
#include "tc_util.cuh"

namespace hg {
namespace {

constexpr int kPos = 16;          // positions a thread holds at a time; the forward keeps every 16th state
constexpr int kMaxWidth = 16384;  // channels of a row
constexpr int kLanes = 16;        // split forms: lanes across a row's piece, so 64 bytes of it
constexpr int kSubs = 16;         // ... and threads along time, kPos positions each
constexpr int kTile = kSubs * kPos;

template <typename T>
constexpr int kVec = 4 / (int)sizeof(T);  // channels of a 4-byte piece

struct Rows {
  const void* p;
  int64_t sn, st;  // strides of a sequence and of a position, in values
};

struct RecurArgs {
  Rows x, g, y, dy, dx, dg;
  const void* bias;
  const int32_t* lens;
  const float* h_in;    // forward, backward: the state before the first position (null: zero)
  float* h_out;
  const float* dh_out;  // backward
  float* dh_in;
  float* saved;         // [n][(T - 1) / kPos][d]: the states before positions kPos, 2 kPos, ...
  float* part;          // backward: partial sums of the bias's gradient, [rows of CTAs][d]
  int64_t n, T, spans;  // spans = (T - 1) / kPos
  int32_t d, blocks;    // split forms: blocks of channels
};

// A piece's channels: two go through one instruction each where there is one for two fp32 numbers.
template <int V>
struct Vec {
  float v[V];
};
#define HG_TWO(name, op)                                                                                        \
  __device__ __forceinline__ Vec<2> name(Vec<2> a, Vec<2> b) {                                                  \
    Vec<2> r;                                                                                                   \
    asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\t" op                       \
        " z, x, y;\n\tmov.b64 {%0, %1}, z;\n\t}"                                                               \
        : "=f"(r.v[0]), "=f"(r.v[1])                                                                            \
        : "f"(a.v[0]), "f"(a.v[1]), "f"(b.v[0]), "f"(b.v[1]));                                                  \
    return r;                                                                                                   \
  }
HG_TWO(add, "add.rn.f32x2")
HG_TWO(mul, "mul.rn.f32x2")
#undef HG_TWO
__device__ __forceinline__ Vec<2> fma(Vec<2> a, Vec<2> b, Vec<2> c) {
  Vec<2> r;
  asm("{\n\t.reg .b64 x, y, z;\n\tmov.b64 x, {%2, %3};\n\tmov.b64 y, {%4, %5};\n\tmov.b64 z, {%6, %7};\n\t"
      "fma.rn.f32x2 z, x, y, z;\n\tmov.b64 {%0, %1}, z;\n\t}"
      : "=f"(r.v[0]), "=f"(r.v[1])
      : "f"(a.v[0]), "f"(a.v[1]), "f"(b.v[0]), "f"(b.v[1]), "f"(c.v[0]), "f"(c.v[1]));
  return r;
}
__device__ __forceinline__ Vec<1> add(Vec<1> a, Vec<1> b) { return {a.v[0] + b.v[0]}; }
__device__ __forceinline__ Vec<1> mul(Vec<1> a, Vec<1> b) { return {a.v[0] * b.v[0]}; }
__device__ __forceinline__ Vec<1> fma(Vec<1> a, Vec<1> b, Vec<1> c) { return {fmaf(a.v[0], b.v[0], c.v[0])}; }
template <int V>
__device__ __forceinline__ Vec<V> all(float x) {
  Vec<V> r;
#pragma unroll
  for (int i = 0; i < V; ++i) r.v[i] = x;
  return r;
}
template <int V>
__device__ __forceinline__ Vec<V> minus(Vec<V> a, Vec<V> b) {  // a - b, rounded once
  return fma(b, all<V>(-1.f), a);
}

// A share z of [0, 1] and 1 - z in one number, each to a few steps of its own size: the smaller of the two, and the sign
// says which: z where it is not negative, -(1 - z) where it is (the gate is open).
__device__ __forceinline__ bool is_open(float code) { return __float_as_int(code) < 0; }
template <int V>
__device__ __forceinline__ Vec<V> pick(Vec<V> code, Vec<V> open, Vec<V> shut) {
  Vec<V> r;
#pragma unroll
  for (int i = 0; i < V; ++i) r.v[i] = is_open(code.v[i]) ? open.v[i] : shut.v[i];
  return r;
}
template <int V>
__device__ __forceinline__ Vec<V> size_of(Vec<V> code) {
  Vec<V> r;
#pragma unroll
  for (int i = 0; i < V; ++i) r.v[i] = fabsf(code.v[i]);
  return r;
}
template <int V>
__device__ __forceinline__ Vec<V> other_of(Vec<V> size) {
  return minus(all<V>(1.f), size);
}
// Of sigmoid(a): e^-|a| / (1 + e^-|a|) is the smaller one (zero from |a| = 87 on).
template <int V>
__device__ __forceinline__ Vec<V> gate_of(Vec<V> a) {
  Vec<V> e, r, c;
#pragma unroll
  for (int i = 0; i < V; ++i) e.v[i] = gate_ex2(fabsf(a.v[i]) * -1.4426950408889634f);
  r = add(e, all<V>(1.f));
#pragma unroll
  for (int i = 0; i < V; ++i) r.v[i] = gate_rcp(r.v[i]);
  r = mul(e, r);
#pragma unroll
  for (int i = 0; i < V; ++i)  // the sign: that of -a; a NaN stays one
    c.v[i] = __int_as_float(__float_as_int(r.v[i]) | (~__float_as_int(a.v[i]) & 0x80000000));
  return c;
}
template <int V>
__device__ __forceinline__ Vec<V> update(Vec<V> h, Vec<V> x, Vec<V> code) {
  return fma(code, minus(x, h), pick(code, x, h));
}

template <typename T>
__device__ __forceinline__ uint32_t ld4(const T* p) {
  return *reinterpret_cast<const uint32_t*>(p);
}
__device__ __forceinline__ Vec<1> piece(uint32_t v, float) { return {__uint_as_float(v)}; }
__device__ __forceinline__ Vec<2> piece(uint32_t v, __nv_bfloat16) {
  return {__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u)};
}
__device__ __forceinline__ void st4(float* p, Vec<1> f) { *p = f.v[0]; }
__device__ __forceinline__ void st4(__nv_bfloat16* p, Vec<2> f) {
  *reinterpret_cast<uint32_t*>(p) = pack2_bf16(f.v[0], f.v[1]);
}
__device__ __forceinline__ void ldf(const float* p, Vec<1>& f) { f.v[0] = *p; }
__device__ __forceinline__ void ldf(const float* p, Vec<2>& f) {
  const float2 v = *reinterpret_cast<const float2*>(p);
  f.v[0] = v.x;
  f.v[1] = v.y;
}
__device__ __forceinline__ void stf(float* p, Vec<1> f) { *p = f.v[0]; }
__device__ __forceinline__ void stf(float* p, Vec<2> f) { *reinterpret_cast<float2*>(p) = make_float2(f.v[0], f.v[1]); }

__device__ __forceinline__ int64_t length(const RecurArgs& a, int64_t i) {
  if (!a.lens) return a.T;
  const int64_t l = a.lens[i];
  return l < 0 ? 0 : l > a.T ? a.T : l;
}

template <typename T>
__device__ __forceinline__ const T* at(const Rows& r, int64_t i, int64_t t, int c) {
  return static_cast<const T*>(r.p) + i * r.sn + t * r.st + c;
}
template <typename T>
__device__ __forceinline__ T* at_out(const Rows& r, int64_t i, int64_t t, int c) {
  return const_cast<T*>(at<T>(r, i, t, c));
}

template <typename T>
__device__ __forceinline__ Vec<kVec<T>> bias_of(const RecurArgs& a, int c) {
  return a.bias ? piece(ld4(static_cast<const T*>(a.bias) + c), T{}) : all<kVec<T>>(0.f);
}
template <int V>
__device__ __forceinline__ Vec<V> state_of(const float* h, const RecurArgs& a, int64_t i, int c) {  // null: zero
  Vec<V> r = all<V>(0.f);
  if (h) ldf(h + i * a.d + c, r);
  return r;
}
// Where the state before position t0 is kept, t0 a multiple of kPos above zero.
__device__ __forceinline__ float* kept(const RecurArgs& a, int64_t i, int64_t t0, int c) {
  return a.saved + (i * a.spans + t0 / kPos - 1) * a.d + c;
}

// Positions in use of the kPos from t0 on.
__device__ __forceinline__ int left_of(int64_t t0, int64_t end) {
  const int64_t l = end - t0;
  return l < 0 ? 0 : l > kPos ? kPos : (int)l;
}
// kPos rows' pieces from position t0 on, zeros from `end` on.
template <typename T>
__device__ __forceinline__ void load_rows(uint32_t (&r)[kPos], const T* p, int64_t st, int64_t t0, int64_t end) {
  const int left = left_of(t0, end);
  p += t0 * st;
#pragma unroll
  for (int u = 0; u < kPos; ++u) {
    r[u] = u < left ? ld4(p) : 0u;
    p += st;
  }
}

// ------------------------------------------------------------------------------------------------------------
// a chain a thread
// ------------------------------------------------------------------------------------------------------------
// kAhead: the next rows' loads run under these ones' updates; histories of one batch do without their registers.
template <typename T, bool kAhead>
__global__ __launch_bounds__(256, kAhead ? 2 : 4) void recur_fwd(RecurArgs a) {
  pdl_begin();
  constexpr int V = kVec<T>;
  const int c = (blockIdx.y * blockDim.x + threadIdx.x) * V;
  const int64_t i = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  if (c >= a.d || i >= a.n) return;
  const int64_t len = length(a, i);
  const T *x = at<T>(a.x, i, 0, c), *g = at<T>(a.g, i, 0, c);
  T* y = at_out<T>(a.y, i, 0, c);
  uint32_t rx[kPos], rg[kPos];
  load_rows(rx, x, a.x.st, 0, len);
  load_rows(rg, g, a.g.st, 0, len);
  const Vec<V> b = bias_of<T>(a, c);
  Vec<V> h = state_of<V>(a.h_in, a, i, c);
  for (int64_t t0 = 0; t0 < len; t0 += kPos) {
    uint32_t nx[kPos], ng[kPos];
    if (kAhead) {
      load_rows(nx, x, a.x.st, t0 + kPos, len);
      load_rows(ng, g, a.g.st, t0 + kPos, len);
      if (a.saved && t0 > 0) stf(kept(a, i, t0, c), h);
    }
    const int left = left_of(t0, len);
#pragma unroll
    for (int u = 0; u < kPos; ++u) {
      if (u >= left) break;
      h = update(h, piece(rx[u], T{}), gate_of(add(piece(rg[u], T{}), b)));
      st4(y, h);
      y += a.y.st;
    }
    if (kAhead) {
#pragma unroll
      for (int u = 0; u < kPos; ++u) {
        rx[u] = nx[u];
        rg[u] = ng[u];
      }
    }
  }
  for (int64_t t = len; t < a.T; ++t, y += a.y.st) st4(y, all<V>(0.f));
  if (a.h_out) stf(a.h_out + i * a.d + c, h);
}

// Sums of a CTA's rows of threads (ty < rows), in a fixed order, to a row of partial sums.
template <int V>
__device__ __forceinline__ void part_sums(Vec<V> sum, float* sh, int tx, int ty, int width, int rows, float* out,
                                          bool in) {
#pragma unroll
  for (int v = 0; v < V; ++v) sh[(ty * width + tx) * V + v] = sum.v[v];
  __syncthreads();
  if (ty != 0 || !in) return;
  Vec<V> s = all<V>(0.f);
  for (int k = 0; k < rows; ++k) {
#pragma unroll
    for (int v = 0; v < V; ++v) s.v[v] += sh[(k * width + tx) * V + v];
  }
  stf(out, s);
}

// A position's part of the backward: what R gives dx and dg, and R for the position before.
template <int V>
__device__ __forceinline__ void back(Vec<V>& R, Vec<V> dy, Vec<V> code, Vec<V> diff, Vec<V>& dx, Vec<V>& dg) {
  const Vec<V> s = size_of(code), o = other_of(s), keep = pick(code, s, o);
  R = add(R, dy);
  dx = mul(pick(code, o, s), R);
  R = mul(keep, R);
  dg = mul(mul(dx, diff), keep);
}

template <typename T, bool kAhead>
__global__ __launch_bounds__(256, kAhead ? 1 : 2) void recur_bwd(RecurArgs a) {
  pdl_begin();
  constexpr int V = kVec<T>;
  __shared__ float sh[256 * V];
  const int c = (blockIdx.y * blockDim.x + threadIdx.x) * V;
  const bool in = c < a.d;
  const Vec<V> zero = all<V>(0.f), b = in ? bias_of<T>(a, c) : zero;
  Vec<V> sum = zero;
  for (int64_t i = (int64_t)blockIdx.x * blockDim.y + threadIdx.y; in && i < a.n;
       i += (int64_t)gridDim.x * blockDim.y) {
    const int64_t len = length(a, i);
    const T *x = at<T>(a.x, i, 0, c), *g = at<T>(a.g, i, 0, c), *dy = at<T>(a.dy, i, 0, c);
    T *dx = at_out<T>(a.dx, i, 0, c), *dg = at_out<T>(a.dg, i, 0, c);
    const int64_t last = len > 0 ? (len - 1) / kPos * kPos : 0;
    uint32_t rx[kPos], rg[kPos], ry[kPos];
    Vec<V> h;
    auto load = [&](int64_t t0, int64_t end) {
      load_rows(rx, x, a.x.st, t0, end);
      load_rows(rg, g, a.g.st, t0, end);
      load_rows(ry, dy, a.dy.st, t0, end);
      if (t0 > 0)
        ldf(kept(a, i, t0, c), h);
      else
        h = state_of<V>(a.h_in, a, i, c);
    };
    load(last, len);
    Vec<V> R = state_of<V>(a.dh_out, a, i, c);
    for (int64_t t = len; t < a.T; ++t) {
      st4(dx + t * a.dx.st, zero);
      st4(dg + t * a.dg.st, zero);
    }
    for (int64_t t0 = last; t0 >= 0 && len > 0; t0 -= kPos) {
      Vec<V> diff[kPos], code[kPos];
#pragma unroll
      for (int u = 0; u < kPos; ++u) {
        code[u] = gate_of(add(piece(rg[u], T{}), b));
        const Vec<V> fx = piece(rx[u], T{});
        diff[u] = minus(fx, h);
        h = fma(code[u], diff[u], pick(code[u], fx, h));
      }
      uint32_t cy[kPos];
#pragma unroll
      for (int u = 0; u < kPos; ++u) cy[u] = ry[u];
      if (kAhead && t0 > 0) load(t0 - kPos, t0);
      Vec<V> here = zero;
      const int left = left_of(t0, len);
      T *px = dx + (t0 + kPos) * a.dx.st, *pg = dg + (t0 + kPos) * a.dg.st;
#pragma unroll
      for (int u = kPos - 1; u >= 0; --u) {
        px -= a.dx.st;
        pg -= a.dg.st;
        if (u < left) {
          Vec<V> ox, og;
          back(R, piece(cy[u], T{}), code[u], diff[u], ox, og);
          here = add(here, og);
          st4(px, ox);
          st4(pg, og);
        }
      }
      sum = add(sum, here);
    }
    if (a.dh_in) stf(a.dh_in + i * a.d + c, R);
  }
  if (a.part)
    part_sums<V>(sum, sh, threadIdx.x, threadIdx.y, blockDim.x, blockDim.y, a.part + (int64_t)blockIdx.x * a.d + c, in);
}

// ------------------------------------------------------------------------------------------------------------
// a chain split over time
// ------------------------------------------------------------------------------------------------------------
// A cluster of CL CTAs takes 64 bytes of a sequence's rows through CL tiles of 256 positions a step; a thread has 16
// positions of a 4-byte piece.  Positions compose: a run of them maps the state h before it to B + K h, B its end from
// a zero state, K the product of its 1 - z (off by a step each, as a state is that is rounded at every position).
// Threads form the runs of their 16 positions and keep B and K of each, a CTA forms that of its tile and hands it to
// the cluster's others (distributed shared memory), and every CTA joins them in the same order, so all carry the same
// state and a call repeats its bits.  One barrier of the cluster a step.
template <int V>
struct Run {
  Vec<V> K, B;
};
template <int V>
struct alignas(8 * V) Pair {  // as it lies in shared memory
  float K[V], B[V];
};
template <int V>
struct SplitSmem {
  Pair<V> run[2][kSubs][kLanes];
  Pair<V> tile[2][8][kLanes];
};
template <int V>
__device__ __forceinline__ void join(Run<V>& a, const Pair<V>& p) {  // a, then p
  Vec<V> K, B;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    K.v[v] = p.K[v];
    B.v[v] = p.B[v];
  }
  a.B = fma(K, a.B, B);
  a.K = mul(a.K, K);
}
template <int V>
__device__ __forceinline__ Pair<V> pair_of(const Run<V>& r) {
  Pair<V> p;
#pragma unroll
  for (int v = 0; v < V; ++v) {
    p.K[v] = r.K.v[v];
    p.B[v] = r.B.v[v];
  }
  return p;
}

template <int CL>
__device__ __forceinline__ uint32_t cluster_rank() {
  uint32_t r = 0;
  if constexpr (CL > 1) asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return r;
}
template <int CL>
__device__ __forceinline__ void cluster_arrive() {
  if constexpr (CL > 1) asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
template <int CL>
__device__ __forceinline__ void cluster_wait() {
  if constexpr (CL > 1)
    asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory");
  else
    __syncthreads();
}
template <int CL, int V>
__device__ __forceinline__ void hand_out(Pair<V>* slot, const Pair<V>& p) {  // to the same place of every CTA
  if constexpr (CL > 1) {
    const uint32_t own = tc::smem_u32(slot);
#pragma unroll
    for (int r = 0; r < CL; ++r) {
      uint32_t there;
      asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(own), "r"(r));
#pragma unroll
      for (int v = 0; v < V; ++v) {
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(there + 4 * v), "f"(p.K[v]) : "memory");
        asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(there + 4 * (V + v)), "f"(p.B[v]) : "memory");
      }
    }
  } else {
    *slot = p;
  }
}

// The joined run of the tiles and threads before this one, from a step's runs: in the order of positions, or from the
// end.  State is carried on to the next step; what enters this thread's positions is returned.
template <int CL, int V, bool kBack>
__device__ __forceinline__ Vec<V> enter(SplitSmem<V>& sm, const Run<V>& mine, Vec<V>& state, int buf, int rank, int sub,
                                        int tx) {
  auto at = [](int k, int count) { return kBack ? count - 1 - k : k; };
  sm.run[buf][sub][tx] = pair_of(mine);
  __syncthreads();
  Run<V> before{all<V>(1.f), all<V>(0.f)};
  if (threadIdx.x < kLanes) {
    Run<V> whole = before;
#pragma unroll
    for (int k = 0; k < kSubs; ++k) join(whole, sm.run[buf][at(k, kSubs)][threadIdx.x]);
    hand_out<CL>(&sm.tile[buf][rank][threadIdx.x], pair_of(whole));
  }
  __syncwarp();
  cluster_arrive<CL>();
  const int ahead = at(sub, kSubs);
  for (int k = 0; k < ahead; ++k) join(before, sm.run[buf][at(k, kSubs)][tx]);
  __syncwarp();
  cluster_wait<CL>();
  Vec<V> got = state;
#pragma unroll
  for (int k = 0; k < CL; ++k) {
    const int r = at(k, CL);
    if (r == rank) got = fma(before.K, state, before.B);
    Run<V> s{all<V>(1.f), state};
    join(s, sm.tile[buf][r][tx]);
    state = s.B;
  }
  return got;
}

template <typename T, int CL>
__cluster_dims__(CL, 1, 1) __global__ void __launch_bounds__(256, 2) recur_fwd_split(RecurArgs a) {
  pdl_begin();
  constexpr int V = kVec<T>;
  __shared__ SplitSmem<V> sm;
  const int rank = cluster_rank<CL>(), tx = threadIdx.x % kLanes, sub = threadIdx.x / kLanes;
  const int64_t item = blockIdx.x / CL, i = item / a.blocks;
  const int c = (int)(item % a.blocks) * kLanes * V + tx * V;
  const bool in = c < a.d;
  const int64_t len = length(a, i);
  const T *x = at<T>(a.x, i, 0, c), *g = at<T>(a.g, i, 0, c);
  T* y = at_out<T>(a.y, i, 0, c);
  const int64_t end = in ? len : 0;  // lanes past the row load and store nothing
  const int64_t steps = (len + CL * kTile - 1) / (CL * kTile);
  const int64_t own = (int64_t)rank * kTile + sub * kPos;
  uint32_t rx[kPos], rg[kPos];
  load_rows(rx, x, a.x.st, own, end);
  load_rows(rg, g, a.g.st, own, end);
  const Vec<V> b = in ? bias_of<T>(a, c) : all<V>(0.f);
  Vec<V> h = in ? state_of<V>(a.h_in, a, i, c) : all<V>(0.f);
  cluster_arrive<CL>();  // every CTA runs before another one writes to it
  cluster_wait<CL>();
  for (int64_t s = 0; s < steps; ++s) {
    const int64_t t0 = s * CL * kTile + own;
    const int left = left_of(t0, end);
    Run<V> run[kPos], now{all<V>(1.f), all<V>(0.f)};
#pragma unroll
    for (int u = 0; u < kPos; ++u) {
      const Vec<V> code = gate_of(add(piece(rg[u], T{}), b)), sz = size_of(code);
      const Vec<V> B = update(now.B, piece(rx[u], T{}), code), K = mul(now.K, pick(code, sz, other_of(sz)));
      if (u < left) now = Run<V>{K, B};
      run[u] = now;
    }
    load_rows(rx, x, a.x.st, t0 + CL * kTile, end);
    load_rows(rg, g, a.g.st, t0 + CL * kTile, end);
    const Vec<V> h0 = enter<CL, V, false>(sm, now, h, s & 1, rank, sub, tx);
    if (a.saved && t0 > 0 && left > 0) stf(kept(a, i, t0, c), h0);
    T* py = y + t0 * a.y.st;
#pragma unroll
    for (int u = 0; u < kPos; ++u) {
      if (u < left) st4(py, fma(run[u].K, h0, run[u].B));
      py += a.y.st;
    }
  }
  if (!in) return;
  for (int64_t t = len + rank * kSubs + sub; t < a.T; t += CL * kSubs) st4(y + t * a.y.st, all<V>(0.f));
  if (a.h_out && rank == 0 && sub == 0) stf(a.h_out + i * a.d + c, h);
}

// The same from the end: a run of positions maps the R that enters from the right to B + K R.  The states before each
// thread's 16 positions are the forward's.
template <typename T, int CL>
__cluster_dims__(CL, 1, 1) __global__ void __launch_bounds__(256, 1) recur_bwd_split(RecurArgs a) {
  pdl_begin();
  constexpr int V = kVec<T>;
  __shared__ SplitSmem<V> sm;
  __shared__ float sh[256 * V];
  const int rank = cluster_rank<CL>(), tx = threadIdx.x % kLanes, sub = threadIdx.x / kLanes;
  const int64_t item = blockIdx.x / CL, i = item / a.blocks;
  const int c = (int)(item % a.blocks) * kLanes * V + tx * V;
  const bool in = c < a.d;
  const int64_t len = length(a, i);
  const T *x = at<T>(a.x, i, 0, c), *g = at<T>(a.g, i, 0, c), *dy = at<T>(a.dy, i, 0, c);
  T *dx = at_out<T>(a.dx, i, 0, c), *dg = at_out<T>(a.dg, i, 0, c);
  const int64_t end = in ? len : 0;
  const int64_t steps = (len + CL * kTile - 1) / (CL * kTile);
  const int64_t own = (int64_t)rank * kTile + sub * kPos;
  const Vec<V> zero = all<V>(0.f);
  uint32_t rx[kPos], rg[kPos], ry[kPos];
  Vec<V> h;
  auto load = [&](int64_t t0) {
    load_rows(rx, x, a.x.st, t0, end);
    load_rows(rg, g, a.g.st, t0, end);
    load_rows(ry, dy, a.dy.st, t0, end);
    h = zero;
    if (t0 < end) {
      if (t0 > 0)
        ldf(kept(a, i, t0, c), h);
      else
        h = state_of<V>(a.h_in, a, i, c);
    }
  };
  if (steps > 0) load((steps - 1) * CL * kTile + own);
  const Vec<V> b = in ? bias_of<T>(a, c) : zero;
  Vec<V> R = in ? state_of<V>(a.dh_out, a, i, c) : zero, sum = zero;
  cluster_arrive<CL>();
  cluster_wait<CL>();
  for (int64_t s = steps - 1; s >= 0; --s) {
    const int64_t t0 = s * CL * kTile + own;
    const int left = left_of(t0, end);
    Vec<V> diff[kPos], code[kPos];
    uint32_t cy[kPos];
#pragma unroll
    for (int u = 0; u < kPos; ++u) {
      const Vec<V> fx = piece(rx[u], T{}), z = gate_of(add(piece(rg[u], T{}), b));
      cy[u] = ry[u];
      code[u] = u < left ? z : zero;  // zero: a position that is not in use
      diff[u] = minus(fx, h);
      h = fma(code[u], diff[u], pick(code[u], fx, h));
    }
    Run<V> run{all<V>(1.f), zero};
#pragma unroll
    for (int u = kPos - 1; u >= 0; --u) {
      const Vec<V> sz = size_of(code[u]), k = pick(code[u], sz, other_of(sz));
      run.B = mul(k, add(run.B, piece(cy[u], T{})));
      run.K = mul(run.K, k);
    }
    if (s > 0) load(t0 - CL * kTile);
    Vec<V> r = enter<CL, V, true>(sm, run, R, s & 1, rank, sub, tx), here = zero;
    T *px = dx + (t0 + kPos) * a.dx.st, *pg = dg + (t0 + kPos) * a.dg.st;
#pragma unroll
    for (int u = kPos - 1; u >= 0; --u) {
      px -= a.dx.st;
      pg -= a.dg.st;
      Vec<V> ox, og;
      back(r, piece(cy[u], T{}), code[u], diff[u], ox, og);
      if (u < left) {
        here = add(here, og);
        st4(px, ox);
        st4(pg, og);
      }
    }
    sum = add(sum, here);
  }
  if (in) {
    for (int64_t t = len + rank * kSubs + sub; t < a.T; t += CL * kSubs) {
      st4(dx + t * a.dx.st, zero);
      st4(dg + t * a.dg.st, zero);
    }
    if (a.dh_in && rank == 0 && sub == 0) stf(a.dh_in + i * a.d + c, R);
  }
  if (a.part) part_sums<V>(sum, sh, tx, sub, kLanes, kSubs, a.part + (i * CL + rank) * a.d + c, in);
}

// ------------------------------------------------------------------------------------------------------------
// the bias's gradient, one snapshot
// ------------------------------------------------------------------------------------------------------------
// Column sums of `rows` partial rows: eight runs a CTA of 32 columns, joined in order.
__global__ __launch_bounds__(256) void recur_bias_sum(const float* part, int64_t rows, int32_t d, float* out) {
  pdl_begin();
  __shared__ float sh[8][32];
  const int tx = threadIdx.x % 32, ty = threadIdx.x / 32, c = blockIdx.x * 32 + tx;
  float s = 0.f;
  if (c < d) {
#pragma unroll 8
    for (int64_t r = ty; r < rows; r += 8) s += part[r * d + c];
  }
  sh[ty][tx] = s;
  __syncthreads();
  if (ty != 0 || c >= d) return;
  for (int k = 1; k < 8; ++k) s += sh[k][tx];
  out[c] = s;
}

// A row of eight values a thread.
template <typename T>
__global__ __launch_bounds__(256) void recur_step(RecurArgs a) {
  pdl_begin();
  constexpr int E = 8, Q = E * sizeof(T) / 16;
  const int c = (blockIdx.y * blockDim.x + threadIdx.x) * E;
  const int64_t i = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  if (c >= a.d || i >= a.n) return;
  const bool live = !a.lens || a.lens[i] > 0;
  float h[E], o[E] = {};
  const float* hi = a.h_in + i * a.d + c;
  unpack(ld16(hi), h, 0.f);
  unpack(ld16(hi + 4), h + 4, 0.f);
  if (live) {
    float x[E], g[E], b[E] = {};
    const T *xp = at<T>(a.x, i, 0, c), *gp = at<T>(a.g, i, 0, c);
#pragma unroll
    for (int q = 0; q < Q; ++q) {
      unpack(ld16(xp + q * E / Q), x + q * E / Q, T{});
      unpack(ld16(gp + q * E / Q), g + q * E / Q, T{});
      if (a.bias) unpack(ld16(static_cast<const T*>(a.bias) + c + q * E / Q), b + q * E / Q, T{});
    }
#pragma unroll
    for (int v = 0; v < E; ++v) o[v] = h[v] = update(Vec<1>{h[v]}, Vec<1>{x[v]}, gate_of(Vec<1>{g[v] + b[v]})).v[0];
  }
  T* yp = at_out<T>(a.y, i, 0, c);
#pragma unroll
  for (int q = 0; q < Q; ++q) st16(yp + q * E / Q, pack(o + q * E / Q, T{}));
  float* ho = a.h_out + i * a.d + c;
  if (live || ho != hi) {
    st16(ho, pack(h, 0.f));
    st16(ho + 4, pack(h + 4, 0.f));
  }
}

// ------------------------------------------------------------------------------------------------------------
// host
// ------------------------------------------------------------------------------------------------------------
struct Shape {
  dim3 block;
  unsigned across;  // CTAs across a row
};
Shape shape_of(int64_t lanes) {  // rows of up to 256 lanes; short ones share a CTA
  const int64_t across = ceil_div(lanes, 256), width = ceil_div(lanes, across);
  return {dim3((unsigned)width, (unsigned)(256 / width)), (unsigned)across};
}

// Split over time, and by a cluster of how many CTAs?
int split_of(const hg_recur_params* p, int64_t n, int64_t T) {
  const int64_t lanes = p->d * (p->dtype == HG_BF16 ? 2 : 4) / 4;
  if (n * lanes >= 152 * 256 || T <= 4 * kPos) return 0;
  const int64_t items = n * ceil_div(lanes, kLanes);
  int cl = 1;
  while (cl < 8 && items * cl < 2 * 152 && cl * kTile < T) cl *= 2;
  return cl;
}

// Rows of partial sums of the bias's gradient.
int64_t part_rows(const hg_recur_params* p, int64_t n, int64_t T) {
  const int cl = split_of(p, n, T);
  if (cl) return n * cl;
  const Shape s = shape_of(p->d * (p->dtype == HG_BF16 ? 2 : 4) / 4);
  const int64_t groups = ceil_div(n, s.block.y), most = std::max<int64_t>(1, 152 * 16 / s.across);
  return std::min(groups, most);
}

hg_status check(const hg_recur_params* p, int64_t n, int64_t T) {
  HG_REQUIRE(p != nullptr, "params must be non-null");
  if (p->d < 8 || p->d > kMaxWidth || p->d % 8 || !(p->dtype == HG_F32 || p->dtype == HG_BF16)) {
    set_error("unsupported d=%d (a multiple of 8 up to %d) / dtype=%d", p->d, kMaxWidth, (int)p->dtype);
    return HG_ERR_UNSUPPORTED;
  }
  HG_REQUIRE(((uintptr_t)p->bias & 15) == 0, "bias must be 16-byte aligned");
  HG_REQUIRE(n >= 0 && n < (int64_t(1) << 28), "n must be in [0, 2^28)");
  HG_REQUIRE(T >= 0 && T < (int64_t(1) << 30), "T must be in [0, 2^30)");
  HG_REQUIRE(n == 0 || T <= (int64_t(1) << 46) / n, "n * T must be at most 2^46");
  return HG_OK;
}

hg_status check_state(const float* h, const char* name) {
  HG_REQUIRE(((uintptr_t)h & 15) == 0, "%s must be 16-byte aligned", name);
  return HG_OK;
}

Rows rows_of(const hg_seq* r, int64_t n, int64_t T) {
  return {r->p, n < 2 ? 0 : r->stride_n, T < 2 ? 0 : r->stride_t};
}

size_t esize(const hg_recur_params* p) { return p->dtype == HG_BF16 ? 2 : 4; }

template <typename T>
hg_status forward(const RecurArgs& a, int cl, cudaStream_t s) {
  if (cl == 0) {
    const Shape sh = shape_of(a.d / kVec<T>);
    const dim3 grid((unsigned)ceil_div(a.n, sh.block.y), sh.across);
    if (a.T <= kPos) return launch("recur_fwd", recur_fwd<T, false>, grid, sh.block, 0, s, a);
    return launch("recur_fwd", recur_fwd<T, true>, grid, sh.block, 0, s, a);
  }
  const dim3 grid((unsigned)(a.n * a.blocks * cl)), block(256);
  if (cl == 1) return launch("recur_fwd_split", recur_fwd_split<T, 1>, grid, block, 0, s, a);
  if (cl == 2) return launch("recur_fwd_split", recur_fwd_split<T, 2>, grid, block, 0, s, a);
  if (cl == 4) return launch("recur_fwd_split", recur_fwd_split<T, 4>, grid, block, 0, s, a);
  return launch("recur_fwd_split", recur_fwd_split<T, 8>, grid, block, 0, s, a);
}

template <typename T>
hg_status backward(const RecurArgs& a, int cl, int64_t rows, cudaStream_t s) {
  if (cl == 0) {
    const Shape sh = shape_of(a.d / kVec<T>);
    const dim3 grid((unsigned)rows, sh.across);
    if (a.T <= kPos) return launch("recur_bwd", recur_bwd<T, false>, grid, sh.block, 0, s, a);
    return launch("recur_bwd", recur_bwd<T, true>, grid, sh.block, 0, s, a);
  }
  const dim3 grid((unsigned)(a.n * a.blocks * cl)), block(256);
  if (cl == 1) return launch("recur_bwd_split", recur_bwd_split<T, 1>, grid, block, 0, s, a);
  if (cl == 2) return launch("recur_bwd_split", recur_bwd_split<T, 2>, grid, block, 0, s, a);
  if (cl == 4) return launch("recur_bwd_split", recur_bwd_split<T, 4>, grid, block, 0, s, a);
  return launch("recur_bwd_split", recur_bwd_split<T, 8>, grid, block, 0, s, a);
}

RecurArgs args_of(const hg_recur_params* p, int64_t n, int64_t T) {
  RecurArgs a{};
  a.bias = p->bias;
  a.n = n;
  a.T = T;
  a.spans = T > 0 ? (T - 1) / kPos : 0;
  a.d = p->d;
  a.blocks = (int32_t)ceil_div(p->d * (int64_t)esize(p) / 4, kLanes);
  return a;
}

size_t saved_bytes_of(const hg_recur_params* p, int64_t n, int64_t T) {
  return T > 0 ? sizeof(float) * (size_t)n * ((T - 1) / kPos) * p->d : 0;
}

}  // namespace
}  // namespace hg

using namespace hg;

extern "C" hg_status hg_recur_workspace_size(const hg_recur_params* params, int64_t n, int64_t T, size_t* saved_bytes,
                                             size_t* scratch_bytes) {
  clear_error();
  HG_REQUIRE(saved_bytes && scratch_bytes, "saved_bytes and scratch_bytes must be non-null");
  HG_TRY(check(params, n, T));
  *saved_bytes = align_up(saved_bytes_of(params, n, T));
  *scratch_bytes = align_up(sizeof(float) * (size_t)part_rows(params, n, T) * params->d);
  return HG_OK;
}

extern "C" hg_status hg_recur_fwd(const hg_recur_params* params, const hg_seq* x, const hg_seq* g, const int32_t* lens,
                                  int64_t n, int64_t T, const float* h_in, const hg_seq* y, float* h_out, void* saved,
                                  hg_stream stream) {
  clear_error();
  HG_TRY(device_guard());
  HG_TRY(check(params, n, T));
  HG_REQUIRE(((uintptr_t)saved & 255) == 0, "saved must be 256-byte aligned");
  if (n == 0) return HG_OK;
  const size_t esz = esize(params);
  const int64_t w = params->d;
  HG_TRY(check_state(h_in, "h_in"));
  HG_TRY(check_state(h_out, "h_out"));
  RecurArgs a = args_of(params, n, T);
  const RowSet hi = block_set(h_in, 4 * n * w), ho = block_set(h_out, 4 * n * w);
  HG_REQUIRE(h_out == h_in || !rows_meet(ho, hi), "h_out and h_in must not overlap");
  if (T > 0) {
    HG_TRY(check_seq(x, "x", n, T, w, esz, false));
    HG_TRY(check_seq(g, "g", n, T, w, esz, false));
    HG_TRY(check_seq(y, "y", n, T, w, esz, true));
    const RowSet sv = block_set(saved, (int64_t)saved_bytes_of(params, n, T));
    const RowSet bias = block_set(params->bias, w * (int64_t)esz), ln = block_set(lens, 4 * n);
    const RowSet rx = seq_set(x, n, T, w, esz), rg = seq_set(g, n, T, w, esz), ry = seq_set(y, n, T, w, esz);
    HG_TRY(check_apart(ry, "y", {rx, rg, hi, ho, sv, bias, ln}));
    HG_TRY(check_apart(ho, "h_out", {rx, rg, sv, bias, ln}));
    HG_TRY(check_apart(sv, "saved", {rx, rg, hi, bias, ln}));
    a.x = rows_of(x, n, T);
    a.g = rows_of(g, n, T);
    a.y = rows_of(y, n, T);
  }
  a.lens = lens;
  a.h_in = h_in;
  a.h_out = h_out;
  a.saved = static_cast<float*>(saved);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const int cl = split_of(params, n, T);
  return params->dtype == HG_BF16 ? forward<__nv_bfloat16>(a, cl, s) : forward<float>(a, cl, s);
}

extern "C" hg_status hg_recur_bwd(const hg_recur_params* params, const hg_seq* x, const hg_seq* g, const int32_t* lens,
                                  int64_t n, int64_t T, const float* h_in, const void* saved, const hg_seq* d_y,
                                  const float* dh_out, const hg_seq* dx, const hg_seq* dg, float* dh_in, float* dbias,
                                  void* scratch, hg_stream stream) {
  clear_error();
  HG_TRY(device_guard());
  HG_TRY(check(params, n, T));
  HG_REQUIRE(((uintptr_t)saved & 255) == 0, "saved must be 256-byte aligned");
  HG_REQUIRE(((uintptr_t)scratch & 255) == 0, "scratch must be 256-byte aligned");
  const size_t saved_bytes = saved_bytes_of(params, n, T), esz = esize(params);
  HG_REQUIRE(saved_bytes == 0 || saved, "saved must be non-null");
  const int64_t w = params->d, rows = part_rows(params, n, T);
  HG_REQUIRE(!dbias || n == 0 || scratch, "scratch must be non-null");
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  RecurArgs a = args_of(params, n, T);
  if (n > 0) {
    HG_TRY(check_state(h_in, "h_in"));
    HG_TRY(check_state(dh_out, "dh_out"));
    HG_TRY(check_state(dh_in, "dh_in"));
    const RowSet hi = block_set(h_in, 4 * n * w), ro = block_set(dh_out, 4 * n * w), ri = block_set(dh_in, 4 * n * w);
    const RowSet sv = block_set(saved, (int64_t)saved_bytes), db = block_set(dbias, 4 * w);
    const RowSet sc = block_set(dbias ? scratch : nullptr, 4 * rows * w), bias = block_set(params->bias, w * (int64_t)esz);
    const RowSet ln = block_set(lens, 4 * n);
    HG_REQUIRE(dh_in == dh_out || !rows_meet(ri, ro), "dh_in and dh_out must not overlap");
    HG_TRY(check_apart(ri, "dh_in", {hi, sv, db, sc, bias, ln}));
    HG_TRY(check_apart(db, "dbias", {hi, ro, sv, sc, bias, ln}));
    HG_TRY(check_apart(sc, "scratch", {hi, ro, sv, bias, ln}));
    if (T > 0) {
      HG_TRY(check_seq(x, "x", n, T, w, esz, false));
      HG_TRY(check_seq(g, "g", n, T, w, esz, false));
      HG_TRY(check_seq(d_y, "d_y", n, T, w, esz, false));
      HG_TRY(check_seq(dx, "dx", n, T, w, esz, true));
      HG_TRY(check_seq(dg, "dg", n, T, w, esz, true));
      const RowSet rx = seq_set(x, n, T, w, esz), rg = seq_set(g, n, T, w, esz), ry = seq_set(d_y, n, T, w, esz);
      const RowSet ox = seq_set(dx, n, T, w, esz), og = seq_set(dg, n, T, w, esz);
      HG_TRY(check_apart(ox, "dx", {rx, rg, ry, og, hi, ro, ri, sv, db, sc, bias, ln}));
      HG_TRY(check_apart(og, "dg", {rx, rg, ry, hi, ro, ri, sv, db, sc, bias, ln}));
      HG_TRY(check_apart(ri, "dh_in", {rx, rg, ry}));
      HG_TRY(check_apart(db, "dbias", {rx, rg, ry}));
      HG_TRY(check_apart(sc, "scratch", {rx, rg, ry}));
      a.x = rows_of(x, n, T);
      a.g = rows_of(g, n, T);
      a.dy = rows_of(d_y, n, T);
      a.dx = rows_of(dx, n, T);
      a.dg = rows_of(dg, n, T);
    }
    a.lens = lens;
    a.h_in = h_in;
    a.saved = const_cast<float*>(static_cast<const float*>(saved));
    a.dh_out = dh_out;
    a.dh_in = dh_in;
    a.part = dbias ? static_cast<float*>(scratch) : nullptr;
    const int cl = split_of(params, n, T);
    HG_TRY(params->dtype == HG_BF16 ? backward<__nv_bfloat16>(a, cl, rows, s) : backward<float>(a, cl, rows, s));
  }
  if (!dbias) return HG_OK;
  return launch("recur_bias_sum", recur_bias_sum, dim3((unsigned)ceil_div(w, 32)), dim3(256), 0, s, a.part,
                n > 0 ? rows : 0, params->d, dbias);
}

extern "C" hg_status hg_recur_step(const hg_recur_params* params, const hg_rows* x, const hg_rows* g,
                                   const int32_t* live, int64_t n, const float* h_in, const hg_rows* y, float* h_out,
                                   hg_stream stream) {
  clear_error();
  HG_TRY(device_guard());
  HG_TRY(check(params, n, 1));
  if (n == 0) return HG_OK;
  const size_t esz = esize(params);
  const int64_t w = params->d;
  const hg_rows* in[3] = {x, g, y};
  const char* names[3] = {"x", "g", "y"};
  hg_seq r[3];
  for (int k = 0; k < 3; ++k) {
    HG_REQUIRE(in[k] != nullptr, "%s must be non-null", names[k]);
    r[k] = hg_seq{in[k]->p, in[k]->stride, 0};
    HG_TRY(check_seq(&r[k], names[k], n, 1, w, esz, k == 2));
  }
  HG_REQUIRE(h_in && h_out, "h_in and h_out must be non-null");
  HG_TRY(check_state(h_in, "h_in"));
  HG_TRY(check_state(h_out, "h_out"));
  const RowSet rx = seq_set(&r[0], n, 1, w, esz), rg = seq_set(&r[1], n, 1, w, esz), ry = seq_set(&r[2], n, 1, w, esz);
  const RowSet hi = block_set(h_in, 4 * n * w), ho = block_set(h_out, 4 * n * w);
  HG_REQUIRE(h_out == h_in || !rows_meet(ho, hi), "h_out and h_in must not overlap");
  const RowSet bias = block_set(params->bias, w * (int64_t)esz), lv = block_set(live, 4 * n);
  HG_TRY(check_apart(ry, "y", {rx, rg, hi, ho, bias, lv}));
  HG_TRY(check_apart(ho, "h_out", {rx, rg, bias, lv}));
  RecurArgs a = args_of(params, n, 1);
  a.x = rows_of(&r[0], n, 1);
  a.g = rows_of(&r[1], n, 1);
  a.y = rows_of(&r[2], n, 1);
  a.lens = live;
  a.h_in = h_in;
  a.h_out = h_out;
  const Shape sh = shape_of(w / 8);
  const dim3 grid((unsigned)ceil_div(n, sh.block.y), sh.across);
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (params->dtype == HG_F32) return launch("recur_step", recur_step<float>, grid, sh.block, 0, s, a);
  return launch("recur_step", recur_step<__nv_bfloat16>, grid, sh.block, 0, s, a);
}
