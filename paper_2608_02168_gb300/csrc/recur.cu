// Gated linear recurrence over whole histories (hg_recur_fwd, hg_recur_bwd) and for one new snapshot
// (hg_recur_step).  A channel's chain:
//   z_t = sigmoid(g_t + b),  h_t = h_(t-1) + z_t (x_t - h_(t-1)),
// and, from the end, with R_t = dy_t + (1 - z_(t+1)) R_(t+1):
//   dx_t = z_t R_t,  dg_t = R_t (x_t - h_(t-1)) z_t (1 - z_t),  db = sum of dg.
// A share z is known to a few steps of its own size, and a state or R goes on by what z changes of it, never by a
// product with a rounded 1 - z, so long memories (z = 1e-5) keep their weights.
//
// Each value is read and written once and costs two special functions and some ten other instructions: all forms are
// bound by HBM, or by latency where there are few chains.
//   recur_fwd, recur_bwd              a thread walks a chain (split_of says when)
//   recur_bwd_short                   the same for histories of at most 16 positions
//   recur_fwd_split, recur_bwd_split  a few long histories: time is split over threads, CTAs and clusters
//   recur_bias_sum                    the CTAs' parts of the bias's gradient, in a fixed order
//   recur_step                        one new snapshot: 1000003 nodes of d 128, one in eight not live: 242 us
// The backward reads x, g, dy and every 16th state, which the forward kept, and forms the states between anew: 0.25
// bytes a value more in either pass, where reading the states (4 bytes) or a second forward pass (2 b) would be more.
#include <algorithm>
#include <cfloat>

#include "ffn_kernels.cuh"
#include "layer_kernels.cuh"
#include "row_sets.cuh"
#include "tc_util.cuh"

namespace hg {
namespace {

constexpr int kPos = 16;          // positions a thread holds at a time; the forward keeps every 16th state
constexpr int kMaxWidth = 16384;  // channels of a row
constexpr int kSplitThr = 256;    // split forms: threads, L across a piece of a row and the others along time
constexpr int kMaxCluster = 8;
template <int L>
constexpr int kSubs = kSplitThr / L;       // threads along time, kPos positions each
template <int L>
constexpr int kTile = kSubs<L> * kPos;     // positions of a CTA's step

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
  int* status;          // split forms: the library's device status word
  float* part;          // backward: partial sums of the bias's gradient, [rows of CTAs][d]
  int64_t n, T, spans;  // spans = (T - 1) / kPos
  int32_t d, blocks;    // split forms: blocks of channels
};

// A piece's channels.  (Instructions on two fp32 numbers at once cost more moves into register pairs, 16 a position of
// two channels, than they save.)
template <int V>
struct Vec {
  float v[V];
};
template <int V>
__device__ __forceinline__ Vec<V> add(Vec<V> a, Vec<V> b) {
#pragma unroll
  for (int i = 0; i < V; ++i) a.v[i] += b.v[i];
  return a;
}
template <int V>
__device__ __forceinline__ Vec<V> mul(Vec<V> a, Vec<V> b) {
#pragma unroll
  for (int i = 0; i < V; ++i) a.v[i] *= b.v[i];
  return a;
}
template <int V>
__device__ __forceinline__ Vec<V> fma(Vec<V> a, Vec<V> b, Vec<V> c) {
#pragma unroll
  for (int i = 0; i < V; ++i) c.v[i] = fmaf(a.v[i], b.v[i], c.v[i]);
  return c;
}
template <int V>
__device__ __forceinline__ Vec<V> all(float x) {
  Vec<V> r;
#pragma unroll
  for (int i = 0; i < V; ++i) r.v[i] = x;
  return r;
}
template <int V>
__device__ __forceinline__ Vec<V> minus(Vec<V> a, Vec<V> b) {
#pragma unroll
  for (int i = 0; i < V; ++i) a.v[i] -= b.v[i];
  return a;
}

// A sum kept as a + rest: as one number and what that leaves of it.
template <int V>
__device__ __forceinline__ void settle(Vec<V>& a, Vec<V>& rest) {
  const Vec<V> sum = add(a, rest);
  rest = minus(rest, minus(sum, a));
  a = sum;
}
template <int V>
__device__ __forceinline__ Vec<V> less(Vec<V> c, Vec<V> a, Vec<V> b) {  // c - a b
#pragma unroll
  for (int i = 0; i < V; ++i) c.v[i] = fmaf(-a.v[i], b.v[i], c.v[i]);
  return c;
}

// z = sigmoid(g + b) and k = 1 - z, with a bias as Gate::bias gives it.
constexpr float kLog2e = 1.4426950408889634f;

// fp32 rows: z and k each to a few steps of their own size.  s = e^-|a| / (1 + e^-|a|) is the smaller of the two (zero
// from |a| = 87 on), 1 - s the other, and an update is the nearer end plus the smaller share of the difference: a state
// that an open gate has just left does not leave its rounding behind.  The bias is added first: its product with log2
// e, rounded, would be |b| 2^-24 of z off, also where g and b cancel.
template <int V, bool kExact>
struct Gate {
  Vec<V> s, big;
  bool open[V];
  // An infinite bias is the largest, so that -infinity plus it stays what it is (NaN too).
  __device__ __forceinline__ static float bias(float b) { return isinf(b) ? copysignf(FLT_MAX, b) : b; }
  __device__ __forceinline__ Gate(Vec<V> g, Vec<V> bias) {
    const Vec<V> a = mul(add(g, bias), all<V>(-kLog2e));
#pragma unroll
    for (int i = 0; i < V; ++i) s.v[i] = gate_ex2(-fabsf(a.v[i]));
    Vec<V> r = add(s, all<V>(1.f));
#pragma unroll
    for (int i = 0; i < V; ++i) {
      r.v[i] = gate_rcp(r.v[i]);
      open[i] = a.v[i] <= 0.f;
    }
    s = mul(s, r);
    big = minus(all<V>(1.f), s);
  }
  __device__ __forceinline__ Vec<V> pick(Vec<V> x, Vec<V> y) const {  // x of an open gate, y of a shut one
    Vec<V> r;
#pragma unroll
    for (int i = 0; i < V; ++i) r.v[i] = open[i] ? x.v[i] : y.v[i];
    return r;
  }
  __device__ __forceinline__ Vec<V> z() const { return pick(big, s); }
  __device__ __forceinline__ Vec<V> k() const { return pick(s, big); }
  __device__ __forceinline__ Vec<V> zk() const { return mul(s, big); }
  __device__ __forceinline__ Vec<V> next(Vec<V> h, Vec<V> x) const { return fma(code(), minus(x, h), pick(x, h)); }
  // The same of a state kept as h + rest, whose sum `sum` is.
  __device__ __forceinline__ void next(Vec<V>& h, Vec<V>& rest, Vec<V> sum, Vec<V> x) const {
    rest = fma(code(), minus(x, sum), pick(x, rest));
    h = pick(all<V>(0.f), h);
  }
  // What a gate lets through of R, z R, and what it leaves, (1 - z) R: the smaller as a product, the other as R without
  // it.
  __device__ __forceinline__ static void part(Vec<V> code, Vec<V> R, Vec<V>& through, Vec<V>& left) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float s = fabsf(code.v[i]), small = s * R.v[i], rest = fmaf(-s, R.v[i], R.v[i]);
      const bool open = __float_as_int(code.v[i]) < 0;
      through.v[i] = open ? rest : small;
      left.v[i] = open ? small : rest;
    }
  }
  // The same of R + rest, whose sum `sum` is: what is left stays in two numbers.
  __device__ __forceinline__ static void part(Vec<V> code, Vec<V>& R, Vec<V>& rest, Vec<V> sum, Vec<V>& through) {
#pragma unroll
    for (int i = 0; i < V; ++i) {
      const float s = fabsf(code.v[i]), small = s * sum.v[i];
      const bool open = __float_as_int(code.v[i]) < 0;
      through.v[i] = open ? sum.v[i] - small : small;
      rest.v[i] = open ? small : fmaf(-s, sum.v[i], rest.v[i]);
      R.v[i] = open ? 0.f : R.v[i];
    }
  }
  // Both in one number: z where it is not negative, -k where it is.
  __device__ __forceinline__ Vec<V> code() const {
    Vec<V> r;
#pragma unroll
    for (int i = 0; i < V; ++i) r.v[i] = open[i] ? -s.v[i] : s.v[i];
    return r;
  }
};

// bf16 rows, whose bytes are half as many and whose instructions therefore count (5 a gate instead of 9): z to a few
// steps of its own size (and |b| 2^-24), 1 - z to a few of one, which is a rounding of the state that it keeps.  The
// logit's product with -log2 e and the sum with the bias's are one instruction.
template <int V>
struct Gate<V, false> {
  Vec<V> e, r;
  // One above 1e38 is as good as that, and its product stays finite, so that -infinity plus it stays what it is (NaN
  // too).
  __device__ __forceinline__ static float bias(float b) {
    return -kLog2e * (fabsf(b) > 1e38f ? copysignf(1e38f, b) : b);
  }
  __device__ __forceinline__ Gate(Vec<V> g, Vec<V> bias) {
    const Vec<V> a = fma(g, all<V>(-kLog2e), bias);
#pragma unroll
    for (int i = 0; i < V; ++i) e.v[i] = gate_ex2(a.v[i]);
    r = add(e, all<V>(1.f));
#pragma unroll
    for (int i = 0; i < V; ++i) r.v[i] = gate_rcp(r.v[i]);
  }
  __device__ __forceinline__ Vec<V> z() const { return r; }
  __device__ __forceinline__ Vec<V> zk() const {  // of its own size, as a gradient that it is
    Vec<V> x;
#pragma unroll
    for (int i = 0; i < V; ++i) {
      x.v[i] = e.v[i];
      asm("min.NaN.f32 %0, %0, %1;" : "+f"(x.v[i]) : "f"(3e38f));  // r is zero where e is infinite
    }
    return mul(mul(x, r), r);
  }
  __device__ __forceinline__ Vec<V> next(Vec<V> h, Vec<V> x) const { return fma(r, minus(x, h), h); }
  __device__ __forceinline__ Vec<V> code() const { return r; }
  __device__ __forceinline__ static void part(Vec<V> code, Vec<V> R, Vec<V>& through, Vec<V>& left) {
    through = mul(code, R);
    left = less(R, code, R);
  }
};
template <typename T>
using GateOf = Gate<4 / (int)sizeof(T), sizeof(T) == 4>;

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
  Vec<kVec<T>> b = all<kVec<T>>(0.f);
  if (a.bias) b = piece(ld4(static_cast<const T*>(a.bias) + c), T{});
#pragma unroll
  for (int v = 0; v < kVec<T>; ++v) b.v[v] = GateOf<T>::bias(b.v[v]);
  return b;
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
// What stands for logits from a sequence's length on: -infinity, so that z = 0 and a position leaves every sum as it
// is.
template <typename T>
__device__ __forceinline__ uint32_t shut() {
  return sizeof(T) == 2 ? 0xFF80FF80u : 0xFF800000u;
}
// kPos rows' pieces from position t0 on, `fill` from `end` on.
template <typename T>
__device__ __forceinline__ void load_rows(uint32_t (&r)[kPos], const T* p, int64_t st, int64_t t0, int64_t end,
                                          uint32_t fill = 0u) {
  const int left = left_of(t0, end);
  p += t0 * st;
  if (left == kPos) {
#pragma unroll
    for (int u = 0; u < kPos; ++u, p += st) r[u] = ld4(p);
  } else {
#pragma unroll
    for (int u = 0; u < kPos; ++u, p += st) r[u] = u < left ? ld4(p) : fill;
  }
}

// ------------------------------------------------------------------------------------------------------------
// a chain a thread
// ------------------------------------------------------------------------------------------------------------
// Forward: a thread has 16 bytes of a row, so that loads, stores and their addresses are few beside the gates (4 bytes
// a thread: 240 us where this takes 203), and four positions, the next four's loads in flight.
constexpr int kWide = 4;
template <typename T>
struct Wide {
  static constexpr int E = 16 / (int)sizeof(T), N = E / 2;
  Vec<2> v[N];
  __device__ __forceinline__ void unpacked(const uint4& r) {
    float f[E];
    unpack(r, f, T{});
#pragma unroll
    for (int k = 0; k < N; ++k) v[k] = {f[2 * k], f[2 * k + 1]};
  }
  __device__ __forceinline__ uint4 packed() const {
    float f[E];
#pragma unroll
    for (int k = 0; k < E; ++k) f[k] = v[k / 2].v[k % 2];
    return pack(f, T{});
  }
  __device__ __forceinline__ void load(const float* p) {
#pragma unroll
    for (int k = 0; k < N; k += 2) {
      float f[4];
      unpack(ld16(p + 2 * k), f, 0.f);
      v[k] = {f[0], f[1]};
      v[k + 1] = {f[2], f[3]};
    }
  }
  __device__ __forceinline__ void store(float* p) const {
#pragma unroll
    for (int k = 0; k < N; k += 2)
      *reinterpret_cast<float4*>(p + 2 * k) = make_float4(v[k].v[0], v[k].v[1], v[k + 1].v[0], v[k + 1].v[1]);
  }
};

// kTwo (fp32 of more than 16 positions): the state in two numbers, joined every four positions, so that what a small z
// adds is not rounded to a step of the state every time (an equal sign there makes z = 1e-6 some 1e-3 off in 30000
// positions; 3000 histories of 1000, d 128: no change in time).  In bf16 that takes 20 % more time (registers), and a
// state is rounded at every position.
// A thread takes sequence after sequence, four positions at a time; the next four's loads, and the next sequence's
// length and state, are on their way while these ones' gates are computed (a sequence a thread: 203 us).  Bound by HBM:
// 150001 ragged histories of up to 12, d 128, bf16, 156 us, 0.94 of the copy rate.
template <typename T, bool kTwo>
__global__ __launch_bounds__(256, 2) void recur_fwd(RecurArgs a) {
  pdl_begin();
  using W = Wide<T>;
  using G = Gate<2, sizeof(T) == 4>;
  const int c = (blockIdx.y * blockDim.x + threadIdx.x) * W::E;
  const int64_t first = (int64_t)blockIdx.x * blockDim.y + threadIdx.y, step = (int64_t)gridDim.x * blockDim.y;
  if (c >= a.d || first >= a.n) return;
  uint4 rx[kWide], rg[kWide], nx[kWide], ng[kWide];  // this batch's rows, and the next one's
  W b, h, enter, rest;
#pragma unroll
  for (int k = 0; k < W::N; ++k) b.v[k] = enter.v[k] = all<2>(0.f);
  if (a.bias) {
    b.unpacked(ld16(static_cast<const T*>(a.bias) + c));
#pragma unroll
    for (int k = 0; k < W::N; ++k) b.v[k] = {G::bias(b.v[k].v[0]), G::bias(b.v[k].v[1])};
  }
  // the loads' place: sequence, position, rows
  int64_t li = first, lt = 0, llen = length(a, li), after = li + step < a.n ? length(a, li + step) : 0;
  const T *x = at<T>(a.x, li, 0, c), *g = at<T>(a.g, li, 0, c);
  int64_t next_len = 0;  // of the sequence that the next batch is of
  auto load = [&]() {
    if (li >= a.n) return;
    next_len = llen;
    if (lt == 0 && a.h_in) enter.load(a.h_in + li * a.d + c);
#pragma unroll
    for (int u = 0; u < kWide; ++u)
      if (lt + u < llen) {
        nx[u] = ld16(x);
        ng[u] = ld16(g);
        x += a.x.st;
        g += a.g.st;
      }
    lt += kWide;
    if (lt < llen) return;
    li += step;
    lt = 0;
    llen = after;
    if (li >= a.n) return;
    x = at<T>(a.x, li, 0, c);
    g = at<T>(a.g, li, 0, c);
    if (li + step < a.n) after = length(a, li + step);
  };
  int64_t i = first, t = 0;
  T* y = at_out<T>(a.y, i, 0, c);
  load();
#pragma unroll 1
  while (true) {
    const int64_t len = next_len;
#pragma unroll
    for (int u = 0; u < kWide; ++u) {
      rx[u] = nx[u];
      rg[u] = ng[u];
    }
    if (t == 0) {
      h = enter;
#pragma unroll
      for (int k = 0; k < W::N; ++k) rest.v[k] = all<2>(0.f);
    }
    load();
    if (a.saved && t > 0 && t % kPos == 0) h.store(kept(a, i, t, c));
#pragma unroll
    for (int u = 0; u < kWide; ++u)
      if (t + u < len) {
        W fx, fg;
        fx.unpacked(rx[u]);
        fg.unpacked(rg[u]);
#pragma unroll
        for (int k = 0; k < W::N; ++k) {
          const G gt(fg.v[k], b.v[k]);
          if constexpr (kTwo) {
            gt.next(h.v[k], rest.v[k], add(h.v[k], rest.v[k]), fx.v[k]);
            fx.v[k] = add(h.v[k], rest.v[k]);
          } else {
            fx.v[k] = h.v[k] = gt.next(h.v[k], fx.v[k]);
          }
        }
        st16(y, fx.packed());
        y += a.y.st;
      }
    if constexpr (kTwo) {
#pragma unroll
      for (int k = 0; k < W::N; ++k) settle(h.v[k], rest.v[k]);
    }
    t += kWide;
    if (t < len) continue;
#pragma unroll 1
    for (int64_t u = len; u < a.T; ++u, y += a.y.st) st16(y, make_uint4(0, 0, 0, 0));
    if (a.h_out) h.store(a.h_out + i * a.d + c);
    i += step;
    if (i >= a.n) return;
    t = 0;
    y = at_out<T>(a.y, i, 0, c);
  }
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

// The backward's forward half: a position's state, and what its gate's gradient is of R: (x - h) z k.
template <int V, bool kExact>
__device__ __forceinline__ Vec<V> slope(Vec<V>& h, Vec<V> x, const Gate<V, kExact>& g) {
  const Vec<V> diff = minus(x, h);
  h = g.next(h, x);
  return mul(diff, g.zk());
}
// And its half from the end: what R gives dx and dg, and R for the position before.
template <typename T, int V>
__device__ __forceinline__ void back(Vec<V>& R, Vec<V> dy, Vec<V> code, Vec<V> slope, Vec<V>& dx, Vec<V>& dg) {
  R = add(R, dy);
  dg = mul(slope, R);
  GateOf<T>::part(code, R, dx, R);
}

// Backward of more than 16 positions: a thread has 4 bytes of a row and 16 positions, whose states it forms from the
// one kept before them; the 16 before them, or the next sequence's last ones, are loaded meanwhile.  CTAs of 128
// threads, three an SM: ragged histories leave fewer threads waiting for the longest one than in 256, and 12 warps hide
// more than 8 (400 of up to 515, d 256, 99 -> 84 us; 2000 of them 347 -> 310 us, 0.88 of the copy rate).  Registers
// bound it: 16 positions' gates and slopes, and the next rows (bf16: 64 bytes of them are spilled).  In fp32 R is kept
// in two numbers, joined every 16 positions, as the forward's state is (3000 of 1000, d 128: 1.21 -> 1.24 ms; not in
// bf16).
constexpr int kBwdThr = 128;
template <typename T>
__global__ __launch_bounds__(kBwdThr, 3) void recur_bwd(RecurArgs a) {
  pdl_begin();
  constexpr int V = kVec<T>;
  constexpr bool kTwo = sizeof(T) == 4;
  __shared__ float sh[kBwdThr * V];
  const int c = (blockIdx.y * blockDim.x + threadIdx.x) * V;
  const bool in = c < a.d;
  const Vec<V> zero = all<V>(0.f), b = in ? bias_of<T>(a, c) : zero;
  Vec<V> sum = zero;
  const int64_t step = (int64_t)gridDim.x * blockDim.y;
  int64_t i = (int64_t)blockIdx.x * blockDim.y + threadIdx.y;
  if (in && i < a.n) {
    uint32_t rx[kPos], rg[kPos], ry[kPos];
    Vec<V> h;
    auto load = [&](int64_t s, int64_t t0, int64_t end) {
      load_rows(rx, at<T>(a.x, s, 0, c), a.x.st, t0, end);
      load_rows(rg, at<T>(a.g, s, 0, c), a.g.st, t0, end, shut<T>());
      load_rows(ry, at<T>(a.dy, s, 0, c), a.dy.st, t0, end);
      if (t0 > 0)
        ldf(kept(a, s, t0, c), h);
      else
        h = state_of<V>(a.h_in, a, s, c);
    };
    auto last_of = [](int64_t len) { return len > 0 ? (len - 1) / kPos * kPos : 0; };
    int64_t len = length(a, i), after = i + step < a.n ? length(a, i + step) : 0;
    load(i, last_of(len), len);
    Vec<V> R = state_of<V>(a.dh_out, a, i, c), rest = zero, next_R = zero;
#pragma unroll 1
    while (true) {
      T *dx = at_out<T>(a.dx, i, 0, c), *dg = at_out<T>(a.dg, i, 0, c);
#pragma unroll 1
      for (int64_t t0 = last_of(len); t0 >= 0; t0 -= kPos) {
        const int left = left_of(t0, len);
        Vec<V> sl[kPos], code[kPos];
#pragma unroll
        for (int half = 0; half < kPos; half += kPos / 2) {  // eight gates at a time: side by side
          if (half > 0 && left <= half) break;
#pragma unroll
          for (int u = half; u < half + kPos / 2; ++u) {
            const GateOf<T> gt(piece(rg[u], T{}), b);
            code[u] = gt.code();
            sl[u] = slope(h, piece(rx[u], T{}), gt);
          }
        }
        uint32_t cy[kPos];
#pragma unroll
        for (int u = 0; u < kPos; ++u) cy[u] = ry[u];
        if (t0 > 0) {
          load(i, t0 - kPos, t0);
        } else if (i + step < a.n) {
          load(i + step, last_of(after), after);
          next_R = state_of<V>(a.dh_out, a, i + step, c);
        }
        Vec<V> here = zero;
        T *px = dx + (t0 + kPos) * a.dx.st, *pg = dg + (t0 + kPos) * a.dg.st;
#pragma unroll
        for (int u = kPos - 1; u >= 0; --u) {
          px -= a.dx.st;
          pg -= a.dg.st;
          if (u < left) {
            Vec<V> ox, og;
            if constexpr (kTwo) {
              rest = add(rest, piece(cy[u], T{}));
              const Vec<V> both = add(R, rest);
              og = mul(sl[u], both);
              GateOf<T>::part(code[u], R, rest, both, ox);
            } else {
              back<T>(R, piece(cy[u], T{}), code[u], sl[u], ox, og);
            }
            here = add(here, og);
            st4(px, ox);
            st4(pg, og);
          }
        }
        if constexpr (kTwo) settle(R, rest);
        sum = add(sum, here);
      }
      // zero rows, 16 bytes at a time: four neighbouring threads take every fourth row each
      const int part = threadIdx.x % 4, back16 = part * V;
#pragma unroll 1
      for (int64_t t = len + part; t < a.T; t += 4) {
        st16(dx + t * a.dx.st - back16, make_uint4(0, 0, 0, 0));
        st16(dg + t * a.dg.st - back16, make_uint4(0, 0, 0, 0));
      }
      if (a.dh_in) stf(a.dh_in + i * a.d + c, R);
      i += step;
      if (i >= a.n) break;
      R = next_R;
      rest = zero;
      len = after;
      if (i + step < a.n) after = length(a, i + step);
    }
  }
  if (a.part)
    part_sums<V>(sum, sh, threadIdx.x, threadIdx.y, blockDim.x, blockDim.y, a.part + (int64_t)blockIdx.x * a.d + c, in);
}

// Backward of at most 16 positions: rows go through shared memory, 16 bytes a copy and a store, the next sequence's on
// their way meanwhile; a thread reads its 4 bytes of them where its positions are, four positions at a time, and leaves
// its gradients in their place.  Fewer instructions for addresses than with loads and stores of 4 bytes, a fourth CTA
// an SM where the next rows were in registers, and only a quad of threads waits for one another.  100000 ragged
// histories of up to 12, d 128, bf16, 221 us, 0.82 of the copy rate (the kernel above: 291); 50000 in fp32 184 (364);
// 150000 of one 142 (347); 50000 of 16, none ragged, 186 (173).  A third stage 261 where two take 223 (three CTAs an SM
// then), five CTAs 246 (96 registers).  Bound by the rows' bytes and by the instructions of gates.
template <int V>
struct ShortStage {  // of shared memory: a sequence's two states, then its rows of x, g and dy, position by position
  static constexpr int kPitch = kBwdThr * 4, kRow = 3 * kPitch + 32;  // a quad's four 16-byte pieces: different banks
  static constexpr int kStates = 2 * kBwdThr * 4 * V;
};
constexpr int kShortStages = 2, kShortCtas = 4, kGroup = 4;
template <typename T>
int short_bytes(int64_t T_) {
  using S = ShortStage<kVec<T>>;
  return kShortStages * (S::kStates + (int)ceil_div(T_, kGroup) * kGroup * S::kRow);
}
template <typename T>
__global__ __launch_bounds__(kBwdThr, kShortCtas) void recur_bwd_short(RecurArgs a) {
  pdl_begin();
  constexpr int V = kVec<T>;
  using S = ShortStage<V>;
  extern __shared__ __align__(128) char smem[];
  __shared__ float sh[kBwdThr * V];
  const int c = (blockIdx.y * blockDim.x + threadIdx.x) * V;
  const int tid = threadIdx.y * blockDim.x + threadIdx.x, part = tid % 4;
  const bool in = c < a.d;
  const uint32_t quad = 0xFu << (tid % 32 - part);
  const Vec<V> zero = all<V>(0.f), b = in ? bias_of<T>(a, c) : zero;
  Vec<V> sum = zero;
  const int n = (int)a.n, T_ = (int)a.T, step = gridDim.x * blockDim.y;
  const int stage_bytes = S::kStates + (T_ + kGroup - 1) / kGroup * kGroup * S::kRow;
  int i = blockIdx.x * blockDim.y + threadIdx.y;
  if (in && i < n) {
    const int c16 = c - part * V;
    auto length_at = [&](int64_t s) { return s < n ? (int)length(a, s) : 0; };
    // a sequence's rows, a quad's 16 bytes of every fourth a thread, and the thread's own states
    auto load = [&](int64_t s, int len, char* to) {
      if (s < n) {
        if (a.h_in) {
          if constexpr (V == 2)
            tc::cp_async8(to + tid * 8, a.h_in + s * a.d + c);
          else
            tc::cp_async4(to + tid * 4, a.h_in + s * a.d + c);
        }
        if (a.dh_out) {
          if constexpr (V == 2)
            tc::cp_async8(to + (kBwdThr + tid) * 8, a.dh_out + s * a.d + c);
          else
            tc::cp_async4(to + (kBwdThr + tid) * 4, a.dh_out + s * a.d + c);
        }
        if (part < len) {
          const T *x = at<T>(a.x, s, part, c16), *g = at<T>(a.g, s, part, c16), *y = at<T>(a.dy, s, part, c16);
          char* row = to + S::kStates + part * S::kRow + (tid - part) * 4;
#pragma unroll
          for (int u = 0; u < kPos; u += 4) {
            if (part + u >= len) break;
            tc::cp_async16(row + u * S::kRow, x, true);
            tc::cp_async16(row + u * S::kRow + S::kPitch, g, true);
            tc::cp_async16(row + u * S::kRow + 2 * S::kPitch, y, true);
            x += 4 * a.x.st;
            g += 4 * a.g.st;
            y += 4 * a.dy.st;
          }
        }
      }
      tc::cp_async_commit();
    };
    int lens[kShortStages + 1];  // of this sequence, of those on their way, and of the next
#pragma unroll
    for (int k = 0; k <= kShortStages; ++k) lens[k] = length_at(i + (int64_t)k * step);
    char *here = smem, *const end = smem + kShortStages * stage_bytes, *free_ = smem + (kShortStages - 1) * stage_bytes;
#pragma unroll
    for (int k = 0; k < kShortStages - 1; ++k) load(i + (int64_t)k * step, lens[k], smem + k * stage_bytes);
#pragma unroll 1
    for (; i < n; i += step) {
      __syncwarp(quad);  // the quad has read its last sequence's gradients
      load(i + (int64_t)(kShortStages - 1) * step, lens[kShortStages - 1], free_);
      const int len = lens[0];
#pragma unroll
      for (int k = 0; k < kShortStages; ++k) lens[k] = lens[k + 1];
      lens[kShortStages] = length_at(i + (int64_t)(kShortStages + 1) * step);
      tc::cp_async_wait<kShortStages - 1>();
      __syncwarp(quad);  // and its pieces of this one are here
      char* const rows = here + S::kStates + tid * 4;
      Vec<V> h = zero, R = zero;
      if (a.h_in) ldf(reinterpret_cast<const float*>(here) + tid * V, h);
      if (a.dh_out) ldf(reinterpret_cast<const float*>(here) + (kBwdThr + tid) * V, R);
      // positions of a group from len on hold what they held before: they change nothing that is used
      Vec<V> sl[kPos], code[kPos];
#pragma unroll
      for (int q = 0; q < kPos; q += kGroup) {
        if (len <= q) break;
#pragma unroll
        for (int u = q; u < q + kGroup; ++u) {
          const char* row = rows + u * S::kRow;
          const GateOf<T> gt(piece(ld4(reinterpret_cast<const T*>(row + S::kPitch)), T{}), b);
          code[u] = gt.code();
          sl[u] = slope(h, piece(ld4(reinterpret_cast<const T*>(row)), T{}), gt);
        }
      }
      Vec<V> partial = zero;
#pragma unroll
      for (int q = kPos - kGroup; q >= 0; q -= kGroup) {
        if (len <= q) continue;
#pragma unroll
        for (int u = q + kGroup - 1; u >= q; --u)
          if (u < len) {
            char* row = rows + u * S::kRow;
            Vec<V> ox, og;
            back<T>(R, piece(ld4(reinterpret_cast<const T*>(row + 2 * S::kPitch)), T{}), code[u], sl[u], ox, og);
            partial = add(partial, og);
            st4(reinterpret_cast<T*>(row), ox);
            st4(reinterpret_cast<T*>(row + S::kPitch), og);
          }
      }
      sum = add(sum, partial);
      if (a.dh_in) stf(a.dh_in + (int64_t)i * a.d + c, R);
      __syncwarp(quad);
      if (part < T_) {
        T *dx = at_out<T>(a.dx, i, part, c16), *dg = at_out<T>(a.dg, i, part, c16);
        const char* row = rows + part * S::kRow - part * 4;
#pragma unroll
        for (int u = 0; u < kPos; u += 4) {
          if (part + u >= T_) break;
          uint4 ox = make_uint4(0, 0, 0, 0), og = ox;
          if (part + u < len) {
            ox = *reinterpret_cast<const uint4*>(row + u * S::kRow);
            og = *reinterpret_cast<const uint4*>(row + u * S::kRow + S::kPitch);
          }
          st16(dx, ox);
          st16(dg, og);
          dx += 4 * a.dx.st;
          dg += 4 * a.dg.st;
        }
      }
      free_ = here;
      here += stage_bytes;
      if (here == end) here = smem;
    }
  }
  if (a.part)
    part_sums<V>(sum, sh, threadIdx.x, threadIdx.y, blockDim.x, blockDim.y, a.part + (int64_t)blockIdx.x * a.d + c, in);
}

// ------------------------------------------------------------------------------------------------------------
// a chain split over time
// ------------------------------------------------------------------------------------------------------------
// A cluster of CL CTAs takes a piece of a sequence's rows (L lanes of 4 bytes) through CL tiles of positions a step: 64
// bytes and 256 positions a tile; where even eight CTAs a piece leave SMs idle, 32 bytes and 512; in the backward,
// whose three arrays in and two out touch half as many lines so, mostly 128 bytes and 128 positions.  A thread has 16
// positions of 4 bytes.  Positions compose: a run of them maps the state h before it to B + K h, B its end from a zero
// state, K the product of its 1 - z.  Threads form the runs of their 16 positions and keep each, a CTA forms that of
// its tile and hands it to the cluster's others (distributed shared memory), and every CTA joins them in the same
// order, so all carry the same state and a call repeats its bits.
//
// A step of a CTA alone takes 1.75 us, one after another: copies into shared memory 0.55, gates 0.5, the join 0.4,
// stores 0.57, barriers 0.6, overlapping in part; two CTAs an SM take 1.3 each.  That bounds it where chains are few: 6
// histories of 32768, d 256, bf16: 82 us forward (HBM: 44).  Half as many positions a thread and twice as many threads
// took 97 us where this took 83; instructions on two numbers at once changed nothing.
//
// K itself would not do for a state: 1 - z rounded, a step of one at every position and of one sign where gates hardly
// change, makes a memory of 10^5 positions a thousandth off (an eighth more instructions an output; 6 histories of
// 32768, d 256, bf16: 78 -> 82 us).  So a run is kept as B and Q = 1 - K, both to some steps of themselves (rounded
// shares of 1 - z only weigh what has been added), and a state goes to h + (B - Q h).  In fp32 K of its own size too,
// and the state goes to B + K h where K is at most a half, as behind an open gate, which leaves no rounding of h.
template <typename T>
struct Run;
template <>
struct Run<__nv_bfloat16> {
  using G = GateOf<__nv_bfloat16>;
  using Kept = Run;
  Vec<2> Q = all<2>(0.f), B = all<2>(0.f);
  __device__ __forceinline__ Vec<2> of(Vec<2> h) const { return add(h, less(B, Q, h)); }
  __device__ __forceinline__ void position(const G& g, Vec<2> x) {  // then this one
    const Vec<2> k = minus(all<2>(1.f), g.z());
    B = fma(k, B, mul(g.z(), x));
    Q = fma(k, Q, g.z());
  }
  __device__ __forceinline__ void before(const G& g, Vec<2> dy) {  // from the end: before it this one
    Q = fma(g.z(), minus(all<2>(1.f), Q), Q);
    B = fma(minus(all<2>(1.f), Q), dy, B);
  }
  __device__ __forceinline__ void join(const Run& p) {  // this, then p
    const Vec<2> k = minus(all<2>(1.f), p.Q);
    B = fma(k, B, p.B);
    Q = fma(k, Q, p.Q);
  }
  __device__ __forceinline__ Kept kept() const { return *this; }
  __device__ __forceinline__ float4 packed() const { return make_float4(Q.v[0], Q.v[1], B.v[0], B.v[1]); }
  __device__ __forceinline__ static Run from(const float4& p) {
    Run r;
    r.Q = {p.x, p.y};
    r.B = {p.z, p.w};
    return r;
  }
};
template <>
struct Run<float> {
  using G = GateOf<float>;
  float K = 1.f, Q = 0.f, B = 0.f;
  struct Kept {  // in two numbers: share is Q, or -K where K is at most a half
    float share, B;
    __device__ __forceinline__ Vec<1> of(Vec<1> h) const {
      const float t = fmaf(-share, h.v[0], B);
      return {t + (__float_as_int(share) < 0 ? 0.f : h.v[0])};
    }
  };
  __device__ __forceinline__ Kept kept() const { return {K <= 0.5f ? -K : Q, B}; }
  __device__ __forceinline__ Vec<1> of(Vec<1> h) const { return kept().of(h); }
  __device__ __forceinline__ float gate(const G& g) {
    const float z = g.z().v[0], k = g.k().v[0];
    K *= k;
    Q = fmaf(k, Q, z);
    return k;
  }
  __device__ __forceinline__ void position(const G& g, Vec<1> x) { B = fmaf(gate(g), B, g.z().v[0] * x.v[0]); }
  __device__ __forceinline__ void before(const G& g, Vec<1> dy) {
    gate(g);
    B = fmaf(K, dy.v[0], B);
  }
  __device__ __forceinline__ void join(const Run& p) {
    B = fmaf(p.K, B, p.B);
    Q = fmaf(p.K, Q, p.Q);
    K *= p.K;
  }
  __device__ __forceinline__ float4 packed() const { return make_float4(Q < 0.5f ? 1.f - Q : K, Q, B, 0.f); }
  __device__ __forceinline__ static Run from(const float4& p) {
    Run r;
    r.K = p.x;
    r.Q = p.y;
    r.B = p.z;
    return r;
  }
};
// Runs that a lane joins one after another; of 32, two lanes join sixteen each, and then theirs.
template <int L>
constexpr int kJoin = kSubs<L> < 16 ? kSubs<L> : 16;
template <int L>
struct SplitSmem {
  float4 run[2][kSubs<L>][L];  // the threads' runs, then what is before each among its sixteen
  float4 half[2][L];           // of the first sixteen of 32
  float4 tile[2][kMaxCluster][L];
  uint64_t bar[2];  // a step's tiles have come
};

__device__ __forceinline__ int cluster_reg_rank() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
  return (int)r;
}
__device__ __forceinline__ int cluster_reg_size() {
  uint32_t r;
  asm volatile("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
  return (int)r;
}
// Every CTA runs before another one writes to it, and is there until the last one has.
__device__ __forceinline__ void cluster_meet() {
  __syncwarp();
  asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// To the same place of every CTA of the cluster, counted by the barrier at the same place there.  (A barrier of the
// whole cluster a step would wait for the rows' stores as well: 1.4 of 6.7 stall cycles an instruction.)
__device__ __forceinline__ void hand_out(float4* slot, uint64_t* bar, const float4& p, int cl) {
  const uint32_t own = tc::smem_u32(slot), own_bar = tc::smem_u32(bar);
  for (int r = 0; r < cl; ++r) {
    uint32_t there, there_bar;
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there) : "r"(own), "r"(r));
    asm volatile("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(there_bar) : "r"(own_bar), "r"(r));
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v4.f32 [%0], {%1, %2, %3, %4}, [%5];"
                 ::"r"(there), "f"(p.x), "f"(p.y), "f"(p.z), "f"(p.w), "r"(there_bar)
                 : "memory");
  }
}

// A bounded wait for a step's tiles: false when it ran out.
__device__ __forceinline__ bool tiles_here(uint64_t* bar, uint32_t parity, uint32_t polls = tc::kSpinLimit) {
  const uint32_t addr = tc::smem_u32(bar);
  for (uint32_t i = 0; i < polls; ++i) {
    uint32_t done;
    asm volatile(
        "{\n\t.reg .pred p;\n\t"
        "mbarrier.try_wait.parity.acquire.cluster.shared::cta.b64 p, [%1], %2;\n\t"
        "selp.u32 %0, 1, 0, p;\n\t}"
        : "=r"(done)
        : "r"(addr), "r"(parity)
        : "memory");
    if (done) return true;
  }
  return false;
}

template <typename T, int L>
struct Split {
  static constexpr int V = kVec<T>;
  SplitSmem<L>& sm;
  int* status;
  int cl, rank, tx, ty;
  uint32_t phase = 0;  // bit b: the parity that bar[b] comes to next; bit 2: a wait has run out
  static constexpr int kGroups = kSubs<L> / kJoin<L>, kJoiners = L * kGroups;
  static_assert(kJoiners <= 32, "the joining lanes are in one warp");

  __device__ __forceinline__ Split(SplitSmem<L>& s, int* st)
      : sm(s), status(st), cl(cluster_reg_size()), rank(cluster_reg_rank()), tx(threadIdx.x % L), ty(threadIdx.x / L) {
    if (threadIdx.x == 0) {
      tc::mbar_init(&sm.bar[0], 1 + kJoiners);
      tc::mbar_init(&sm.bar[1], 1 + kJoiners);
      tc::fence_mbar_init();
    }
    __syncthreads();
  }
  // The state that enters this thread's run, in the order of positions or from the end; `state`, of the step before, is
  // carried on.  `then` is done by all threads when all have formed their runs.  A CTA hands out step s + 1 after all
  // its threads have read step s, and enters s + 2 after every other one has handed out s + 1: two places are enough.
  template <bool kBack, typename F>
  __device__ __forceinline__ Vec<V> enter(const Run<T>& mine, Vec<V>& state, int buf, F then) {
    auto at = [](int k, int count) { return kBack ? count - 1 - k : k; };
    sm.run[buf][ty][tx] = mine.packed();
    if (cl > 1 && phase < 4 && threadIdx.x == 0) tc::mbar_expect_tx(&sm.bar[buf], (uint32_t)(cl * L * sizeof(float4)));
    __syncthreads();
    if (threadIdx.x < kJoiners) {
      const int group = threadIdx.x / L;
      Run<T> whole;
#pragma unroll
      for (int k = 0; k < kJoin<L>; ++k) {
        float4& p = sm.run[buf][at(group * kJoin<L> + k, kSubs<L>)][tx];
        const Run<T> own = Run<T>::from(p);
        p = whole.packed();
        whole.join(own);
      }
      if constexpr (kGroups == 2) {
        float4 w = whole.packed();
        if (group == 0) sm.half[buf][tx] = w;
        w.x = __shfl_xor_sync(0xffffu, w.x, L);
        w.y = __shfl_xor_sync(0xffffu, w.y, L);
        w.z = __shfl_xor_sync(0xffffu, w.z, L);
        w.w = __shfl_xor_sync(0xffffu, w.w, L);
        Run<T> first = Run<T>::from(w);
        first.join(whole);
        whole = first;
      }
      if (cl == 1) {
        if (group == kGroups - 1) sm.tile[buf][0][tx] = whole.packed();
      } else if (phase < 4) {
        if (group == kGroups - 1) hand_out(&sm.tile[buf][rank][tx], &sm.bar[buf], whole.packed(), cl);
        tc::mbar_arrive(&sm.bar[buf]);
      }
    }
    then();
    if (cl == 1) {
      __syncthreads();
    } else if (phase < 4) {
      if (tiles_here(&sm.bar[buf], phase >> buf & 1)) {
        phase ^= 1u << buf;
      } else {  // this call's results are invalid; this thread neither waits nor arrives any more, and every loop ends
        phase |= 4;
        record_device_error(status, tc::kErrTimeout);
      }
    }
    const float4* t = &sm.tile[buf][0][tx];
    auto tile = [&](int k) { return Run<T>::from(t[at(k, cl) * L]); };
    int k = 0;
    for (; at(k, cl) != rank; ++k) state = tile(k).of(state);
    Vec<V> got = state;
    if (kGroups == 2 && at(ty, kSubs<L>) >= kJoin<L>) got = Run<T>::from(sm.half[buf][tx]).of(got);
    got = Run<T>::from(sm.run[buf][ty][tx]).of(got);
    for (; k < cl; ++k) state = tile(k).of(state);
    return got;
  }
  // When every CTA has handed out its last: what is on its way to this one comes before it ends.  (Each step has waited
  // for it; after a wait that ran out, a while.)
  __device__ __forceinline__ void finish() {
    __syncwarp();
    cluster_meet();
    if (phase >= 4)
      for (int b = 0; b < 2; ++b) tiles_here(&sm.bar[b], phase >> b & 1, 1u << 12);
  }
};

// A tile of rows' pieces in shared memory, 4 L bytes a row: rows change places within groups of 32 / L by the thread
// along time that they are of, which puts the rows that a warp's threads along time read together into different banks.
constexpr int kTileBytes = kSplitThr * kPos * 4;
template <int L>
__device__ __forceinline__ int tile_row(int r) {
  return (r ^ (r / kPos & (32 / L - 1))) * L * 4;
}
template <int L>
struct RunRows {  // a thread's rows
  static constexpr int M = 32 / L;
  const char* p[M];
  __device__ __forceinline__ RunRows(const char* tile, int ty, int tx) {
#pragma unroll
    for (int m = 0; m < M; ++m) p[m] = tile + (ty * kPos + (m ^ (ty & (M - 1)))) * L * 4 + tx * 4;
  }
  __device__ __forceinline__ uint32_t operator[](int u) const {
    return *reinterpret_cast<const uint32_t*>(p[u % M] + u / M * M * L * 4);
  }
};

// kStreams arrays' tiles, each step's asked for kStages - 1 steps ahead.  Array 1 is the gates': from the sequence's
// length on its logits are -infinity and the others' values zero, so no position needs a look at the length.
template <typename T, int L, int kStreams, int kStages>
struct Stages {
  static constexpr size_t kBytes = (size_t)kStages * kStreams * kTileBytes;
  static constexpr int kPieces = L / 4;                 // 16-byte pieces of a row
  static constexpr int kApart = kSplitThr / kPieces;    // a thread's rows' distance
  static constexpr int kRows = kTile<L> / kApart;       // ... and number
  char* smem;               // of this thread's first row
  const char* p[kStreams];  // its row of the next tile
  int64_t left;             // rows in use from that row on
  int stage = 0;
  bool in;
  __device__ __forceinline__ explicit Stages(char* base)
      : smem(base + tile_row<L>(threadIdx.x / kPieces) + threadIdx.x % kPieces * 16) {}
  // A sequence's tiles begin at t0.
  __device__ __forceinline__ void begin(const Rows (&r)[kStreams], int64_t i, int64_t t0, int64_t len, int c0, int d) {
    const int r0 = threadIdx.x / kPieces, c = c0 + threadIdx.x % kPieces * (16 / (int)sizeof(T));
    in = c < d;
    left = len - t0 - r0;
#pragma unroll
    for (int k = 0; k < kStreams; ++k) p[k] = reinterpret_cast<const char*>(at<T>(r[k], i, t0 + r0, c));
  }
  // The next tile of each array, `by` rows before the one after it.
  __device__ __forceinline__ void ask(const Rows (&rows)[kStreams], int64_t by) {
    char* const to = smem + stage * kStreams * kTileBytes;
#pragma unroll
    for (int k = 0; k < kStreams; ++k) {
      const char* from = p[k];
      const int64_t row = kApart * rows[k].st * (int64_t)sizeof(T);
      if (in && left > kApart * (kRows - 1)) {
#pragma unroll
        for (int m = 0; m < kRows; ++m, from += row)
          tc::cp_async16(to + k * kTileBytes + m * kApart * L * 4, from, true);
      } else {
        const uint32_t f = k == 1 ? shut<T>() : 0u;
#pragma unroll
        for (int m = 0; m < kRows; ++m, from += row) {
          if (in && left > kApart * m)
            tc::cp_async16(to + k * kTileBytes + m * kApart * L * 4, from, true);
          else
            st16(to + k * kTileBytes + m * kApart * L * 4, make_uint4(f, f, f, f));
        }
      }
      p[k] += by * rows[k].st * (int64_t)sizeof(T);
    }
    left -= by;
    stage = stage + 1 == kStages ? 0 : stage + 1;
  }
};

constexpr int kFwdStages = 3, kBwdStages = 4;

template <typename T, int L>
__global__ __launch_bounds__(kSplitThr, 2) void recur_fwd_split(RecurArgs a) {
  pdl_begin();
  constexpr int V = kVec<T>;
  extern __shared__ __align__(128) char smem[];
  __shared__ SplitSmem<L> sm;
  Split<T, L> sp(sm, a.status);
  const Rows in_rows[2] = {a.x, a.g};
  const int CL = sp.cl, rank = sp.rank, tx = sp.tx, sub = sp.ty;
  const int items = (int)(a.n * a.blocks), stride = gridDim.x / CL, first = blockIdx.x / CL;
  auto steps_of = [&](int64_t len) { return (int)((len + CL * kTile<L> - 1) / (CL * kTile<L>)); };
  // The loads run ahead from piece to piece; a piece's length, bias and state are asked for a piece ahead.
  Stages<T, L, 2, kFwdStages> tiles(smem);
  int l_item = first, l_steps = 0;
  auto begin = [&]() {
    const int64_t i = l_item / a.blocks, len = length(a, i);
    l_steps = steps_of(len);
    tiles.begin(in_rows, i, rank * kTile<L>, len, l_item % a.blocks * L * V, a.d);
  };
  if (l_item < items) begin();
  auto ask = [&]() {
    while (l_steps == 0 && l_item < items) {
      l_item += stride;
      if (l_item < items) begin();
    }
    if (l_item < items) {
      tiles.ask(in_rows, CL * kTile<L>);
      --l_steps;
    }
    tc::cp_async_commit();
  };
  int64_t next_len = 0;
  Vec<V> next_b = all<V>(0.f), next_h = next_b;
  auto fetch = [&](int item) {
    if (item >= items) return;
    const int64_t i = item / a.blocks;
    const int c = item % a.blocks * L * V + tx * V;
    next_len = length(a, i);
    if (c >= a.d) return;
    next_b = bias_of<T>(a, c);
    next_h = state_of<V>(a.h_in, a, i, c);
  };
  fetch(first);
#pragma unroll 1
  for (int s = 0; s < kFwdStages - 1; ++s) ask();
  tc::cp_async_wait<kFwdStages - 2>();
  cluster_meet();
  int stage = 0, buf = 0;
#pragma unroll 1
  for (int item = first; item < items; item += stride) {
    const int64_t i = item / a.blocks, len = next_len;
    const int c = item % a.blocks * L * V + tx * V, steps = steps_of(len);
    const bool in = c < a.d;
    T* const y = at_out<T>(a.y, i, 0, c);
    const Vec<V> b = next_b;
    Vec<V> h = next_h;
    fetch(item + stride);
#pragma unroll 1
    for (int s = 0; s < steps; ++s, buf ^= 1) {
      const int64_t t0 = ((int64_t)s * CL + rank) * kTile<L> + sub * kPos;
      const char* const tile = smem + stage * 2 * kTileBytes;
      stage = stage + 1 == kFwdStages ? 0 : stage + 1;
      const RunRows<L> px(tile, sub, tx), pg(tile + kTileBytes, sub, tx);
      Run<T> now;
      typename Run<T>::Kept run[kPos];
#pragma unroll
      for (int u = 0; u < kPos; ++u) {
        now.position(GateOf<T>(piece(pg[u], T{}), b), piece(px[u], T{}));
        run[u] = now.kept();
      }
      tc::cp_async_wait<kFwdStages - 3>();
      const Vec<V> h0 = sp.template enter<false>(now, h, buf, ask);
      const int left = in ? left_of(t0, len) : 0;
      if (a.saved && t0 > 0 && left > 0) stf(kept(a, i, t0, c), h0);
      T* py = y + t0 * a.y.st;
      if (left == kPos) {
#pragma unroll
        for (int u = 0; u < kPos; ++u, py += a.y.st) st4(py, run[u].of(h0));
      } else {
#pragma unroll
        for (int u = 0; u < kPos; ++u, py += a.y.st)
          if (u < left) st4(py, run[u].of(h0));
      }
    }
    if (!in) continue;
#pragma unroll 1
    for (int64_t t = len + rank * kSubs<L> + sub; t < a.T; t += CL * kSubs<L>) st4(y + t * a.y.st, all<V>(0.f));
    if (a.h_out && rank == 0 && sub == 0) stf(a.h_out + i * a.d + c, h);
  }
  sp.finish();
}

// The same from the end: a run of positions maps the R that enters from the right to B + K R.  The states before each
// thread's 16 positions are the forward's.
template <typename T, int L>
__global__ __launch_bounds__(kSplitThr, 1) void recur_bwd_split(RecurArgs a) {
  pdl_begin();
  constexpr int V = kVec<T>;
  extern __shared__ __align__(128) char smem[];
  __shared__ SplitSmem<L> sm;
  __shared__ float sh[256 * V];
  Split<T, L> sp(sm, a.status);
  const Rows in_rows[3] = {a.x, a.g, a.dy};
  const int CL = sp.cl, rank = sp.rank, tx = sp.tx, sub = sp.ty;
  const int64_t item = blockIdx.x / CL, i = item / a.blocks;
  const int c0 = (int)(item % a.blocks) * L * V, c = c0 + tx * V;
  const bool in = c < a.d;
  const int64_t len = length(a, i), steps = (len + CL * kTile<L> - 1) / (CL * kTile<L>);
  auto start = [&](int64_t s) { return ((steps - 1 - s) * CL + rank) * kTile<L>; };  // steps from the end
  Stages<T, L, 3, kBwdStages> tiles(smem);
  tiles.begin(in_rows, i, start(0), len, c0, a.d);
  auto ask = [&](int64_t s) {
    if (s < steps) tiles.ask(in_rows, -CL * kTile<L>);
    tc::cp_async_commit();
  };
  const Vec<V> zero = all<V>(0.f);
  auto before = [&](int64_t t0) {  // the state before this thread's positions
    Vec<V> h = zero;
    if (in && t0 < len) {
      if (t0 > 0)
        ldf(kept(a, i, t0, c), h);
      else
        h = state_of<V>(a.h_in, a, i, c);
    }
    return h;
  };
  for (int s = 0; s < kBwdStages - 1; ++s) ask(s);
  T *dx = at_out<T>(a.dx, i, 0, c), *dg = at_out<T>(a.dg, i, 0, c);
  const Vec<V> b = in ? bias_of<T>(a, c) : zero;
  Vec<V> R = in ? state_of<V>(a.dh_out, a, i, c) : zero, sum = zero;
  Vec<V> ahead = steps > 0 ? before(start(0) + sub * kPos) : zero;
  tc::cp_async_wait<kBwdStages - 2>();
  cluster_meet();
  int stage = 0;
  for (int64_t s = 0; s < steps; ++s) {
    const int64_t t0 = start(s) + sub * kPos;
    const int left = in ? left_of(t0, len) : 0;
    const char* const tile = smem + stage * 3 * kTileBytes;
    stage = stage + 1 == kBwdStages ? 0 : stage + 1;
    const RunRows<L> qx(tile, sub, tx), qg(tile + kTileBytes, sub, tx), qy(tile + 2 * kTileBytes, sub, tx);
    Vec<V> h = ahead;
    if (s + 1 < steps) ahead = before(start(s + 1) + sub * kPos);
    Vec<V> sl[kPos], code[kPos];
    Run<T> run;  // B = sum of dy_u times the product of 1 - z up to u
#pragma unroll
    for (int u = 0; u < kPos; ++u) {
      const GateOf<T> gt(piece(qg[u], T{}), b);
      code[u] = gt.code();
      sl[u] = slope(h, piece(qx[u], T{}), gt);
      run.before(gt, piece(qy[u], T{}));
    }
    tc::cp_async_wait<kBwdStages - 3>();
    Vec<V> r = sp.template enter<true>(run, R, s & 1, [&] { ask(s + kBwdStages - 1); }), here = zero;
    T *px = dx + (t0 + kPos) * a.dx.st, *pg = dg + (t0 + kPos) * a.dg.st;
#pragma unroll
    for (int u = kPos - 1; u >= 0; --u) {
      px -= a.dx.st;
      pg -= a.dg.st;
      Vec<V> ox, og;
      back<T>(r, piece(qy[u], T{}), code[u], sl[u], ox, og);
      if (u < left) {
        here = add(here, og);
        st4(px, ox);
        st4(pg, og);
      }
    }
    sum = add(sum, here);
  }
  sp.finish();
  if (in) {
    for (int64_t t = len + rank * kSubs<L> + sub; t < a.T; t += CL * kSubs<L>) {
      st4(dx + t * a.dx.st, zero);
      st4(dg + t * a.dg.st, zero);
    }
    if (a.dh_in && rank == 0 && sub == 0) stf(a.dh_in + i * a.d + c, R);
  }
  if (a.part) part_sums<V>(sum, sh, tx, sub, L, kSubs<L>, a.part + (i * CL + rank) * a.d + c, in);
}

// ------------------------------------------------------------------------------------------------------------
// the bias's gradient, one snapshot
// ------------------------------------------------------------------------------------------------------------
// Column sums of `rows` partial rows: 32 runs a CTA of 32 columns, joined in order.
__global__ __launch_bounds__(1024) void recur_bias_sum(const float* part, int64_t rows, int32_t d, float* out) {
  pdl_begin();
  __shared__ float sh[32][32];
  const int tx = threadIdx.x % 32, ty = threadIdx.x / 32, c = blockIdx.x * 32 + tx;
  float s = 0.f;
  if (c < d) {
#pragma unroll 8
    for (int64_t r = ty; r < rows; r += 32) s += part[r * d + c];
  }
  sh[ty][tx] = s;
  __syncthreads();
  if (ty != 0 || c >= d) return;
  for (int k = 1; k < 32; ++k) s += sh[k][tx];
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
    for (int v = 0; v < E; ++v) {
      using G = Gate<1, true>;
      o[v] = h[v] = G(Vec<1>{g[v]}, Vec<1>{G::bias(b[v])}).next(Vec<1>{h[v]}, Vec<1>{x[v]}).v[0];
    }
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
// Rows of up to `threads` lanes a CTA; short ones share it.
Shape shape_of(int64_t lanes, int threads = 256, int unit = 1) {
  const int64_t across = ceil_div(lanes, threads), width = ceil_div(ceil_div(lanes, across), unit) * unit;
  return {dim3((unsigned)width, (unsigned)(threads / width)), (unsigned)across};
}

// Split over time, and how (lanes 0: a chain a thread)?  The least time by a model of the measured parts, in us: a
// chain takes 0.2 a position forward and 0.085 backward; a split step some 1.5 forward and 2 backward, longer with more
// CTAs to hand runs to, and longer where two CTAs share an SM; a CTA's beginning 0.5 and 3 (the forward's go on to the
// next piece), and the kernel's 2.5 more than a chain's.  `held` is how many clusters of each size the GPU holds at
// once.  Measured, chain / split: 77 fp32 histories of up to 1001, d 200, forward 192 / 36 us; 400 of up to 515, d 256,
// 112 / 66; 1000 of 100, d 128, 28 / 50; backward 80 / 57, 85 / 109, 31 / 72.  By clusters of 1, 2, 3, 4, 6 and 8, 6
// histories of 32768, d 256: forward 191, 105, 84, 77 (with runs as 1 - K: 82), 134, 99; backward with pieces of 128
// bytes 474, 246, 172, 132, 185, 148 (64 bytes: 262, 139, 146, 146, 168, 199).
constexpr int64_t kMaxPartRows = 4096;  // of the split backward (some 3000 sequences and more are faster as chains)
struct SplitHow {
  int lanes, cl, held;  // lanes 0: a chain a thread
};
SplitHow split_of(const hg_recur_params* p, int64_t n, int64_t T, bool back) {
  static const int held[2][kMaxCluster] = {{304, 152, 97, 74, 58, 46, 38, 36}, {152, 76, 46, 36, 28, 23, 15, 15}};
  SplitHow how{0, 0, 0};
  if (T <= kPos || n == 0) return how;
  const int64_t lanes = p->d * (p->dtype == HG_BF16 ? 2 : 4) / 4;
  const Shape s = back ? shape_of(lanes, kBwdThr, 4) : shape_of(lanes / 4);
  const int64_t ctas = ceil_div(n, s.block.y) * s.across;
  double best = 3 + (back ? 0.085 : 0.2) * T * ceil_div(ctas, back ? 456 : 304);
  auto waves = [](int64_t count, int c) {  // of `count` clusters at once: how long beside one CTA an SM
    const double full = count * c / 152.0;
    return full <= 1 ? 1.0 : c == 1 ? 0.4 + 0.6 * full : full;
  };
  for (int L = back ? 32 : 16; L >= 8; L /= 2) {
    const int64_t items = n * ceil_div(lanes, L), tile = kSplitThr / L * kPos;
    if (items >= int64_t(1) << 28) break;
    for (int c = 1; c <= kMaxCluster; ++c) {
      if (back && n * c > kMaxPartRows) break;
      const int h = held[back][c - 1];
      const double step = (back ? 2.05 + 0.06 * (c - 1) : 1.5 + 0.09 * (c - 1)) + (L == 8 ? 0.2 : L == 32 ? -0.2 : 0);
      const double w = items / h * waves(h, c) + (items % h ? waves(items % h, c) : 0);
      const double cost = ceil_div(T, c * tile) * step * w + (back ? 3 : 0.5) * ceil_div(items, h) + 2.5;
      if (cost < best) {
        best = cost;
        how = {L, c, h};
      }
    }
  }
  return how;
}

// CTAs of short histories that an SM holds.
int short_ctas(const hg_recur_params* p, int64_t T) {
  const int bytes = p->dtype == HG_BF16 ? short_bytes<__nv_bfloat16>(T) : short_bytes<float>(T);
  return std::min(kShortCtas, (227 << 10) / (bytes + (2 << 10)));
}
// Rows of partial sums of the bias's gradient: chains' CTAs.  Short histories: as many as run at once, each from one to
// the next; long ones differ too much for that.
int64_t chain_rows(const hg_recur_params* p, int64_t n, int64_t T) {
  const Shape s = shape_of(p->d * (p->dtype == HG_BF16 ? 2 : 4) / 4, kBwdThr, 4);
  const int64_t most = T <= kPos ? 152 * short_ctas(p, T) : T <= 64 ? 152 * 3 : 152 * 16;
  return std::min(ceil_div(n, s.block.y), std::max<int64_t>(1, most / s.across));
}
int64_t part_rows(const hg_recur_params* p, int64_t n, int64_t T) {
  const SplitHow how = split_of(p, n, T, true);
  return how.lanes ? n * how.cl : chain_rows(p, n, T);
}
// No fewer than of any n and T up to these.
int64_t most_part_rows(const hg_recur_params* p, int64_t n, int64_t T) {
  int64_t rows = std::max(chain_rows(p, n, std::min<int64_t>(T, 1)), chain_rows(p, n, T));
  if (T > kPos) rows = std::max(rows, std::min(n * kMaxCluster, kMaxPartRows));
  return rows;
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

// A kernel's dynamic shared memory, allowed once for each kernel.
template <auto* kKernel>
hg_status allow_smem(size_t bytes) {
  static bool done = false;
  if (!done) HG_CUDA(cudaFuncSetAttribute(kKernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)bytes));
  done = true;
  return HG_OK;
}

template <typename T, int L>
hg_status forward_split(const RecurArgs& a, int cl, int held, cudaStream_t s) {
  constexpr size_t smem = Stages<T, L, 2, kFwdStages>::kBytes;
  HG_TRY((allow_smem<recur_fwd_split<T, L>>(smem)));
  return launch_clusters("recur_fwd_split", recur_fwd_split<T, L>,
                         dim3((unsigned)(std::min<int64_t>(a.n * a.blocks, held) * cl)), dim3(kSplitThr),
                         smem, s, cl, a);
}
template <typename T>
hg_status forward(RecurArgs& a, SplitHow how, cudaStream_t s) {
  const int64_t lanes = a.d / kVec<T>;
  if (how.lanes == 0) {
    const Shape sh = shape_of(a.d / Wide<T>::E);
    const int64_t groups = ceil_div(a.n, sh.block.y), most = std::max<int64_t>(1, 2 * 152 / sh.across);
    const dim3 grid((unsigned)std::min(groups, most), sh.across);
    if constexpr (sizeof(T) == 4)
      if (a.T > kPos) return launch("recur_fwd", recur_fwd<T, true>, grid, sh.block, 0, s, a);
    return launch("recur_fwd", recur_fwd<T, false>, grid, sh.block, 0, s, a);
  }
  a.blocks = (int32_t)ceil_div(lanes, how.lanes);
  return how.lanes == 16 ? forward_split<T, 16>(a, how.cl, how.held, s) : forward_split<T, 8>(a, how.cl, how.held, s);
}

template <typename T, int L>
hg_status backward_split(const RecurArgs& a, int cl, cudaStream_t s) {
  constexpr size_t smem = Stages<T, L, 3, kBwdStages>::kBytes;
  HG_TRY((allow_smem<recur_bwd_split<T, L>>(smem)));
  return launch_clusters("recur_bwd_split", recur_bwd_split<T, L>, dim3((unsigned)(a.n * a.blocks * cl)),
                         dim3(kSplitThr), smem, s, cl, a);
}
template <typename T>
hg_status backward(RecurArgs& a, SplitHow how, int64_t rows, cudaStream_t s) {
  const int64_t lanes = a.d / kVec<T>;
  if (how.lanes == 0) {
    const Shape sh = shape_of(lanes, kBwdThr, 4);
    const dim3 grid((unsigned)rows, sh.across);
    if (a.T <= kPos) {
      HG_TRY((allow_smem<recur_bwd_short<T>>((size_t)short_bytes<T>(kPos))));
      return launch("recur_bwd_short", recur_bwd_short<T>, grid, sh.block, (size_t)short_bytes<T>(a.T), s, a);
    }
    return launch("recur_bwd", recur_bwd<T>, grid, sh.block, 0, s, a);
  }
  a.blocks = (int32_t)ceil_div(lanes, how.lanes);
  if (how.lanes == 32) return backward_split<T, 32>(a, how.cl, s);
  return how.lanes == 16 ? backward_split<T, 16>(a, how.cl, s) : backward_split<T, 8>(a, how.cl, s);
}

RecurArgs args_of(const hg_recur_params* p, int64_t n, int64_t T) {
  RecurArgs a{};
  a.bias = p->bias;
  a.n = n;
  a.T = T;
  a.spans = T > 0 ? (T - 1) / kPos : 0;
  a.d = p->d;
  a.status = device_status_ptr();
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
  *scratch_bytes = align_up(sizeof(float) * (size_t)most_part_rows(params, n, T) * params->d);
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
  const SplitHow how = split_of(params, n, T, false);
  return params->dtype == HG_BF16 ? forward<__nv_bfloat16>(a, how, s) : forward<float>(a, how, s);
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
    const RowSet sc = block_set(dbias ? scratch : nullptr, 4 * rows * w), ln = block_set(lens, 4 * n);
    const RowSet bias = block_set(params->bias, w * (int64_t)esz);
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
    const SplitHow how = split_of(params, n, T, true);
    HG_TRY(params->dtype == HG_BF16 ? backward<__nv_bfloat16>(a, how, rows, s) : backward<float>(a, how, rows, s));
  }
  if (!dbias) return HG_OK;
  return launch("recur_bias_sum", recur_bias_sum, dim3((unsigned)ceil_div(w, 32)), dim3(1024), 0, s, a.part,
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
