// A whole layer of experts for a few rows (hg_moe_fwd):
//   moe_router    l = x W_router, the top_k largest, their weights; a CTA a row
//   moe_experts   (act(x W_gate[e]) * (x W_up[e])) W_down[e] for each expert e and the rows that chose it
//   moe_sum       Y = sum of a row's w_j times what expert e_j gave it (+ x); one or two rows: often moe_experts
//
// With a few rows an expert the weights are the work: 3 d f values of every expert that a row chose are read once, with
// one multiplication and addition a row for each (16 rows of bf16: 16 flops a byte, where the tensor pipe has 280 a
// byte of HBM).  So moe_experts is a stream of weights: the chosen experts' hidden features in chunks of 64 bytes of a
// W_gate row are one list, cut into equal shares, a CTA a share, with some 100 KB of copies ahead of the products.  A
// share may begin and end inside an expert; a pass over an expert's chunks serves up to 64 of its rows.  What a share
// gives a pass's rows (d sums each, fp32) goes to scratch and is added up in the order of the list, whichever CTA was
// last.  mma.sync has the room: a tile of sixteen rows is what few rows fill, and an instruction on 128 would run at an
// eighth of its rate.
//
// 64 rows, two of 64 experts each, d 256, f 1024, bf16: 24 us for the 87 MB that they chose; of that 3 us for the list
// and the rows, 2 us until the first chunks are there, 13 us of weights; f 4096: 66 us, so beyond the beginning the
// weights come at 6.3 TB/s (0.93 of the copy rate).  300 rows, four of 32 experts each, f 704 (33 rows a pass): 21 us,
// bound by a pass's products (1.4 us a chunk, half of it the second product with its two terms of H).
#include <algorithm>

#include "ffn_kernels.cuh"
#include "layer_kernels.cuh"
#include "row_sets.cuh"
#include "tc_util.cuh"

namespace hg {
namespace {

constexpr int kSms = 152;
constexpr int kThr = 256;
constexpr int kMaxRows = 1024, kMaxExperts = 256, kMaxTop = 8, kMaxF = 16384;
constexpr int kGroup = 64;  // rows of an expert that a pass over its weights serves
// The CTA that brings a row's last share adds the shares up, one launch less, where the rows that may come to one CTA
// take it at most two rounds: it has one row after another, and kThr / d of a row's experts at a time, of which a
// launch of its own has all at once.  Calls in a graph, weights from HBM, without / with that launch, f 1024 and 4096
// (and 16384):
//   one row     two of 8 experts, d 128 (one round): 17.5 / 19.6, 21.6 / 25.8 (25.7 / 29.9) us;  d 256 (two): 19.6 /
//               19.6, 25.7 / 25.8 (33.9 / 34.0);  eight of 64, d 128 (four): 21.6 / 19.6, 27.7 / 25.8 (44 / 40), d 256
//               (eight): 28 / 26, 38 / 34
//   two rows    one of two, d 256 (two): 17.5 / 18.6, 21.7 / 26.8 (34 / 35);  two of two, d 128 (two): 19.6 / 19.6,
//               25.7 / 24.7 (29.9 / 29.8), d 256 (four): 21.6 / 19.6, 31.9 / 25.7 (40 / 34)
//   three rows  of one expert, d 128 (three): 19.6 / 17.6, 29.8 / 25.8 (36 / 30) us
constexpr int kMaxRounds = 2;
constexpr int kMaxPasses = kMaxExperts + kMaxRows * kMaxTop / kGroup;

struct MoeArgs {
  const void *x, *wr, *wg, *wu, *wd;
  const int32_t* live;
  void* y;
  int32_t* experts_out;  // null: not wanted
  float* weights_out;
  int32_t* sel;      // [n][top] chosen expert, -1: none
  float* w;          // [n][top]
  int32_t* row_in;   // [n] shares that have arrived
  int32_t* place;    // [n][top] pass * group + row in it
  int32_t* items;    // chunks of all passes
  int* status;       // the library's device status word
  float* part;       // [CTA + pass][group][d]
  int32_t n, d, f, experts, top, renorm, residual, group;
  int32_t last;      // the CTA that brings a row's last share adds them up (else moe_sum does)
};

// ------------------------------------------------------------------------------------------------------------
// router
// ------------------------------------------------------------------------------------------------------------
// The choice hangs on differences of logits, so these are sums of two fp32 numbers: a product and what it lost, a sum
// and what it lost.  Off by d 2^-48 of the sum of the terms' sizes.
struct Two {
  float hi = 0.f, lo = 0.f;
  __device__ __forceinline__ void add(float v, float rest) {
    const float s = __fadd_rn(hi, v), b = __fsub_rn(s, hi);
    lo = __fadd_rn(lo, __fadd_rn(__fadd_rn(__fsub_rn(hi, __fsub_rn(s, b)), __fsub_rn(v, b)), rest));
    hi = s;
  }
  template <bool kExact>  // the product of two bf16 numbers is an fp32 number
  __device__ __forceinline__ void add_product(float a, float b) {
    const float p = __fmul_rn(a, b);
    if constexpr (kExact) {
      const float s = __fadd_rn(hi, p), c = __fsub_rn(s, hi);
      lo = __fadd_rn(lo, __fadd_rn(__fsub_rn(hi, __fsub_rn(s, c)), __fsub_rn(p, c)));
      hi = s;
    } else {
      add(p, fmaf(a, b, -p));
    }
  }
  // As one number in two parts that do not overlap; an infinity has no rest, NaN counts as more than an infinity.
  __device__ __forceinline__ float2 key() const {
    if (isnan(hi)) return make_float2(INFINITY, INFINITY);
    if (isinf(hi)) return make_float2(hi, 0.f);
    const float s = __fadd_rn(hi, lo);
    return make_float2(s, __fsub_rn(lo, __fsub_rn(s, hi)));
  }
};

// A CTA a row: an expert's logit is summed by `parts` threads, sixteen weights' loads in flight each.
constexpr int kRouterThr = 1024, kMaxParts = 16;
template <typename T>
__global__ __launch_bounds__(kRouterThr) void moe_router(MoeArgs a, int width, int parts) {
  pdl_begin();
  pdl_next();
  __shared__ __align__(16) float xs[256];
  __shared__ float2 sums[kRouterThr], keys[kMaxExperts];
  __shared__ float warp_sum[kMaxExperts / 32];
  __shared__ int chosen[kMaxTop], before[kMaxExperts];
  __shared__ float pw[kMaxTop];
  __shared__ float raw[kMaxExperts];
  const int row = blockIdx.x, tid = threadIdx.x, d = a.d, E = a.experts, top = a.top;
  if (tid == 0) a.row_in[row] = 0;
  if (a.live && a.live[row] <= 0) {
    if (tid < top) {
      a.sel[row * top + tid] = -1;
      if (a.experts_out) a.experts_out[row * top + tid] = -1;
      if (a.weights_out) a.weights_out[row * top + tid] = 0.f;
    }
    if (tid < d) static_cast<T*>(a.y)[(int64_t)row * d + tid] = from_f32<T>(0.f);
    return;
  }
  const int e = tid % width, part = tid / width, per = d / parts;
  if (tid < d) xs[tid] = to_f32(static_cast<const T*>(a.x)[(int64_t)row * d + tid]);
  if (tid < E) before[tid] = 0;
  const bool mine = part < parts && e < E;
  const T* wr = static_cast<const T*>(a.wr) + (int64_t)part * per * E + e;
  T v[16];
  auto fetch = [&](int k0) {  // per is a multiple of four
#pragma unroll
    for (int k = 0; k < 16; k += 4)
      if (k0 + k < per) {
#pragma unroll
        for (int j = 0; j < 4; ++j) v[k + j] = wr[(k0 + k + j) * E];
      }
  };
  if (mine) fetch(0);
  __syncthreads();
  if (mine) {
    Two l;
#pragma unroll 1
    for (int k0 = 0; k0 < per; k0 += 16) {
      if (k0 > 0) fetch(k0);
#pragma unroll
      for (int k = 0; k < 16; k += 4)
        if (k0 + k < per) {
          const float4 x = *reinterpret_cast<const float4*>(&xs[part * per + k0 + k]);
          l.add_product<sizeof(T) == 2>(x.x, to_f32(v[k]));
          l.add_product<sizeof(T) == 2>(x.y, to_f32(v[k + 1]));
          l.add_product<sizeof(T) == 2>(x.z, to_f32(v[k + 2]));
          l.add_product<sizeof(T) == 2>(x.w, to_f32(v[k + 3]));
        }
    }
    sums[tid] = make_float2(l.hi, l.lo);
  }
  __syncthreads();
  if (tid < E) {
    Two l;
#pragma unroll 4
    for (int p = 0; p < parts; ++p) l.add(sums[p * width + tid].x, sums[p * width + tid].y);
    raw[tid] = l.hi;
    keys[tid] = l.key();
  }
  __syncthreads();
  // an expert's place is the number of those before it
  if (mine) {
    const float2 me = keys[e];
    int n = 0;
#pragma unroll 4
    for (int j = part; j < E; j += parts) {
      const float2 o = keys[j];
      n += o.x > me.x || (o.x == me.x && (o.y > me.y || (o.y == me.y && j < e)));
    }
    if (n > 0) atomicAdd(&before[e], n);
  }
  __syncthreads();
  if (tid < E && before[tid] < top) chosen[before[tid]] = tid;
  __syncthreads();
  // the largest is taken off in both parts; with a NaN among the logits every weight is NaN
  const float2 most = keys[chosen[0]];
  const bool finite = isfinite(most.x);
  auto power = [&](int j) {
    const float2 l = keys[j];
    return expf(finite ? (l.x - most.x) + (l.y - most.y) : raw[j] - raw[chosen[0]]);
  };
  if (tid < top) pw[tid] = power(chosen[tid]);
  float sum = 0.f;
  if (!a.renorm && tid < (E + 31) / 32 * 32) {
    sum = tid < E ? power(tid) : 0.f;
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, o);
    if (tid % 32 == 0) warp_sum[tid / 32] = sum;
  }
  __syncthreads();
  if (tid >= top) return;
  sum = 0.f;
  if (a.renorm) {
#pragma unroll 1
    for (int j = 0; j < top; ++j) sum += pw[j];
  } else {
#pragma unroll 1
    for (int j = 0; j < (E + 31) / 32; ++j) sum += warp_sum[j];
  }
  const float w = pw[tid] / sum;
  a.sel[row * top + tid] = chosen[tid];
  a.w[row * top + tid] = w;
  if (a.experts_out) a.experts_out[row * top + tid] = chosen[tid];
  if (a.weights_out) a.weights_out[row * top + tid] = w;
}

// ------------------------------------------------------------------------------------------------------------
// experts
// ------------------------------------------------------------------------------------------------------------
template <typename T, int D>
struct MoeCfg {
  static constexpr int FC = 64 / (int)sizeof(T);     // hidden features of a chunk: 64 bytes of a W_gate row
  static constexpr int EP = 16 / (int)sizeof(T);     // values of a 16-byte piece
  static constexpr int kGate = D * 64;               // bytes of a chunk of W_gate; W_up and W_down have as many
  static constexpr int kStage = 3 * kGate;
  static constexpr int XS = sizeof(T) == 2 ? D : D + 4;    // values between two rows of X, and of H (fp32: padded)
  static constexpr int HS = sizeof(T) == 2 ? FC : FC + 4;
  static constexpr int kX = kGroup * XS * (int)sizeof(T);
  // H of one of two places; bf16: the rounded rows, then what they lost.  fp32: and 8 KB for the parts of its sums.
  static constexpr int kTerm = kGroup * HS * (int)sizeof(T), kH = sizeof(T) == 2 ? 2 * kTerm : kTerm;
  static constexpr int kRed = sizeof(T) == 2 ? 0 : 16 * 4 * 16 * 8;
  static_assert(2 * kH >= kMaxTop * D * 4, "a row's experts' sums have the same place");
  static constexpr int kIdx = kMaxRows * kMaxTop * 2;
  static constexpr int kFit = (222 * 1024 - kX - 2 * kH - kIdx - kRed) / kStage;
  static constexpr int kStages = kFit > 8 ? 8 : kFit;
  static constexpr size_t kSmem = (size_t)kStages * kStage + kX + 2 * kH + kIdx + kRed;
};

// Byte offset of piece c of row r, N pieces a row, such that eight rows' pieces lie in different banks (N = 4: as the
// 64-byte swizzle of a copied box has them).
template <int N>
__device__ __forceinline__ uint32_t place16(int r, int c) {
  return (uint32_t)(r * N + (c ^ (N == 4 ? (r >> 1) & 3 : r & 7))) * 16u;
}
// Of W_down's chunk, which comes in boxes of 128 bytes a row.
__device__ __forceinline__ uint32_t down16(int r, int c) {
  return (uint32_t)(c / 8 * 32 * 128 + r * 128 + ((c % 8) ^ (r & 7)) * 16);
}
__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0, %1, %2, %3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3])
               : "r"(addr)
               : "memory");
}
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm volatile(
      "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, "
      "%3};"
      : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
      : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}

// A CTA's sums of up to 64 rows: tensor instructions in bf16, FMAs in fp32.
template <typename T, int D, int kAct>
struct Sums;

template <int D, int kAct>
struct Sums<__nv_bfloat16, D, kAct> {
  using C = MoeCfg<__nv_bfloat16, D>;
  static constexpr int NT = D / 64;  // a warp has an eighth of the columns, in tiles of 8
  float acc[kGroup / 16][NT][4];
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < kGroup / 16; ++i)
#pragma unroll
      for (int j = 0; j < NT; ++j)
#pragma unroll
        for (int k = 0; k < 4; ++k) acc[i][j][k] = 0.f;
  }
  // H: a warp has 8 of the chunk's features, of every other tile of 16 rows; G and U share the rows' fragments, two
  // tiles the weights'.  H is kept as a sum of two bf16 numbers (16 bits), the operands of the next product: rounded
  // once to 8 bits it would add 1.8e-3 of a row to the 1.7e-3 of Y's own rounding, and the product is not what takes
  // the time.
  template <int NR>
  __device__ __forceinline__ void hidden_of(const char* st, const char* X, char* H, int rt) {
    const int lane = threadIdx.x % 32, ft = threadIdx.x / 32 % 4;
    const uint32_t w = tc::smem_u32(st) + (lane < 16 ? 0 : C::kGate), xa = tc::smem_u32(X);
    float g[NR][4] = {}, u[NR][4] = {};
#pragma unroll(D / 16 < 8 / NR ? D / 16 : 8 / NR)
    for (int ks = 0; ks < D / 16; ++ks) {
      uint32_t b[4], x[NR][4];
      ldsm4t(w + place16<4>(ks * 16 + lane % 16, ft), b);
#pragma unroll
      for (int i = 0; i < NR; ++i) ldsm4(xa + place16<D / 8>((rt + 2 * i) * 16 + lane % 16, ks * 2 + lane / 16), x[i]);
#pragma unroll
      for (int i = 0; i < NR; ++i) {
        mma(g[i], x[i], b[0], b[1]);
        mma(u[i], x[i], b[2], b[3]);
      }
    }
#pragma unroll
    for (int i = 0; i < NR; ++i)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const float a = gate<kAct>(g[i][2 * h]) * u[i][2 * h], c = gate<kAct>(g[i][2 * h + 1]) * u[i][2 * h + 1];
        const uint32_t v = pack2_bf16(a, c);
        char* to = H + place16<4>((rt + 2 * i) * 16 + lane / 4 + 8 * h, ft) + lane % 4 * 4;
        *reinterpret_cast<uint32_t*>(to) = v;
        *reinterpret_cast<uint32_t*>(to + C::kTerm) =
            pack2_bf16(a - __uint_as_float(v << 16), c - __uint_as_float(v & 0xFFFF0000u));
      }
  }
  __device__ __forceinline__ void hidden(const char* st, const char* X, char* H, int rows, float2*) {
    const int half = threadIdx.x / 128, tiles = (rows + 15) / 16;
    if (half + 2 < tiles)
      hidden_of<2>(st, X, H, half);
    else if (half < tiles)
      hidden_of<1>(st, X, H, half);
  }
  __device__ __forceinline__ void out(const char* st, const char* H, int rows) {
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32, tiles = (rows + 15) / 16;
    const uint32_t w = tc::smem_u32(st) + 2 * C::kGate, ha = tc::smem_u32(H);
#pragma unroll
    for (int ks = 0; ks < 2; ++ks) {
      uint32_t b[(NT + 1) / 2][4];
#pragma unroll
      for (int j = 0; j < (NT + 1) / 2; ++j)  // one tile: the second half of the fragment is not used
        ldsm4t(w + down16(ks * 16 + lane % 16, warp * NT + 2 * j + (NT > 1 ? lane / 16 : 0)), b[j]);
#pragma unroll
      for (int rt = 0; rt < kGroup / 16; ++rt) {
        if (rt >= tiles) break;
        uint32_t h[4], l[4];
        ldsm4(ha + place16<4>(rt * 16 + lane % 16, ks * 2 + lane / 16), h);
        ldsm4(ha + C::kTerm + place16<4>(rt * 16 + lane % 16, ks * 2 + lane / 16), l);
#pragma unroll
        for (int j = 0; j < NT; ++j) mma(acc[rt][j], l, b[j / 2][j % 2 * 2], b[j / 2][j % 2 * 2 + 1]);
#pragma unroll
        for (int j = 0; j < NT; ++j) mma(acc[rt][j], h, b[j / 2][j % 2 * 2], b[j / 2][j % 2 * 2 + 1]);
      }
    }
  }
  // Row r of the pass to row at(r) of `part`.
  template <typename F>
  __device__ __forceinline__ void store(float* part, int rows, F at) const {
    const int lane = threadIdx.x % 32, warp = threadIdx.x / 32;
#pragma unroll
    for (int rt = 0; rt < kGroup / 16; ++rt)
#pragma unroll
      for (int h = 0; h < 2; ++h) {
        const int r = rt * 16 + lane / 4 + 8 * h;
        if (r >= rows) continue;
#pragma unroll
        for (int j = 0; j < NT; ++j)
          *reinterpret_cast<float2*>(part + at(r) * D + (warp * NT + j) * 8 + lane % 4 * 2) =
              make_float2(acc[rt][j][2 * h], acc[rt][j][2 * h + 1]);
      }
  }
};

template <int D, int kAct>
struct Sums<float, D, kAct> {
  using C = MoeCfg<float, D>;
  static constexpr int kCols = kThr / D;            // rows side by side: thread t has column t % D of rows t / D + ...
  static constexpr int kPer = kGroup / kCols;       // rows a thread
  float acc[kPer];
  __device__ __forceinline__ void zero() {
#pragma unroll
    for (int i = 0; i < kPer; ++i) acc[i] = 0.f;
  }
  // Sixteen rows at a time.  A thread has one feature of four rows and a share of the sum, which is the finer the fewer
  // rows there are (1, 2 or 4 times four rows: a 16th, an 8th or a 4th); the shares are added in shared memory.
  __device__ __forceinline__ void hidden(const char* st, const char* X, char* H, int rows, float2* red) {
    const int ft = threadIdx.x % 16, of = threadIdx.x / 16;
    const float *wg = reinterpret_cast<const float*>(st) + ft, *wu = wg + C::kGate / 4;
#pragma unroll 1
    for (int t0 = 0; t0 < rows; t0 += 16) {
      const int left = rows - t0, blocks = left <= 4 ? 1 : left <= 8 ? 2 : 4, shares = 16 / blocks;
      const float* x = reinterpret_cast<const float*>(X) + (t0 + of % blocks * 4) * C::XS;
      float g[4] = {}, u[4] = {};
#pragma unroll 2
      for (int k = of / blocks * 4; k < D; k += shares * 4) {
        float a[4], b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
          a[i] = wg[(k + i) * 16];
          b[i] = wu[(k + i) * 16];
        }
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          const float4 v = *reinterpret_cast<const float4*>(x + r * C::XS + k);
          g[r] = fmaf(v.x, a[0], fmaf(v.y, a[1], fmaf(v.z, a[2], fmaf(v.w, a[3], g[r]))));
          u[r] = fmaf(v.x, b[0], fmaf(v.y, b[1], fmaf(v.z, b[2], fmaf(v.w, b[3], u[r]))));
        }
      }
      if (t0 > 0) __syncthreads();  // the parts of the rows before have been added
#pragma unroll
      for (int r = 0; r < 4; ++r) red[(of * 4 + r) * 16 + ft] = make_float2(g[r], u[r]);
      __syncthreads();
      if (of < 4 * blocks) {  // row `of` of the sixteen
        float2 s = make_float2(0.f, 0.f);
#pragma unroll 4
        for (int q = 0; q < shares; ++q) {
          const float2 p = red[((q * blocks + of / 4) * 4 + of % 4) * 16 + ft];
          s.x += p.x;
          s.y += p.y;
        }
        reinterpret_cast<float*>(H)[(t0 + of) * C::HS + ft] = gate<kAct>(s.x) * s.y;
      }
    }
  }
  __device__ __forceinline__ void out(const char* st, const char* H, int rows) {
    const int c = threadIdx.x % D, r0 = threadIdx.x / D;
    const float* w = reinterpret_cast<const float*>(st + 2 * C::kGate) + c;
    const float* h = reinterpret_cast<const float*>(H) + r0 * C::HS;
#pragma unroll 1
    for (int k = 0; k < 16; k += 4) {
      const float w0 = w[k * D], w1 = w[(k + 1) * D], w2 = w[(k + 2) * D], w3 = w[(k + 3) * D];
#pragma unroll
      for (int i = 0; i < kPer; ++i) {
        if (i % 4 == 0 && i * kCols >= rows) break;
        const float4 v = *reinterpret_cast<const float4*>(h + i * kCols * C::HS + k);
        acc[i] = fmaf(v.x, w0, fmaf(v.y, w1, fmaf(v.z, w2, fmaf(v.w, w3, acc[i]))));
      }
    }
  }
  template <typename F>
  __device__ __forceinline__ void store(float* part, int rows, F at) const {
    const int c = threadIdx.x % D, r0 = threadIdx.x / D;
#pragma unroll
    for (int i = 0; i < kPer; ++i)
      if (r0 + i * kCols < rows) part[at(r0 + i * kCols) * D + c] = acc[i];
  }
};

// Shares of `items` chunks: CTA b of `ctas` has [first_of(b), first_of(b + 1)).
__device__ __forceinline__ int first_of(int b, int items, int ctas) {
  return (int)((uint32_t)b * (uint32_t)items / (uint32_t)ctas);
}
__device__ __forceinline__ int owner_of(int item, int items, int ctas) {  // (at most 384 passes of 1024 chunks)
  return (int)(((uint32_t)(item + 1) * (uint32_t)ctas - 1u) / (uint32_t)items);
}

// A column of what an expert gave a row: the shares of its pass, in the order of the list, at row r of each.
template <int D>
__device__ __forceinline__ float share_sum(const MoeArgs& a, int pass, int r, int c, int chunks, int items, int ctas) {
  const int b0 = owner_of(pass * chunks, items, ctas), b1 = owner_of((pass + 1) * chunks - 1, items, ctas);
  const float* p = a.part + ((int64_t)(b0 + pass) * a.group + r) * D + c;
  float s = 0.f;
#pragma unroll 1
  for (int k = b0; k <= b1; k += 8, p += 8 * a.group * D) {
    float v[8];
#pragma unroll
    for (int m = 0; m < 8; ++m) v[m] = k + m <= b1 ? __ldcg(p + m * a.group * D) : 0.f;
#pragma unroll
    for (int m = 0; m < 8; ++m) s += v[m];
  }
  return s;
}
// A column of a row of Y.
template <typename T, int D>
__device__ __forceinline__ void row_out(const MoeArgs& a, int row, int c, const float* sums, float x) {
#pragma unroll 1
  for (int j = 0; j < a.top; ++j) x = fmaf(a.w[row * a.top + j], sums[j * D + c], x);
  static_cast<T*>(a.y)[(int64_t)row * D + c] = from_f32<T>(x);
}
template <typename T, int D>
__device__ __forceinline__ float row_in(const MoeArgs& a, int row, int c) {
  return a.residual ? to_f32(static_cast<const T*>(a.x)[(int64_t)row * D + c]) : 0.f;
}

// A CTA a row: a thread has a column of one of the row's experts, so that all their shares' loads are in flight
// together.
template <typename T, int D>
__global__ __launch_bounds__(D * kMaxTop > 1024 ? 1024 : D * kMaxTop) void moe_sum(MoeArgs a, int grid) {
  pdl_begin();
  __shared__ float sums[kMaxTop * D];
  const int row = blockIdx.x, c = threadIdx.x, chunks = (a.f + MoeCfg<T, D>::FC - 1) / MoeCfg<T, D>::FC;
  const int items = *a.items, ctas = min(grid, items);
  if (a.sel[row * a.top] < 0) return;  // not live: zeros already
  const float x = row_in<T, D>(a, row, c);
#pragma unroll 1
  for (int j = threadIdx.y; j < a.top; j += blockDim.y) {
    // (no place of this call's: moe_experts gave up a wait, and its results are invalid)
    const int at = a.place[row * a.top + j];
    const bool there = (uint32_t)at < (uint32_t)(items / chunks * a.group);
    sums[j * D + c] = there ? share_sum<D>(a, at / a.group, at % a.group, c, chunks, items, ctas) : NAN;
  }
  __syncthreads();
  if (threadIdx.y == 0) row_out<T, D>(a, row, c, sums, x);
}

template <typename T, int D, int kAct>
__global__ __launch_bounds__(kThr, 1) void moe_experts(MoeArgs a, const __grid_constant__ CUtensorMap wg,
                                                       const __grid_constant__ CUtensorMap wu,
                                                       const __grid_constant__ CUtensorMap wd) {
  pdl_begin();
  using C = MoeCfg<T, D>;
  extern __shared__ __align__(1024) char smem[];
  char* const X = smem + C::kStages * C::kStage;
  char* const H = X + C::kX;
  uint16_t* const idx = reinterpret_cast<uint16_t*>(H + 2 * C::kH);
  float2* const red = reinterpret_cast<float2*>(H + 2 * C::kH + C::kIdx);
  __shared__ int count[kMaxExperts];      // rows of an expert
  __shared__ int first[kMaxExperts + 1];  // its first pass
  __shared__ uint8_t expert[kMaxPasses];  // of a pass
  __shared__ int warp_part[kThr / 32], list[kGroup], row_of[kGroup];  // a pass's slots, and their rows
  __shared__ bool last[kGroup];
  __shared__ uint64_t full[C::kStages];  // a chunk has come
  const int tid = threadIdx.x, lane = tid % 32, warp = tid / 32, slots = a.n * a.top, E = a.experts, group = a.group;

  // ---- the list: passes of up to `group` rows of an expert, experts in order; chunks of f in a pass
#pragma unroll 1
  for (int i = tid; i < E; i += kThr) count[i] = 0;
  if (tid == 0) {
    tc::prefetch_tmap(&wg);
    tc::prefetch_tmap(&wu);
    tc::prefetch_tmap(&wd);
#pragma unroll 1
    for (int i = 0; i < C::kStages; ++i) tc::mbar_init(&full[i], 1);
    tc::fence_mbar_init();
  }
  __syncthreads();
#pragma unroll 1
  for (int i0 = tid * 4; i0 < slots; i0 += kThr * 8) {  // two loads of four in flight
    int4 v[2];
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      v[k] = make_int4(-1, -1, -1, -1);
      if (i0 + k * kThr * 4 < slots) v[k] = *reinterpret_cast<const int4*>(a.sel + i0 + k * kThr * 4);
    }
#pragma unroll
    for (int k = 0; k < 2; ++k) {
      const int e[4] = {v[k].x, v[k].y, v[k].z, v[k].w}, i = i0 + k * kThr * 4;
#pragma unroll
      for (int j = 0; j < 4; ++j)
        if (i + j < slots) {
          idx[i + j] = (uint16_t)e[j];  // none: 0xFFFF
          if (e[j] >= 0) atomicAdd(&count[e[j]], 1);
        }
    }
  }
  __syncthreads();
  int passes = tid < E ? (count[tid] + group - 1) / group : 0;
  int scan = passes;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const int v = __shfl_up_sync(0xffffffffu, scan, o);
    if (lane >= o) scan += v;
  }
  if (lane == 31) warp_part[warp] = scan;
  __syncthreads();
#pragma unroll 1
  for (int k = 0; k < warp; ++k) scan += warp_part[k];
  if (tid < E) first[tid + 1] = scan;
#pragma unroll 1
  for (int k = scan - passes; k < scan; ++k) expert[k] = (uint8_t)tid;
  if (tid == 0) first[0] = 0;
  __syncthreads();
  const int chunks = (a.f + C::FC - 1) / C::FC, items = first[E] * chunks;
  const int ctas = min((int)gridDim.x, items), b = blockIdx.x;
  if (b == 0 && tid == 0) *a.items = items;
  if (b >= ctas) return;
  if (!a.last) pdl_next();
  const int lo = first_of(b, items, ctas), hi = first_of(b + 1, items, ctas);

  // ---- a cursor of the loads and one of the products
  struct At {
    int pass, chunk, e;
  };
  auto next = [&](At& c) {
    if (++c.chunk < chunks) return;
    c.chunk = 0;
    c.e = expert[++c.pass];
  };
  At ahead{lo / chunks, lo % chunks, expert[lo / chunks]}, now = ahead;
  int ahead_item = lo;
  auto load = [&]() {  // thread 0: the next chunk, into the place of its number; columns and rows past f are zeros
    if (ahead_item >= hi) return;
    const int stage = (ahead_item - lo) % C::kStages, f0 = ahead.chunk * C::FC;
    char* st = smem + stage * C::kStage;
    tc::mbar_expect_tx(&full[stage], C::kStage);
    tc::tma_load_2d(st, &wg, f0, ahead.e * D, &full[stage]);
    tc::tma_load_2d(st + C::kGate, &wu, f0, ahead.e * D, &full[stage]);
    constexpr int kBox = sizeof(T) == 2 ? 64 : D;
#pragma unroll
    for (int k = 0; k < D / kBox; ++k)
      tc::tma_load_3d(st + 2 * C::kGate + k * 32 * 128, &wd, k * kBox, f0, ahead.e, &full[stage]);
    if (++ahead_item < hi) next(ahead);
  };
  Sums<T, D, kAct> sums;
  int rows = 0, tiles = 0;
  bool gave_up = false;
#pragma unroll 1
  for (int item = lo; item < hi; ++item) {
    if (item == lo || now.chunk == 0) {  // a pass begins: its rows
      const int skip = (now.pass - first[now.e]) * group;
      rows = min(group, count[now.e] - skip);
      tiles = (rows + 15) / 16;
      const int per = (slots + kThr - 1) / kThr * 32, s0 = warp * per, s1 = min(slots, s0 + per);
      int found = 0;
#pragma unroll 1
      for (int s = s0; s < s1; s += 32)
        found += __popc(__ballot_sync(0xffffffffu, s + lane < s1 && idx[s + lane] == now.e));
      if (lane == 0) warp_part[warp] = found;
      __syncthreads();
      int at = -skip;
#pragma unroll 1
      for (int k = 0; k < warp; ++k) at += warp_part[k];
#pragma unroll 1
      for (int s = s0; s < s1; s += 32) {
        const bool mine = s + lane < s1 && idx[s + lane] == now.e;
        const uint32_t m = __ballot_sync(0xffffffffu, mine);
        const int r = at + __popc(m & ((1u << lane) - 1));
        if (mine && r >= 0 && r < group) {
          list[r] = s + lane;
          row_of[r] = (s + lane) / a.top;
        }
        at += __popc(m);
      }
      __syncthreads();
      constexpr int N = D / C::EP, kTileLoads = 16 * N / kThr > 0 ? 16 * N / kThr : 1;  // a thread's of 16 rows
      uint4 v[4 * kTileLoads];
#pragma unroll
      for (int m = 0; m < 4 * kTileLoads; ++m) {
        const int p = tid + m * kThr, r = p / N, q = p % N;
        v[m] = make_uint4(0, 0, 0, 0);
        if (r < rows) v[m] = ld16(static_cast<const T*>(a.x) + (int64_t)row_of[r] * D + q * C::EP);
      }
      if (item == lo && tid == 0)  // the first chunks: behind the rows' loads, which would wait for them some 3 us
#pragma unroll 1
        for (int i = 0; i < C::kStages; ++i) load();
#pragma unroll
      for (int m = 0; m < 4 * kTileLoads; ++m) {
        const int p = tid + m * kThr, r = p / N, q = p % N;
        if (r < tiles * 16)
          st16(X + (sizeof(T) == 2 ? place16<N>(r, q) : (uint32_t)(r * C::XS + q * C::EP) * 4u), v[m]);
      }
      sums.zero();
      __syncthreads();
    }
    const int at = item - lo, stage = at % C::kStages;
    const char* st = smem + stage * C::kStage;
    char* const h = H + at % 2 * C::kH;
    const bool here = tc::mbar_wait(&full[stage], at / C::kStages & 1);
    sums.hidden(st, X, h, rows, red);
    if (__syncthreads_or(!here)) {  // H is there, and nobody reads the chunk before any more
      gave_up = true;
      break;
    }
    if (tid == 0 && at > 0) load();
    sums.out(st, h, rows);
    const At was = now;
    if (item + 1 < hi) next(now);
    if (item + 1 < hi && now.chunk != 0) continue;

    // ---- the share's end of a pass: its sums
    float* part = a.part + (int64_t)(b + was.pass) * group * D;
    if (!a.last) {  // moe_sum follows
      sums.store(part, rows, [](int r) { return r; });
      if (tid < rows) a.place[list[tid]] = was.pass * group + tid;
      continue;
    }
    // few rows: one pass an expert, at the rows' own places; whose last share this is
    sums.store(part, rows, [&](int r) { return row_of[r]; });
    __threadfence();
    __syncthreads();
    if (tid < rows) {
      const int row = row_of[tid];
      int shares = 0;
#pragma unroll 1
      for (int j = 0; j < a.top; ++j) {
        const int pass = first[idx[row * a.top + j]];
        shares += owner_of((pass + 1) * chunks - 1, items, ctas) - owner_of(pass * chunks, items, ctas) + 1;
      }
      last[tid] = atomicAdd(&a.row_in[row], 1) == shares - 1;
    }
    __syncthreads();
    __threadfence();
#pragma unroll 1
    for (int r = 0; r < rows; ++r) {
      if (!last[r]) continue;
      const int row = row_of[r], c = tid % D;
      float* const all = reinterpret_cast<float*>(H);
      const float x = row_in<T, D>(a, row, c);
#pragma unroll 1
      for (int j = tid / D; j < a.top; j += kThr / D)
        all[j * D + c] = share_sum<D>(a, first[idx[row * a.top + j]], row, c, chunks, items, ctas);
      __syncthreads();
      if (tid < D) row_out<T, D>(a, row, c, all, x);
      __syncthreads();
    }
    __syncthreads();  // list, last and X are free
  }
  if (gave_up && tid == 0) {  // a copy did not come: nor wait for the others without end
    record_device_error(a.status, tc::kErrTimeout);
#pragma unroll 1
    for (int at = max(0, ahead_item - lo - C::kStages); at < ahead_item - lo; ++at)
      tc::mbar_wait(&full[at % C::kStages], at / C::kStages & 1);
  }
}

// ------------------------------------------------------------------------------------------------------------
// host
// ------------------------------------------------------------------------------------------------------------
struct MoeLayout {
  int32_t *sel, *row_in, *place, *items;
  float *w, *part;
  int group;
};
size_t carve(void* scratch, const hg_moe_params* p, int64_t n, MoeLayout* L) {
  Carve c(scratch);
  const size_t slots = (size_t)n * p->top_k;
  L->group = (int)std::min<int64_t>(kGroup, (n + 15) / 16 * 16);
  L->sel = c.take<int32_t>(slots);
  L->row_in = c.take<int32_t>(n);
  L->place = c.take<int32_t>(slots);
  L->w = c.take<float>(slots);
  L->items = c.take<int32_t>(1);
  // a pass has its own rows, or 64 of an expert's: at most that many, and a CTA begins at most one more
  const size_t passes = n > 0 ? std::min<size_t>(p->experts, slots) + slots / L->group : 0;
  L->part = c.take<float>((kSms + passes) * L->group * p->d);
  return n > 0 ? c.used : 0;
}

hg_status check(const hg_moe_params* p, int64_t n) {
  HG_REQUIRE(p != nullptr, "params must be non-null");
  if (!(p->d == 64 || p->d == 128 || p->d == 256) || !(p->dtype == HG_F32 || p->dtype == HG_BF16)) {
    set_error("unsupported d=%d / dtype=%d", p->d, (int)p->dtype);
    return HG_ERR_UNSUPPORTED;
  }
  HG_REQUIRE(p->f >= 8 && p->f <= kMaxF && p->f % 8 == 0, "f must be a multiple of 8 in [8, %d]", kMaxF);
  HG_REQUIRE(p->experts >= 1 && p->experts <= kMaxExperts, "experts must be in [1, %d]", kMaxExperts);
  HG_REQUIRE(p->top_k >= 1 && p->top_k <= kMaxTop && p->top_k <= p->experts,
             "top_k must be in [1, %d], at most experts", kMaxTop);
  HG_REQUIRE(p->act == HG_ACT_RELU || p->act == HG_ACT_GELU_TANH || p->act == HG_ACT_NONE || p->act == HG_ACT_SILU,
             "unknown activation %d", (int)p->act);
  HG_REQUIRE(n >= 0, "n must not be negative");
  if (n > kMaxRows) {
    set_error("n=%lld: a call takes up to %d rows (larger batches: hg_ffn_fwd on each expert's rows)", (long long)n,
              kMaxRows);
    return HG_ERR_UNSUPPORTED;
  }
  return HG_OK;
}

struct MoeMaps {
  CUtensorMap wg, wu, wd;
};
template <typename T, int D>
hg_status encode(const MoeArgs& a, MoeMaps* m) {
  using C = MoeCfg<T, D>;
  const bool f32 = sizeof(T) == 4;
  const uint64_t gate[2] = {(uint64_t)a.f, (uint64_t)a.experts * D}, down[3] = {D, (uint64_t)a.f, (uint64_t)a.experts};
  const uint32_t gate_box[2] = {C::FC, D}, down_box[3] = {f32 ? D : 64, C::FC, 1};
  HG_TRY(make_tmap(&m->wg, a.wg, f32, 2, gate, gate_box, f32 ? 0 : 64));
  m->wu = m->wg;
  HG_TRY(move_tmap(&m->wu, a.wu));
  return make_tmap(&m->wd, a.wd, f32, 3, down, down_box, f32 ? 0 : 128);
}

template <typename T, int D, int kAct>
hg_status experts_act(const MoeArgs& a, int grid, cudaStream_t s) {
  using C = MoeCfg<T, D>;
  static bool once = false;
  if (!once) {
    HG_CUDA(cudaFuncSetAttribute(moe_experts<T, D, kAct>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)C::kSmem));
    once = true;
  }
  MoeMaps m;
  HG_TRY((encode<T, D>(a, &m)));
  HG_TRY(launch("moe_experts", moe_experts<T, D, kAct>, dim3(grid), dim3(kThr), C::kSmem, s, a, m.wg, m.wu, m.wd));
  if (a.last) return HG_OK;
  return launch("moe_sum", moe_sum<T, D>, dim3(a.n), dim3(D, std::min(a.top, 1024 / D)), 0, s, a, grid);
}
template <typename T, int D>
hg_status experts_d(const MoeArgs& a, hg_act act, int grid, cudaStream_t s) {
  if (act == HG_ACT_RELU) return experts_act<T, D, HG_ACT_RELU>(a, grid, s);
  if (act == HG_ACT_GELU_TANH) return experts_act<T, D, HG_ACT_GELU_TANH>(a, grid, s);
  if (act == HG_ACT_SILU) return experts_act<T, D, HG_ACT_SILU>(a, grid, s);
  return experts_act<T, D, HG_ACT_NONE>(a, grid, s);
}
template <typename T>
hg_status layer(const MoeArgs& a, hg_act act, cudaStream_t s) {
  int width = 1;  // threads side by side, an expert each
  while (width < a.experts) width *= 2;
  const int parts = std::min(kRouterThr / width, kMaxParts);
  HG_TRY(launch("moe_router", moe_router<T>, dim3(a.n), dim3(std::max(width * parts, a.d)), 0, s, a, width, parts));
  // no more CTAs than chunks there can be
  const int64_t slots = (int64_t)a.n * a.top, chunks = ceil_div(a.f, 64 / (int)sizeof(T));
  const int64_t passes = std::min<int64_t>(a.experts, slots) + slots / a.group;
  const int grid = (int)std::min<int64_t>(kSms, passes * chunks);
  if (a.d == 64) return experts_d<T, 64>(a, act, grid, s);
  if (a.d == 128) return experts_d<T, 128>(a, act, grid, s);
  return experts_d<T, 256>(a, act, grid, s);
}

}  // namespace
}  // namespace hg

using namespace hg;

extern "C" hg_status hg_moe_workspace_size(const hg_moe_params* params, int64_t n, size_t* scratch_bytes) {
  clear_error();
  HG_REQUIRE(scratch_bytes != nullptr, "scratch_bytes must be non-null");
  HG_TRY(check(params, n));
  MoeLayout L;
  *scratch_bytes = carve(nullptr, params, n, &L);
  return HG_OK;
}

extern "C" hg_status hg_moe_fwd(const hg_moe_params* params, const void* X, const int32_t* live, int64_t n, void* Y,
                                int32_t* experts, float* weights, void* scratch, hg_stream stream) {
  clear_error();
  HG_TRY(device_guard());
  HG_TRY(check(params, n));
  const hg_moe_params& p = *params;
  HG_REQUIRE(p.W_router && p.W_gate && p.W_up && p.W_down, "every weight pointer must be non-null");
  HG_REQUIRE((((uintptr_t)p.W_router | (uintptr_t)p.W_gate | (uintptr_t)p.W_up | (uintptr_t)p.W_down) & 15) == 0,
             "weights must be 16-byte aligned");
  if (n == 0) return HG_OK;
  HG_REQUIRE(X && Y && scratch, "X, Y and scratch must be non-null");
  HG_REQUIRE((((uintptr_t)X | (uintptr_t)Y) & 15) == 0, "X and Y must be 16-byte aligned");
  HG_REQUIRE((((uintptr_t)live | (uintptr_t)experts | (uintptr_t)weights) & 3) == 0,
             "live, experts and weights must be 4-byte aligned");
  HG_REQUIRE(((uintptr_t)scratch & 255) == 0, "scratch must be 256-byte aligned");
  const int64_t esz = p.dtype == HG_BF16 ? 2 : 4, rows = n * p.d * esz, slots = n * p.top_k;
  MoeLayout L;
  const RowSet sc = block_set(scratch, (int64_t)carve(scratch, params, n, &L));
  const RowSet x = block_set(X, rows), y = block_set(Y, rows), lv = block_set(live, 4 * n);
  const RowSet oe = block_set(experts, 4 * slots), ow = block_set(weights, 4 * slots);
  const RowSet r = block_set(p.W_router, p.experts * p.d * esz);
  const int64_t w = esz * p.experts * p.d * p.f;
  const RowSet g = block_set(p.W_gate, w), u = block_set(p.W_up, w), d = block_set(p.W_down, w);
  HG_TRY(check_apart(y, "Y", {x, lv, oe, ow, sc, r, g, u, d}));
  HG_TRY(check_apart(sc, "scratch", {x, lv, oe, ow, r, g, u, d}));
  HG_TRY(check_apart(oe, "experts", {x, lv, ow, r, g, u, d}));
  HG_TRY(check_apart(ow, "weights", {x, lv, r, g, u, d}));
  MoeArgs a{};
  a.x = X;
  a.wr = p.W_router;
  a.wg = p.W_gate;
  a.wu = p.W_up;
  a.wd = p.W_down;
  a.live = live;
  a.y = Y;
  a.experts_out = experts;
  a.weights_out = weights;
  a.sel = L.sel;
  a.w = L.w;
  a.row_in = L.row_in;
  a.place = L.place;
  a.part = L.part;
  a.items = L.items;
  a.status = device_status_ptr();
  a.last = n * ceil_div((int64_t)p.top_k * p.d, kThr) <= kMaxRounds;
  a.n = (int32_t)n;
  a.d = p.d;
  a.f = p.f;
  a.experts = p.experts;
  a.top = p.top_k;
  a.renorm = p.renorm;
  a.residual = p.residual;
  a.group = L.group;
  cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  if (p.dtype == HG_F32) return layer<float>(a, p.act, s);
  return layer<__nv_bfloat16>(a, p.act, s);
}
