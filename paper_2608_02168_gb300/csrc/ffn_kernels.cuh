// Internal declarations of the gated feed-forward block (ffn.cu, ffn_tc.cu, ffn_bwd_tc.cu); not part of the public ABI.
#pragma once

#include "hg_internal.cuh"

namespace hg {

// 2^x and 1/x by the special-function unit, each within two steps of fp32, for both storage types: fp32 rows end 4.2e-7
// of themselves off, most of it by the sums' order, and 3.4e-7 in PyTorch's own operations.
__device__ __forceinline__ float gate_ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float gate_rcp(float x) {
  float y;
  asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}

// The logistic function of z as s (s r) and its complement as r, from s = e^(z / 2), r = 1 / (1 + s^2): the
// exponent is halved, so a gate as small as the smallest fp32 number comes out as it is.  Above z = 41 (half_log2 = 30,
// where the caller ends it) the logistic function is 1 to the last bit.
struct Logistic {
  float s, r;
  __device__ __forceinline__ explicit Logistic(float half_log2) {
    s = gate_ex2(half_log2);
    r = gate_rcp(fmaf(s, s, 1.f));
  }
};

// (z / 2) log2 e for the gate's z: SiLU z = x; GELU (tanh form) (1 + tanh(z / 2)) / 2 with
// z = 2 sqrt(2 / pi) (x + 0.044715 x^3).
template <int kAct>
__device__ __forceinline__ float gate_half(float x) {
  if (kAct == HG_ACT_GELU_TANH) {
    const float k = 0.7213475204444817f * 1.5957691216057308f;
    return x * fmaf(x * x, 0.044715f * k, k);
  }
  return 0.7213475204444817f * x;
}

// The positive part, NaN as it is.
__device__ __forceinline__ float gate_relu(float x) {
  asm("max.NaN.f32 %0, %0, 0f00000000;" : "+f"(x));
  return x;
}

// kAct: hg_act.  The gate's value; s r is at most 1/2, so no factor carries a large x past the largest number.
template <int kAct>
__device__ __forceinline__ float gate(float x) {
  if (kAct == HG_ACT_RELU) return gate_relu(x);
  if (kAct == HG_ACT_NONE) return x;
  const Logistic l(fminf(gate_half<kAct>(x), 30.f));
  return (x * (l.s * l.r)) * l.s;
}

// The gate's value x p and derivative p (1 + r x dz/dx), p = s^2 r (one below 2^-126 loses bits here). r ends at 2^-60
// where it should go on to 0, and what it is multiplied with grows like x, or x^3: the functions are taken at x's
// nearest in the range outside of which p is 1 or 0 to the last bit (NaN stays).
template <int kAct>
__device__ __forceinline__ float gate_grad(float x, float* d) {
  if (kAct == HG_ACT_RELU) {
    *d = x > 0.f ? 1.f : 0.f;
    return gate_relu(x);
  }
  if (kAct == HG_ACT_NONE) {
    *d = 1.f;
    return x;
  }
  float xb = x;
  asm("min.NaN.f32 %0, %0, %1;" : "+f"(xb) : "f"(kAct == HG_ACT_GELU_TANH ? 7.45f : 41.5f));
  if (kAct == HG_ACT_GELU_TANH) asm("max.NaN.f32 %0, %0, %1;" : "+f"(xb) : "f"(-16.f));
  const Logistic l(gate_half<kAct>(xb));
  const float sr = l.s * l.r, p = l.s * sr;
  float k = xb * l.r;
  if (kAct == HG_ACT_GELU_TANH) k *= fmaf(xb * xb, 3.f * 0.044715f * 1.5957691216057308f, 1.5957691216057308f);
  *d = fmaf(p, k, p);
  return x * p;
}

}  // namespace hg
