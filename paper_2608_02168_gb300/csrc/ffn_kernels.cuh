// Internal declarations of the gated feed-forward block (ffn.cu, ffn_tc.cu, ffn_bwd_tc.cu); not part of the public ABI.
#pragma once

#include "hg_internal.cuh"

namespace hg {

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

// The logistic function as s r and its complement as t r, from s = e^(z / 2), t = e^(-z / 2), r = 1 / (s + t): the
// exponents are halved, so a gate as small as the smallest fp32 number comes out as it is and none of the factors
// leaves the range.  (Above z = 277 both are at their limits.)
struct Logistic {
  float s, t, r;
  __device__ __forceinline__ explicit Logistic(float half_log2) {
    const float h = fminf(half_log2, 100.f);
    s = gate_ex2(h);
    t = gate_ex2(-h);
    r = gate_rcp(s + t);
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

// kAct: hg_act.  The gate's value.
template <int kAct>
__device__ __forceinline__ float gate(float x) {
  if (kAct == HG_ACT_RELU) return x > 0.f ? x : 0.f;
  if (kAct == HG_ACT_NONE) return x;
  const Logistic l(gate_half<kAct>(x));
  return x * l.s * l.r;
}

// The gate's value and derivative.
template <int kAct>
__device__ __forceinline__ float gate_grad(float x, float* d) {
  if (kAct == HG_ACT_RELU) {
    *d = x > 0.f ? 1.f : 0.f;
    return x > 0.f ? x : 0.f;
  }
  if (kAct == HG_ACT_NONE) {
    *d = 1.f;
    return x;
  }
  const Logistic l(gate_half<kAct>(x));
  const float p = l.s * l.r;
  float k = x * (l.t * l.r);
  if (kAct == HG_ACT_GELU_TANH) k *= fmaf(x * x, 3.f * 0.044715f * 1.5957691216057308f, 1.5957691216057308f);
  *d = fmaf(p, k, p);
  return x * p;
}

}  // namespace hg
