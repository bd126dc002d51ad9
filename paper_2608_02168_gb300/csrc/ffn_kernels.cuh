// Internal declarations of the gated feed-forward block (ffn.cu, ffn_tc.cu); not part of the public ABI.
#pragma once

#include "hg_internal.cuh"

namespace hg {

// x sigmoid(x) and its derivative.  e^-|x| <= 1, so neither form overflows or loses a small gate.
__device__ __forceinline__ float sigm_of(float x, float* comp) {
  const float e = __expf(-fabsf(x));
  const float r = __fdividef(1.f, 1.f + e);
  const float s = e * r;
  *comp = x >= 0.f ? s : r;  // 1 - sigmoid
  return x >= 0.f ? r : s;
}

// kAct: hg_act.  The gate's value.
template <int kAct>
__device__ __forceinline__ float gate(float x) {
  if (kAct == HG_ACT_RELU) return x > 0.f ? x : 0.f;
  if (kAct == HG_ACT_SILU) {
    float c;
    return x * sigm_of(x, &c);
  }
  if (kAct == HG_ACT_GELU_TANH) {  // (1 + tanh z) / 2 = sigmoid(2 z)
    float c;
    return x * sigm_of(1.5957691216057308f * (x + 0.044715f * x * x * x), &c);
  }
  return x;
}

// e^-|x| and the gate's argument of the logistic function
template <int kAct>
__device__ __forceinline__ float gate_arg(float x) {
  return kAct == HG_ACT_GELU_TANH ? 1.5957691216057308f * x * fmaf(0.044715f, x * x, 1.f) : x;
}

// The gates of two features with one reciprocal: 1 / (1 + e0) = (1 + e1) / ((1 + e0) (1 + e1)), both factors
// in [1, 2].
template <int kAct>
__device__ __forceinline__ void gate2(float x0, float x1, float* a0, float* a1) {
  if (kAct == HG_ACT_SILU || kAct == HG_ACT_GELU_TANH) {
    const float z0 = gate_arg<kAct>(x0), z1 = gate_arg<kAct>(x1);
    const float e0 = __expf(-fabsf(z0)), e1 = __expf(-fabsf(z1));
    const float d0 = 1.f + e0, d1 = 1.f + e1;
    const float r = __fdividef(1.f, d0 * d1);
    *a0 = x0 * (z0 >= 0.f ? 1.f : e0) * (r * d1);
    *a1 = x1 * (z1 >= 0.f ? 1.f : e1) * (r * d0);
  } else {
    *a0 = gate<kAct>(x0);
    *a1 = gate<kAct>(x1);
  }
}

// The gate's value and derivative.
template <int kAct>
__device__ __forceinline__ float gate_grad(float x, float* d) {
  if (kAct == HG_ACT_RELU) {
    *d = x > 0.f ? 1.f : 0.f;
    return x > 0.f ? x : 0.f;
  }
  if (kAct == HG_ACT_SILU) {
    float c;
    const float s = sigm_of(x, &c);
    *d = s * fmaf(x, c, 1.f);
    return x * s;
  }
  if (kAct == HG_ACT_GELU_TANH) {
    float c;
    const float x2 = x * x;
    const float s = sigm_of(1.5957691216057308f * x * fmaf(0.044715f, x2, 1.f), &c);
    *d = s * fmaf(x * c, 1.5957691216057308f * fmaf(3.f * 0.044715f, x2, 1.f), 1.f);
    return x * s;
  }
  *d = 1.f;
  return x;
}

// Gates and derivatives of two features, one reciprocal.
template <int kAct>
__device__ __forceinline__ void gate_grad2(float x0, float x1, float* a0, float* a1, float* d0, float* d1) {
  if (kAct == HG_ACT_SILU || kAct == HG_ACT_GELU_TANH) {
    const float z0 = gate_arg<kAct>(x0), z1 = gate_arg<kAct>(x1);
    const float e0 = __expf(-fabsf(z0)), e1 = __expf(-fabsf(z1));
    const float n0 = 1.f + e0, n1 = 1.f + e1;
    const float r = __fdividef(1.f, n0 * n1);
    const float r0 = r * n1, r1 = r * n0;
    const float s0 = z0 >= 0.f ? r0 : e0 * r0, c0 = z0 >= 0.f ? e0 * r0 : r0;
    const float s1 = z1 >= 0.f ? r1 : e1 * r1, c1 = z1 >= 0.f ? e1 * r1 : r1;
    float k0 = c0, k1 = c1;
    if (kAct == HG_ACT_GELU_TANH) {
      k0 *= 1.5957691216057308f * fmaf(3.f * 0.044715f, x0 * x0, 1.f);
      k1 *= 1.5957691216057308f * fmaf(3.f * 0.044715f, x1 * x1, 1.f);
    }
    *a0 = x0 * s0;
    *a1 = x1 * s1;
    *d0 = s0 * fmaf(x0, k0, 1.f);
    *d1 = s1 * fmaf(x1, k1, 1.f);
  } else {
    *a0 = gate_grad<kAct>(x0, d0);
    *a1 = gate_grad<kAct>(x1, d1);
  }
}

}  // namespace hg
