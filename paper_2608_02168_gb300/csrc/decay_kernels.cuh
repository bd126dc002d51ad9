// Internal declarations of the linear attention with decay (decay.cu, decay_mma.cu); not part of the public ABI.
#pragma once

#include "hg_internal.cuh"

namespace hg {

// One causal scan over n sequences and their heads.  With tau = t + shift and gamma = exp(log_decay):
//   S = gamma^shift-decayed state before position t plus c_in k_t v_t^T,   o_t = c_out q_t S
// i.e. shift = 1: S_t = gamma S_(t-1) + c_in k_t v_t^T with S_(-1) = init;  shift = 0: the state given is
// already decayed at the first position, and the one left behind is decayed once more.  reverse: position
// t of the scan is row len - 1 - t of its sequence.
//   forward              q, k, v  -> o       shift 1, init S_in
//   dq_t = c S_t do_t    do, v, k -> dq      shift 1, init S_in^T
//   dk_t = R_t v_t       v, do, q -> dk      reverse, shift 0, init dS_out^T     (R_t = gamma R_(t+1) + c q_t do_t^T)
//   dv_t = R_t^T k_t     k, q, do -> dv      reverse, shift 0, init dS_out; leaves dS_in
struct ScanRows {
  const void* p;
  int64_t sn, st;
};
struct ScanArgs {
  ScanRows q, k, v, o;
  const int32_t* lens;
  const float* ld;
  const float* init;  // [n][heads][d_h][d_h] or null
  int init_t;         // read transposed
  float* last;        // state left behind, or null
  uint32_t* claims;   // counter, zero before the launch: items are claimed instead of dealt out (null: dealt out)
  float* seg;         // [n][heads][nseg][d_h][d_h]: states of the segments (nseg > 1)
  int64_t n, T, seg_len;
  int nseg, heads;
  int shift, reverse;
  float c_in, c_out;
};

// Scans over the same sequences (n, T, lens, ld, segments and claims agree), run side by side.
struct ScanBatch {
  ScanArgs s[3];
  int count;
};

// log_decay as the kernels take it
__device__ __forceinline__ float clamp_ld(float x) { return x < 0.f ? fmaxf(x, -200.f) : 0.f; }

__device__ __forceinline__ int64_t scan_len(const ScanArgs& a, int64_t i) {
  const int64_t len = a.lens ? (int64_t)a.lens[i] : a.T;
  return len < 0 ? 0 : len > a.T ? a.T : len;
}

// A state is kept in a frame: S = gamma^(tau - b) F with a base time b, so that no position multiplies it;
// additions are scaled by gamma^(b - tau), at most e^kFrame.  Beyond that the frame moves on.
// A state multiplied at each of thousands of positions would gather the rounding of gamma itself; a wider frame
// would magnify the rounding of the exponents.
constexpr float kFrame = 5.f;

// bf16 scan on the tensor cores (decay_mma.cu); local: the segments' own states into a.seg, no rows.
hg_status scan_mma(const ScanBatch& b, int d_h, bool local, cudaStream_t s);
// warps that scan_mma runs for one sequence and segment, and warps that an SM holds
int scan_mma_warps(int heads, int d_h);
int scan_mma_resident(int d_h);

}  // namespace hg
