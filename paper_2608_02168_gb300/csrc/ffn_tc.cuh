// Internal declarations of the gated feed-forward block's tensor-core path (bf16); not part of the public ABI.
#pragma once

#include "tc_util.cuh"

namespace hg {

// 16 consecutive 32-bit columns of this thread's tensor-memory lane; valid after ld_wait
__device__ __forceinline__ void ld16_issue(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, "
      "[%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
__device__ __forceinline__ void ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }


hg_status ffn_fwd_tc(const hg_ffn_params* w, const void* X, int64_t n, void* Y, cudaStream_t s);
// dX null or g null: that part is left out
hg_status ffn_bwd_tc(const hg_ffn_params* w, const void* X, int64_t n, const void* dY, void* dX, const hg_ffn_grads* g,
                     void* scratch, cudaStream_t s);
size_t ffn_bwd_tc_scratch(const hg_ffn_params* w, int64_t n);

}  // namespace hg
