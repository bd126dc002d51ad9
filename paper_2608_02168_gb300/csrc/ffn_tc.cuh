// Internal declarations of the gated feed-forward block's tensor-core path (bf16); not part of the public ABI.
#pragma once

#include "tc_util.cuh"

namespace hg {

hg_status ffn_fwd_tc(const hg_ffn_params* w, const void* X, int64_t n, void* Y, cudaStream_t s);
// dX null or g null: that part is left out
hg_status ffn_bwd_tc(const hg_ffn_params* w, const void* X, int64_t n, const void* dY, void* dX, const hg_ffn_grads* g,
                     void* scratch, cudaStream_t s);
// the weights' gradients from the row shares' sums, part[splits] = [dW_gate | dW_up | dW_down] of df values each
hg_status ffn_sum_shares(const float* part, int splits, int64_t df, const hg_ffn_grads* g, cudaStream_t s);
size_t ffn_bwd_tc_scratch(const hg_ffn_params* w, int64_t n);

// 16 consecutive 32-bit columns of this thread's tensor-memory lane; valid after ld_wait
__device__ __forceinline__ void ld16_issue(uint32_t taddr, uint32_t (&r)[16]) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, "
      "[%16];"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(taddr));
}
__device__ __forceinline__ void ld8_issue(uint32_t taddr, uint32_t (&r)[8]) {
  asm volatile("tcgen05.ld.sync.aligned.32x32b.x8.b32 {%0, %1, %2, %3, %4, %5, %6, %7}, [%8];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7])
               : "r"(taddr));
}
__device__ __forceinline__ void ld_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ void st16_issue(uint32_t taddr, const float* v) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16};" ::"r"(taddr),
      "f"(v[0]), "f"(v[1]), "f"(v[2]), "f"(v[3]), "f"(v[4]), "f"(v[5]), "f"(v[6]), "f"(v[7]), "f"(v[8]), "f"(v[9]),
      "f"(v[10]), "f"(v[11]), "f"(v[12]), "f"(v[13]), "f"(v[14]), "f"(v[15])
      : "memory");
}
__device__ __forceinline__ void st_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

// A descriptor `bytes` further on.
__device__ __forceinline__ uint64_t desc_at(uint64_t desc, uint32_t bytes) { return desc + (bytes >> 4); }

// One arrival for the warp, after what all its lanes did before.
__device__ __forceinline__ void warp_arrive(uint64_t* bar) {
  __syncwarp();
  if ((threadIdx.x & 31) == 0) tc::mbar_arrive(bar);
}

// The issuing warp of a CTA (CL = 1) or of a pair of CTAs (CL = 2, a cluster): all its lanes run the role, so that
// descriptors are warp-uniform values, and one elected lane issues.  A pair's product has 256 rows, 128 of each CTA
// from the same places of its shared memory to the same columns of its tensor memory; the second operand lies half in
// each.  The first CTA issues, and a commit arrives at the same barrier of both.
template <int CL>
struct Issuer {
  uint32_t lead;
  __device__ __forceinline__ Issuer() {
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(lead));
  }
  // D[tmem] (+)= A[smem] B[smem]
  __device__ __forceinline__ void mma(uint32_t d_tmem, uint64_t adesc, uint64_t bdesc, uint32_t idesc,
                                      uint32_t accumulate) const {
    if constexpr (CL == 1)
      asm volatile(
          "{\n\t.reg .pred p, q;\n\t"
          "setp.ne.b32 p, %4, 0;\n\t"
          "setp.ne.b32 q, %5, 0;\n\t"
          "@q tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
          ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(lead)
          : "memory");
    else
      asm volatile(
          "{\n\t.reg .pred p, q;\n\t"
          "setp.ne.b32 p, %4, 0;\n\t"
          "setp.ne.b32 q, %5, 0;\n\t"
          "@q tcgen05.mma.cta_group::2.kind::f16 [%0], %1, %2, %3, p;\n\t}"
          ::"r"(d_tmem), "l"(adesc), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(lead)
          : "memory");
  }
  // D += A[tmem] B[smem]: A's lane = row, each 32-bit column two bf16 along K
  __device__ __forceinline__ void mma_ts(uint32_t d_tmem, uint32_t a_tmem, uint64_t bdesc, uint32_t idesc,
                                         uint32_t accumulate) const {
    static_assert(CL == 1);
    asm volatile(
        "{\n\t.reg .pred p, q;\n\t"
        "setp.ne.b32 p, %4, 0;\n\t"
        "setp.ne.b32 q, %5, 0;\n\t"
        "@q tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
        ::"r"(d_tmem), "r"(a_tmem), "l"(bdesc), "r"(idesc), "r"(accumulate), "r"(lead)
        : "memory");
  }
  __device__ __forceinline__ void commit(uint64_t* bar) const {
    if (!lead) return;
    if constexpr (CL == 1)
      tc::mma_commit(bar);
    else
      asm volatile(
          "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
              tc::smem_u32(bar)),
          "h"((uint16_t)3)
          : "memory");
  }
  // After a give-up: the products issued so far end (the arrival is this CTA's alone: the other one may be gone).
  __device__ __forceinline__ void drain(uint64_t* bar) const {
    if (!lead) return;
    if constexpr (CL == 1)
      tc::mma_commit(bar);
    else
      asm volatile(
          "tcgen05.commit.cta_group::2.mbarrier::arrive::one.shared::cluster.multicast::cluster.b64 [%0], %1;" ::"r"(
              tc::smem_u32(bar)),
          "h"((uint16_t)1)
          : "memory");
    tc::mbar_wait(bar, 0);
  }

  // The other roles of the CTAs.
  static __device__ __forceinline__ uint32_t rank() {
    if constexpr (CL == 1) return 0;
    uint32_t r;
    asm volatile("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
  }
  static __device__ __forceinline__ void sync_all() {
    __syncwarp();
    if constexpr (CL == 1)
      __syncthreads();
    else
      asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
  }
  // address of the first CTA's barrier
  static __device__ __forceinline__ uint32_t first(uint64_t* bar) {
    uint32_t a;
    asm volatile("mapa.shared::cluster.u32 %0, %1, 0;" : "=r"(a) : "r"(tc::smem_u32(bar)));
    return a;
  }
  // one arrival for the warp at the first CTA's barrier, after what all its lanes did before
  static __device__ __forceinline__ void arrive(uint64_t* bar) {
    if constexpr (CL == 1) {
      warp_arrive(bar);
    } else {
      __syncwarp();
      if ((threadIdx.x & 31) == 0)
        asm volatile("mbarrier.arrive.shared::cluster.b64 _, [%0];" ::"r"(first(bar)) : "memory");
    }
  }
  // tile load into this CTA's shared memory, counted on the first CTA's barrier
  static __device__ __forceinline__ void load(void* dst, const CUtensorMap* map, int x, int y, uint64_t* bar) {
    if constexpr (CL == 1)
      tc::tma_load_2d(dst, map, x, y, bar);
    else
      asm volatile(
          "cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes.cta_group::2 [%0], [%1, "
          "{%2, %3}], [%4];" ::"r"(tc::smem_u32(dst)),
          "l"(map), "r"(x), "r"(y), "r"(first(bar))
          : "memory");
  }
  static __device__ __forceinline__ void alloc(uint32_t* slot, uint32_t ncols) {
    if constexpr (CL == 1) {
      tc::tmem_alloc(slot, ncols);
    } else {
      asm volatile("tcgen05.alloc.cta_group::2.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(tc::smem_u32(slot)),
                   "r"(ncols)
                   : "memory");
      asm volatile("tcgen05.relinquish_alloc_permit.cta_group::2.sync.aligned;" ::: "memory");
    }
  }
  static __device__ __forceinline__ void dealloc(uint32_t taddr, uint32_t ncols) {
    if constexpr (CL == 1)
      tc::tmem_dealloc(taddr, ncols);
    else
      asm volatile("tcgen05.dealloc.cta_group::2.sync.aligned.b32 %0, %1;" ::"r"(taddr), "r"(ncols) : "memory");
  }
};

// A bounded wait of a role: false, and the give-up recorded once, when it runs out.
struct Waiter {
  int* status;
  bool ok = true;
  __device__ __forceinline__ bool operator()(uint64_t* b, uint32_t parity) {
    if (ok && !tc::mbar_wait(b, parity)) {
      ok = false;
      record_device_error(status, tc::kErrTimeout);
    }
    if (ok) tc::fence_after_sync();
    return ok;
  }
};

// A warp's bounded wait: false on every lane, and the give-up recorded, once it has run out on one of them.
struct WarpWaiter {
  int* status;
  bool ok = true;
  __device__ __forceinline__ bool operator()(uint64_t* b, uint32_t parity) {
    if (ok && !tc::mbar_wait(b, parity)) {
      ok = false;
      record_device_error(status, tc::kErrTimeout);
    }
    ok = __all_sync(0xffffffffu, ok);
    if (ok) tc::fence_after_sync();
    return ok;
  }
};

}  // namespace hg
