// Internal declarations of the gated feed-forward block's tensor-core path (bf16); not part of the public ABI.
#pragma once

#include "hg_internal.cuh"

namespace hg {

hg_status ffn_fwd_tc(const hg_ffn_params* w, const void* X, int64_t n, void* Y, cudaStream_t s);
// dX null or g null: that part is left out
hg_status ffn_bwd_tc(const hg_ffn_params* w, const void* X, int64_t n, const void* dY, void* dX, const hg_ffn_grads* g,
                     void* scratch, cudaStream_t s);
size_t ffn_bwd_tc_scratch(const hg_ffn_params* w, int64_t n);

}  // namespace hg
