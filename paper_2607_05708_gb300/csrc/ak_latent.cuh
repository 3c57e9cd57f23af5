// Attention over the latent cache: what its kernels share.
#pragma once

#include "ak_attend.cuh"

namespace ak {

template <typename S>
constexpr bool is_bf16 = false;
template <>
constexpr bool is_bf16<__nv_bfloat16> = true;

// One call's arguments.  Absorbed: one key head, all query heads its group; expanded: a key head a
// query head.
struct LatentParams {
    AttendParams a;
    int R, P;                         // latent and rotated values of a row
    bool bf16;                        // else fp16
    // expanded
    int nope, value;
    const void *w_k, *w_v;
    int64_t k_head, k_row, v_head, v_row;
};

int64_t latent_absorbed_scratch(const LatentParams &p);
int64_t latent_expanded_scratch(const LatentParams &p);
cudaError_t launch_latent_absorbed(LatentParams &p, void *scratch, cudaStream_t st);
cudaError_t launch_latent_expanded(LatentParams &p, void *scratch, cudaStream_t st);

}  // namespace ak
