// Attention over the latent cache: what its kernels share.
#pragma once

#include "ak_attend.cuh"
#include "ak_sm100.cuh"

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

// The expanded form's keys and values of a group of heads: row (head, sequence, token) at (head *
// n_seq + sequence) * seq_rows + token.
struct LatentSpace {
    void *k, *v;                      // [rows][nope], [rows][value]
    int64_t seq_rows, rows;           // seq_rows: a multiple of 128
    int64_t k_step, v_step;           // rows of w_k and w_v from one head to the next
    int head0, heads;
};

// Scratch of the joins, the tokens of a box of the copies from the cache (boxes do not cross blocks), and
// the cache's tensor map: boxes of 64 values.
int64_t latent_joins_bytes(int ctas);
int latent_box(const LatentParams &p);
cudaError_t latent_rows_map(const LatentParams &p, CUtensorMap *map);

int64_t latent_absorbed_scratch(const LatentParams &p);
int64_t latent_expanded_scratch(const LatentParams &p);  // -1: too many tokens
cudaError_t launch_latent_absorbed(LatentParams &p, void *scratch, cudaStream_t st);
cudaError_t launch_latent_expand(const LatentParams &p, const LatentSpace &sp, cudaStream_t st);
cudaError_t launch_latent_expanded(LatentParams &p, void *scratch, cudaStream_t st);

}  // namespace ak
