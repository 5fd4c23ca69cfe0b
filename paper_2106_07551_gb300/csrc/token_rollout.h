// Token policies, the rollout's side, and dropout: what the entry points give the kernels.
#pragma once

#include "token_common.cuh"

namespace malib {

enum : int { kListTop = 0, kListDraw = 1, kListDrawAll = 2 };

struct ListArgs : TokenArgs {                        // tokens: null, every row is live
    int32_t K;                                       // entries of the list
    // the list
    int32_t* top_ids;                                // [n][K]
    float* top_logp;                                 // [n][K]
    int32_t* rank;                                   // [n]
    // the draw
    int32_t* drawn;                                  // [n]
    float* draw_logp;                                // [n]
    const float* uniform;                            // [n]; null: by (seed; sequence, step, agent)
    const int64_t* sequence;                         // [n]
    const int32_t* step;                             // [n]
    uint64_t seed;
    uint32_t agent;
    float top_p;
};
// Lists and draws (token_list.cuh), by type.
cudaError_t launch_token_list_f32(const ListArgs& a, int op, int n_sm, cudaStream_t s);
cudaError_t launch_token_list_bf16(const ListArgs& a, int op, int n_sm, cudaStream_t s);
cudaError_t launch_token_list_f16(const ListArgs& a, int op, int n_sm, cudaStream_t s);
inline cudaError_t launch_token_list(const ListArgs& a, int op, int n_sm, cudaStream_t s) {
    if (a.dtype == MALIB_F32) return launch_token_list_f32(a, op, n_sm, s);
    if (a.dtype == MALIB_BF16) return launch_token_list_bf16(a, op, n_sm, s);
    return launch_token_list_f16(a, op, n_sm, s);
}

struct DropArgs {
    const void *x, *residual;                        // residual: null: none
    void* out;
    int64_t n, ld_x, ld_res, ld_out;
    int32_t d, dtype;
    const int64_t* sequence;                         // [n]
    const int32_t* step;                             // [n]
    uint64_t seed;
    uint32_t counter;                                // 2^31 | site << 16
    uint32_t least;                                  // p 2^16: smaller halves drop their column
    float scale;
    // vectors of a row; how far a block's next tile is on; ceil(2^32 / per_row)
    int32_t per_row, step_i;
    int64_t step_r;
    uint32_t magic;
};
cudaError_t launch_dropout(const DropArgs& a, int n_sm, cudaStream_t s);

}  // namespace malib
