// Arguments of the kernels that score rows, and their launches per element type (rsd_score_f32.cu, rsd_score_bf16.cu).
#pragma once
#include <cuda_runtime.h>
#include <stdint.h>

namespace rsd {

struct ScoreArgs {
    const void* data;
    int64_t seq_stride, row_stride;
    int R, V, T, K, num_rows;
    const int32_t* row_index;      // [B][R] or null
    const int32_t* token;          // [B][R][T] or null
    // the path that a verification accepted, in place of row_index and token (R = L + 1, T = 1)
    const int32_t *accepted_len, *accepted_node, *accepted_token, *last_token;
    float inv_temp, k;             // 1 / temperature, log2(e) / temperature; finite
    float *out_logprob, *out_entropy, *out_top_logprob;
    int32_t *out_token, *out_top_token, *status;
    // gradient
    const float *g_logprob, *g_entropy;
    void* grad;
};

struct DivergenceArgs {
    const void *draft, *target;
    int64_t draft_seq, draft_row, target_seq, target_row;    // strides in entries
    int R, V;
    float k_draft, k_target;                                 // log2(e) / temperature
    float inv_draft_temp;
    float *out_kl, *out_reverse, *out_overlap;
    int32_t* status;
    const float *g_kl, *g_reverse;
    void* grad;
};

// `slots` rows (or pairs of rows), a block or a cluster of blocks each.  aligned: rows (and gradient rows) start on 16-byte boundaries.
void launch_score_f32(bool aligned, unsigned slots, const ScoreArgs& a, cudaStream_t s);
void launch_score_bf16(bool aligned, unsigned slots, const ScoreArgs& a, cudaStream_t s);
void launch_score_grad_f32(bool aligned, unsigned slots, const ScoreArgs& a, cudaStream_t s);
void launch_score_grad_bf16(bool aligned, unsigned slots, const ScoreArgs& a, cudaStream_t s);
void launch_divergence_f32(bool aligned, unsigned slots, const DivergenceArgs& a, cudaStream_t s);
void launch_divergence_bf16(bool aligned, unsigned slots, const DivergenceArgs& a, cudaStream_t s);
void launch_divergence_grad_f32(bool aligned, unsigned slots, const DivergenceArgs& a, cudaStream_t s);
void launch_divergence_grad_bf16(bool aligned, unsigned slots, const DivergenceArgs& a, cudaStream_t s);

}  // namespace rsd
