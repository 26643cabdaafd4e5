// Launches of the kernels that score rows for one element type; each type is a translation unit of its own (rsd_score_f32.cu,
// rsd_score_bf16.cu), which keeps the compiles short.
#pragma once
#include "../../include/rsd.h"
#include "rsd_api_common.h"
#include "rsd_divergence.cuh"
#include "rsd_score.cuh"

namespace rsd {

template <typename T>
void launch_score_of(bool aligned, unsigned slots, const ScoreArgs& a, cudaStream_t s) {
    const size_t smem = a.K ? (size_t)tiles::tiles_of<T>(a.V, score::kWords) * 32 * sizeof(float) : 0;
    rsd_host::launch_overlapped(aligned ? score::score_rows_kernel<T, true> : score::score_rows_kernel<T, false>, slots, score::kThreads, smem, s, 0, a);
}
template <typename T>
void launch_score_grad_of(bool aligned, unsigned slots, const ScoreArgs& a, cudaStream_t s) {
    if (a.g_entropy) rsd_host::launch_overlapped(aligned ? score::score_grad_kernel<T, true, true> : score::score_grad_kernel<T, false, true>, slots, score::kThreads, 0, s, 0, a);
    else rsd_host::launch_overlapped(aligned ? score::score_grad_kernel<T, true, false> : score::score_grad_kernel<T, false, false>, slots, score::kThreads, 0, s, 0, a);
}
template <typename T>
void launch_divergence_of(bool aligned, unsigned slots, const DivergenceArgs& a, cudaStream_t s) {
    rsd_host::launch_overlapped(aligned ? divergence::divergence_kernel<T, true> : divergence::divergence_kernel<T, false>, slots, divergence::kThreads, 0, s, 0, a);
}
template <typename T>
void launch_divergence_grad_of(bool aligned, unsigned slots, const DivergenceArgs& a, cudaStream_t s) {
    namespace d = divergence;
    if (a.g_reverse) rsd_host::launch_overlapped(aligned ? d::divergence_grad_kernel<T, true, true> : d::divergence_grad_kernel<T, false, true>, slots, d::kThreads, 0, s, 0, a);
    else rsd_host::launch_overlapped(aligned ? d::divergence_grad_kernel<T, true, false> : d::divergence_grad_kernel<T, false, false>, slots, d::kThreads, 0, s, 0, a);
}

}  // namespace rsd
