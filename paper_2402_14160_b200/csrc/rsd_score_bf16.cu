// The kernels that score rows of bf16 entries.
#include "rsd_score_launch.cuh"

namespace rsd {

void launch_score_bf16(bool aligned, unsigned slots, const ScoreArgs& a, cudaStream_t s) { launch_score_of<__nv_bfloat16>(aligned, slots, a, s); }
void launch_score_grad_bf16(bool aligned, unsigned slots, const ScoreArgs& a, cudaStream_t s) { launch_score_grad_of<__nv_bfloat16>(aligned, slots, a, s); }
void launch_divergence_bf16(bool aligned, unsigned slots, const DivergenceArgs& a, cudaStream_t s) { launch_divergence_of<__nv_bfloat16>(aligned, slots, a, s); }
void launch_divergence_grad_bf16(bool aligned, unsigned slots, const DivergenceArgs& a, cudaStream_t s) { launch_divergence_grad_of<__nv_bfloat16>(aligned, slots, a, s); }

}  // namespace rsd
