// The kernels that score rows of fp32 entries.
#include "rsd_score_launch.cuh"

namespace rsd {

void launch_score_f32(bool aligned, unsigned slots, const ScoreArgs& a, cudaStream_t s) { launch_score_of<float>(aligned, slots, a, s); }
void launch_score_grad_f32(bool aligned, unsigned slots, const ScoreArgs& a, cudaStream_t s) { launch_score_grad_of<float>(aligned, slots, a, s); }
void launch_divergence_f32(bool aligned, unsigned slots, const DivergenceArgs& a, cudaStream_t s) { launch_divergence_of<float>(aligned, slots, a, s); }
void launch_divergence_grad_f32(bool aligned, unsigned slots, const DivergenceArgs& a, cudaStream_t s) { launch_divergence_grad_of<float>(aligned, slots, a, s); }

}  // namespace rsd
