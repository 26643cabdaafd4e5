// Launches of the kernels that score rows for one element type; each type is a translation unit of its own (rsd_score_f32.cu,
// rsd_score_bf16.cu), which keeps the compiles short.
#pragma once
#include "../../include/rsd.h"
#include <algorithm>
#include <cstdlib>
#include "rsd_api_common.h"
#include "rsd_divergence.cuh"
#include "rsd_score.cuh"

namespace rsd {

// Blocks that share a row: few rows leave most of the chip idle, so that their tiles are dealt to the blocks of a cluster.
inline int row_blocks(unsigned slots, int n_tiles, int warps) {
    const int sms = rsd_host::sm_count();
    int blocks = 1;
    while (blocks < tiles::kMaxBlocks && (int64_t)slots * blocks * 2 <= 2 * sms && n_tiles > blocks * warps) blocks *= 2;
    return blocks;
}
template <typename A>
void launch_rows(void (*kernel)(A), unsigned slots, int blocks, int threads, size_t smem, cudaStream_t s, const A& a) {
    rsd_host::launch_overlapped(kernel, slots * (unsigned)blocks, (unsigned)threads, smem, s, blocks > 1 ? blocks : 0, a);
}

inline int env_int(const char* n, int d) { const char* e = getenv(n); return e ? atoi(e) : d; }
template <typename T, bool ALIGNED, bool TOP, int NW>
void launch_score_as(unsigned slots, int blocks, const ScoreArgs& a, cudaStream_t s) {
    const int n_tiles = tiles::tiles_of<T>(a.V, score::kWords);
    const size_t smem = score::sums_bytes(n_tiles) + (TOP ? (size_t)((n_tiles + blocks - 1) / blocks) * 32 * sizeof(float) : 0);
    launch_rows(score::score_rows_kernel<T, ALIGNED, TOP, NW>, slots, blocks, NW * 32, smem, s, a);
}
template <typename T, bool ALIGNED, bool TOP>
void launch_score_warps(unsigned slots, const ScoreArgs& a, cudaStream_t s) {
    const int blocks = row_blocks(slots, tiles::tiles_of<T>(a.V, score::kWords), 8);
    const int nw = env_int("NW", 8);
    if (blocks > 1 || nw == 8) launch_score_as<T, ALIGNED, TOP, 8>(slots, blocks, a, s);
    else if (nw == 4) launch_score_as<T, ALIGNED, TOP, 4>(slots, 1, a, s);
    else if (nw == 2) launch_score_as<T, ALIGNED, TOP, 2>(slots, 1, a, s);
    else launch_score_as<T, ALIGNED, TOP, 1>(slots, 1, a, s);
}
template <typename T>
void launch_score_of(bool aligned, unsigned slots, const ScoreArgs& a, cudaStream_t s) {
    if (a.K) {
        if (aligned) launch_score_warps<T, true, true>(slots, a, s);
        else launch_score_warps<T, false, true>(slots, a, s);
    } else {
        if (aligned) launch_score_warps<T, true, false>(slots, a, s);
        else launch_score_warps<T, false, false>(slots, a, s);
    }
}
// Blocks of a row whose tiles they keep in shared memory: as few as leave three blocks on an SM, and more where few rows leave SMs idle.
constexpr int kHeldBytes = 68 * 1024, kMostHeldBytes = 200 * 1024;
inline int holding_blocks(unsigned slots, int n_tiles, int tile_bytes, int warps) {
    int blocks = row_blocks(slots, n_tiles, warps);
    while (blocks < tiles::kMaxBlocks && (n_tiles + blocks - 1) / blocks * tile_bytes > kHeldBytes) blocks *= 2;
    return blocks;
}
template <typename T, bool ALIGNED, bool ENTROPY, int NW>
void launch_score_grad_as(unsigned slots, int blocks, const ScoreArgs& a, cudaStream_t s) {
    const int n_tiles = tiles::tiles_of<T>(a.V, score::kWords);
    const size_t smem = (size_t)((n_tiles + blocks - 1) / blocks) * tiles::kHeldTile<score::kWords> + score::sums_bytes(n_tiles);
    if (!rsd_host::raise_shared_memory<score::score_grad_kernel<T, ALIGNED, ENTROPY, NW>>(kMostHeldBytes)) return;
    launch_rows(score::score_grad_kernel<T, ALIGNED, ENTROPY, NW>, slots, blocks, NW * 32, smem, s, a);
}
template <typename T, bool ALIGNED, bool ENTROPY>
void launch_score_grad_warps(unsigned slots, const ScoreArgs& a, cudaStream_t s) {
    const int n_tiles = tiles::tiles_of<T>(a.V, score::kWords), blocks = holding_blocks(slots, n_tiles, tiles::kHeldTile<score::kWords>, 8);
    const int nw = env_int("NW", 8);
    if (blocks > 1 || nw == 8) launch_score_grad_as<T, ALIGNED, ENTROPY, 8>(slots, blocks, a, s);
    else if (nw == 4) launch_score_grad_as<T, ALIGNED, ENTROPY, 4>(slots, 1, a, s);
    else launch_score_grad_as<T, ALIGNED, ENTROPY, 2>(slots, 1, a, s);
}
template <typename T>
void launch_score_grad_of(bool aligned, unsigned slots, const ScoreArgs& a, cudaStream_t s) {
    if (a.g_entropy) {
        if (aligned) launch_score_grad_warps<T, true, true>(slots, a, s);
        else launch_score_grad_warps<T, false, true>(slots, a, s);
    } else {
        if (aligned) launch_score_grad_warps<T, true, false>(slots, a, s);
        else launch_score_grad_warps<T, false, false>(slots, a, s);
    }
}
template <typename T, bool ALIGNED, int NW>
void launch_divergence_as(unsigned slots, const DivergenceArgs& a, cudaStream_t s) {
    namespace d = divergence;
    const int n_tiles = tiles::tiles_of<T>(a.V, d::kWords), blocks = env_int("GB", 0) ? env_int("GB", 0) : row_blocks(slots, n_tiles, NW);
    launch_rows(d::divergence_kernel<T, ALIGNED, NW>, slots, blocks, NW * 32, (size_t)n_tiles * sizeof(d::Sums), s, a);
}
template <typename T>
void launch_divergence_of(bool aligned, unsigned slots, const DivergenceArgs& a, cudaStream_t s) {
    const int nw = env_int("NW", 8);
    if (aligned) nw == 8 ? launch_divergence_as<T, true, 8>(slots, a, s) : launch_divergence_as<T, true, 4>(slots, a, s);
    else nw == 8 ? launch_divergence_as<T, false, 8>(slots, a, s) : launch_divergence_as<T, false, 4>(slots, a, s);
}
template <typename T, bool ALIGNED, bool REVERSE, int NW>
void launch_divergence_grad_as(unsigned slots, const DivergenceArgs& a, cudaStream_t s) {
    namespace d = divergence;
    const int n_tiles = tiles::tiles_of<T>(a.V, d::kWords), blocks = env_int("GB", 0) ? env_int("GB", 0) : row_blocks(slots, n_tiles, NW);
    launch_rows(d::divergence_grad_kernel<T, ALIGNED, REVERSE, NW>, slots, blocks, NW * 32, (size_t)n_tiles * sizeof(d::Sums), s, a);
}
template <typename T, bool REVERSE>
void launch_divergence_grad_warps(bool aligned, unsigned slots, const DivergenceArgs& a, cudaStream_t s) {
    const int nw = env_int("NW", 8);
    if (aligned) nw == 8 ? launch_divergence_grad_as<T, true, REVERSE, 8>(slots, a, s) : launch_divergence_grad_as<T, true, REVERSE, 4>(slots, a, s);
    else nw == 8 ? launch_divergence_grad_as<T, false, REVERSE, 8>(slots, a, s) : launch_divergence_grad_as<T, false, REVERSE, 4>(slots, a, s);
}
template <typename T>
void launch_divergence_grad_of(bool aligned, unsigned slots, const DivergenceArgs& a, cudaStream_t s) {
    if (a.g_reverse) launch_divergence_grad_warps<T, true>(aligned, slots, a, s);
    else launch_divergence_grad_warps<T, false>(aligned, slots, a, s);
}

}  // namespace rsd
