// Launches of the kernels that score rows for one element type; each type is a translation unit of its own (rsd_score_f32.cu,
// rsd_score_bf16.cu), which keeps the compiles short.
#pragma once
#include <algorithm>

#include "../../include/rsd.h"
#include "rsd_api_common.h"
#include "rsd_divergence.cuh"
#include "rsd_score.cuh"

namespace rsd {

// Blocks that share a row: few rows leave most of the chip idle, so that their tiles are dealt to the blocks of a cluster, up to three blocks an SM and as long as
// every warp has a tile.  (us a call, 1 / 2 / 4 / 8 blocks: likeliest 5 of 1 / 100 / 200 / 400 rows of 128,000 bf16 14.4 / 10.8 / 8.9 / 7.3, 16.5 / 14.0 / 12.9 / 17.1,
// 20.9 / 18.1 / 23.4 / 28.3, 26.3 / 31.0 / 35.9 / 49.3; divergence of 37 pairs of 32,000 fp32 19.6 / 14.0 / 10.6 / 9.3.)
inline int row_blocks(unsigned slots, int n_tiles, int warps) {
    const int sms = rsd_host::sm_count();
    int blocks = 1;
    while (blocks < tiles::kMaxBlocks && (int64_t)slots * blocks * 2 <= 3 * sms && n_tiles > blocks * warps) blocks *= 2;
    return blocks;
}
template <typename A>
void launch_rows(void (*kernel)(A), unsigned slots, int blocks, int threads, size_t smem, cudaStream_t s, const A& a) {
    rsd_host::launch_overlapped(kernel, slots * (unsigned)blocks, (unsigned)threads, smem, s, blocks > 1 ? blocks : 0, a);
}

// Warps per row where a row has one block.  As many as leave all rows resident at 32 warps an SM; rows beyond that take turns, and long turns of few warps leave SMs
// idle at the end where short ones of many warps pay for their barriers.  (us, 1 / 2 / 4 / 8 warps, bf16 without likeliest tokens: 300 / 700 / 1500 / 7000 rows of 32,000
// 18.3 / 11.8 / 8.6 / 8.0, 21.2 / 14.9 / 12.5 / 13.7, 25.1 / 22.3 / 22.1 / 21.5, 80.6 / 73.4 / 71.3 / 79.2; 7000 of 8000 23.4 / 24.3 / 27.5 / 42.9; with the
// likeliest 5, which warps spend more time apart on, 7000 of 32,000 101 / 93 / 97 / 115; 3000 of 128,000 fp32 410 / 307 / 270 / 233.)
inline int score_warps(unsigned slots, int n_tiles, bool top) {
    const int sms = rsd_host::sm_count();
    const int most = n_tiles >= 8 ? 8 : n_tiles >= 4 ? 4 : n_tiles >= 2 ? 2 : 1;
    const int least = n_tiles <= 4 ? 1 : n_tiles > 40 ? (slots > 8u * sms ? 8 : 4) : top ? (n_tiles <= 20 ? 2 : 4) : n_tiles <= 8 ? 2 : 4;
    int warps = most;
    while (warps > least && slots > (unsigned)(sms * 32 / warps)) warps /= 2;
    return std::max(warps, std::min(least, most));
}

template <typename T, bool ALIGNED, bool TOP, int NW>
void launch_score_as(unsigned slots, int blocks, const ScoreArgs& a, cudaStream_t s) {
    const int n_tiles = tiles::tiles_of<T>(a.V, score::kWords);
    const size_t smem = score::sums_bytes(n_tiles) + (TOP ? (size_t)((n_tiles + blocks - 1) / blocks) * 32 * sizeof(float) : 0);
    launch_rows(score::score_rows_kernel<T, ALIGNED, TOP, NW>, slots, blocks, NW * 32, smem, s, a);
}
template <typename T, bool ALIGNED, bool TOP>
void launch_score_warps(unsigned slots, const ScoreArgs& a, cudaStream_t s) {
    const int n_tiles = tiles::tiles_of<T>(a.V, score::kWords), blocks = row_blocks(slots, n_tiles, 8), warps = blocks > 1 ? 8 : score_warps(slots, n_tiles, TOP);
    if (warps == 8) launch_score_as<T, ALIGNED, TOP, 8>(slots, blocks, a, s);
    else if (warps == 4) launch_score_as<T, ALIGNED, TOP, 4>(slots, 1, a, s);
    else if (warps == 2) launch_score_as<T, ALIGNED, TOP, 2>(slots, 1, a, s);
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

// Gradients of scores: blocks keep their tiles in shared memory, as few blocks a row as leave three of them on an SM (more for few rows).  Short rows have fewer warps (us, 2 / 4 / 8 warps,
// 7000 bf16 rows of 1500 / 8000 / 32,000: 36 / 59 / 131, 55 / 57 / 90, 262 / 194 / 173).
constexpr int kHeldBytes = 68 * 1024, kMostHeldBytes = 200 * 1024;
template <typename T, bool ALIGNED, bool ENTROPY, int NW>
void launch_score_grad_as(unsigned slots, int blocks, const ScoreArgs& a, cudaStream_t s) {
    const int n_tiles = tiles::tiles_of<T>(a.V, score::kWords);
    const size_t smem = (size_t)((n_tiles + blocks - 1) / blocks) * tiles::kHeldTile<score::kWords> + score::sums_bytes(n_tiles);
    if (!rsd_host::raise_shared_memory<score::score_grad_kernel<T, ALIGNED, ENTROPY, NW>>(kMostHeldBytes)) return;
    launch_rows(score::score_grad_kernel<T, ALIGNED, ENTROPY, NW>, slots, blocks, NW * 32, smem, s, a);
}
template <typename T, bool ALIGNED, bool ENTROPY>
void launch_score_grad_warps(unsigned slots, const ScoreArgs& a, cudaStream_t s) {
    const int n_tiles = tiles::tiles_of<T>(a.V, score::kWords);
    int blocks = row_blocks(slots, n_tiles, 8);
    while (blocks < tiles::kMaxBlocks && (n_tiles + blocks - 1) / blocks * tiles::kHeldTile<score::kWords> > kHeldBytes) blocks *= 2;
    if (blocks > 1 || n_tiles > 8) launch_score_grad_as<T, ALIGNED, ENTROPY, 8>(slots, blocks, a, s);
    else if (n_tiles > 2) launch_score_grad_as<T, ALIGNED, ENTROPY, 4>(slots, 1, a, s);
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

// Divergences: short rows have fewer warps (us, 2 / 4 / 8 warps: 7000 pairs of 1500 bf16 48 / 58 / 99, of 8000 fp32 140 / 115 / 137, of 32,000 bf16 284 / 291 / 293), and so
// have many pairs of which no second sweep is asked for (KL alone, 700 / 7000 pairs of 32,000 bf16 32 / 24 / 25, 170 / 164 / 176).
inline int divergence_warps(unsigned slots, int n_tiles, bool one_sweep) {
    const int sms = rsd_host::sm_count();
    if (n_tiles <= 3) return 2;
    if (n_tiles <= 8 || (n_tiles <= 16 && slots > 2u * sms) || (one_sweep && slots > 4u * sms)) return 4;
    return 8;
}
template <typename T, bool ALIGNED, bool OVERLAP, int NW>
void launch_divergence_as(unsigned slots, int blocks, const DivergenceArgs& a, cudaStream_t s) {
    launch_rows(divergence::divergence_kernel<T, ALIGNED, OVERLAP, NW>, slots, blocks, NW * 32, (size_t)tiles::tiles_of<T>(a.V, divergence::kWords) * sizeof(divergence::Sums), s, a);
}
template <typename T, bool ALIGNED, bool OVERLAP>
void launch_divergence_warps(unsigned slots, const DivergenceArgs& a, cudaStream_t s) {
    const int n_tiles = tiles::tiles_of<T>(a.V, divergence::kWords), blocks = row_blocks(slots, n_tiles, 8), warps = blocks > 1 ? 8 : divergence_warps(slots, n_tiles, !OVERLAP);
    if (warps == 8) launch_divergence_as<T, ALIGNED, OVERLAP, 8>(slots, blocks, a, s);
    else if (warps == 4) launch_divergence_as<T, ALIGNED, OVERLAP, 4>(slots, 1, a, s);
    else launch_divergence_as<T, ALIGNED, OVERLAP, 2>(slots, 1, a, s);
}
template <typename T>
void launch_divergence_of(bool aligned, unsigned slots, const DivergenceArgs& a, cudaStream_t s) {
    if (a.out_overlap) {
        if (aligned) launch_divergence_warps<T, true, true>(slots, a, s);
        else launch_divergence_warps<T, false, true>(slots, a, s);
    } else {
        if (aligned) launch_divergence_warps<T, true, false>(slots, a, s);
        else launch_divergence_warps<T, false, false>(slots, a, s);
    }
}

// Gradients of divergences read their rows twice, the second time from L2, which does not hold the pairs under way beside the gradient's words where they are long: those are shared by two or four
// blocks, so that fewer are under way at a time (us, 1 / 2 / 4 / 8 blocks: 1000 pairs of 32,000 fp32 91 / 89 / 108 / 150, of 60,000 fp32 180 / 159 / 159 / 201, of 128,000 bf16
// 193 / 179 / 184 / 229, of 128,000 fp32 390 / 355 / 328 / 337; 5000 of 60,000 bf16 387 / 405 / 506 / 713).
constexpr int64_t kReadAgainBytes = 120 * 1000 * 1000;
template <typename T, bool ALIGNED, bool REVERSE, int NW>
void launch_divergence_grad_as(unsigned slots, int blocks, const DivergenceArgs& a, cudaStream_t s) {
    launch_rows(divergence::divergence_grad_kernel<T, ALIGNED, REVERSE, NW>, slots, blocks, NW * 32, (size_t)tiles::tiles_of<T>(a.V, divergence::kWords) * sizeof(divergence::Sums), s, a);
}
template <typename T, bool ALIGNED, bool REVERSE>
void launch_divergence_grad_warps(unsigned slots, const DivergenceArgs& a, cudaStream_t s) {
    const int n_tiles = tiles::tiles_of<T>(a.V, divergence::kWords);
    int blocks = row_blocks(slots, n_tiles, 8);
    const int64_t under_way = std::min<int64_t>(slots, 3 * rsd_host::sm_count()) * a.V * 2 * (int64_t)sizeof(T);
    while (blocks < 4 && under_way / blocks > kReadAgainBytes) blocks *= 2;
    const int warps = blocks > 1 ? 8 : divergence_warps(slots, n_tiles, false);
    if (warps == 8) launch_divergence_grad_as<T, ALIGNED, REVERSE, 8>(slots, blocks, a, s);
    else if (warps == 4) launch_divergence_grad_as<T, ALIGNED, REVERSE, 4>(slots, 1, a, s);
    else launch_divergence_grad_as<T, ALIGNED, REVERSE, 2>(slots, 1, a, s);
}
template <typename T>
void launch_divergence_grad_of(bool aligned, unsigned slots, const DivergenceArgs& a, cudaStream_t s) {
    if (a.g_reverse) {
        if (aligned) launch_divergence_grad_warps<T, true, true>(slots, a, s);
        else launch_divergence_grad_warps<T, false, true>(slots, a, s);
    } else {
        if (aligned) launch_divergence_grad_warps<T, true, false>(slots, a, s);
        else launch_divergence_grad_warps<T, false, false>(slots, a, s);
    }
}

}  // namespace rsd
