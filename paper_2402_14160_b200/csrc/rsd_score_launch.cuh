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
// every warp has a tile.  (us a call, 1 / 2 / 4 / 8 blocks: likeliest 5 of 1 / 100 / 200 / 400 rows of 128,000 bf16 14.7 / 10.7 / 8.9 / 7.6, 16.9 / 14.4 / 13.7 / 18.1,
// 20.9 / 18.2 / 23.7 / 28.9, 26.5 / 31.4 / 36.8 / 50.3; divergence of 37 pairs of 32,000 fp32 17.6 / 13.2 / 10.6 / 9.2.)
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
// 19.8 / 12.4 / 8.9 / 8.5, 21.8 / 15.1 / 12.6 / 13.7, 25.6 / 22.2 / 21.4 / 21.4, 82.8 / 74.3 / 71.5 / 79.9; 7000 of 8000 23.7 / 24.7 / 27.8 / 43.6; with the
// likeliest 5, which warps spend more time apart on, 7000 of 32,000 104 / 94 / 97 / 116; 3000 of 128,000 fp32 218 / 266 / 222 / 220.)
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
// 7000 bf16 rows of 1500 / 8000 / 32,000: 41 / 71 / 129, 56 / 60 / 94, 271 / 197 / 175).
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

// Divergences: short rows have fewer warps (us, 2 / 4 / 8 warps: 7000 pairs of 1500 bf16 47 / 61 / 106, of 8000 fp32 111 / 117 / 153), long ones eight, which reads them again from L2
// (7000 pairs of 32,000 fp32 491 / 442 / 401, bf16 257 / 258 / 260).  Where no second sweep is asked for, many pairs have four (KL alone, 700 / 7000 pairs of 32,000 bf16
// 33 / 24 / 25, 152 / 148 / 159).  How many blocks are resident is not looked at: a little more than a wave of them (640 pairs of 32,001 bf16 65 / 44 / 46, 700 of 32,000 56 / 42 / 46)
// would be faster with four warps, two waves (1300 pairs 70 / 66 / 59) are not.
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
// blocks, so that fewer are under way at a time (us, 1 / 2 / 4 / 8 blocks: 1000 pairs of 32,000 fp32 92 / 90 / 108 / 149, of 60,000 fp32 182 / 159 / 161 / 203, of 128,000 bf16
// 191 / 177 / 183 / 228, of 128,000 fp32 390 / 357 / 325 / 328; 5000 of 60,000 bf16 386 / 412 / 506 / 702).  The bytes under way are taken as those of three pairs an SM, or of all pairs if there
// are fewer, over the blocks a pair; between one and three pairs an SM that is too little (192 pairs of 128,000 fp32 88 / 73 / 67 / 72, and it takes two blocks).
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
