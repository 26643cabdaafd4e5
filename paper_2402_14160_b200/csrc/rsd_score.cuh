// Log-probabilities of given tokens, entropy and the likeliest tokens of rows (score_rows_kernel), and the gradient of weighted
// log-probabilities and entropies (score_grad_kernel).
//
// With z = v / T, m = max z, y = (v - max v) log2(e) / T:   Z = sum 2^y,   log p_x = z_x - m - ln Z,   H = ln Z - ln 2 (sum 2^y y) / Z.
// Both terms of H are positive: nothing cancels.  One pass over the row, one exponential per entry.
//
// Sums, maxima and norms are fp32 throughout; a gradient is rounded to the rows' type once, where it is stored.
#pragma once
#include "../../include/rsd.h"
#include "rsd_score_args.h"
#include "rsd_tiles.cuh"

namespace rsd {

namespace score {

constexpr int kWords = 8;
constexpr int kBuckets = 64;       // samples that bound the K-th largest entry: two per lane
constexpr int kList = 512;         // groups opened, and entries taken from them
static_assert(kBuckets >= RSD_MAX_K, "");

struct Sums {                      // of a row's n tiles, relative to each tile's largest entry; every block of the row has all of them
    float *m, *s, *w;
    __device__ __forceinline__ Sums(float* at, int n) : m(at), s(at + n), w(at + 2 * n) {}
};
constexpr size_t sums_bytes(int n) { return (size_t)n * 3 * sizeof(float); }
struct RowTotals {
    float m, s, w;                 // largest entry; sum of 2^y, of 2^y y
};

// Sum of 2^y and of 2^y y over a tile, y = (v - m) k, to all blocks of the row; lane_max: the lane's largest entry.  refill(i) reads word i of
// the warp's next tile into its place as soon as it is free, so that half of the work and the sums over the warp go on while the words are on their way.
template <typename T, bool ENTROPY, typename F>
__device__ __forceinline__ void tile_sums(uint4 (&w)[kWords], float k, int t, int lane, uint32_t blocks, const Sums& sums, float& lane_max, bool& bad, F refill) {
    using P = tiles::Packed16<T>;
    float mx = P::largest(w), m = tiles::warp_max_nan(mx);
    unsigned long long s = tiles::both(0.0f), e = s;
    if (tiles::plain_tile(m, k)) {
        const unsigned long long ref = tiles::both(-(m * k)), kk = tiles::both(k);
#pragma unroll
        for (int half = 0; half < kWords; half += kWords / 2) {
#pragma unroll
            for (int i = half; i < half + kWords / 2; ++i)
                P::pairs(ENTROPY ? P::raised(w[i]) : w[i], [&](unsigned long long v) {
                    const unsigned long long y = fma_f32x2(v, kk, ref);
                    float a, b;
                    split_f32x2(y, a, b);
                    const unsigned long long x = f32x2(ex2_approx(a), ex2_approx(b));
                    s = add_f32x2(s, x);
                    if (ENTROPY) e = fma_f32x2(x, y, e);
                });
            refill(half);
        }
    } else {                                        // no entry, NaN, +inf, or values or a scale near the end of the range
        if (!(m < __builtin_huge_valf())) {
#pragma unroll
            for (int i = 0; i < kWords; ++i) P::clean(w[i], bad);
            mx = P::largest(w), m = tiles::warp_max_nan(mx);
        }
        if (m > kNegInf) {
            const bool plain = tiles::plain_tile(m, k);   // (as the join takes it)
            const float half = tiles::part_of(k);
            const unsigned long long part = tiles::both(half), minus_m = tiles::both(plain ? 0.0f : -m * half), ref = tiles::both(plain ? -(m * k) : 0.0f),
                                     kk = tiles::both(tiles::scale_of_part(k));
#pragma unroll
            for (int i = 0; i < kWords; ++i)
                P::pairs(w[i], [&](unsigned long long v) {
                    float a, b;
                    split_f32x2(fma_f32x2(fma_f32x2(v, part, minus_m), kk, ref), a, b);
                    a = fmaxf(a, tiles::kFarBelow), b = fmaxf(b, tiles::kFarBelow);
                    const unsigned long long x = f32x2(ex2_approx(a), ex2_approx(b));
                    s = add_f32x2(s, x);
                    e = fma_f32x2(x, f32x2(a, b), e);
                });
        }
        refill(0);
        refill(kWords / 2);
    }
    lane_max = mx;
    float s0, s1, e0, e1;
    split_f32x2(s, s0, s1);
    split_f32x2(e, e0, e1);
    const float sum = tiles::warp_sum_two(s0 + s1, e0 + e1, lane);   // lanes 0 to 15 the first, the others the second
    if (blocks == 1) {
        if (lane == 0) sums.m[t] = m, sums.s[t] = sum;
        if (ENTROPY && lane == 16) sums.w[t] = sum;
        return;
    }
    const uint32_t to = lane & 7;
    if (to < blocks) {
        if (lane < 8) tiles::store_at(&sums.s[t], to, sum);
        else if (lane < 16) tiles::store_at(&sums.m[t], to, m);
        else if (lane < 24) tiles::store_at(&sums.w[t], to, sum);
    }
}

// Half of the words of a tile; nothing where there is no such tile.
template <typename T, bool ALIGNED>
__device__ __forceinline__ void load_half(uint4 (&w)[kWords], const tiles::View& view, int t, int half, int lane, int V) {
    constexpr int kHalf = kWords / 2, E = tiles::Packed16<T>::kEntries;
    const int from = t * tiles::tile_entries<T>(kWords) + half * 32 * E;
    if (t * tiles::tile_entries<T>(kWords) >= V) return;
    uint4 h[kHalf];
    tiles::load_words<T, ALIGNED, kHalf>(h, view, from + lane * E, from + tiles::tile_entries<T>(kHalf) <= V, V);
#pragma unroll
    for (int i = 0; i < kHalf; ++i) w[half + i] = h[i];
}

// The tiles' sums joined by one warp; every lane gets the result.
template <bool ENTROPY>
__device__ __forceinline__ RowTotals join(const Sums& sums, int n, float k, int lane) {
    float m = kNegInf;
    for (int t = lane; t < n; t += 32) m = fmaxf(m, sums.m[t]);
    m = tiles::warp_max_nan(m);
    float s = 0.0f, w = 0.0f;
    for (int t = lane; t < n; t += 32) {
        const float mt = sums.m[t];
        if (mt == kNegInf) continue;
        const float d = fmaxf(tiles::distance(mt, m, k), tiles::kFarBelow) - tiles::rounded_off(mt, k), f = ex2_approx(d);
        s = fmaf(f, sums.s[t], s);
        if (ENTROPY) w = fmaf(f, fmaf(d, sums.s[t], sums.w[t]), w);
    }
    const float sum = tiles::warp_sum_two(s, w, lane);
    return {m, __shfl_sync(0xFFFFFFFFu, sum, 0), __shfl_sync(0xFFFFFFFFu, sum, 16)};
}

template <typename T>
__device__ __forceinline__ float entry(const void* row, int x) {   // -inf where it is none
    const float v = RowIO<T>::scalar(row, x);
    return v < __builtin_huge_valf() ? v : kNegInf;
}

// ---- the K largest entries of a row ----------------------------------------------------------------------------------------------
// Every lane knows its largest entry of each tile (a group of up to 64 entries).  The largest of a block's even and of its odd tiles in each lane are
// kBuckets distinct entries: the K-th largest of them is at most the K-th largest entry of the block's tiles.  Only groups that reach that bound are read again
// (they lie in L2), a word a thread; the entries that reach it, about 1.4 K of a block, go to the row's first block, which ranks those that reach
// the largest of the blocks' bounds.
template <int NW>
struct TopSmem {
    float bucket[NW][kBuckets];
    float bound, bounds[tiles::kMaxBlocks];   // the block's; in the first block those of all
    int32_t group[kList];
    unsigned long long key[kList];            // in the first block: the entries of all, by value, then by token (the smaller one is larger)
    int groups, count, kept, overflow;
    float best_value[NW];
    int best_token[NW];
};
__device__ __forceinline__ unsigned long long key_of(float v, int x) { return (unsigned long long)float_to_ordered(v + 0.0f) << 32 | (uint32_t)~x; }   // (-0 is 0)
__device__ __forceinline__ float value_of(unsigned long long key) { return ordered_to_float((uint32_t)(key >> 32)); }
__device__ __forceinline__ int token_of(unsigned long long key) { return (int)~(uint32_t)key; }

// K-th largest of 64 values, two per lane, from below: exact in its upper 16 bits, found two bits at a time.
__device__ __forceinline__ float bound_of_kth(float a, float b, int K) {
    const uint32_t ca = a > kNegInf ? float_to_ordered(a) >> 16 : 0u, cb = b > kNegInf ? float_to_ordered(b) >> 16 : 0u;
    uint32_t code = 0;
#pragma unroll 1
    for (int at = 14; at >= 0; at -= 2) {
        int reached = 0;
#pragma unroll
        for (uint32_t i = 1; i < 4; ++i) {
            const uint32_t c = code | i << at;
            reached += __popc(__ballot_sync(0xFFFFFFFFu, ca >= c)) + __popc(__ballot_sync(0xFFFFFFFFu, cb >= c)) >= K;
        }
        code |= (uint32_t)reached << at;
    }
    return code ? ordered_to_float(code << 16) : kNegInf;      // (fewer than K buckets hold an entry: no bound)
}

// Beyond the list: the entries one after the other, each the best below the one before.
template <typename T, int NW>
__device__ __noinline__ void top_one_by_one(const void* row, int V, int K, TopSmem<NW>& sm) {
    float last_v = __builtin_huge_valf();
    int last_x = -1, found = 0;
    for (; found < K; ++found) {
        float v = kNegInf;
        int at = -1;
        for (int x = threadIdx.x; x < V; x += NW * 32) {
            const float u = entry<T>(row, x);
            if (u > v && (u < last_v || (u == last_v && x > last_x))) v = u, at = x;
        }
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) {
            const float ov = __shfl_xor_sync(0xFFFFFFFFu, v, o);
            const int ox = __shfl_xor_sync(0xFFFFFFFFu, at, o);
            if (ox >= 0 && (at < 0 || ov > v || (ov == v && ox < at))) v = ov, at = ox;
        }
        __syncthreads();
        if ((threadIdx.x & 31) == 0) sm.best_value[threadIdx.x >> 5] = v, sm.best_token[threadIdx.x >> 5] = at;
        __syncthreads();
        v = sm.best_value[0], at = sm.best_token[0];
        for (int j = 1; j < NW; ++j)
            if (sm.best_token[j] >= 0 && (at < 0 || sm.best_value[j] > v || (sm.best_value[j] == v && sm.best_token[j] < at))) v = sm.best_value[j], at = sm.best_token[j];
        if (at < 0) break;
        last_v = v, last_x = at;
        if (threadIdx.x == 0) sm.key[found] = key_of(v, at);
    }
    __syncthreads();
    if (threadIdx.x == 0) sm.count = found;
    __syncthreads();
}

// The entries of the block's tiles that reach its bound, in the first block's list.  even, odd: the lane's largest entries.
template <typename T, bool ALIGNED, int NW>
__device__ __forceinline__ void gather_top(const ScoreArgs& a, const tiles::View& view, int n_groups, int first_tile, int tile_step, float even, float odd, const float* group_max,
                                           TopSmem<NW>& sm, uint32_t blocks) {
    using P = tiles::Packed16<T>;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (NW > 1) sm.bucket[warp][lane] = even, sm.bucket[warp][lane + 32] = odd;
    __syncthreads();
    if (warp == 0) {
        for (int i = 1; i < NW; ++i) even = fmaxf(even, sm.bucket[i][lane]), odd = fmaxf(odd, sm.bucket[i][lane + 32]);
        const float b = bound_of_kth(even, odd, a.K);
        if (lane == 0) {
            sm.bound = b;
            if (blocks > 1) tiles::store_at(&sm.bounds[first_tile], 0, b);
        }
    }
    __syncthreads();
    const float bound = sm.bound;
    for (int i = tid; i < n_groups; i += NW * 32)
        if (group_max[i] >= bound && group_max[i] > kNegInf) {
            const int at = atomicAdd(&sm.groups, 1);
            if (at < kList) sm.group[at] = i;
        }
    __syncthreads();
    const int groups = sm.groups;
    if (groups > kList) {
        if (tid == 0) tiles::store_at(&sm.overflow, 0, 1);
        return;
    }
    for (int i = tid; i < groups * kWords; i += NW * 32) {
        // group i: lane i & 31 of the block's (i >> 5)-th tile
        const int g = sm.group[i / kWords], t = first_tile + (g >> 5) * tile_step, x0 = ((t * kWords + i % kWords) * 32 + (g & 31)) * P::kEntries;
        const uint4 w = tiles::load_word<T, ALIGNED>(view, x0, a.V);
        uint32_t reach = 0;
#pragma unroll
        for (int j = 0; j < P::kEntries; ++j) {
            const float v = P::get(w, j);
            if (v >= bound && v > kNegInf && v < __builtin_huge_valf()) reach |= 1u << j;
        }
        if (!reach) continue;
        int at = blocks > 1 ? tiles::add_at(&sm.count, 0, __popc(reach)) : atomicAdd(&sm.count, __popc(reach));
#pragma unroll
        for (int j = 0; j < P::kEntries; ++j)
            if (reach >> j & 1) {
                if (at < kList) {
                    if (blocks > 1) tiles::store_at(&sm.key[at], 0, key_of(P::get(w, j), x0 + j));
                    else sm.key[at] = key_of(P::get(w, j), x0 + j);
                }
                ++at;
            }
    }
}

// In the first block: what is left of the list at the largest of the blocks' bounds, in order of no kind, in place of the groups' list.
template <int NW>
__device__ __forceinline__ int keep_top(TopSmem<NW>& sm, uint32_t blocks) {
    if (blocks == 1) return sm.count;
    float bound = sm.bounds[0];
    for (uint32_t i = 1; i < blocks; ++i) bound = fmaxf(bound, sm.bounds[i]);
    for (int i = threadIdx.x; i < sm.count; i += NW * 32)
        if (value_of(sm.key[i]) >= bound) sm.group[atomicAdd(&sm.kept, 1)] = i;
    __syncthreads();
    return sm.kept;
}

// Row r of sequence b, and the token that the accepted path has there; false: the slot is empty.
__device__ __forceinline__ bool slot_of(const ScoreArgs& a, int64_t slot, int64_t b, int r, const char*& row, int elem, int32_t& path_token, int& status) {
    int64_t at = r;
    bool there = true;
    path_token = -1;
    if (a.accepted_len) {                          // (what the slot needs is read before it is known whether the path reaches it)
        const int L = a.R - 1, len = a.accepted_len[b], node = r > 0 ? a.accepted_node[b * L + r - 1] : 0;
        path_token = r < L ? a.accepted_token[b * L + r] : -1;
        const int last = a.last_token[b];
        if (r >= len) path_token = last;
        at = len >= 0 && len <= L && r <= len ? node : -1;
    } else if (a.row_index) {
        at = a.row_index[slot];
    }
    if (at < 0) there = false;
    else if (at >= a.num_rows) there = false, status |= RSD_ST_BAD_INDEX;
    row = (const char*)a.data + (b * a.seq_stride + (there ? at : 0) * a.row_stride) * elem;
    return there;
}

// Tiles of a row are dealt to the warps of its blocks in turn: tile t to warp t / blocks mod NW of block t mod blocks.
//
// 14,592 rows of 32,000 bf16 with 8 tokens and the entropy: 170 us = 5.5 TB/s back to back, where the chip draws 1000 W and the SMs go down to 1.6 GHz (142 us, the measured copy
// bandwidth, as long as it is below its power limit).  Issue slots 54 % busy, special-function unit 67 % (7560 warp instructions a row, 4650 of them
// the least that unpacking, bounding, scaling, exponentials and the two sums take).  Few rows are bound by what follows on each other: one row of 32,000 3.9 us, with five likeliest
// tokens 6.5; 2560 of them 39 and 49 us (floor 25), where the rows that start last have the chip to themselves.
template <typename T, bool ALIGNED, bool TOP, int NW>
__global__ void __launch_bounds__(NW * 32, 32 / NW) score_rows_kernel(const __grid_constant__ ScoreArgs a) {
    extern __shared__ float dynamic[];             // the tiles' sums, and [tiles of the block][32] largest entries where the likeliest tokens are asked for
    __shared__ RowTotals total_of_row;
    __shared__ int status_of_row;
    __shared__ typename std::conditional<TOP, TopSmem<NW>, int>::type top_store;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t rank = tiles::cluster_rank(), blocks = tiles::cluster_blocks();
    if (tid == 0) {
        status_of_row = 0;
        if constexpr (TOP) top_store.groups = top_store.count = top_store.kept = top_store.overflow = 0;
    }
    if (blocks > 1) tiles::cluster_arrive();       // (the row's other blocks have started, and their words above are set, behind the wait below)
    grid_wait();
    const uint32_t slot_word = blockIdx.x / blocks, sequence = slot_word / (uint32_t)a.R;
    const int64_t slot = slot_word, b = sequence;
    const int r = (int)(slot_word - sequence * (uint32_t)a.R);
    int status = 0;
    int32_t path_token;
    const char* row;
    const bool there = slot_of(a, slot, b, r, row, (int)sizeof(T), path_token, status);
    const tiles::View view = tiles::view_of<T>(row, a.V);
    const int all_tiles = tiles::tiles_of<T>(a.V, kWords), n_tiles = there ? all_tiles : 0;
    const Sums sums(dynamic, all_tiles);
    float* const group_max = dynamic + 3 * all_tiles;
    uint4 w[kWords];
    const int step = NW * (int)blocks;
    int t = warp * (int)blocks + (int)rank;
    load_half<T, ALIGNED>(w, view, t, 0, lane, there ? a.V : 0), load_half<T, ALIGNED>(w, view, t, kWords / 2, lane, there ? a.V : 0);
    int32_t token = path_token;
    if (rank == 0 && tid < a.T && !a.accepted_len) token = a.token[slot * a.T + tid];
    if (blocks > 1) tiles::cluster_wait();
    else __syncthreads();
    float even = kNegInf, odd = kNegInf;
    bool bad = false;
#pragma unroll 1
    for (int i = warp; t < n_tiles; i += NW, t += step) {   // i: the tile's place in the block
        float lane_max;
        tile_sums<T, true>(w, a.k, t, lane, blocks, sums, lane_max, bad, [&](int half) { load_half<T, ALIGNED>(w, view, t + step, half, lane, a.V); });
        if (TOP) {
            group_max[i * 32 + lane] = lane_max;
            if (i & 1) odd = fmaxf(odd, lane_max);
            else even = fmaxf(even, lane_max);
        }
    }
    float value = kNegInf;
    if (rank == 0 && tid < a.T) {
        if (token >= a.V) token = -1, status |= RSD_ST_BAD_INDEX;
        if (there && token >= 0) value = entry<T>(row, token);
    }
    if (bad) status |= RSD_ST_NAN_INPUT;
    if (status) tiles::or_at(&status_of_row, 0, status);
    if constexpr (TOP)
        gather_top<T, ALIGNED, NW>(a, view, there ? (n_tiles - (int)rank + (int)blocks - 1) / (int)blocks * 32 : 0, (int)rank, (int)blocks, even, odd, group_max, top_store, blocks);
    tiles::row_barrier(blocks);
    if (rank != 0) {
        grid_started();
        return;
    }
    if (warp == 0) {
        const RowTotals t = join<true>(sums, n_tiles, a.k, lane);
        if (lane == 0) total_of_row = t;
    }
    int kept = 0;
    if constexpr (TOP) {
        const bool beyond = top_store.overflow || top_store.count > kList;
        if (beyond) top_one_by_one<T, NW>(row, a.V, a.K, top_store);
        kept = keep_top<NW>(top_store, beyond ? 1 : blocks);
    }
    __syncthreads();
    const RowTotals total = total_of_row;
    const bool none = !there || total.m == kNegInf;
    const float lnz = none ? 0.0f : logf(total.s);
    auto logprob = [&](float v) { return v == kNegInf ? kNegInf : tiles::distance(v, total.m, a.inv_temp, -lnz); };
    if (tid < a.T) {
        if (a.out_logprob) a.out_logprob[slot * a.T + tid] = there && token >= 0 ? logprob(value) : 0.0f;
        if (a.out_token) a.out_token[slot] = there ? token : -1;
    }
    bool few = false;
    if constexpr (TOP) {
        const TopSmem<NW>& top = top_store;
        const bool in_place = blocks == 1 || top.overflow || top.kept == 0;
        const int n = there ? kept : 0;
        few = there && n < a.K;
        for (int i = tid; i < n; i += NW * 32) {
            const unsigned long long key = top.key[in_place ? i : top.group[i]];
            int place = 0;
#pragma unroll 4
            for (int j = 0; j < n; ++j) place += top.key[in_place ? j : top.group[j]] > key;
            if (place < a.K) {
                a.out_top_token[slot * a.K + place] = token_of(key);
                a.out_top_logprob[slot * a.K + place] = logprob(value_of(key));
            }
        }
        for (int i = n + tid; i < a.K; i += NW * 32) a.out_top_token[slot * a.K + i] = -1, a.out_top_logprob[slot * a.K + i] = kNegInf;
    }
    if (tid == 0) {
        if (a.out_entropy) a.out_entropy[slot] = none ? 0.0f : max_nan(lnz - 0.69314718f * __fdividef(total.w, total.s), 0.0f);
        a.status[slot] = status_of_row | (there && none ? RSD_ST_EMPTY_ROW : 0) | (few ? RSD_ST_FEWER_THAN_K : 0);
    }
    grid_started();
}

// d / dv_x of  sum_t g_t log p(token_t) + h H  =  ( sum_{t: token_t = x} g_t - p_x (G + h (log p_x + H)) ) / T,   G = sum_t g_t.
// A block has consecutive tiles of its row and keeps them in shared memory for the second sweep (read again from L2, the
// gradient's own words pushed two thirds of the rows out to memory); words of the gradient are written on their own 16-byte boundaries.
//
// 8192 rows of 32,000 bf16 with an entropy term: 221 us = 4.7 TB/s read and written back to back, 0.72 of the measured copy bandwidth (201 below the power limit).  Three rows an SM are what
// shared memory holds, 24 warps; two exponentials an entry keep the special-function unit 59 % busy, and the warps wait for each other at the two barriers (15 % of
// the stalls) and for the unit's queue.  Slower: blocks that stay for several rows and ask for the next one early (by 7 %: without arithmetic 180 us against 159), 4 warps a row (by 7 %).
// Rows that are not plain, or whose factors are not ordinary, are written entry by entry in 64 bits (4096 rows 343 us, the others 105).
struct Slope {                     // gradient of an entry without a token: p (c0 + c1 log2 p),   log2 p = (v - m) k - c, m = 0 in a plain row
    float m, c, c0, c1, inv_temp;
    double wide_c0, wide_c1;       // the factors of rows that are not plain, or where products in fp32 might leave its range
    int plain, none;
};
__device__ __forceinline__ Slope slope_of(const RowTotals& total, float G, float h, float inv_temp, float k) {
    Slope f;
    f.inv_temp = inv_temp;
    f.none = total.m == kNegInf;
    const bool plain = f.none || tiles::plain_tile(total.m, k);
    f.m = plain ? 0.0f : total.m;
    const float log2s = f.none ? 0.0f : log2f(total.s), H = f.none ? 0.0f : 0.69314718f * (log2s - __fdividef(total.w, total.s));
    // what c loses when it is rounded goes into the factors
    f.c = plain && !f.none ? fmaf(total.m, k, log2s) : log2s;
    const float off = plain && !f.none ? -(fmaf(total.m, k, -f.c) + log2s) : 0.0f, scale = ex2_approx(off);
    f.c1 = f.none ? 0.0f : -h * 0.69314718f * inv_temp;
    f.c0 = f.none ? 0.0f : fmaf(f.c1, off, -(G + h * H) * inv_temp) * scale;
    f.c1 *= scale;
    f.plain = plain && tiles::ordinary_factor(f.c0) && tiles::ordinary_factor(f.c1);
    if (!f.plain) {
        const double c1 = -(double)h * 0.693147180559945309 * (double)inv_temp;
        f.wide_c0 = (c1 * (double)off - ((double)G + (double)h * (double)H) * (double)inv_temp) * (double)scale;
        f.wide_c1 = c1 * (double)scale;
    }
    return f;
}
// The gradient of an entry in 64 bits, and of a row's entries from..to - 1: a weight of 0 makes every finite factor 0, and factors that are not finite reach every entry.
template <bool ENTROPY>
__device__ __forceinline__ double wide_slope(float v, float k, const Slope& f) {
    float x = tiles::distance(v, f.m, k, -f.c);
    if (ENTROPY) x = fmaxf(x, tiles::kNoWeight);
    const double p = (double)ex2_approx(x);
    return p * (ENTROPY ? fma((double)x, f.wide_c1, f.wide_c0) : f.wide_c0);
}
template <typename T, bool ENTROPY>
__device__ __noinline__ void write_wide(const void* row, void* grad, int from, int to, float k, const Slope& f) {
    for (int x = from + (int)threadIdx.x; x < to; x += (int)blockDim.x) tiles::Packed16<T>::store(grad, x, (float)wide_slope<ENTROPY>(entry<T>(row, x), k, f));
}

template <typename T, bool ALIGNED, bool ENTROPY, int NW>
__global__ void __launch_bounds__(NW * 32, 24 / NW) score_grad_kernel(const __grid_constant__ ScoreArgs a) {
    using P = tiles::Packed16<T>;
    constexpr int E = P::kEntries, kTile = tiles::tile_entries<T>(kWords), kHeld = tiles::kHeldTile<kWords>;
    extern __shared__ __align__(16) unsigned char dynamic_bytes[];   // the block's tiles, then all tiles' sums
    __shared__ Slope slope_of_row;
    __shared__ int status_of_row;
    __shared__ int32_t tokens[RSD_MAX_K];          // absent: -1
    __shared__ float weights[RSD_MAX_K];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t rank = tiles::cluster_rank(), blocks = tiles::cluster_blocks();
    if (tid == 0) status_of_row = 0;
    if (blocks > 1) tiles::cluster_arrive();
    else __syncthreads();
    grid_wait();
    const uint32_t slot = blockIdx.x / blocks, sequence = slot / (uint32_t)a.R;
    const char* row = (const char*)a.data + (sequence * a.seq_stride + (slot - sequence * (uint32_t)a.R) * a.row_stride) * (int64_t)sizeof(T);
    const tiles::View view = tiles::view_of<T>(row, a.V);
    const int n_tiles = tiles::tiles_of<T>(a.V, kWords), each = (n_tiles + (int)blocks - 1) / (int)blocks;   // tiles of a block
    const int t0 = min((int)rank * each, n_tiles), t1 = min(t0 + each, n_tiles);
    const uint32_t held = smem_u32(dynamic_bytes);
    const Sums sums((float*)(dynamic_bytes + each * kHeld), n_tiles);
    for (int t = t0 + warp; t < t1; t += NW) {
        tiles::fetch_tile<ALIGNED, kWords>(held + (t - t0) * kHeld, view, t, lane);
        tiles::copies_sent();
    }
    int32_t token = -1;                            // lane t of the first warp has token t
    float weight = 0.0f, h = 0.0f;
    if (tid < a.T) token = a.token[(int64_t)slot * a.T + tid], weight = a.g_logprob[(int64_t)slot * a.T + tid];
    if (ENTROPY && warp == 0) h = a.g_entropy[slot];
    if (blocks > 1) tiles::cluster_wait();
    bool bad = false;
#pragma unroll 1
    for (int t = t0 + warp; t < t1; t += NW) {
        uint4 w[kWords];
        tiles::copies_landed((t1 - 1 - t) / NW);
        __syncwarp();
        tiles::read_tile<T, ALIGNED, kWords>(w, held + (t - t0) * kHeld, view, t, lane, a.V);
        float lane_max;
        tile_sums<T, ENTROPY>(w, a.k, t, lane, blocks, sums, lane_max, bad, [](int) {});
    }
    int status = bad ? RSD_ST_NAN_INPUT : 0;
    if (token >= a.V) token = -1, status |= RSD_ST_BAD_INDEX;
    if (token < 0) weight = 0.0f;
    if (tid < a.T) tokens[tid] = token, weights[tid] = weight;
    if (status)
        for (uint32_t i = 0; i < blocks; ++i) tiles::or_at(&status_of_row, i, status);
    float G = weight;
    if (warp == 0) {
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) G += __shfl_xor_sync(0xFFFFFFFFu, G, o);
    }
    tiles::row_barrier(blocks);
    if (warp == 0) {
        const Slope f = slope_of(join<ENTROPY>(sums, n_tiles, a.k, lane), G, h, a.inv_temp, a.k);
        if (lane == 0) {
            slope_of_row = f;
            if (rank == 0) a.status[slot] = status_of_row | (f.none ? RSD_ST_EMPTY_ROW : 0);
        }
    }
    __syncthreads();
    const Slope f = slope_of_row;
    bad = status_of_row & RSD_ST_NAN_INPUT;
    char* const grad = (char*)a.grad + (int64_t)slot * a.V * (int64_t)sizeof(T);
    if (!f.plain) {
        const int from = t0 * kTile, to = min(t1 * kTile, a.V);
        write_wide<T, ENTROPY>(row, grad, from, to, a.k, slope_of_row);
        __syncthreads();
        const int32_t mine = warp == 0 && lane < a.T ? tokens[lane] : -1;
        if (mine >= from && mine < to) {           // (as below)
            double own = wide_slope<ENTROPY>(entry<T>(row, mine), a.k, f);
            bool first = true;
            for (int i = 0; i < a.T; ++i)
                if (tokens[i] == mine) own = fma((double)weights[i], (double)f.inv_temp, own), first = first && i >= lane;
            if (first) P::store(grad, mine, (float)own);
        }
        grid_started();
        return;
    }
    const unsigned long long kk = tiles::both(a.k), minus_c = tiles::both(-f.c), c0 = tiles::both(f.c0), c1 = tiles::both(f.c1);
    auto slope = [&](unsigned long long v) {
        float x, y;
        const unsigned long long l = fma_f32x2(v, kk, minus_c);
        split_f32x2(l, x, y);
        if (ENTROPY) x = fmaxf(x, tiles::kNoWeight), y = fmaxf(y, tiles::kNoWeight);
        const unsigned long long p = f32x2(ex2_approx(x), ex2_approx(y));
        return tiles::mul_f32x2(p, ENTROPY ? fma_f32x2(f32x2(x, y), c1, c0) : c0);
    };
    const int head = ALIGNED ? 0 : (int)((uintptr_t)grad & 15u) / (int)sizeof(T);   // entries between the boundary and the gradient's first one
    auto word = [&](const uint4& v) {
        return P::make([&](int i) { return slope(P::pair(v, i)); });
    };
    const int last = t1 == n_tiles ? tiles::tiles_of<T>(head + a.V, kWords) : t1;   // tiles of the gradient: `head` entries ahead of the row's
#pragma unroll 1
    for (int t = t0 + warp; t < last && t0 < t1; t += NW) {
        const int x = t * kTile - head + lane * E;
        char* const to = grad + (int64_t)x * (int)sizeof(T);
        const bool whole = t * kTile >= head && (t + 1) * kTile - head <= a.V;
        uint4 w[kWords];
        tiles::held_words<T, ALIGNED, kWords>(w, held, view, t0, t1, x, a.V);
        if (bad) {
            bool ignored = false;
#pragma unroll
            for (int k = 0; k < kWords; ++k) P::clean(w[k], ignored);
        }
        if (whole) {
#pragma unroll
            for (int k = 0; k < kWords; ++k) __stcs((uint4*)(to + k * 512), word(w[k]));
        } else {
#pragma unroll
            for (int k = 0; k < kWords; ++k) {
                const int at = x + k * 32 * E;
                if (at >= 0 && at + E <= a.V) {
                    __stcs((uint4*)(to + k * 512), word(w[k]));
                } else if (at + E > 0 && at < a.V) {
                    const uint4 g = word(w[k]);
                    for (int i = 0; i < E; ++i)
                        if (at + i >= 0 && at + i < a.V) P::store(grad, at + i, P::get(g, i));
                }
            }
        }
        __syncwarp();
        // The entries of the tokens in this tile again, with their weights: a token given twice has both, and its first lane stores it.
        const int32_t mine = lane < a.T ? tokens[lane] : -1;
        if (mine >= 0 && (mine + head) / kTile == t) {
            float own = 0.0f;
            bool first = true;
            for (int i = 0; i < a.T; ++i)
                if (tokens[i] == mine) own += weights[i], first = first && i >= lane;
            if (first) {
                const int at = view.first + mine * (int)sizeof(T) - t0 * kWords * 512, tile = min(at / (kWords * 512), t1 - t0 - 1);
                const float v = at >= 0 ? entry<T>(dynamic_bytes + at + tile * 16, 0) : entry<T>(view.base + view.first, mine);
                float rest, ignored;
                split_f32x2(slope(tiles::both(v)), rest, ignored);
                P::store(grad, mine, f.none ? 0.0f : fmaf(own, f.inv_temp, rest));
            }
        }
    }
    grid_started();
}

}  // namespace score
}  // namespace rsd
