// Log-probabilities of given tokens, entropy and the likeliest tokens of rows (score_rows_kernel), and the gradient of weighted
// log-probabilities and entropies (score_grad_kernel).
//
// With z = v / T, m = max z, y = (v - max v) log2(e) / T:   Z = sum 2^y,   log p_x = z_x - m - ln Z,   H = ln Z - ln 2 (sum 2^y y) / Z.
// Both terms of H are positive: nothing cancels.  One pass over the row, one exponential per entry.
#pragma once
#include "../../include/rsd.h"
#include "rsd_score_args.h"
#include "rsd_tiles.cuh"

namespace rsd {

namespace score {

constexpr int kThreads = 256, kWarps = kThreads / 32, kWords = 8;
constexpr int kMaxTiles = RSD_MAX_VOCAB / tiles::tile_entries<float>(kWords);
constexpr int kBuckets = 64;       // samples that bound the K-th largest entry; at least RSD_MAX_K
constexpr int kList = 512;         // groups opened, and entries taken from them
static_assert(kBuckets >= RSD_MAX_K && kThreads % kBuckets == 0, "");

struct Sums {                      // of a row's tiles, relative to each tile's largest entry
    float m[kMaxTiles], s[kMaxTiles], w[kMaxTiles];
};
struct RowTotals {
    float m, s, w;                 // largest entry; sum of 2^y, of 2^y y
};

// Sum of 2^y and of 2^y y over a tile, y = (v - m) k; the largest entry in m (-inf: no entry at all).
template <typename T, bool ENTROPY>
__device__ __forceinline__ void tile_sums(uint4 (&w)[kWords], float k, int t, int lane, Sums& sums, float& lane_max, bool& bad) {
    using P = tiles::Packed16<T>;
    float mx, mn;
    P::bounds(w, mx, mn);
    float m = tiles::warp_max_nan(mx);
    if (!(m < __builtin_huge_valf())) {   // NaN or +inf somewhere in the tile
#pragma unroll
        for (int i = 0; i < kWords; ++i) P::clean(w[i], bad);
        P::bounds(w, mx, mn);
        m = tiles::warp_max_nan(mx);
    }
    lane_max = mx;
    unsigned long long s = tiles::both(0.0f), e = s;
    if (m > kNegInf) {
        const unsigned long long minus_m = tiles::both(-m), kk = tiles::both(k);
        const bool plain = (mn - m) * k > tiles::kFarBelow;
        if (__all_sync(0xFFFFFFFFu, plain) || !ENTROPY) {
#pragma unroll
            for (int i = 0; i < kWords; ++i)
                P::pairs(w[i], [&](unsigned long long v) {
                    const unsigned long long y = tiles::mul_f32x2(add_f32x2(v, minus_m), kk);
                    float a, b;
                    split_f32x2(y, a, b);
                    const unsigned long long x = f32x2(ex2_approx(a), ex2_approx(b));
                    s = add_f32x2(s, x);
                    if (ENTROPY) e = fma_f32x2(x, y, e);
                });
        } else {
#pragma unroll
            for (int i = 0; i < kWords; ++i)
                P::pairs(w[i], [&](unsigned long long v) {
                    float a, b;
                    split_f32x2(tiles::mul_f32x2(add_f32x2(v, minus_m), kk), a, b);
                    a = fmaxf(a, tiles::kFarBelow), b = fmaxf(b, tiles::kFarBelow);
                    const unsigned long long x = f32x2(ex2_approx(a), ex2_approx(b));
                    s = add_f32x2(s, x);
                    e = fma_f32x2(x, f32x2(a, b), e);
                });
        }
    }
    float s0, s1, e0, e1;
    split_f32x2(s, s0, s1);
    split_f32x2(e, e0, e1);
    const float sum = tiles::warp_sum_two(s0 + s1, e0 + e1, lane);
    if (lane == 0) sums.m[t] = m, sums.s[t] = sum;
    if (lane == 16) sums.w[t] = sum;
}

// The tiles' sums joined by one warp; every lane gets the result.
__device__ __forceinline__ RowTotals join(const Sums& sums, int n, float k, int lane) {
    float m = kNegInf;
    for (int t = lane; t < n; t += 32) m = fmaxf(m, sums.m[t]);
    m = warp_max(m);
    float s = 0.0f, w = 0.0f;
    for (int t = lane; t < n; t += 32) {
        if (sums.m[t] == kNegInf) continue;
        const float d = fmaxf((sums.m[t] - m) * k, tiles::kFarBelow), f = ex2_approx(d);
        s = fmaf(f, sums.s[t], s);
        w = fmaf(f, fmaf(d, sums.s[t], sums.w[t]), w);
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
// Every lane knows its largest entry of each tile (a group of up to 64 entries).  The threads' largest entries, taken together into
// kBuckets buckets, are distinct entries: the K-th largest of them is at most the K-th largest entry.  Only groups that reach it are read again (they lie in
// L2), a word a thread, and only entries that reach it are ranked: about 1.4 K of them.
struct TopSmem {
    float bucket[kThreads];
    float value[kList];
    int32_t token[kList];
    int32_t group[kList];
    int groups, count;
    float bound;
};

// K-th largest of 64 values, two per lane, from below: exact in its upper 16 bits.
__device__ __forceinline__ float bound_of_kth(float a, float b, int K) {
    const uint32_t ca = a > kNegInf ? float_to_ordered(a) >> 16 : 0u, cb = b > kNegInf ? float_to_ordered(b) >> 16 : 0u;
    uint32_t code = 0;
#pragma unroll 1
    for (uint32_t bit = 0x8000u; bit; bit >>= 1) {
        const uint32_t c = code | bit;
        if (__popc(__ballot_sync(0xFFFFFFFFu, ca >= c)) + __popc(__ballot_sync(0xFFFFFFFFu, cb >= c)) >= K) code = c;
    }
    return code ? ordered_to_float(code << 16) : kNegInf;      // (fewer than K buckets hold an entry: no bound)
}

// Beyond the list: the entries one after the other, each the best below the one before.
template <typename T>
__device__ void top_one_by_one(const void* row, int V, int K, TopSmem& sm, float* value, int32_t* token) {
    __shared__ float best_v[kWarps];
    __shared__ int best_x[kWarps];
    float last_v = __builtin_huge_valf();
    int last_x = -1;
    for (int i = 0; i < K; ++i) {
        float v = kNegInf;
        int at = -1;
        for (int x = threadIdx.x; x < V; x += kThreads) {
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
        if ((threadIdx.x & 31) == 0) best_v[threadIdx.x >> 5] = v, best_x[threadIdx.x >> 5] = at;
        __syncthreads();
        v = best_v[0], at = best_x[0];
        for (int j = 1; j < kWarps; ++j)
            if (best_x[j] >= 0 && (at < 0 || best_v[j] > v || (best_v[j] == v && best_x[j] < at))) v = best_v[j], at = best_x[j];
        if (at < 0) break;
        last_v = v, last_x = at;
        if (threadIdx.x == 0) value[i] = v, token[i] = at, sm.count = i + 1;
    }
    __syncthreads();
}

template <typename T, bool ALIGNED>
__device__ void top_entries(const ScoreArgs& a, const void* row, const tiles::View& view, int n_tiles, float thread_max, const float* group_max, TopSmem& sm) {
    using P = tiles::Packed16<T>;
    const int tid = threadIdx.x;
    sm.bucket[tid] = thread_max;
    if (tid == 0) sm.groups = 0, sm.count = 0;
    __syncthreads();
    if (tid < 32) {
        float u = kNegInf, v = kNegInf;
#pragma unroll
        for (int i = 0; i < kThreads; i += kBuckets) u = fmaxf(u, sm.bucket[i + tid]), v = fmaxf(v, sm.bucket[i + 32 + tid]);
        const float b = bound_of_kth(u, v, a.K);
        if (tid == 0) sm.bound = b;
    }
    __syncthreads();
    const float bound = sm.bound;
    for (int i = tid; i < n_tiles * 32; i += kThreads)
        if (group_max[i] >= bound && group_max[i] > kNegInf) {
            const int at = atomicAdd(&sm.groups, 1);
            if (at < kList) sm.group[at] = i;
        }
    __syncthreads();
    const int groups = sm.groups;
    if (groups <= kList) {
        for (int i = tid; i < groups * kWords; i += kThreads) {
            const int g = sm.group[i / kWords], x0 = (((g >> 5) * kWords + i % kWords) * 32 + (g & 31)) * P::kEntries;
            const uint4 w = tiles::load_word<T, ALIGNED>(view, x0, a.V);
#pragma unroll
            for (int j = 0; j < P::kEntries; ++j) {
                const float v = P::get(w, j);
                if (v >= bound && v > kNegInf && v < __builtin_huge_valf()) {
                    const int at = atomicAdd(&sm.count, 1);
                    if (at < kList) sm.value[at] = v, sm.token[at] = x0 + j;
                }
            }
        }
    }
    __syncthreads();
    if (groups > kList || sm.count > kList) top_one_by_one<T>(row, a.V, a.K, sm, sm.value, sm.token);
}

struct Smem {
    Sums sums;
    RowTotals total;
    int status;
};

// Row r of sequence b, and the token that the accepted path has there; false: the slot is empty.
__device__ __forceinline__ bool slot_of(const ScoreArgs& a, int64_t slot, int64_t b, int r, const char*& row, int elem, int32_t& path_token, int& status) {
    int64_t at = r;
    bool there = true;
    path_token = -1;
    if (a.accepted_len) {
        const int len = a.accepted_len[b], L = a.R - 1;
        if (len < 0 || len > L || r > len) return false;
        if (r > 0) at = a.accepted_node[b * L + r - 1];
        path_token = r < len ? a.accepted_token[b * L + r] : a.last_token[b];
    } else if (a.row_index) {
        at = a.row_index[slot];
    }
    if (at < 0) there = false;
    else if (at >= a.num_rows) there = false, status |= RSD_ST_BAD_INDEX;
    row = (const char*)a.data + (b * a.seq_stride + (there ? at : 0) * a.row_stride) * elem;
    return there;
}

template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(kThreads) score_rows_kernel(const __grid_constant__ ScoreArgs a) {
    extern __shared__ float group_max[];           // [tiles][32] where the largest entries are asked for
    __shared__ Smem sm;
    __shared__ TopSmem top;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (a.own_status) grid_wait();                 // (otherwise the kernel ahead is the one that clears the status: waited for below)
    const int64_t slot = blockIdx.x, b = slot / a.R;
    const int r = (int)(slot - b * a.R);
    int status = 0;
    int32_t path_token;
    const char* row;
    const bool there = slot_of(a, slot, b, r, row, (int)sizeof(T), path_token, status);
    int32_t token = -1;
    float value = kNegInf;
    if (tid < a.T) {
        token = a.accepted_len ? path_token : a.token ? a.token[slot * a.T + tid] : -1;
        if (token >= a.V) token = -1, status |= RSD_ST_BAD_INDEX;
        if (there && token >= 0) value = entry<T>(row, token);
    }
    const tiles::View view = tiles::view_of<T>(row, a.V);
    const int n_tiles = there ? tiles::tiles_of<T>(a.V, kWords) : 0;
    if (tid == 0) sm.status = 0;
    float thread_max = kNegInf;
    bool bad = false;
    for (int t = warp; t < n_tiles; t += kWarps) {
        uint4 w[kWords];
        tiles::load_tile<T, ALIGNED, kWords>(w, view, t, lane, a.V);
        float lane_max;
        tile_sums<T, true>(w, a.k, t, lane, sm.sums, lane_max, bad);
        thread_max = fmaxf(thread_max, lane_max);
        if (a.K) group_max[t * 32 + lane] = lane_max;
    }
    __syncthreads();
    if (bad) status |= RSD_ST_NAN_INPUT;
    if (warp == 0) {
        const RowTotals t = join(sm.sums, n_tiles, a.k, lane);
        if (lane == 0) sm.total = t;
    }
    if (there && a.K) top_entries<T, ALIGNED>(a, row, view, n_tiles, thread_max, group_max, top);
    else __syncthreads();
    const RowTotals total = sm.total;
    const bool none = !there || total.m == kNegInf;
    const float lnz = none ? 0.0f : logf(total.s);
    if (there && none) status |= RSD_ST_EMPTY_ROW;
    auto logprob = [&](float v) { return v == kNegInf ? kNegInf : (v - total.m) / a.temp - lnz; };
    if (tid < a.T) {
        if (a.out_logprob) a.out_logprob[slot * a.T + tid] = there && token >= 0 ? logprob(value) : 0.0f;
        if (a.out_token) a.out_token[slot] = there ? token : -1;
    }
    if (tid == 0 && a.out_entropy) a.out_entropy[slot] = none ? 0.0f : fmaxf(lnz - 0.69314718f * (total.w / total.s), 0.0f);
    if (a.K) {
        const int n = there ? min(top.count, kList) : 0;
        for (int i = tid; i < n; i += kThreads) {
            const float v = top.value[i];
            const int x = top.token[i];
            int rank = 0;
            for (int j = 0; j < n; ++j) rank += top.value[j] > v || (top.value[j] == v && top.token[j] < x);
            if (rank < a.K) {
                a.out_top_token[slot * a.K + rank] = x;
                a.out_top_logprob[slot * a.K + rank] = logprob(v);
            }
        }
        if (there && n < a.K) status |= RSD_ST_FEWER_THAN_K;
        for (int i = n + tid; i < a.K; i += kThreads) a.out_top_token[slot * a.K + i] = -1, a.out_top_logprob[slot * a.K + i] = kNegInf;
    }
    if (status) atomicOr(&sm.status, status);
    __syncthreads();
    grid_started();
    if (!a.own_status) grid_wait();
    if (tid == 0) {
        if (a.own_status) a.status[b] = sm.status;
        else if (sm.status) atomicOr(&a.status[b], sm.status);
    }
}

// d / dv_x of  sum_t g_t log p(token_t) + h H  =  ( sum_{t: token_t = x} g_t - p_x (G + h (log p_x + H)) ) / T,   G = sum_t g_t.
// The row is read twice, the second time from L2; words of the gradient are written on their own 16-byte boundaries.
template <typename T, bool ALIGNED, bool ENTROPY>
__global__ void __launch_bounds__(kThreads) score_grad_kernel(const __grid_constant__ ScoreArgs a) {
    using P = tiles::Packed16<T>;
    constexpr int E = P::kEntries;
    __shared__ Smem sm;
    __shared__ int32_t tokens[RSD_MAX_K];
    __shared__ float weights[RSD_MAX_K];
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (a.own_status) grid_wait();
    const int64_t slot = blockIdx.x, b = slot / a.R;
    const int r = (int)(slot - b * a.R);
    const char* row = (const char*)a.data + (b * a.seq_stride + r * a.row_stride) * (int64_t)sizeof(T);
    char* grad = (char*)a.grad + slot * a.V * (int64_t)sizeof(T);
    int status = 0;
    if (tid < a.T) {
        int32_t token = a.token[slot * a.T + tid];
        if (token >= a.V) token = -1, status |= RSD_ST_BAD_INDEX;
        tokens[tid] = token;
        weights[tid] = token >= 0 ? a.g_logprob[slot * a.T + tid] : 0.0f;
    }
    const float h = ENTROPY ? a.g_entropy[slot] : 0.0f;
    const tiles::View view = tiles::view_of<T>(row, a.V);
    const int n_tiles = tiles::tiles_of<T>(a.V, kWords);
    if (tid == 0) sm.status = 0;
    bool bad = false;
    for (int t = warp; t < n_tiles; t += kWarps) {
        uint4 w[kWords];
        tiles::load_tile<T, ALIGNED, kWords>(w, view, t, lane, a.V);
        float lane_max;
        tile_sums<T, ENTROPY>(w, a.k, t, lane, sm.sums, lane_max, bad);
    }
    if (__syncthreads_or(bad)) bad = true;
    if (bad) status |= RSD_ST_NAN_INPUT;
    if (warp == 0) {
        const RowTotals t = join(sm.sums, n_tiles, a.k, lane);
        if (lane == 0) sm.total = t;
    }
    __syncthreads();
    const RowTotals total = sm.total;
    const bool none = total.m == kNegInf;
    if (none) status |= RSD_ST_EMPTY_ROW;
    float G = 0.0f;
    for (int t = 0; t < a.T; ++t) G += weights[t];
    const float log2z = none ? 0.0f : log2f(total.s), inv_temp = fminf(1.0f / a.temp, 3.0e38f);
    // gradient of an entry without a token: p (c0 + c1 log2 p)
    const float H = ENTROPY && !none ? 0.69314718f * (log2z - total.w / total.s) : 0.0f;
    const float c0 = none ? 0.0f : -(G + h * H) * inv_temp, c1 = none ? 0.0f : -h * 0.69314718f * inv_temp;
    const unsigned long long minus_m = tiles::both(none ? 0.0f : -total.m), kk = tiles::both(a.k), minus_l = tiles::both(-log2z), cc0 = tiles::both(c0), cc1 = tiles::both(c1);
    auto slope = [&](unsigned long long v) {
        float x, y;
        split_f32x2(fma_f32x2(add_f32x2(v, minus_m), kk, minus_l), x, y);
        if (ENTROPY) x = fmaxf(x, tiles::kFarBelow), y = fmaxf(y, tiles::kFarBelow);
        const unsigned long long p = f32x2(ex2_approx(x), ex2_approx(y));
        return tiles::mul_f32x2(p, ENTROPY ? fma_f32x2(f32x2(x, y), cc1, cc0) : cc0);
    };
    const int head = (int)((uintptr_t)grad & 15u) / (int)sizeof(T);   // entries between the boundary and the gradient's first one
    const int words = (head + a.V + E - 1) / E;
    for (int j = tid; j < words; j += kThreads) {
        const int x0 = j * E - head;
        uint4 w = tiles::load_word<T, ALIGNED>(view, x0, a.V);
        if (bad) {
            bool ignored = false;
            P::clean(w, ignored);
        }
        const uint4 g = P::make([&](int i) { return slope(P::pair(w, i)); });
        if (x0 >= 0 && x0 + E <= a.V) {
            *(uint4*)(grad + (int64_t)x0 * (int)sizeof(T)) = g;
        } else {
            for (int i = 0; i < E; ++i)
                if (x0 + i >= 0 && x0 + i < a.V) P::store(grad, x0 + i, P::get(g, i));
        }
    }
    __syncthreads();
    if (tid < a.T && tokens[tid] >= 0) {       // the tokens' entries again, with their own weights; a token given twice has both
        const int32_t x = tokens[tid];
        float own = 0.0f;
        bool first = true;
        for (int t = 0; t < a.T; ++t)
            if (tokens[t] == x) own += weights[t], first = first && t >= tid;
        if (first) {
            const float v = entry<T>(row, x);
            float rest, ignored;
            split_f32x2(slope(tiles::both(v)), rest, ignored);
            P::store(grad, x, none ? 0.0f : fmaf(own, inv_temp, rest));
        }
    }
    if (status) atomicOr(&sm.status, status);
    __syncthreads();
    grid_started();
    if (!a.own_status) grid_wait();
    if (tid == 0) {
        if (a.own_status) a.status[b] = sm.status;
        else if (sm.status) atomicOr(&a.status[b], sm.status);
    }
}

}  // namespace score
}  // namespace rsd
