// How far draft rows are from target rows (divergence_kernel), and the gradient of that with respect to the draft rows
// (divergence_grad_kernel).
//
// With a = (v_t - max v_t) log2(e) / T_t for the target row and b alike for the draft row, q = 2^a / S_q, p = 2^b / S_p:
//   KL(q||p) = ln 2 [ (sum 2^a (a - b)) / S_q - log2 S_q + log2 S_p ]       KL(p||q) = ln 2 [ (sum 2^b (b - a)) / S_p - log2 S_p + log2 S_q ]
// so both come from one pass with one exponential per entry and row; what cancels is of the size of 1, not of the size of a logit.
// The overlap sum min(p, q) needs the normalisers first: a second pass (from L2) with one exponential per pair, 2^min(log2 p, log2 q).
#pragma once
#include "../../include/rsd.h"
#include "rsd_score_args.h"
#include "rsd_tiles.cuh"

namespace rsd {

namespace divergence {

constexpr int kThreads = 256, kWarps = kThreads / 32, kWords = 4;
constexpr int kMaxTiles = RSD_MAX_VOCAB / tiles::tile_entries<float>(kWords);

struct Sums {   // of the rows' tiles, relative to each tile's largest entries
    float mq[kMaxTiles], mp[kMaxTiles], sq[kMaxTiles], sp[kMaxTiles], dq[kMaxTiles], dp[kMaxTiles];
    // overlap of a tile takes the place of mq
};
struct Totals {
    float mq, mp, sq, sp, dq, dp;   // largest entries, sums of weights, of weight times a - b (q), b - a (p)
};
struct Smem {
    Sums sums;
    Totals total;
    float alone_q[kWarps], alone_p[kWarps];   // largest target entry whose token the draft lacks, and the other way round
    int status;
};

template <typename T>
__device__ __forceinline__ float largest(uint4 (&w)[kWords], float& mn, bool& bad) {   // over the tile; NaN and +inf are no entries
    using P = tiles::Packed16<T>;
    float mx;
    P::bounds(w, mx, mn);
    float m = tiles::warp_max_nan(mx);
    if (!(m < __builtin_huge_valf())) {
#pragma unroll
        for (int i = 0; i < kWords; ++i) P::clean(w[i], bad);
        P::bounds(w, mx, mn);
        m = tiles::warp_max_nan(mx);
    }
    return m;
}

template <typename T, bool BOTH>   // BOTH: the sums of weight times difference too
__device__ __forceinline__ void tile_sums(uint4 (&p)[kWords], uint4 (&q)[kWords], float kp, float kq, int t, int lane, Sums& sums, float& alone_q, float& alone_p, bool& bad) {
    using P = tiles::Packed16<T>;
    float np, nq;
    const float mp = largest<T>(p, np, bad), mq = largest<T>(q, nq, bad);
    const float zp = mp > kNegInf ? mp : 0.0f, zq = mq > kNegInf ? mq : 0.0f;
    const unsigned long long minus_p = tiles::both(-zp), minus_q = tiles::both(-zq), kkp = tiles::both(kp), kkq = tiles::both(kq), minus_one = tiles::both(-1.0f);
    unsigned long long sp = tiles::both(0.0f), sq = sp, dp = sp, dq = sp;
    const bool plain = (np - zp) * kp > tiles::kFarBelow && (nq - zq) * kq > tiles::kFarBelow;
    if (__all_sync(0xFFFFFFFFu, plain)) {
#pragma unroll
        for (int i = 0; i < kWords; ++i)
#pragma unroll
            for (int j = 0; j < P::kEntries / 2; ++j) {
                const unsigned long long b = tiles::mul_f32x2(add_f32x2(P::pair(p[i], j), minus_p), kkp), a = tiles::mul_f32x2(add_f32x2(P::pair(q[i], j), minus_q), kkq);
                float x, y;
                split_f32x2(b, x, y);
                const unsigned long long wp = f32x2(ex2_approx(x), ex2_approx(y));
                split_f32x2(a, x, y);
                const unsigned long long wq = f32x2(ex2_approx(x), ex2_approx(y));
                sp = add_f32x2(sp, wp), sq = add_f32x2(sq, wq);
                if (BOTH) {
                    const unsigned long long d = fma_f32x2(b, minus_one, a);
                    dq = fma_f32x2(wq, d, dq);
                    dp = fma_f32x2(wp, d, dp);                     // (its sign is turned below)
                }
            }
    } else {
#pragma unroll 1
        for (int i = 0; i < kWords; ++i) {
            const uint4 pw = i == 0 ? p[0] : i == 1 ? p[1] : i == 2 ? p[2] : p[3], qw = i == 0 ? q[0] : i == 1 ? q[1] : i == 2 ? q[2] : q[3];
#pragma unroll
            for (int j = 0; j < P::kEntries; ++j) {
                const float vp = P::get(pw, j), vq = P::get(qw, j), b = (vp - zp) * kp, a = (vq - zq) * kq;
                const bool in_p = b > kNegInf, in_q = a > kNegInf;
                const float wp = ex2_approx(b), wq = ex2_approx(a), d = in_p && in_q ? a - b : 0.0f;
                if (in_q && !in_p) alone_q = fmaxf(alone_q, vq);
                if (in_p && !in_q) alone_p = fmaxf(alone_p, vp);
                sp = add_f32x2(sp, f32x2(wp, 0.0f)), sq = add_f32x2(sq, f32x2(wq, 0.0f));
                dq = fma_f32x2(f32x2(wq, 0.0f), tiles::both(d), dq), dp = fma_f32x2(f32x2(wp, 0.0f), tiles::both(d), dp);
            }
        }
    }
    float x, y;
    split_f32x2(sp, x, y);
    const float s_p = x + y;
    split_f32x2(sq, x, y);
    const float s_q = x + y;
    split_f32x2(dp, x, y);
    const float d_p = -(x + y);
    split_f32x2(dq, x, y);
    const float d_q = x + y;
    const float sum = tiles::warp_sum_four(s_p, s_q, d_p, d_q, lane);
    if (lane == 0) sums.mp[t] = mp, sums.mq[t] = mq, sums.sp[t] = sum;
    if (lane == 8) sums.sq[t] = sum;
    if (lane == 16) sums.dp[t] = sum;
    if (lane == 24) sums.dq[t] = sum;
}

// The tiles' sums joined by one warp; every lane gets the result.  A tile without an entry in one of the rows has its largest entry counted as 0 there.
__device__ __forceinline__ Totals join(const Sums& sums, int n, float kp, float kq, int lane) {
    float mp = kNegInf, mq = kNegInf;
    for (int t = lane; t < n; t += 32) mp = fmaxf(mp, sums.mp[t]), mq = fmaxf(mq, sums.mq[t]);
    mp = warp_max(mp), mq = warp_max(mq);
    float sp = 0.0f, sq = 0.0f, dp = 0.0f, dq = 0.0f;
    for (int t = lane; t < n; t += 32) {
        const bool has_p = sums.mp[t] > kNegInf, has_q = sums.mq[t] > kNegInf;
        const float bp = has_p ? fmaxf((sums.mp[t] - mp) * kp, tiles::kFarBelow) : 0.0f, bq = has_q ? fmaxf((sums.mq[t] - mq) * kq, tiles::kFarBelow) : 0.0f;
        const float fp = has_p ? ex2_approx(bp) : 0.0f, fq = has_q ? ex2_approx(bq) : 0.0f;
        const float d = has_p && has_q ? bq - bp : 0.0f;
        sp = fmaf(fp, sums.sp[t], sp), sq = fmaf(fq, sums.sq[t], sq);
        dp = fmaf(fp, fmaf(-d, sums.sp[t], sums.dp[t]), dp), dq = fmaf(fq, fmaf(d, sums.sq[t], sums.dq[t]), dq);
    }
    const float sum = tiles::warp_sum_four(sp, sq, dp, dq, lane);
    return {mq, mp, __shfl_sync(0xFFFFFFFFu, sum, 8), __shfl_sync(0xFFFFFFFFu, sum, 0), __shfl_sync(0xFFFFFFFFu, sum, 24), __shfl_sync(0xFFFFFFFFu, sum, 16)};
}

// sum of the tiles' overlaps, by one warp
__device__ __forceinline__ float join_overlap(const Sums& sums, int n, int lane) {
    float s = 0.0f;
    for (int t = lane; t < n; t += 32) s += sums.mq[t];
    return tiles::warp_sum_two(s, 0.0f, lane);
}

// Both rows of a block, read into the tiles' sums; everything else of a row follows from what this leaves in shared memory.
template <typename T, bool ALIGNED, bool BOTH>
__device__ __forceinline__ bool read_rows(const DivergenceArgs& a, const tiles::View& draft, const tiles::View& target, int n_tiles, Smem& sm) {
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    float alone_q = kNegInf, alone_p = kNegInf;
    bool bad = false;
    if (tid == 0) sm.status = 0;
    for (int t = warp; t < n_tiles; t += kWarps) {
        uint4 p[kWords], q[kWords];
        tiles::load_tile<T, ALIGNED, kWords>(p, draft, t, lane, a.V);
        tiles::load_tile<T, ALIGNED, kWords>(q, target, t, lane, a.V);
        tile_sums<T, BOTH>(p, q, a.k_draft, a.k_target, t, lane, sm.sums, alone_q, alone_p, bad);
    }
    alone_q = warp_max(alone_q), alone_p = warp_max(alone_p);
    if (lane == 0) sm.alone_q[warp] = alone_q, sm.alone_p[warp] = alone_p;
    bad = __syncthreads_or(bad);
    if (warp == 0) {
        const Totals t = join(sm.sums, n_tiles, a.k_draft, a.k_target, lane);
        if (lane == 0) sm.total = t;
    }
    __syncthreads();
    return bad;
}

struct RowResult {
    bool empty, kl_infinite, reverse_infinite;
    float log2_sp, log2_sq, kl, reverse;
};
// A weight below 2^-126 of its row's largest counts as none.
__device__ __forceinline__ RowResult result_of(const DivergenceArgs& a, const Smem& sm) {
    const Totals& t = sm.total;
    RowResult r;
    r.empty = t.mp == kNegInf || t.mq == kNegInf;
    r.kl_infinite = r.reverse_infinite = false;
    r.log2_sp = r.log2_sq = r.kl = r.reverse = 0.0f;
    if (r.empty) return r;
    float alone_q = kNegInf, alone_p = kNegInf;
#pragma unroll
    for (int w = 0; w < kWarps; ++w) alone_q = fmaxf(alone_q, sm.alone_q[w]), alone_p = fmaxf(alone_p, sm.alone_p[w]);
    r.kl_infinite = (alone_q - t.mq) * a.k_target >= -126.0f;
    r.reverse_infinite = (alone_p - t.mp) * a.k_draft >= -126.0f;
    const double lp = log2((double)t.sp), lq = log2((double)t.sq), ln2 = 0.693147180559945309;
    r.log2_sp = (float)lp, r.log2_sq = (float)lq;
    r.kl = r.kl_infinite ? __builtin_huge_valf() : fmaxf((float)(ln2 * ((double)t.dq / (double)t.sq - lq + lp)), 0.0f);
    r.reverse = r.reverse_infinite ? __builtin_huge_valf() : fmaxf((float)(ln2 * ((double)t.dp / (double)t.sp - lp + lq)), 0.0f);
    return r;
}
__device__ __forceinline__ int status_of(const RowResult& r, bool bad) {
    return (bad ? RSD_ST_NAN_INPUT : 0) | (r.empty ? RSD_ST_EMPTY_ROW : 0) | (r.kl_infinite ? RSD_ST_ZERO_DRAFT_PROB : 0) | (r.reverse_infinite ? RSD_ST_ZERO_TARGET_PROB : 0);
}

__device__ __forceinline__ void store_status(const DivergenceArgs& a, int64_t b, int status) {   // every thread calls it; thread 0's word counts
    grid_started();
    if (!a.own_status) grid_wait();
    if (threadIdx.x == 0) {
        if (a.own_status) a.status[b] = status;
        else if (status) atomicOr(&a.status[b], status);
    }
}

template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(kThreads) divergence_kernel(const __grid_constant__ DivergenceArgs a) {
    using P = tiles::Packed16<T>;
    __shared__ Smem sm;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    if (a.own_status) grid_wait();
    const int64_t slot = blockIdx.x, b = slot / a.R;
    const int r = (int)(slot - b * a.R);
    const tiles::View draft = tiles::view_of<T>((const T*)a.draft + b * a.draft_seq + r * a.draft_row, a.V);
    const tiles::View target = tiles::view_of<T>((const T*)a.target + b * a.target_seq + r * a.target_row, a.V);
    const int n_tiles = tiles::tiles_of<T>(a.V, kWords);
    const bool bad = read_rows<T, ALIGNED, true>(a, draft, target, n_tiles, sm);
    const RowResult res = result_of(a, sm);
    if (tid == 0) {
        if (a.out_kl) a.out_kl[slot] = res.kl;
        if (a.out_reverse) a.out_reverse[slot] = res.reverse;
    }
    if (a.out_overlap) {
        const float mp = res.empty ? 0.0f : sm.total.mp, mq = res.empty ? 0.0f : sm.total.mq;
        __syncthreads();                                            // (mq is read no more: the overlaps take its place)
        const unsigned long long minus_p = tiles::both(-mp), minus_q = tiles::both(-mq), kkp = tiles::both(a.k_draft), kkq = tiles::both(a.k_target);
        const unsigned long long lp = tiles::both(-res.log2_sp), lq = tiles::both(-res.log2_sq);
        for (int t = warp; t < n_tiles && !res.empty; t += kWarps) {
            uint4 p[kWords], q[kWords];
            tiles::load_tile<T, ALIGNED, kWords>(p, draft, t, lane, a.V);
            tiles::load_tile<T, ALIGNED, kWords>(q, target, t, lane, a.V);
            unsigned long long s = tiles::both(0.0f);
#pragma unroll
            for (int i = 0; i < kWords; ++i) {
                if (bad) {
                    bool ignored = false;
                    P::clean(p[i], ignored), P::clean(q[i], ignored);
                }
#pragma unroll
                for (int j = 0; j < P::kEntries / 2; ++j) {
                    float x, y, u, v;
                    split_f32x2(fma_f32x2(add_f32x2(P::pair(p[i], j), minus_p), kkp, lp), x, y);
                    split_f32x2(fma_f32x2(add_f32x2(P::pair(q[i], j), minus_q), kkq, lq), u, v);
                    s = add_f32x2(s, f32x2(ex2_approx(fminf(x, u)), ex2_approx(fminf(y, v))));
                }
            }
            float x, y;
            split_f32x2(s, x, y);
            const float sum = tiles::warp_sum_two(x + y, 0.0f, lane);
            if (lane == 0) sm.sums.mq[t] = sum;
        }
        __syncthreads();
        if (warp == 0) {
            const float sum = res.empty ? 0.0f : join_overlap(sm.sums, n_tiles, lane);
            if (lane == 0) a.out_overlap[slot] = fminf(sum, 1.0f);
        }
    }
    store_status(a, b, status_of(res, bad));
}

// d KL(q||p) / dv_x = (p_x - q_x) / T,   d KL(p||q) / dv_x = p_x (log p_x - log q_x - KL(p||q)) / T,   v the draft row, T its temperature.
// A row whose KL(p||q) is infinite has no gradient of it.  The rows are read twice, the second time from L2.
template <typename T, bool ALIGNED, bool REVERSE>
__global__ void __launch_bounds__(kThreads) divergence_grad_kernel(const __grid_constant__ DivergenceArgs a) {
    using P = tiles::Packed16<T>;
    constexpr int E = P::kEntries;
    __shared__ Smem sm;
    const int tid = threadIdx.x;
    if (a.own_status) grid_wait();
    const int64_t slot = blockIdx.x, b = slot / a.R;
    const int r = (int)(slot - b * a.R);
    const tiles::View draft = tiles::view_of<T>((const T*)a.draft + b * a.draft_seq + r * a.draft_row, a.V);
    const tiles::View target = tiles::view_of<T>((const T*)a.target + b * a.target_seq + r * a.target_row, a.V);
    char* grad = (char*)a.grad + slot * a.V * (int64_t)sizeof(T);
    const float g = a.g_kl ? a.g_kl[slot] : 0.0f, h = REVERSE ? a.g_reverse[slot] : 0.0f;
    const bool bad = read_rows<T, ALIGNED, REVERSE>(a, draft, target, tiles::tiles_of<T>(a.V, kWords), sm);
    const RowResult res = result_of(a, sm);
    const float inv_temp = fminf(1.0f / a.draft_temp, 3.0e38f), gt = res.empty ? 0.0f : g * inv_temp, ht = res.empty || res.reverse_infinite ? 0.0f : h * inv_temp;
    const unsigned long long minus_p = tiles::both(res.empty ? 0.0f : -sm.total.mp), minus_q = tiles::both(res.empty ? 0.0f : -sm.total.mq);
    const unsigned long long kkp = tiles::both(a.k_draft), kkq = tiles::both(a.k_target), lp = tiles::both(-res.log2_sp), lq = tiles::both(-res.log2_sq);
    // p (gt + ht (ln 2 (log2 p - log2 q) - KL)) - gt q
    const unsigned long long c0 = tiles::both(gt - (ht != 0.0f ? ht * res.reverse : 0.0f)), c1 = tiles::both(ht * 0.69314718f), cq = tiles::both(-gt), minus_one = tiles::both(-1.0f);
    const int head = (int)((uintptr_t)grad & 15u) / (int)sizeof(T);
    const int words = (head + a.V + E - 1) / E;
    for (int j = tid; j < words; j += kThreads) {
        const int x0 = j * E - head;
        uint4 p = tiles::load_word<T, ALIGNED>(draft, x0, a.V), q = tiles::load_word<T, ALIGNED>(target, x0, a.V);
        if (bad) {
            bool ignored = false;
            P::clean(p, ignored), P::clean(q, ignored);
        }
        const uint4 out = P::make([&](int i) {
            float x, y, u, v;
            split_f32x2(fma_f32x2(add_f32x2(P::pair(p, i), minus_p), kkp, lp), x, y);
            split_f32x2(fma_f32x2(add_f32x2(P::pair(q, i), minus_q), kkq, lq), u, v);
            const unsigned long long wp = f32x2(ex2_approx(x), ex2_approx(y)), wq = f32x2(ex2_approx(u), ex2_approx(v));
            unsigned long long c = c0;
            if (REVERSE) {
                x = fmaxf(x, tiles::kFarBelow), y = fmaxf(y, tiles::kFarBelow), u = fmaxf(u, tiles::kFarBelow), v = fmaxf(v, tiles::kFarBelow);
                c = fma_f32x2(fma_f32x2(f32x2(u, v), minus_one, f32x2(x, y)), c1, c0);
            }
            return fma_f32x2(wp, c, tiles::mul_f32x2(wq, cq));
        });
        if (x0 >= 0 && x0 + E <= a.V) {
            *(uint4*)(grad + (int64_t)x0 * (int)sizeof(T)) = out;
        } else {
            for (int i = 0; i < E; ++i)
                if (x0 + i >= 0 && x0 + i < a.V) P::store(grad, x0 + i, P::get(out, i));
        }
    }
    store_status(a, b, status_of(res, bad));
}

}  // namespace divergence
}  // namespace rsd
