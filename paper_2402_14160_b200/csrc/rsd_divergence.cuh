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

struct Sums {   // of the rows' tiles, relative to each tile's largest entries; every block of the pair has all of them
    float mp[kMaxTiles], mq[kMaxTiles], sp[kMaxTiles], sq[kMaxTiles], dp[kMaxTiles], dq[kMaxTiles];
};
struct Totals {
    float mp, mq, sp, sq, dp, dq;   // largest entries, sums of weights, of weight times b - a (p), a - b (q)
};
struct Smem {
    Sums sums;
    Totals total;
    uint32_t alone_p, alone_q;      // largest entry whose token the other row lacks, as an ordered word (0: none)
    int status;
};

// Four pairs of sums of a lane
struct LaneSums {
    unsigned long long sp, sq, dp, dq;
};
// MASKED: entries without mass are raised, so that their terms are 0
template <typename T, bool BOTH, bool MASKED>
__device__ __forceinline__ void add_tile(const uint4 (&p)[kWords], const uint4 (&q)[kWords], float mp, float mq, float kp, float kq, LaneSums& l) {
    using P = tiles::Packed16<T>;
    const unsigned long long ref_p = tiles::both(-(mp * kp)), ref_q = tiles::both(-(mq * kq)), kkp = tiles::both(kp), kkq = tiles::both(kq), minus_one = tiles::both(-1.0f);
#pragma unroll
    for (int i = 0; i < kWords; ++i) {
        const uint4 pw = MASKED && BOTH ? P::raised(p[i]) : p[i], qw = MASKED && BOTH ? P::raised(q[i]) : q[i];
#pragma unroll
        for (int j = 0; j < P::kEntries / 2; ++j) {
            const unsigned long long b = fma_f32x2(P::pair(pw, j), kkp, ref_p), a = fma_f32x2(P::pair(qw, j), kkq, ref_q);
            float x, y;
            split_f32x2(b, x, y);
            const unsigned long long wp = f32x2(ex2_approx(x), ex2_approx(y));
            split_f32x2(a, x, y);
            const unsigned long long wq = f32x2(ex2_approx(x), ex2_approx(y));
            l.sp = add_f32x2(l.sp, wp), l.sq = add_f32x2(l.sq, wq);
            if (BOTH) {
                const unsigned long long d = fma_f32x2(b, minus_one, a);
                l.dq = fma_f32x2(wq, d, l.dq);
                l.dp = fma_f32x2(wp, d, l.dp);                     // (its sign is turned below)
            }
        }
    }
}

// A tile whose rows have mass at different tokens, or entries near the end of the range: one pair after the other.
struct Words {
    uint4 w[kWords];
};
struct CarefulSums {
    float sp, sq, dp, dq, alone_p, alone_q;
};
template <typename T>
__device__ __noinline__ CarefulSums add_tile_careful(Words p, Words q, float mp, float mq, float kp, float kq) {
    using P = tiles::Packed16<T>;
    const bool plain_p = tiles::plain_tile(mp, kp), plain_q = tiles::plain_tile(mq, kq);   // (as the join takes it)
    const float zp = mp > kNegInf && !plain_p ? mp : 0.0f, zq = mq > kNegInf && !plain_q ? mq : 0.0f, rp = plain_p ? mp * kp : 0.0f, rq = plain_q ? mq * kq : 0.0f;
    CarefulSums l = {0.0f, 0.0f, 0.0f, 0.0f, kNegInf, kNegInf};
#pragma unroll 1
    for (int i = 0; i < kWords; ++i) {
        const uint4 pw = i == 0 ? p.w[0] : i == 1 ? p.w[1] : i == 2 ? p.w[2] : p.w[3], qw = i == 0 ? q.w[0] : i == 1 ? q.w[1] : i == 2 ? q.w[2] : q.w[3];
#pragma unroll
        for (int j = 0; j < P::kEntries; ++j) {
            const float vp = P::get(pw, j), vq = P::get(qw, j), b = fmaf(vp - zp, kp, -rp), a = fmaf(vq - zq, kq, -rq);
            const bool in_p = b > kNegInf, in_q = a > kNegInf;
            const float wp = ex2_approx(b), wq = ex2_approx(a), d = in_p && in_q ? a - b : 0.0f;
            if (in_q && !in_p) l.alone_q = fmaxf(l.alone_q, vq);
            if (in_p && !in_q) l.alone_p = fmaxf(l.alone_p, vp);
            l.sp += wp, l.sq += wq, l.dp = fmaf(wp, d, l.dp), l.dq = fmaf(wq, d, l.dq);
        }
    }
    return l;
}

template <typename T, bool BOTH>   // BOTH: the sums of weight times difference too
__device__ __forceinline__ void tile_sums(uint4 (&p)[kWords], uint4 (&q)[kWords], float kp, float kq, int t, int lane, uint32_t blocks, Smem& sm, float& alone_p, float& alone_q,
                                          bool& bad) {
    using P = tiles::Packed16<T>;
    float mp = tiles::warp_max_nan(P::largest(p)), mq = tiles::warp_max_nan(P::largest(q));
    if (!(mp < __builtin_huge_valf()) || !(mq < __builtin_huge_valf())) {   // NaN or +inf: no entries
#pragma unroll
        for (int i = 0; i < kWords; ++i) P::clean(p[i], bad), P::clean(q[i], bad);
        mp = tiles::warp_max_nan(P::largest(p)), mq = tiles::warp_max_nan(P::largest(q));
    }
    LaneSums l = {tiles::both(0.0f), tiles::both(0.0f), tiles::both(0.0f), tiles::both(0.0f)};
    const bool plain = tiles::plain_tile(mp, kp) && tiles::plain_tile(mq, kq);
    if (plain && (!BOTH || __all_sync(0xFFFFFFFFu, fminf(P::smallest(p), P::smallest(q)) > tiles::kLow))) {
        add_tile<T, BOTH, false>(p, q, mp, mq, kp, kq, l);
    } else {
        bool alike = true;
#pragma unroll
        for (int i = 0; i < kWords; ++i) alike = alike && !P::differ(p[i], q[i]);
        if (BOTH && plain && __all_sync(0xFFFFFFFFu, alike)) {
            add_tile<T, BOTH, true>(p, q, mp, mq, kp, kq, l);
        } else {
            Words pw, qw;
#pragma unroll
            for (int i = 0; i < kWords; ++i) pw.w[i] = p[i], qw.w[i] = q[i];
            const CarefulSums c = add_tile_careful<T>(pw, qw, mp, mq, kp, kq);
            l = {f32x2(c.sp, 0.0f), f32x2(c.sq, 0.0f), f32x2(c.dp, 0.0f), f32x2(c.dq, 0.0f)};
            alone_p = fmaxf(alone_p, c.alone_p), alone_q = fmaxf(alone_q, c.alone_q);
        }
    }
    float x, y;
    split_f32x2(l.sp, x, y);
    const float sp = x + y;
    split_f32x2(l.sq, x, y);
    const float sq = x + y;
    split_f32x2(l.dp, x, y);
    const float dp = -(x + y);
    split_f32x2(l.dq, x, y);
    const float dq = x + y;
    const uint32_t to = lane & 7;
    if (BOTH) {
        const float sum = tiles::warp_sum_four(sp, sq, dp, dq, lane);   // eight lanes each
        if (to < blocks) {
            float* const at = lane < 8 ? sm.sums.sp : lane < 16 ? sm.sums.sq : lane < 24 ? sm.sums.dp : sm.sums.dq;
            tiles::store_at(at + t, to, sum);
            if (lane < 16) tiles::store_at((lane < 8 ? sm.sums.mp : sm.sums.mq) + t, to, lane < 8 ? mp : mq);
        }
    } else {
        const float sum = tiles::warp_sum_two(sp, sq, lane);            // sixteen lanes each
        if (to < blocks) {
            float* const at = lane < 8 ? sm.sums.sp : lane < 16 ? sm.sums.mp : lane < 24 ? sm.sums.sq : sm.sums.mq;
            tiles::store_at(at + t, to, lane < 8 || (lane >= 16 && lane < 24) ? sum : lane < 16 ? mp : mq);
        }
    }
}

// The tiles' sums joined by one warp; every lane gets the result.
template <bool BOTH>
__device__ __forceinline__ Totals join(const Sums& sums, int n, float kp, float kq, int lane) {
    float mp = kNegInf, mq = kNegInf;
    for (int t = lane; t < n; t += 32) mp = fmaxf(mp, sums.mp[t]), mq = fmaxf(mq, sums.mq[t]);
    mp = warp_max(mp), mq = warp_max(mq);
    float sp = 0.0f, sq = 0.0f, dp = 0.0f, dq = 0.0f;
    for (int t = lane; t < n; t += 32) {
        const float mtp = sums.mp[t], mtq = sums.mq[t];
        const bool has_p = mtp > kNegInf, has_q = mtq > kNegInf;
        const float bp = has_p ? fmaxf((mtp - mp) * kp, tiles::kFarBelow) - tiles::rounded_off(mtp, kp) : 0.0f;
        const float bq = has_q ? fmaxf((mtq - mq) * kq, tiles::kFarBelow) - tiles::rounded_off(mtq, kq) : 0.0f;
        const float fp = has_p ? ex2_approx(bp) : 0.0f, fq = has_q ? ex2_approx(bq) : 0.0f;
        sp = fmaf(fp, sums.sp[t], sp), sq = fmaf(fq, sums.sq[t], sq);
        if (BOTH) {
            const float d = has_p && has_q ? bq - bp : 0.0f;
            dp = fmaf(fp, fmaf(-d, sums.sp[t], sums.dp[t]), dp), dq = fmaf(fq, fmaf(d, sums.sq[t], sums.dq[t]), dq);
        }
    }
    const float sum = tiles::warp_sum_four(sp, sq, dp, dq, lane);
    return {mp, mq, __shfl_sync(0xFFFFFFFFu, sum, 0), __shfl_sync(0xFFFFFFFFu, sum, 8), __shfl_sync(0xFFFFFFFFu, sum, 16), __shfl_sync(0xFFFFFFFFu, sum, 24)};
}

// A pair of rows and the tiles of it that this warp has: tile t belongs to warp t / blocks mod kWarps of block t mod blocks.
struct Pair {
    tiles::View draft, target;
    int64_t slot;
    uint32_t rank, blocks;
    int n_tiles, first, step;
};
template <typename T>
__device__ __forceinline__ Pair pair_of(const DivergenceArgs& a) {
    Pair w;
    w.rank = tiles::cluster_rank(), w.blocks = tiles::cluster_blocks();
    const uint32_t slot = blockIdx.x / w.blocks, sequence = slot / (uint32_t)a.R;
    const int64_t b = sequence;
    const int r = (int)(slot - sequence * (uint32_t)a.R);
    w.slot = slot;
    w.draft = tiles::view_of<T>((const T*)a.draft + b * a.draft_seq + r * a.draft_row, a.V);
    w.target = tiles::view_of<T>((const T*)a.target + b * a.target_seq + r * a.target_row, a.V);
    w.n_tiles = tiles::tiles_of<T>(a.V, kWords);
    w.first = (int)(threadIdx.x >> 5) * (int)w.blocks + (int)w.rank, w.step = kWarps * (int)w.blocks;
    return w;
}

// Both rows, read into the tiles' sums; everything else of a pair follows from what this leaves in every block's shared memory.  True: there were NaN or +inf.
template <typename T, bool ALIGNED, bool BOTH>
__device__ __forceinline__ bool read_rows(const DivergenceArgs& a, const Pair& w, Smem& sm) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) sm.status = 0, sm.alone_p = sm.alone_q = 0;
    if (w.blocks > 1) tiles::cluster_arrive();     // (the pair's other blocks have started, and their words above are set, behind the wait below)
    grid_wait();
    if (w.blocks > 1) tiles::cluster_wait();
    else __syncthreads();
    float alone_p = kNegInf, alone_q = kNegInf;
    bool bad = false;
    for (int t = w.first; t < w.n_tiles; t += w.step) {
        uint4 p[kWords], q[kWords];
        tiles::load_tile<T, ALIGNED, kWords>(p, w.draft, t, lane, a.V);
        tiles::load_tile<T, ALIGNED, kWords>(q, w.target, t, lane, a.V);
        tile_sums<T, BOTH>(p, q, a.k_draft, a.k_target, t, lane, w.blocks, sm, alone_p, alone_q, bad);
    }
    if (bad || alone_p > kNegInf || alone_q > kNegInf)
        for (uint32_t i = 0; i < w.blocks; ++i) {
            if (bad) tiles::or_at(&sm.status, i, RSD_ST_NAN_INPUT);
            if (alone_p > kNegInf) tiles::max_at(&sm.alone_p, i, float_to_ordered(alone_p));
            if (alone_q > kNegInf) tiles::max_at(&sm.alone_q, i, float_to_ordered(alone_q));
        }
    tiles::row_barrier(w.blocks);
    if (warp == 0) {
        const Totals t = join<BOTH>(sm.sums, w.n_tiles, a.k_draft, a.k_target, lane);
        if (lane == 0) sm.total = t;
    }
    __syncthreads();
    return sm.status != 0;
}

struct Result {
    bool empty, kl_infinite, reverse_infinite;
    float log2_sp, log2_sq;
};
// A weight below 2^-126 of its row's largest counts as none.
__device__ __forceinline__ Result result_of(const DivergenceArgs& a, const Smem& sm) {
    const Totals& t = sm.total;
    Result r;
    r.empty = t.mp == kNegInf || t.mq == kNegInf;
    r.kl_infinite = r.reverse_infinite = false;
    r.log2_sp = r.log2_sq = 0.0f;
    if (r.empty) return r;
    r.kl_infinite = sm.alone_q && (ordered_to_float(sm.alone_q) - t.mq) * a.k_target >= -126.0f;
    r.reverse_infinite = sm.alone_p && (ordered_to_float(sm.alone_p) - t.mp) * a.k_draft >= -126.0f;
    r.log2_sp = log2f(t.sp), r.log2_sq = log2f(t.sq);
    return r;
}
__device__ __forceinline__ int status_of(const Result& r, bool bad) {
    return (bad ? RSD_ST_NAN_INPUT : 0) | (r.empty ? RSD_ST_EMPTY_ROW : 0) | (r.kl_infinite ? RSD_ST_ZERO_DRAFT_PROB : 0) | (r.reverse_infinite ? RSD_ST_ZERO_TARGET_PROB : 0);
}

// The divergences themselves in 64 bits: logarithms of sums cancel against each other.
__device__ __forceinline__ float divergence_of(float d, float s, float other) {
    return fmaxf((float)(0.693147180559945309 * ((double)d / (double)s + log2((double)other / (double)s))), 0.0f);
}

// log2 of a row's probabilities: v k - c + off in a plain row, (v - m) k - c otherwise; off is what c loses when it is rounded.
struct LogProb {
    bool plain;
    float c, off;
    unsigned long long kk, minus_c, minus_m;
    template <bool PLAIN>
    __device__ __forceinline__ unsigned long long of(unsigned long long v) const { return fma_f32x2(PLAIN ? v : add_f32x2(v, minus_m), kk, minus_c); }
};
__device__ __forceinline__ LogProb log_prob(float m, float k, float log2s, bool empty) {
    LogProb l;
    l.plain = tiles::plain_tile(m, k);
    const double exact = l.plain ? (double)m * (double)k + (double)log2s : (double)log2s;
    l.c = (float)exact, l.off = (float)((double)l.c - exact);
    l.kk = tiles::both(k), l.minus_c = tiles::both(-l.c), l.minus_m = tiles::both(l.plain || empty ? 0.0f : -m);
    return l;
}

template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(kThreads, 3) divergence_kernel(const __grid_constant__ DivergenceArgs a) {
    using P = tiles::Packed16<T>;
    __shared__ Smem sm;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const Pair w = pair_of<T>(a);
    const bool bad = read_rows<T, ALIGNED, true>(a, w, sm);
    const Result res = result_of(a, sm);
    if (w.rank == 0 && tid == 0) {
        const Totals& t = sm.total;
        const float inf = __builtin_huge_valf();
        if (a.out_kl) a.out_kl[w.slot] = res.empty ? 0.0f : res.kl_infinite ? inf : divergence_of(t.dq, t.sq, t.sp);
        if (a.out_reverse) a.out_reverse[w.slot] = res.empty ? 0.0f : res.reverse_infinite ? inf : divergence_of(t.dp, t.sp, t.sq);
        a.status[w.slot] = status_of(res, bad);
    }
    if (a.out_overlap) {
        const LogProb p = log_prob(sm.total.mp, a.k_draft, res.log2_sp, res.empty), q = log_prob(sm.total.mq, a.k_target, res.log2_sq, res.empty);
        const unsigned long long shift = tiles::both(q.off - p.off);
        const float scale = exp2f(p.off);
        tiles::row_barrier(w.blocks);                               // (the tiles' sums are read no more: the overlaps take the place of mp)
        auto sweep = [&](auto plain) {
            constexpr bool PLAIN = decltype(plain)::value;
            for (int t = w.first; t < w.n_tiles; t += w.step) {
                uint4 pw[kWords], qw[kWords];
                tiles::load_tile<T, ALIGNED, kWords>(pw, w.draft, t, lane, a.V);
                tiles::load_tile<T, ALIGNED, kWords>(qw, w.target, t, lane, a.V);
                if (bad) {
                    bool ignored = false;
#pragma unroll
                    for (int i = 0; i < kWords; ++i) P::clean(pw[i], ignored), P::clean(qw[i], ignored);
                }
                unsigned long long s = tiles::both(0.0f);
#pragma unroll
                for (int i = 0; i < kWords; ++i)
#pragma unroll
                    for (int j = 0; j < P::kEntries / 2; ++j) {
                        float x, y, u, v;
                        split_f32x2(p.of<PLAIN>(P::pair(pw[i], j)), x, y);
                        split_f32x2(add_f32x2(q.of<PLAIN>(P::pair(qw[i], j)), shift), u, v);
                        s = add_f32x2(s, f32x2(ex2_approx(fminf(x, u)), ex2_approx(fminf(y, v))));
                    }
                float x, y;
                split_f32x2(s, x, y);
                const float sum = tiles::warp_sum_two(x + y, 0.0f, lane);
                if (lane == 0) tiles::store_at(&sm.sums.mp[t], 0, sum);
            }
        };
        if (!res.empty) {
            if (p.plain && q.plain) sweep(std::true_type());
            else sweep(std::false_type());
        }
        tiles::row_barrier(w.blocks);
        if (w.rank == 0 && warp == 0) {
            float s = 0.0f;
            for (int t = lane; t < w.n_tiles; t += 32) s += sm.sums.mp[t];
            s = tiles::warp_sum_two(s, 0.0f, lane);
            if (lane == 0) a.out_overlap[w.slot] = res.empty ? 0.0f : fminf(s * scale, 1.0f);
        }
    }
    grid_started();
}

// d KL(q||p) / dv_x = (p_x - q_x) / T,   d KL(p||q) / dv_x = p_x (log p_x - log q_x - KL(p||q)) / T,   v the draft row, T its temperature.
// A row whose KL(p||q) is infinite has no gradient of it.  The rows are read twice, the second time from L2.
template <typename T, bool ALIGNED, bool REVERSE>
__global__ void __launch_bounds__(kThreads, 3) divergence_grad_kernel(const __grid_constant__ DivergenceArgs a) {
    using P = tiles::Packed16<T>;
    constexpr int E = P::kEntries;
    __shared__ Smem sm;
    const int tid = threadIdx.x, lane = tid & 31;
    const Pair w = pair_of<T>(a);
    char* grad = (char*)a.grad + w.slot * a.V * (int64_t)sizeof(T);
    const bool bad = read_rows<T, ALIGNED, REVERSE>(a, w, sm);
    const Result res = result_of(a, sm);
    const float g = a.g_kl ? a.g_kl[w.slot] : 0.0f, h = REVERSE ? a.g_reverse[w.slot] : 0.0f;
    const float inv_temp = a.inv_draft_temp, gt = res.empty ? 0.0f : g * inv_temp, ht = res.empty || (REVERSE && res.reverse_infinite) ? 0.0f : h * inv_temp;
    const LogProb lp = log_prob(sm.total.mp, a.k_draft, res.log2_sp, res.empty), lq = log_prob(sm.total.mq, a.k_target, res.log2_sq, res.empty);
    const float scale_p = exp2f(lp.off), scale_q = exp2f(lq.off);
    // gt (p - q) + p ht (ln 2 (log2 p - log2 q) - KL(p||q)); rows that are equal give 0
    const float reverse = ht != 0.0f ? 0.69314718f * (sm.total.dp / sm.total.sp + log2f(sm.total.sq / sm.total.sp)) : 0.0f;
    const float c1f = ht * 0.69314718f, c0f = fmaf(c1f, lp.off - lq.off, -ht * reverse);
    const unsigned long long c0 = tiles::both(c0f * scale_p), c1 = tiles::both(c1f * scale_p), cg = tiles::both(gt * scale_p), minus_ratio = tiles::both(-(scale_q / scale_p)),
                             minus_one = tiles::both(-1.0f);
    const int head = (int)((uintptr_t)grad & 15u) / (int)sizeof(T);
    const int out_tiles = tiles::tiles_of<T>(head + a.V, kWords);
    auto write = [&](auto plain) {
        constexpr bool PLAIN = decltype(plain)::value;
        for (int t = w.first; t < out_tiles; t += w.step) {
            const int x0 = t * tiles::tile_entries<T>(kWords) + lane * E - head, from = x0 - lane * E;
            const bool whole = from >= 0 && from + tiles::tile_entries<T>(kWords) <= a.V;
            uint4 pw[kWords], qw[kWords];
            tiles::load_words<T, ALIGNED, kWords>(pw, w.draft, x0, whole, a.V);
            tiles::load_words<T, ALIGNED, kWords>(qw, w.target, x0, whole, a.V);
#pragma unroll
            for (int k = 0; k < kWords; ++k) {
                if (bad) {
                    bool ignored = false;
                    P::clean(pw[k], ignored), P::clean(qw[k], ignored);
                }
                const uint4 pr = REVERSE && PLAIN ? P::raised(pw[k]) : pw[k], qr = REVERSE && PLAIN ? P::raised(qw[k]) : qw[k];
                uint4 out = P::make([&](int i) {
                    float x, y, u, v;
                    split_f32x2(lp.of<PLAIN>(P::pair(pr, i)), x, y);
                    split_f32x2(lq.of<PLAIN>(P::pair(qr, i)), u, v);
                    const unsigned long long wp = f32x2(ex2_approx(x), ex2_approx(y)), wq = f32x2(ex2_approx(u), ex2_approx(v));
                    const unsigned long long apart = tiles::mul_f32x2(fma_f32x2(wq, minus_ratio, wp), cg);
                    if (!REVERSE) return apart;
                    if (!PLAIN) x = fmaxf(x, tiles::kFarBelow), y = fmaxf(y, tiles::kFarBelow), u = fmaxf(u, tiles::kFarBelow), v = fmaxf(v, tiles::kFarBelow);
                    return fma_f32x2(wp, fma_f32x2(fma_f32x2(f32x2(u, v), minus_one, f32x2(x, y)), c1, c0), apart);
                });
                const int x = x0 + k * 32 * E;
                if (res.empty) out = make_uint4(0, 0, 0, 0);
                if (whole || (x >= 0 && x + E <= a.V)) {
                    *(uint4*)(grad + (int64_t)x * (int)sizeof(T)) = out;
                } else {
                    for (int i = 0; i < E; ++i)
                        if (x + i >= 0 && x + i < a.V) P::store(grad, x + i, P::get(out, i));
                }
            }
        }
    };
    if (lp.plain && lq.plain) write(std::true_type());
    else write(std::false_type());
    if (w.rank == 0 && tid == 0) {
        Result said = res;
        said.kl_infinite = false;                                   // (its gradient is finite)
        if (!REVERSE) said.reverse_infinite = false;
        a.status[w.slot] = status_of(said, bad);
    }
    grid_started();
}

}  // namespace divergence
}  // namespace rsd
