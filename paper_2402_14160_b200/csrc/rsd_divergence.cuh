// How far draft rows are from target rows (divergence_kernel), and the gradient of that with respect to the draft rows
// (divergence_grad_kernel).
//
// With a = (v_t - max v_t) log2(e) / T_t for the target row and b alike for the draft row, q = 2^a / S_q, p = 2^b / S_p:
//   KL(q||p) = ln 2 [ (sum 2^a (a - b)) / S_q - log2 S_q + log2 S_p ]       KL(p||q) = ln 2 [ (sum 2^b (b - a)) / S_p - log2 S_p + log2 S_q ]
// so both come from one pass with one exponential per entry and row; what cancels is of the size of 1, not of the size of a logit.
// The overlap sum min(p, q) needs the normalisers first: a second pass (from L2) with one exponential per pair, 2^min(log2 p, log2 q).
//
// 7296 pairs of 32,000 bf16: 280 us back to back (259 below the power limit; floor 143); 7000 pairs without the overlap 149 (floor 137).  With it three exponentials a pair of entries and
// 26,400 warp instructions a pair of rows keep the special-function unit and the issue slots 61 to 63 % busy.  7000 fp32 pairs 375 (floor 273).  Rows that are not plain: 4096 pairs 258 us
// (150).
// Slower: the rows held in shared memory, which takes clusters of two blocks (401), halves of the next tile read in between (its conditions cost more than the wait), a prefetch of
// whole rows into L2 (a tenth), edges of rows out of line (3 %).
#pragma once
#include "../../include/rsd.h"
#include "rsd_score_args.h"
#include "rsd_tiles.cuh"

namespace rsd {

namespace divergence {

constexpr int kWords = 4;

// Sums of weight times difference are kept in units of 2^20: a difference may be anything that fp32 holds, and up to 262,144 of them are added.
constexpr float kUnit = 1.0f / 1048576.0f;

struct Sums {   // of a tile of both rows, relative to its largest entries; every block of the pair has those of all tiles
    float sp, sq, dp, dq, mp, mq, overlap, unused;
};
struct Totals {
    float sp, sq, dp, dq, mp, mq;   // sums of weights, of weight times b - a (p), a - b (q), in units, largest entries
    float alone_p, alone_q;         // largest entries of tiles that are missing in the other row
};
struct Smem {
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
            const float vp = P::get(pw, j), vq = P::get(qw, j), b = tiles::distance(vp, zp, kp, -rp), a = tiles::distance(vq, zq, kq, -rq);
            const bool in_p = b > kNegInf, in_q = a > kNegInf;
            const float wp = ex2_approx(b), wq = ex2_approx(a), d = in_p && in_q ? a - b : 0.0f;
            if (in_q && !in_p) l.alone_q = fmaxf(l.alone_q, vq);
            if (in_p && !in_q) l.alone_p = fmaxf(l.alone_p, vp);
            l.sp += wp, l.sq += wq, l.dp = fmaf(wp, d * kUnit, l.dp), l.dq = fmaf(wq, d * kUnit, l.dq);
        }
    }
    return l;
}

// masked: a tile of this warp had entries without mass, so that this one is looked through for them at once.
// next() reads the warp's next tile into the words' places, ahead of the sums over the warp.  What is rare goes straight to the blocks' shared memory, and takes no registers of the loop.
template <typename T, bool BOTH, typename F>   // BOTH: the sums of weight times difference too
__device__ __forceinline__ void tile_sums(uint4 (&p)[kWords], uint4 (&q)[kWords], float kp, float kq, int t, int lane, uint32_t blocks, Sums* sums, Smem& sm,
                                          bool& masked, F next) {
    using P = tiles::Packed16<T>;
    float mp = tiles::warp_max_nan(P::largest(p)), mq = tiles::warp_max_nan(P::largest(q));
    if (!(mp < __builtin_huge_valf()) || !(mq < __builtin_huge_valf())) {   // NaN or +inf: no entries
        bool bad = false;
        if (lane < blocks) tiles::or_at(&sm.status, lane, RSD_ST_NAN_INPUT);
#pragma unroll
        for (int i = 0; i < kWords; ++i) P::clean(p[i], bad), P::clean(q[i], bad);
        mp = tiles::warp_max_nan(P::largest(p)), mq = tiles::warp_max_nan(P::largest(q));
    }
    LaneSums l = {tiles::both(0.0f), tiles::both(0.0f), tiles::both(0.0f), tiles::both(0.0f)};
    const bool plain = tiles::plain_tile(mp, kp) && tiles::plain_tile(mq, kq);
    float x, y, sp, sq, dp, dq;
    auto halves = [&](float unit) {
        split_f32x2(l.sp, x, y), sp = x + y;
        split_f32x2(l.sq, x, y), sq = x + y;
        split_f32x2(l.dp, x, y), dp = -(x + y) * unit;
        split_f32x2(l.dq, x, y), dq = (x + y) * unit;
    };
    // Which form a tile is summed in depends on the tile alone (where the same entries have no mass in both rows the first two give the same bits).
    auto alike = [&] {
        bool same = true;
#pragma unroll
        for (int i = 0; i < kWords; ++i) same = same && !P::differ(p[i], q[i]);
        return __all_sync(0xFFFFFFFFu, same) != 0;
    };
    const bool known = BOTH && plain && masked && alike();
    bool done = false;
    if (plain && !known) {
        add_tile<T, BOTH, false>(p, q, mp, mq, kp, kq, l);
        halves(kUnit);
        done = !BOTH || !__any_sync(0xFFFFFFFFu, !(fabsf(dp + dq) < __builtin_huge_valf()));   // (an entry without mass gives 0 times infinity, one far below may give infinity)
    }
    if (!done) {
        masked = true;
        if (BOTH && plain && (known || alike())) {
            l = {tiles::both(0.0f), tiles::both(0.0f), tiles::both(0.0f), tiles::both(0.0f)};
            add_tile<T, BOTH, true>(p, q, mp, mq, kp, kq, l);
            halves(kUnit);
        } else {
            Words pw, qw;
#pragma unroll
            for (int i = 0; i < kWords; ++i) pw.w[i] = p[i], qw.w[i] = q[i];
            const CarefulSums c = add_tile_careful<T>(pw, qw, mp, mq, kp, kq);
            l = {f32x2(c.sp, 0.0f), f32x2(c.sq, 0.0f), f32x2(c.dp, 0.0f), f32x2(c.dq, 0.0f)};
            const float alone_p = tiles::warp_max_nan(c.alone_p), alone_q = tiles::warp_max_nan(c.alone_q);
            if (lane < blocks && alone_p > kNegInf) tiles::max_at(&sm.alone_p, lane, float_to_ordered(alone_p));
            if (lane < blocks && alone_q > kNegInf) tiles::max_at(&sm.alone_q, lane, float_to_ordered(alone_q));
            halves(1.0f);
        }
    }
    next();
    // Sums::sp, sq, dp, dq are in eight lanes each (without the last two in sixteen each); four lanes store them and two the largest entries, in every block.
    const float sum = BOTH ? tiles::warp_sum_four(sp, sq, dp, dq, lane) : tiles::warp_sum_two(sp, sq, lane);
    const int member = (lane & 4) ? 4 + (lane >> 4) : BOTH ? lane >> 3 : lane >> 4;
    const float value = (lane & 4) ? (lane < 16 ? mp : mq) : sum;
    float* const to = (float*)&sums[t] + member;
    if (blocks == 1) {
        if ((lane & 3) == 0) *to = value;          // (several lanes store the same)
    } else {
        for (uint32_t r = lane & 3; r < blocks; r += 4) tiles::store_at(to, r, value);
    }
}

// The tiles' sums joined by one warp; every lane gets the result.
template <bool BOTH>
__device__ __forceinline__ Totals join(const Sums* sums, int n, float kp, float kq, int lane) {
    float mp = kNegInf, mq = kNegInf;
    for (int t = lane; t < n; t += 32) mp = fmaxf(mp, sums[t].mp), mq = fmaxf(mq, sums[t].mq);
    mp = tiles::warp_max_nan(mp), mq = tiles::warp_max_nan(mq);
    float sp = 0.0f, sq = 0.0f, dp = 0.0f, dq = 0.0f, alone_p = kNegInf, alone_q = kNegInf;
    for (int t = lane; t < n; t += 32) {
        const float mtp = sums[t].mp, mtq = sums[t].mq, far_p = tiles::distance(mtp, mp, kp), far_q = tiles::distance(mtq, mq, kq);
        const bool has_p = far_p > kNegInf, has_q = far_q > kNegInf;   // (a tile whose distance leaves fp32's range is missing, like single entries)
        const float bp = has_p ? far_p - tiles::rounded_off(mtp, kp) : 0.0f, bq = has_q ? far_q - tiles::rounded_off(mtq, kq) : 0.0f;
        if (has_p && !has_q) alone_p = fmaxf(alone_p, mtp);
        if (has_q && !has_p) alone_q = fmaxf(alone_q, mtq);
        const float fp = has_p ? ex2_approx(bp) : 0.0f, fq = has_q ? ex2_approx(bq) : 0.0f;
        sp = fmaf(fp, sums[t].sp, sp), sq = fmaf(fq, sums[t].sq, sq);
        if (BOTH) {
            const float d = has_p && has_q ? fmaxf(fminf(bq - bp, -tiles::kLowest), tiles::kLowest) * kUnit : 0.0f;
            dp = fmaf(fp, fmaf(-d, sums[t].sp, sums[t].dp), dp), dq = fmaf(fq, fmaf(d, sums[t].sq, sums[t].dq), dq);
        }
    }
    const float sum = tiles::warp_sum_four(sp, sq, dp, dq, lane);
    if (BOTH) alone_p = tiles::warp_max_nan(alone_p), alone_q = tiles::warp_max_nan(alone_q);
    return {__shfl_sync(0xFFFFFFFFu, sum, 0), __shfl_sync(0xFFFFFFFFu, sum, 8), __shfl_sync(0xFFFFFFFFu, sum, 16), __shfl_sync(0xFFFFFFFFu, sum, 24), mp, mq, alone_p, alone_q};
}

// A pair of rows and the tiles of it that this warp has: tile t belongs to warp t / blocks mod NW of block t mod blocks.
struct Pair {
    tiles::View draft, target;
    int64_t slot;
    uint32_t rank, blocks;
    int n_tiles, first, step;
    Sums* sums;
};
template <typename T, int NW>
__device__ __forceinline__ Pair pair_of(const DivergenceArgs& a, unsigned char* dynamic_bytes) {
    Pair w;
    w.rank = tiles::cluster_rank(), w.blocks = tiles::cluster_blocks();
    const uint32_t slot = blockIdx.x / w.blocks, sequence = slot / (uint32_t)a.R;
    const int64_t b = sequence;
    const int r = (int)(slot - sequence * (uint32_t)a.R);
    w.slot = slot;
    w.draft = tiles::view_of<T>((const T*)a.draft + b * a.draft_seq + r * a.draft_row, a.V);
    w.target = tiles::view_of<T>((const T*)a.target + b * a.target_seq + r * a.target_row, a.V);
    w.n_tiles = tiles::tiles_of<T>(a.V, kWords);
    w.first = (int)(threadIdx.x >> 5) * (int)w.blocks + (int)w.rank, w.step = NW * (int)w.blocks;
    w.sums = (Sums*)dynamic_bytes;
    return w;
}

// Both rows, read into the tiles' sums; everything else of a pair follows from what this leaves in every block's shared memory.  True: there were NaN or +inf.
template <typename T, bool ALIGNED, bool BOTH, int NW, int USE>
__device__ __forceinline__ bool read_rows(const DivergenceArgs& a, const Pair& w, Smem& sm) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    if (threadIdx.x == 0) sm.status = 0, sm.alone_p = sm.alone_q = 0;
    if (w.blocks > 1) tiles::cluster_arrive();     // (the pair's other blocks have started, and their words above are set, behind the wait below)
    else __syncthreads();
    grid_wait();
    uint4 p[kWords], q[kWords];
    auto load = [&](int t) {
        if (t >= w.n_tiles) return;
        tiles::load_tile<T, ALIGNED, kWords, USE>(p, w.draft, t, lane, a.V);
        tiles::load_tile<T, ALIGNED, kWords, USE>(q, w.target, t, lane, a.V);
    };
    load(w.first);
    if (w.blocks > 1) tiles::cluster_wait();
    bool masked = false;
#pragma unroll 1
    for (int t = w.first; t < w.n_tiles; t += w.step)
        tile_sums<T, BOTH>(p, q, a.k_draft, a.k_target, t, lane, w.blocks, w.sums, sm, masked, [&] { load(t + w.step); });
    tiles::row_barrier(w.blocks);
    if (warp == 0) {
        const Totals t = join<BOTH>(w.sums, w.n_tiles, a.k_draft, a.k_target, lane);
        if (lane == 0) {
            sm.total = t;
            if (BOTH && t.alone_p > kNegInf) sm.alone_p = max(sm.alone_p, float_to_ordered(t.alone_p));
            if (BOTH && t.alone_q > kNegInf) sm.alone_q = max(sm.alone_q, float_to_ordered(t.alone_q));
        }
    }
    __syncthreads();
    return sm.status != 0;
}

// The warp's last tile of n (negative: it has none).  Second sweeps go from there to the first one: what was read last is in L2 even where the pairs under way do not all fit.
__device__ __forceinline__ int last_tile(const Pair& w, int n) { return w.first < n ? w.first + (n - 1 - w.first) / w.step * w.step : -1; }

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
    r.kl_infinite = sm.alone_q && tiles::distance(ordered_to_float(sm.alone_q), t.mq, a.k_target) >= -126.0f;
    r.reverse_infinite = sm.alone_p && tiles::distance(ordered_to_float(sm.alone_p), t.mp, a.k_draft) >= -126.0f;
    r.log2_sp = log2f(t.sp), r.log2_sq = log2f(t.sq);
    return r;
}
__device__ __forceinline__ int status_of(const Result& r, bool bad) {
    return (bad ? RSD_ST_NAN_INPUT : 0) | (r.empty ? RSD_ST_EMPTY_ROW : 0) | (r.kl_infinite ? RSD_ST_ZERO_DRAFT_PROB : 0) | (r.reverse_infinite ? RSD_ST_ZERO_TARGET_PROB : 0);
}

// The divergences themselves in 64 bits: logarithms of sums cancel against each other.
__device__ __forceinline__ float divergence_of(float d, float s, float other) {
    return max_nan((float)(0.693147180559945309 * ((double)d / ((double)kUnit * (double)s) + log2((double)other / (double)s))), 0.0f);
}

// log2 of a row's probabilities: v k - c + off in a plain row, (v - m) k - c otherwise; off is what c loses when it is rounded.
struct LogProb {
    bool plain;
    float m, k, c, off;                            // (m is 0 in a plain row)
    __device__ __forceinline__ unsigned long long of(unsigned long long v) const { return fma_f32x2(v, tiles::both(k), tiles::both(-c)); }   // of a plain row
    __device__ __forceinline__ float at(float v) const { return tiles::distance(v, m, k, -c); }
};
__device__ __forceinline__ LogProb log_prob(float m, float k, float log2s, bool empty) {
    LogProb l;
    l.plain = tiles::plain_tile(m, k);
    l.m = l.plain || empty ? 0.0f : m, l.k = k;
    l.c = l.plain ? __fmaf_ru(m, k, log2s) : log2s;   // (rounded up: no weight is above 1, so that its product with any finite number is finite)
    l.off = l.plain ? -(fmaf(m, k, -l.c) + log2s) : 0.0f;
    return l;
}

template <typename T>
__device__ __forceinline__ float entry_of(const void* row, int x) {   // -inf where it is none
    const float v = RowIO<T>::scalar(row, x);
    return v < __builtin_huge_valf() ? v : kNegInf;
}
// The overlap's sums of this warp's tiles where a row is not plain (out of line: the kernel waits for its instructions as it is).
template <typename T>
__device__ __noinline__ void overlap_of_far_rows(const void* draft, const void* target, int first, int step, int V, LogProb p, LogProb q, Sums* sums) {
    constexpr int kTile = tiles::tile_entries<T>(kWords);
    const int lane = threadIdx.x & 31, n = tiles::tiles_of<T>(V, kWords);
    for (int t = first; t < n; t += step) {
        float s = 0.0f;
        for (int x = t * kTile + lane; x < min((t + 1) * kTile, V); x += 32)
            s += ex2_approx(fminf(p.at(entry_of<T>(draft, x)), q.at(entry_of<T>(target, x)) + (q.off - p.off)));
        s = tiles::warp_sum_two(s, 0.0f, lane);
        if (lane == 0) tiles::store_at(&sums[t].overlap, 0, s);
    }
}

template <typename T, bool ALIGNED, bool OVERLAP, int NW>
__global__ void __launch_bounds__(NW * 32, 32 / NW) divergence_kernel(const __grid_constant__ DivergenceArgs a) {
    using P = tiles::Packed16<T>;
    extern __shared__ __align__(16) unsigned char dynamic_bytes[];   // all tiles' sums
    __shared__ Smem sm;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const Pair w = pair_of<T, NW>(a, dynamic_bytes);
    const bool bad = read_rows<T, ALIGNED, true, NW, OVERLAP ? tiles::kReadFirst : tiles::kReadOnce>(a, w, sm);
    const Result res = result_of(a, sm);
    if (w.rank == 0 && tid == 0) {
        const Totals& t = sm.total;
        const float inf = __builtin_huge_valf();
        if (a.out_kl) a.out_kl[w.slot] = res.empty ? 0.0f : res.kl_infinite ? inf : divergence_of(t.dq, t.sq, t.sp);
        if (a.out_reverse) a.out_reverse[w.slot] = res.empty ? 0.0f : res.reverse_infinite ? inf : divergence_of(t.dp, t.sp, t.sq);
        a.status[w.slot] = status_of(res, bad);
    }
    if constexpr (OVERLAP) {
        const LogProb p = log_prob(sm.total.mp, a.k_draft, res.log2_sp, res.empty), q = log_prob(sm.total.mq, a.k_target, res.log2_sq, res.empty);
        const unsigned long long shift = tiles::both(q.off - p.off);
        if (!res.empty && !(p.plain && q.plain)) {
            overlap_of_far_rows<T>(w.draft.base + w.draft.first, w.target.base + w.target.first, w.first, w.step, a.V, p, q, w.sums);
        } else if (!res.empty) {
            uint4 pw[kWords], qw[kWords];
            auto load = [&](int t) {
                if (t < 0) return;
                tiles::load_tile<T, ALIGNED, kWords, tiles::kReadLast>(pw, w.draft, t, lane, a.V);
                tiles::load_tile<T, ALIGNED, kWords, tiles::kReadLast>(qw, w.target, t, lane, a.V);
            };
            const int last = last_tile(w, w.n_tiles);
            load(last);
#pragma unroll 1
            for (int t = last; t >= 0; t -= w.step) {
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
                        split_f32x2(p.of(P::pair(pw[i], j)), x, y);
                        split_f32x2(add_f32x2(q.of(P::pair(qw[i], j)), shift), u, v);
                        s = add_f32x2(s, f32x2(ex2_approx(fminf(x, u)), ex2_approx(fminf(y, v))));
                    }
                load(t - w.step);
                float x, y;
                split_f32x2(s, x, y);
                const float sum = tiles::warp_sum_two(x + y, 0.0f, lane);
                if (lane == 0) tiles::store_at(&w.sums[t].overlap, 0, sum);
            }
        }
        tiles::row_barrier(w.blocks);
        if (w.rank == 0 && warp == 0) {
            float s = 0.0f;
            for (int t = lane; t < w.n_tiles; t += 32) s += w.sums[t].overlap;
            s = tiles::warp_sum_two(s, 0.0f, lane);
            if (lane == 0) a.out_overlap[w.slot] = res.empty ? 0.0f : min_nan(s * ex2_approx(p.off), 1.0f);
        }
    }
    grid_started();
}

// The gradient of rows that are not plain, or where products of weights and factors might leave fp32's range, in 64 bits: a weight of 0 makes every finite factor 0, and
// factors that are not finite reach every entry.
struct WideSlope {
    LogProb p, q;
    double g, h, scale_p, scale_q, mean;           // weights over the temperature
};
template <typename T, bool REVERSE>
__device__ __noinline__ void write_wide(const void* draft, const void* target, void* grad, int first, int step, int V, WideSlope f) {
    for (int i = first; i < V; i += step) {
        float x = f.p.at(entry_of<T>(draft, i)), u = f.q.at(entry_of<T>(target, i));
        const double wp = (double)ex2_approx(x) * f.scale_p, wq = (double)ex2_approx(u) * f.scale_q;
        double slope = (wp - wq) * f.g;
        if (REVERSE) {
            x = fmaxf(x, tiles::kLowest), u = fmaxf(u, tiles::kLowest);
            slope += wp * f.h * 0.693147180559945309 * ((double)x - (double)u + ((double)f.p.off - (double)f.q.off) - f.mean);
        }
        tiles::Packed16<T>::store(grad, i, (float)slope);
    }
}

// d KL(q||p) / dv_x = (p_x - q_x) / T,   d KL(p||q) / dv_x = p_x (log p_x - log q_x - KL(p||q)) / T,   v the draft row, T its temperature.
// A row whose KL(p||q) is infinite has no gradient of it.  Words of the gradient are written on their own 16-byte boundaries.
//
// 4096 pairs of 32,000 bf16, KL(q||p): 180 us back to back (167 below the power limit; floor 120): four exponentials a pair of entries, the special-function unit 73 % busy.  (A quarter of the second sweep's exponentials by a
// polynomial on the multiplying pipe: 2 % faster with KL(q||p) alone, 3 % slower with both.)  fp32 pairs are bound by memory: where the pairs under way do not stay in L2 beside the
// gradient's words they are read twice (7000 pairs of 32,000: 535 us, floor 410; 192 of 128,000 with both divergences 77, floor 45).
template <typename T, bool ALIGNED, bool REVERSE, int NW>
__global__ void __launch_bounds__(NW * 32, 24 / NW) divergence_grad_kernel(const __grid_constant__ DivergenceArgs a) {
    using P = tiles::Packed16<T>;
    constexpr int E = P::kEntries, kTile = tiles::tile_entries<T>(kWords);
    extern __shared__ __align__(16) unsigned char dynamic_bytes[];   // all tiles' sums
    __shared__ Smem sm;
    const int tid = threadIdx.x, lane = tid & 31;
    const Pair w = pair_of<T, NW>(a, dynamic_bytes);
    const bool bad = read_rows<T, ALIGNED, REVERSE, NW, tiles::kReadFirst>(a, w, sm);
    const float g = a.g_kl ? a.g_kl[w.slot] : 0.0f, h = REVERSE ? a.g_reverse[w.slot] : 0.0f;
    const Result res = result_of(a, sm);
    const float gt = res.empty ? 0.0f : g * a.inv_draft_temp, ht = res.empty || (REVERSE && res.reverse_infinite) ? 0.0f : h * a.inv_draft_temp;
    // p = 2^x scale_p with x relative to the row's largest entry, q = 2^u scale_q alike; then  ln p - ln q - KL(p||q) = ln 2 (x - u - sum p (x - u)),  where no term is as large as ln V.
    // Rows that are equal give 0.
    const LogProb lp = log_prob(sm.total.mp, a.k_draft, 0.0f, res.empty), lq = log_prob(sm.total.mq, a.k_target, 0.0f, res.empty);
    const float scale_p = ex2_approx(lp.off) / sm.total.sp, scale_q = ex2_approx(lq.off) / sm.total.sq;
    const float mean = REVERSE && ht != 0.0f ? sm.total.dp / sm.total.sp * (1.0f / kUnit) : 0.0f;
    const float c1f = ht * 0.69314718f * scale_p, c0f = c1f * (lp.off - lq.off - mean), cgf = gt * scale_p;
    char* const grad = (char*)a.grad + w.slot * a.V * (int64_t)sizeof(T);
    const int head = ALIGNED ? 0 : (int)((uintptr_t)grad & 15u) / (int)sizeof(T);   // entries between the boundary and the gradient's first one
    auto finish = [&] {
        if (w.rank == 0 && tid == 0) {
            Result said = res;
            said.kl_infinite = false;                               // (its gradient is finite)
            if (!REVERSE) said.reverse_infinite = false;
            a.status[w.slot] = status_of(said, bad);
        }
        grid_started();
    };
    if (!res.empty && !(lp.plain && lq.plain && tiles::ordinary_factor(c0f) && tiles::ordinary_factor(c1f) && tiles::ordinary_factor(cgf))) {
        WideSlope f;
        f.p = lp, f.q = lq;
        f.g = (double)g * (double)a.inv_draft_temp, f.h = ht == 0.0f ? 0.0 : (double)h * (double)a.inv_draft_temp;
        f.scale_p = (double)scale_p, f.scale_q = (double)scale_q, f.mean = (double)mean;
        const int threads = NW * 32;
        write_wide<T, REVERSE>(w.draft.base + w.draft.first, w.target.base + w.target.first, grad, (int)w.rank * threads + tid, (int)w.blocks * threads, a.V, f);
        finish();
        return;
    }
    const unsigned long long c0 = tiles::both(c0f), c1 = tiles::both(c1f), cg = tiles::both(cgf), minus_ratio = tiles::both(-scale_q / scale_p), minus_one = tiles::both(-1.0f);
    auto word = [&](const uint4& pw, const uint4& qw) {
        return P::make([&](int i) {
            float x, y, u, v;
            split_f32x2(lp.of(P::pair(pw, i)), x, y);
            split_f32x2(lq.of(P::pair(qw, i)), u, v);
            const unsigned long long wp = f32x2(ex2_approx(x), ex2_approx(y)), wq = f32x2(ex2_approx(u), ex2_approx(v));
            const unsigned long long apart = tiles::mul_f32x2(fma_f32x2(wq, minus_ratio, wp), cg);
            if (!REVERSE) return apart;
            x = fmaxf(x, tiles::kLowest), y = fmaxf(y, tiles::kLowest), u = fmaxf(u, tiles::kLowest), v = fmaxf(v, tiles::kLowest);
            // (the weight first: the target's logarithm may be as low as it likes where the draft has mass, and is of no account where it has none)
            const unsigned long long far = tiles::mul_f32x2(wp, fma_f32x2(f32x2(u, v), minus_one, f32x2(x, y)));
            return fma_f32x2(far, c1, fma_f32x2(wp, c0, apart));
        });
    };
    // tiles of the gradient: `head` entries ahead of the rows'
#pragma unroll 1
    for (int t = last_tile(w, tiles::tiles_of<T>(head + a.V, kWords)); t >= 0; t -= w.step) {
        const int x = t * kTile - head + lane * E;
        char* const to = grad + (int64_t)x * (int)sizeof(T);
        const bool whole = t * kTile >= head && (t + 1) * kTile - head <= a.V;
        uint4 pw[kWords], qw[kWords];
        tiles::load_words<T, ALIGNED, kWords, tiles::kReadLast>(pw, w.draft, x, whole, a.V);
        tiles::load_words<T, ALIGNED, kWords, tiles::kReadLast>(qw, w.target, x, whole, a.V);
        if (bad) {
            bool ignored = false;
#pragma unroll
            for (int k = 0; k < kWords; ++k) P::clean(pw[k], ignored), P::clean(qw[k], ignored);
        }
#pragma unroll
        for (int k = 0; k < kWords; ++k) {
            const int at = x + k * 32 * E;
            if (!whole && (at >= a.V || at + E <= 0)) continue;
            uint4 out = word(pw[k], qw[k]);
            if (res.empty) out = make_uint4(0, 0, 0, 0);
            if (whole || (at >= 0 && at + E <= a.V)) {
                __stcs((uint4*)(to + k * 512), out);
            } else {
                for (int i = 0; i < E; ++i)
                    if (at + i >= 0 && at + i < a.V) P::store(grad, at + i, P::get(out, i));
            }
        }
    }
    finish();
}

}  // namespace divergence
}  // namespace rsd
