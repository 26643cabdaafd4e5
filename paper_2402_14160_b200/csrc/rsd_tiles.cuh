// Rows dealt out in tiles to warps: what the kernels that score rows share.
//
// A tile is KW words of 16 bytes per lane: word k of lane l of tile t holds the entries that start at ((t KW + k) 32 + l) E of the row, E entries a word.
// Everything that is summed is summed per tile, relative to the tile's own maximum, by one warp in a fixed order, and the tiles' sums
// are joined in the order of the tiles.  So a row gives the same bits whatever the number of warps or blocks that share it, the rows beside it
// and the address that it starts at.
#pragma once
#include <type_traits>

#include "rsd_device.cuh"
#include "rsd_scan.cuh"   // ex2_approx, packed arithmetic

namespace rsd {
namespace tiles {

// A row as 16-byte granules from the one that holds its first entry (an allocation holds whole granules, so that what lies around the row in its first and last
// granule may be read; it is masked).
struct View {
    const char* base;     // 16-byte aligned
    int first;            // bytes from base to the first entry
    int last;             // index of the granule that holds the last entry
};
template <typename T>
__device__ __forceinline__ View view_of(const void* row, int V) {
    const int first = (int)((uintptr_t)row & 15u);
    return {(const char*)row - first, first, (first + V * (int)sizeof(T) - 1) >> 4};
}

// bytes shift .. shift + 15 of two adjacent granules, shift = 4 Q + bits / 8
template <int Q>
__device__ __forceinline__ uint4 shifted(const uint4& a, const uint4& b, int bits) {
    const uint32_t w[8] = {a.x, a.y, a.z, a.w, b.x, b.y, b.z, b.w};
    return make_uint4(__funnelshift_r(w[Q], w[Q + 1], bits), __funnelshift_r(w[Q + 1], w[Q + 2], bits), __funnelshift_r(w[Q + 2], w[Q + 3], bits),
                      __funnelshift_r(w[Q + 3], w[(Q + 4) & 7], bits));
}
// f(Q) for a shift that is the same for all threads
template <typename F>
__device__ __forceinline__ void with_shift(int shift, F f) {
    switch (shift >> 2) {
        case 0: f(std::integral_constant<int, 0>()); break;
        case 1: f(std::integral_constant<int, 1>()); break;
        case 2: f(std::integral_constant<int, 2>()); break;
        default: f(std::integral_constant<int, 3>()); break;
    }
}

// Entries are raised to this where 0 times -inf would not be a number: their weight stays 0.  Plain arithmetic holds where a tile's largest entry is far above it
// and the exponents' scale keeps it finite, and where the product of both is so small that it loses no more than half when it is rounded (see plain_tile).
// (kLeastScale: below it an entry of kLow would have a weight.)
constexpr float kLow = -1e30f, kPlainProduct = 16777216.0f, kPlainScale = 1e6f, kLeastScale = 1e-20f;

template <typename T>
struct Packed16;   // one word as entries

template <>
struct Packed16<float> {
    static constexpr int kEntries = 4;
    static constexpr uint32_t kMasked = 0xFF800000u;
    __device__ static __forceinline__ float get(const uint4& w, int i) { return __uint_as_float(i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w); }
    // entries outside [from, to) become -inf
    __device__ static __forceinline__ void keep(uint4& w, int from, int to) {
        if (from > 0 || to < 1) w.x = kMasked;
        if (from > 1 || to < 2) w.y = kMasked;
        if (from > 2 || to < 3) w.z = kMasked;
        if (from > 3 || to < 4) w.w = kMasked;
    }
    __device__ static __forceinline__ uint32_t clean_entry(uint32_t u, bool& bad) {   // NaN and +inf are no entries
        const bool b = !(__uint_as_float(u) < __builtin_huge_valf());
        bad |= b;
        return b ? kMasked : u;
    }
    __device__ static __forceinline__ void clean(uint4& w, bool& bad) {
        w.x = clean_entry(w.x, bad), w.y = clean_entry(w.y, bad), w.z = clean_entry(w.z, bad), w.w = clean_entry(w.w, bad);
    }
    __device__ static __forceinline__ uint4 masked() { return make_uint4(kMasked, kMasked, kMasked, kMasked); }
    template <int KW>
    __device__ static __forceinline__ float largest(const uint4 (&w)[KW]) {   // NaN if there is one
        float a = max_nan(__uint_as_float(w[0].x), __uint_as_float(w[0].y));
        a = max_nan(a, max_nan(__uint_as_float(w[0].z), __uint_as_float(w[0].w)));
#pragma unroll
        for (int k = 1; k < KW; ++k)
            a = max_nan(a, max_nan(max_nan(__uint_as_float(w[k].x), __uint_as_float(w[k].y)), max_nan(__uint_as_float(w[k].z), __uint_as_float(w[k].w))));
        return a;
    }
    __device__ static __forceinline__ uint32_t raised_entry(uint32_t u) { return __float_as_uint(fmaxf(__uint_as_float(u), kLow)); }
    __device__ static __forceinline__ uint4 raised(const uint4& w) { return make_uint4(raised_entry(w.x), raised_entry(w.y), raised_entry(w.z), raised_entry(w.w)); }
    // whether one of two words has an entry above kLow where the other has none
    __device__ static __forceinline__ bool differ(uint32_t a, uint32_t b) { return (__uint_as_float(a) > kLow) != (__uint_as_float(b) > kLow); }
    __device__ static __forceinline__ bool differ(const uint4& a, const uint4& b) { return differ(a.x, b.x) | differ(a.y, b.y) | differ(a.z, b.z) | differ(a.w, b.w); }
    // f(pair of entries) for the pairs of a word
    template <typename F>
    __device__ static __forceinline__ void pairs(const uint4& w, F f) {
        f(f32x2(__uint_as_float(w.x), __uint_as_float(w.y)));
        f(f32x2(__uint_as_float(w.z), __uint_as_float(w.w)));
    }
    // a word from its entries
    template <typename F>
    __device__ static __forceinline__ uint4 make(F f) {
        float a[4];
#pragma unroll
        for (int i = 0; i < 2; ++i) split_f32x2(f(i), a[2 * i], a[2 * i + 1]);
        return make_uint4(__float_as_uint(a[0]), __float_as_uint(a[1]), __float_as_uint(a[2]), __float_as_uint(a[3]));
    }
    __device__ static __forceinline__ unsigned long long pair(const uint4& w, int i) {
        return i == 0 ? f32x2(__uint_as_float(w.x), __uint_as_float(w.y)) : f32x2(__uint_as_float(w.z), __uint_as_float(w.w));
    }
    __device__ static __forceinline__ void store(void* row, int x, float v) { ((float*)row)[x] = v; }
};

template <>
struct Packed16<__nv_bfloat16> {
    static constexpr int kEntries = 8;
    static constexpr uint32_t kMasked = 0xFF80FF80u;
    __device__ static __forceinline__ float get(const uint4& w, int i) {
        const uint32_t u = (i >> 1) == 0 ? w.x : (i >> 1) == 1 ? w.y : (i >> 1) == 2 ? w.z : w.w;
        return __uint_as_float((i & 1) ? (u & 0xFFFF0000u) : (u << 16));
    }
    __device__ static __forceinline__ uint32_t keep_entry(uint32_t u, int i, int from, int to) {
        if (from > i || to <= i) u = (u & 0xFFFF0000u) | 0xFF80u;
        if (from > i + 1 || to <= i + 1) u = (u & 0xFFFFu) | 0xFF800000u;
        return u;
    }
    __device__ static __forceinline__ void keep(uint4& w, int from, int to) {
        w.x = keep_entry(w.x, 0, from, to), w.y = keep_entry(w.y, 2, from, to), w.z = keep_entry(w.z, 4, from, to), w.w = keep_entry(w.w, 6, from, to);
    }
    __device__ static __forceinline__ uint32_t clean_entry(uint32_t u, bool& bad) {
        const bool lo = !(__uint_as_float(u << 16) < __builtin_huge_valf()), hi = !(__uint_as_float(u & 0xFFFF0000u) < __builtin_huge_valf());
        bad |= lo | hi;
        if (lo) u = (u & 0xFFFF0000u) | 0xFF80u;
        if (hi) u = (u & 0xFFFFu) | 0xFF800000u;
        return u;
    }
    __device__ static __forceinline__ void clean(uint4& w, bool& bad) {
        w.x = clean_entry(w.x, bad), w.y = clean_entry(w.y, bad), w.z = clean_entry(w.z, bad), w.w = clean_entry(w.w, bad);
    }
    __device__ static __forceinline__ uint4 masked() { return make_uint4(kMasked, kMasked, kMasked, kMasked); }
    template <int KW>
    __device__ static __forceinline__ float largest(const uint4 (&w)[KW]) {
        uint32_t a = bf162_max_nan(bf162_max_nan(w[0].x, w[0].y), bf162_max_nan(w[0].z, w[0].w));
#pragma unroll
        for (int k = 1; k < KW; ++k) a = bf162_max_nan(a, bf162_max_nan(bf162_max_nan(w[k].x, w[k].y), bf162_max_nan(w[k].z, w[k].w)));
        return max_nan(__uint_as_float(a << 16), __uint_as_float(a & 0xFFFF0000u));
    }
    static constexpr uint32_t kLow2 = 0xF149F149u;   // kLow rounded to this type, twice
    __device__ static __forceinline__ uint32_t raised_entry(uint32_t u) {
        uint32_t r;
        asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(u), "r"(kLow2));
        return r;
    }
    __device__ static __forceinline__ uint4 raised(const uint4& w) { return make_uint4(raised_entry(w.x), raised_entry(w.y), raised_entry(w.z), raised_entry(w.w)); }
    __device__ static __forceinline__ uint32_t none(uint32_t u) {   // 0xFFFF per half without an entry above kLow
        uint32_t r;
        asm("set.le.u32.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(u), "r"(kLow2));
        return r;
    }
    __device__ static __forceinline__ bool differ(const uint4& a, const uint4& b) {
        return ((none(a.x) ^ none(b.x)) | (none(a.y) ^ none(b.y)) | (none(a.z) ^ none(b.z)) | (none(a.w) ^ none(b.w))) != 0;
    }
    __device__ static __forceinline__ unsigned long long unpack(uint32_t u) { return f32x2(__uint_as_float(u << 16), __uint_as_float(u & 0xFFFF0000u)); }
    template <typename F>
    __device__ static __forceinline__ void pairs(const uint4& w, F f) {
        f(unpack(w.x)), f(unpack(w.y)), f(unpack(w.z)), f(unpack(w.w));
    }
    __device__ static __forceinline__ uint32_t pack(unsigned long long v) {   // rounded to nearest even, once
        float lo, hi;
        split_f32x2(v, lo, hi);
        uint32_t r;
        asm("cvt.rn.bf16x2.f32 %0, %1, %2;" : "=r"(r) : "f"(hi), "f"(lo));
        return r;
    }
    template <typename F>
    __device__ static __forceinline__ uint4 make(F f) { return make_uint4(pack(f(0)), pack(f(1)), pack(f(2)), pack(f(3))); }
    __device__ static __forceinline__ unsigned long long pair(const uint4& w, int i) { return unpack(i == 0 ? w.x : i == 1 ? w.y : i == 2 ? w.z : w.w); }
    __device__ static __forceinline__ void store(void* row, int x, float v) { ((__nv_bfloat16*)row)[x] = __float2bfloat16_rn(v); }
};

__device__ __forceinline__ unsigned long long mul_f32x2(unsigned long long a, unsigned long long b) {
    unsigned long long r;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
    return r;
}
__device__ __forceinline__ unsigned long long both(float v) { return f32x2(v, v); }

template <typename T>
__host__ __device__ constexpr int tile_entries(int KW) { return KW * 32 * (16 / (int)sizeof(T)); }
template <typename T>
__host__ __device__ constexpr int tiles_of(int V, int KW) { return (V + tile_entries<T>(KW) - 1) / tile_entries<T>(KW); }

// What L2 is told about a row's words: nothing, that they are read again soon, or that they are read for the last time.  (Two sweeps over more rows than fit beside what is written:
// gradients of 7000 pairs of 32,000 bf16 319 -> 278 us, divergences of as many fp32 pairs 457 -> 375; rows read once are 4 % slower when they are to be kept, and so are rows off the boundaries.)
enum { kReadOnce = 0, kReadFirst = 1, kReadLast = 2 };
template <int USE>
__device__ __forceinline__ uint64_t l2_policy() {
    uint64_t policy;
    if (USE == kReadFirst) asm("createpolicy.fractional.L2::evict_last.b64 %0, 1.0;" : "=l"(policy));
    else asm("createpolicy.fractional.L2::evict_first.b64 %0, 1.0;" : "=l"(policy));
    return policy;
}
template <int USE>
__device__ __forceinline__ uint4 ld_use(const void* p) {
    if (USE == kReadOnce) return ld_stream(p);
    uint4 v;
    asm volatile("ld.global.nc.L1::no_allocate.L2::cache_hint.v4.u32 {%0,%1,%2,%3}, [%4], %5;"
                 : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w)
                 : "l"(p), "l"(l2_policy<USE>()));
    return v;
}
// The word that starts at entry x0 (which may lie before or behind the row), entries outside the row as -inf.
// ALIGNED: x0 lies on a 16-byte boundary.
template <typename T, bool ALIGNED>
__device__ __forceinline__ uint4 load_word(const View& v, int x0, int V) {
    constexpr int E = Packed16<T>::kEntries;
    if (x0 >= V || x0 + E <= 0) return Packed16<T>::masked();
    const int at = v.first + x0 * (int)sizeof(T), g = at >> 4, shift = at & 15;
    uint4 w = make_uint4(0, 0, 0, 0);
    if (ALIGNED || shift == 0) {
        w = ld_stream(v.base + (int64_t)g * 16);
    } else {
        uint4 b = w;
        if (g >= 0) w = ld_shared_word(v.base + (int64_t)g * 16);
        if (g < v.last) b = ld_shared_word(v.base + (int64_t)(g + 1) * 16);
        with_shift(shift, [&](auto q) { w = shifted<decltype(q)::value>(w, b, (shift & 3) * 8); });
    }
    if (x0 < 0 || x0 + E > V) Packed16<T>::keep(w, -x0, V - x0);
    return w;
}

// KW words of a lane, 32 words apart, from entry x0 on
template <typename T, bool ALIGNED, int KW, int USE = kReadOnce>
__device__ __forceinline__ void load_words(uint4 (&w)[KW], const View& v, int x0, bool whole, int V) {   // whole: every word of the warp lies in the row
    constexpr int E = Packed16<T>::kEntries;
    if (whole) {
        const int at = v.first + x0 * (int)sizeof(T), shift = at & 15;
        const char* p = v.base + (at & ~15);
        if (ALIGNED || shift == 0) {
#pragma unroll
            for (int k = 0; k < KW; ++k) w[k] = ld_use<ALIGNED ? USE : kReadOnce>(p + k * 512);
        } else {                                   // (the word's last entry lies in the second granule)
            with_shift(shift, [&](auto q) {
#pragma unroll
                for (int k = 0; k < KW; ++k) w[k] = shifted<decltype(q)::value>(ld_shared_word(p + k * 512), ld_shared_word(p + k * 512 + 16), (shift & 3) * 8);
            });
        }
    } else {
#pragma unroll
        for (int k = 0; k < KW; ++k) w[k] = load_word<T, ALIGNED>(v, x0 + k * 32 * E, V);
    }
}
template <typename T, bool ALIGNED, int KW, int USE = kReadOnce>
__device__ __forceinline__ void load_tile(uint4 (&w)[KW], const View& v, int t, int lane, int V) {
    load_words<T, ALIGNED, KW, USE>(w, v, t * tile_entries<T>(KW) + lane * Packed16<T>::kEntries, (t + 1) * tile_entries<T>(KW) <= V, V);
}

// ---- tiles held in shared memory ---------------------------------------------------------------------------------------------------
// A held tile is KW * 32 granules of the row and, so that a row off the boundaries can be shifted, the first granule of the next tile.  The copies go on without
// registers: a block asks for all its tiles at once and a warp waits for its own.
template <int KW>
constexpr int kHeldTile = KW * 512 + 16;
__device__ __forceinline__ void copy_granule(uint32_t to, const char* from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_sent() { asm volatile("cp.async.commit_group;" ::: "memory"); }
__device__ __forceinline__ void copies_landed(int later) {   // all but (at most) the last `later` groups of this thread
    if (later >= 3) asm volatile("cp.async.wait_group 3;" ::: "memory");
    else if (later == 2) asm volatile("cp.async.wait_group 2;" ::: "memory");
    else if (later == 1) asm volatile("cp.async.wait_group 1;" ::: "memory");
    else asm volatile("cp.async.wait_group 0;" ::: "memory");
}
template <bool ALIGNED, int KW>
__device__ __forceinline__ void fetch_tile(uint32_t to, const View& v, int t, int lane) {
    const int g = t * KW * 32 + lane;
    const char* from = v.base + (int64_t)g * 16;
    if ((t + 1) * KW * 32 <= v.last) {
#pragma unroll
        for (int k = 0; k < KW; ++k) copy_granule(to + (k * 32 + lane) * 16, from + k * 512);
        if (!ALIGNED && lane == 0) copy_granule(to + KW * 512, from + KW * 512);
    } else {
#pragma unroll
        for (int k = 0; k < KW; ++k)
            if (g + k * 32 <= v.last) copy_granule(to + (k * 32 + lane) * 16, from + k * 512);
    }
}
__device__ __forceinline__ uint4 held_granule(uint32_t at) {
    uint4 w;
    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "r"(at) : "memory");
    return w;
}
// The words of a held tile, entries outside the row as -inf.  (The warp's copies have landed for all its lanes.)
template <typename T, bool ALIGNED, int KW>
__device__ __forceinline__ void read_tile(uint4 (&w)[KW], uint32_t at, const View& v, int t, int lane, int V) {
    constexpr int E = Packed16<T>::kEntries;
    at += lane * 16;
#pragma unroll
    for (int k = 0; k < KW; ++k) w[k] = held_granule(at + k * 512);
    if (!ALIGNED && v.first) {
        with_shift(v.first, [&](auto q) {
#pragma unroll
            for (int k = 0; k < KW; ++k) w[k] = shifted<decltype(q)::value>(w[k], held_granule(at + k * 512 + 16), (v.first & 3) * 8);
        });
    }
    if ((t + 1) * tile_entries<T>(KW) > V) {
#pragma unroll
        for (int k = 0; k < KW; ++k) {
            const int x0 = ((t * KW + k) * 32 + lane) * E;
            if (x0 >= V) w[k] = Packed16<T>::masked();
            else if (x0 + E > V) Packed16<T>::keep(w[k], 0, V - x0);
        }
    }
}
// Tiles t0 .. t1 - 1 of a row as a block holds them, read by words of another boundary: KW words of a lane, 32 words apart, from entry x0 on, where x0 lies
// `shift` bytes behind a granule.  Entries outside the row are undefined.
template <typename T, bool ALIGNED, int KW>
__device__ __forceinline__ void held_words(uint4 (&w)[KW], uint32_t held, const View& v, int t0, int t1, int x0, int V) {
    constexpr int kPerTile = KW * 32;
    const int at = v.first + x0 * (int)sizeof(T), shift = at & 15, local = (at >> 4) - t0 * kPerTile;   // granule of the block
    const int last = (t1 - t0) * kPerTile + (shift == 0 ? -1 : 0) - (KW - 1) * 32;                    // (the granule behind a tile's last one is held with it)
    if (ALIGNED || (local >= 0 && local <= last - 1)) {
        constexpr int kGap = kHeldTile<KW> - kPerTile * 16;
        const uint32_t a = held + local * 16 + local / kPerTile * kGap;
        if (ALIGNED || shift == 0) {
            // words of one tile, or of two where the lane's words cross into the next one
            const int inside = local % kPerTile;
#pragma unroll
            for (int k = 0; k < KW; ++k) w[k] = held_granule(a + k * 512 + (ALIGNED || inside + k * 32 < kPerTile ? 0 : kGap));
        } else {
            const int inside = local % kPerTile;
            with_shift(shift, [&](auto q) {
#pragma unroll
                for (int k = 0; k < KW; ++k) {
                    const uint32_t b = a + k * 512 + (inside + k * 32 < kPerTile ? 0 : kGap);
                    w[k] = shifted<decltype(q)::value>(held_granule(b), held_granule(b + 16), (shift & 3) * 8);
                }
            });
        }
    } else {                                       // some of them another block's
#pragma unroll
        for (int k = 0; k < KW; ++k) w[k] = load_word<T, ALIGNED>(v, x0 + k * 32 * Packed16<T>::kEntries, V);
    }
}

// ---- a row's blocks: one, or a cluster of up to eight that deal out its tiles -----------------------------------------------------------------
constexpr int kMaxBlocks = 8;
__device__ __forceinline__ uint32_t cluster_rank() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_ctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t cluster_blocks() {
    uint32_t r;
    asm("mov.u32 %0, %%cluster_nctarank;" : "=r"(r));
    return r;
}
__device__ __forceinline__ uint32_t remote(const void* p, uint32_t rank) {   // the same place in another block's shared memory
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(smem_u32(p)), "r"(rank));
    return r;
}
__device__ __forceinline__ void store_at(float* p, uint32_t rank, float v) { asm volatile("st.shared::cluster.f32 [%0], %1;" ::"r"(remote(p, rank)), "f"(v) : "memory"); }
__device__ __forceinline__ void store_at(int* p, uint32_t rank, int v) { asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(remote(p, rank)), "r"(v) : "memory"); }
__device__ __forceinline__ void store_at(unsigned long long* p, uint32_t rank, unsigned long long v) {
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(remote(p, rank)), "l"(v) : "memory");
}
__device__ __forceinline__ void or_at(int* p, uint32_t rank, int v) { asm volatile("red.shared::cluster.or.b32 [%0], %1;" ::"r"(remote(p, rank)), "r"(v) : "memory"); }
__device__ __forceinline__ void max_at(uint32_t* p, uint32_t rank, uint32_t v) { asm volatile("red.shared::cluster.max.u32 [%0], %1;" ::"r"(remote(p, rank)), "r"(v) : "memory"); }
__device__ __forceinline__ int add_at(int* p, uint32_t rank, int v) {
    int r;
    asm volatile("atom.shared::cluster.add.u32 %0, [%1], %2;" : "=r"(r) : "r"(remote(p, rank)), "r"(v) : "memory");
    return r;
}
__device__ __forceinline__ void cluster_arrive() { asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory"); }
__device__ __forceinline__ void cluster_wait() { asm volatile("barrier.cluster.wait.acquire.aligned;" ::: "memory"); }
// Every thread of the row's blocks; what they wrote before is visible behind it.
__device__ __forceinline__ void row_barrier(uint32_t blocks) {
    if (blocks > 1) {
        cluster_arrive();
        cluster_wait();
    } else {
        __syncthreads();
    }
}

__device__ __forceinline__ float warp_max_nan(float v) {   // NaN if any lane has one
    float r;
    asm volatile("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(r) : "f"(v));
    return r;
}

// Two sums over the warp at once, in an order of their own: the first in lanes 0 to 15, the second in the others.
__device__ __forceinline__ float warp_sum_two(float a, float b, int lane) {
    const bool high = lane & 16;
    float mine = high ? b : a;
    const float other = high ? a : b;
    mine += __shfl_xor_sync(0xFFFFFFFFu, other, 16);
#pragma unroll
    for (int o = 8; o > 0; o >>= 1) mine += __shfl_xor_sync(0xFFFFFFFFu, mine, o);
    return mine;
}
// Four sums: lanes 0 to 7, 8 to 15, 16 to 23, 24 to 31.
__device__ __forceinline__ float warp_sum_four(float a, float b, float c, float d, int lane) {
    const bool high = lane & 16, second = lane & 8;
    float p = high ? c : a, q = high ? d : b;
    p += __shfl_xor_sync(0xFFFFFFFFu, high ? a : c, 16);
    q += __shfl_xor_sync(0xFFFFFFFFu, high ? b : d, 16);
    float mine = second ? q : p;
    mine += __shfl_xor_sync(0xFFFFFFFFu, second ? p : q, 8);
#pragma unroll
    for (int o = 4; o > 0; o >>= 1) mine += __shfl_xor_sync(0xFFFFFFFFu, mine, o);
    return mine;
}

// (v - m) k + c.  The difference of two entries may leave fp32's range where its product with k < 1 does not: halves are subtracted there (the same bits otherwise).
__device__ __forceinline__ float part_of(float k) { return k < 1.0f ? 0.5f : 1.0f; }
__device__ __forceinline__ float scale_of_part(float k) { return k < 1.0f ? 2.0f * k : k; }
__device__ __forceinline__ float distance(float v, float m, float k, float c = 0.0f) {
    const float part = part_of(k);
    return fmaf(fmaf(v, part, -m * part), scale_of_part(k), c);
}

// Exponents below this give weights of 0 and may be replaced by it; kLowest: the lowest finite one, where the exponent itself counts.
constexpr float kFarBelow = -1e30f, kLowest = -3.402823466e38f;
// The same where an exponent is multiplied by a gradient's factor of at most kMostFactor: their product stays finite, so that a weight of 0 makes it 0.  Rows with larger factors, and
// with factors that are not finite, are written in 64 bits.
constexpr float kNoWeight = -1e4f, kMostFactor = 1e33f;
__device__ __forceinline__ bool ordinary_factor(float v) { return fabsf(v) <= kMostFactor; }   // (NaN is none)

// What m k loses when it is rounded: plain tiles take their weights relative to the rounded m k, the others to m k itself (m subtracted first).  Half a step of m k is 0.5 at
// the most below 2^24, so that a plain tile's weights reach 2^0.5; at 2^31 it would be 64, and the largest weight infinite or 0.
__device__ __forceinline__ bool plain_tile(float m, float k) { return fabsf(m) * k < kPlainProduct && k < kPlainScale && k > kLeastScale; }
__device__ __forceinline__ float rounded_off(float m, float k) { return plain_tile(m, k) ? fmaf(m, k, -(m * k)) : 0.0f; }

}  // namespace tiles
}  // namespace rsd
