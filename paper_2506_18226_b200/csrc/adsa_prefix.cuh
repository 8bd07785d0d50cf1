// What the kernels of adsa_shared_prefix_attn share: their arguments, lengths and groups as the device finds them, copies.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>
#include <type_traits>

#include "adsa_async.cuh"
#include "adsa_half.cuh"

namespace adsa {

constexpr int kWideQueries = 256;           // query rows of an item of the wide kernel: 128 for each of its two groups
constexpr int kWideTile = 128;              // cached rows of a unit of the wide kernel

struct PrefixArgs {
    const void *q, *k_pool, *v_pool;
    long long q_row, q_head;                // element strides of q
    const int32_t *table, *n_rows;          // [batch][max_pages], [batch]
    const int32_t *p_table, *p_rows, *start;   // [groups][max_p_pages], [groups], [groups + 1]
    uint32_t *status;
    int batch, groups, kv_heads, per_kv;    // per_kv: query heads of a key head
    int max_pages, max_p_pages, page_rows, n_pages, box_rows;
    int d, row_stride;
    float scale_log2e;
    void *out;                              // 16-bit, or null
    float *out_f32, *lse;                   // or null
    // workspace
    uint4 *plan;                            // [batch][3] for the merge: {first own unit, tiles, units, group's first slot}, {group's first unit,
                                            // tiles, first batch row, query rows}, {units of the wide kernel}
    float *p_state, *p_ml, *o_state, *o_ml; // prefix slots, own-row slots: rows of d_pad floats, (m, l) pairs
    int n_p_slots, n_o_slots;
    // groups with more query rows per key head than this go to the wide kernel, with a plan and slots of its own
    int wide_above;
    float *w_state, *w_ml;                  // slots of kWideQueries rows
    int n_w_slots, w_resident;              // w_resident: blocks of the wide kernel that fit the GPU at a time; 0: it does not run
    int resident;                           // blocks of the sweep kernel that the cut counts on at a time: two per SM, one for rows of
                                            // more than 128 elements (with over some 2000 batch rows + twice the groups the plan
                                            // leaves room for one: runs then start later, with the same results)
    int split;                              // blocks of a cluster, which share an item's cached rows (1: no cluster)
};

__device__ __forceinline__ int clamp_rows(int n, int max_pages, int page_rows)
{
    const long long most = (long long)max_pages * page_rows;
    return n < 0 ? 0 : n > most ? (int)most : n;
}
__device__ __forceinline__ int group_begin(const PrefixArgs &a, int g) { return min(max(a.start[g], 0), a.batch); }
__device__ __forceinline__ int group_members(const PrefixArgs &a, int g) { return max(group_begin(a, g + 1) - group_begin(a, g), 0); }

// A number no larger item of an earlier group reaches, with items of `queries` rows: the sum of ceil(rows / queries) over
// groups 0 .. g-1 is at most begin per_kv / queries + g
__device__ __forceinline__ int first_group_item(const PrefixArgs &a, int g, int begin, int queries)
{
    return (int)(((long long)begin * a.per_kv / queries + g) * a.kv_heads);
}

__device__ __forceinline__ void pa_tma(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar) : "memory");
}

__device__ __forceinline__ float pa_exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}

// P enters the second product as two 16-bit values, hi + lo: one would round every weight to 8 (11) bits, and the output with
// it (rms error against 64 bits 0.0018 .. 0.0023 where rounding the output alone costs 0.0016).  P lies in 0 .. 1 relative to the running
// maximum; the half type has a fixed step below 2^-14, so there P is scaled by 2^8 (it cancels in o / l; the states carry it in m).
template <typename T> struct WeightBias { static constexpr float value = 0.f; };
template <> struct WeightBias<__half> { static constexpr float value = 8.f; };

// Two weights (>= 0) as hi, cut to the type's bits, and lo, what that leaves, rounded: together 16 bits of a weight for bfloat16, 22 for
// half.  Neither is below zero, and lo is above it wherever hi is, so that an infinity of V under a weight stays that infinity in the
// sum of both products: for bfloat16 lo takes 2^-23 of the weight more; the half type cannot hold that, so there lo is its least number
// at least (2^-24, which is 2^-30 .. 2^-32 of the largest weight).
template <typename T> struct WeightSplit { static constexpr uint32_t kept = 0xffff0000u; static constexpr float one = 1.f + 1.f / 8388608.f; };
template <> struct WeightSplit<__half> { static constexpr uint32_t kept = 0xffffe000u; static constexpr float one = 1.f; };
__device__ __forceinline__ uint32_t above_zero(uint32_t lo, uint32_t hi)
{
    const uint32_t least = 0x00010001u;
    const __half2 x = __hmax2(reinterpret_cast<const __half2 &>(lo), __hmin2(reinterpret_cast<const __half2 &>(hi), reinterpret_cast<const __half2 &>(least)));
    return reinterpret_cast<const uint32_t &>(x);
}
__device__ __forceinline__ float weight_bits(float p, uint32_t kept, uint32_t sign) { return __uint_as_float((__float_as_uint(p) & kept) ^ sign); }
template <typename T>
__device__ __forceinline__ void split_weights(float2 p, uint32_t &hi, uint32_t &lo)
{
    typedef WeightSplit<T> S;
    const float hx = weight_bits(p.x, S::kept, 0u), hy = weight_bits(p.y, S::kept, 0u);
    lo = pack2<T>(fmaf(p.x, S::one, -hx), fmaf(p.y, S::one, -hy));
    if constexpr (std::is_same<T, __half>::value) {
        hi = pack2<T>(hx, hy);
        lo = above_zero(lo, hi);
    } else {
        hi = __byte_perm(__float_as_uint(p.x), __float_as_uint(p.y), 0x7632);
    }
}
// The same where a lane wants one of the two: hi (whole = 0, sign = 0) or lo (whole = WeightSplit<T>::one, sign = 0x80000000).
template <typename T>
__device__ __forceinline__ uint32_t weights_of_lane(float2 p, float whole, uint32_t sign)
{
    typedef WeightSplit<T> S;
    const float2 x = fma2(p, make_float2(whole, whole), make_float2(weight_bits(p.x, S::kept, sign), weight_bits(p.y, S::kept, sign)));
    const uint32_t w = pack2<T>(x.x, x.y);
    if constexpr (std::is_same<T, __half>::value) return above_zero(w, pack2<T>(p.x, p.y));
    else return w;
}

// How a list of units is cut into runs: `resident` runs of 2^(K-2) pieces, as many of half that, .. of one piece, and
// as many of one piece again (K = 1: a run a block).  Blocks that are quick take more of the shrinking runs, and all end
// within a short one.  A piece has at least four units, as a run costs about two (its state, its first queries); K is at
// most 5.
struct Cut {
    uint32_t resident, runs, half, base, rem;   // half = 2^(K-1); piece p begins at unit p base + min(p, rem)
    __device__ __forceinline__ Cut(uint32_t total, uint32_t resident_) : resident(resident_)
    {
        const uint32_t fours = min(total / (4u * resident), 16u);
        const uint32_t K = fours < 2u ? 1u : 32u - __clz(fours);
        half = 1u << (K - 1u);
        uint32_t pieces = half * resident;
        runs = K * resident;
        if (total < resident) pieces = runs = max(total, 1u);
        base = total / pieces;
        rem = total - base * pieces;
        if (total == 0u) runs = 0u;
    }
    __device__ __forceinline__ uint32_t begin_of(uint32_t run) const
    {
        uint32_t p = run;
        if (half > 1u) {
            const uint32_t k = run / resident;
            p = (half - (half >> k)) * resident + (run - k * resident) * max(1u, half >> (k + 1u));
            p = min(p, half * resident);
        }
        return p * base + min(p, rem);
    }
    __device__ __forceinline__ uint32_t run_of(uint32_t unit) const
    {
        const uint32_t big = rem * (base + 1u), p = unit < big ? unit / (base + 1u) : rem + (unit - big) / max(base, 1u);
        if (half == 1u) return min(p, runs - 1u);
        const uint32_t left = half - p / resident;       // half >> (k+1) < left <= half >> k
        const uint32_t k = 31u - __clz(half) - (32u - __clz(left - 1u));
        return min(k * resident + (p - (half - (half >> k)) * resident) / max(1u, half >> (k + 1u)), runs - 1u);
    }
};

// Items of a key head in the wide kernel's list: 256 query rows each, two units a tile; the last one, if it has 128 rows or
// fewer, one unit a tile.
struct WideItems {
    int items;
    uint32_t tiles, head_units;
    __device__ __forceinline__ WideItems(int m, int n) : items((m + kWideQueries - 1) / kWideQueries), tiles((uint32_t)(n + kWideTile - 1) / kWideTile)
    {
        head_units = (uint32_t)(m + 127) / 128u * tiles;
    }
};
// Even runs of the wide kernel's list: one per block, two units or more (so the first unit of a tile).  (Leaving out blocks so
// that no run goes over the end of an item changed nothing: the sweep of the own rows begins where the other blocks have ended.)
struct WideCut {
    uint32_t total, runs;
    __device__ __forceinline__ WideCut(uint32_t total_, uint32_t resident) : total(total_), runs(min(resident, total_ / 2u))
    {
        if (total > 0u && runs == 0u) runs = 1u;
    }
    __device__ __forceinline__ uint32_t begin_of(uint32_t run) const { return (uint32_t)((unsigned long long)run * total / runs); }
    __device__ __forceinline__ uint32_t run_of(uint32_t unit) const { return (uint32_t)((((unsigned long long)unit + 1u) * runs - 1u) / total); }
};

cudaError_t launch_prefix_wide(int dtype, int nsub, const PrefixArgs &a, const CUtensorMap &km, const CUtensorMap &vm, cudaStream_t st);

}  // namespace adsa
