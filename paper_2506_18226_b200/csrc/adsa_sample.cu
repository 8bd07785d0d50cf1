// The draw of the next token: temperature, the top_k largest logits, the smallest head of them that holds top_p of their mass,
// weights of min_p of the largest at least, and one of what is left by a given uniform number.
//
// All three rules keep a head of the ids in the order (logit descending, id ascending), so what is kept is one border: a key and how
// many of the ids with just that logit.  Keys are the logits' bits in an order that integers have.  Weights are made in 64 bits and added up
// as whole multiples of 2^-42 of the largest (2^20 of them fit 63 bits): sums do not depend on their order.  One of n weights is off by n 2^-43
// of the largest at most, where a sum of 32-bit weights would be by n 2^-24 of itself; within that of its edge an id may be kept or drawn otherwise
// than the real numbers say.
//
// A block per row; keys lie in shared memory, as many as fit.  A border is found by a histogram of 2048 steps between the largest and the
// lowest logit, of counts or of masses, and a sort of the step that holds it (where one step holds over 2048 ids: by steps between its own
// ends).  Where up to 2048 ids can be kept, they are listed in order of their ids once, and the rest works on the list; else over the row.
// (Sorting 2048 of them, by logit and then by id, took 30000 clocks each time: 46 us for one row of 16384, 29 by the list.)  Few by top_k, or by
// min_p, are gathered in one pass and sorted both ways (64 rows of 50001 floats, top_k 50: 44 us by histogram and list, 25 so; 22 with a range of
// keys before the steps).
//
// One row of 16384 with guidance, top_k 2000 and top_p: 26 us, of which 3 are its reading; some 20 steps follow one another, each a barrier or
// two of 1024 threads and code that runs once.  256 rows of 131072, top_p and min_p: 174 .. 181 us in two rounds of 148 blocks.  128 rows of 131072: the largest
// logit 38 us, top_p 0.9 150 us (the masses of all ids), with min_p 67, where 32 bits show that top_p cuts nothing.
#include <float.h>
#include <math.h>

#include "adsa_half.cuh"

namespace adsa {

constexpr int kDrawThreads = 1024, kDrawWarps = kDrawThreads / 32;
constexpr int kDrawShort = 256;              // top_k up to which the threads' largest keys show where it lies
constexpr int kDrawBins = 2048, kDrawList = 2048;   // steps of a histogram; entries that are sorted
constexpr int kDrawMaxVocab = 1 << 20;       // so that 2^20 weights of 2^42 fit 63 bits
constexpr double kDrawOne = 4398046511104.0;   // 2^42

struct DrawArgs {
    const void *logits, *uncond;
    long long row, uncond_row;              // element strides
    int rows, vocab, wide;                  // wide: rows begin on 16 bytes
    float guidance, temperature, top_p, min_p;
    int top_k;
    const float *temperatures, *top_ps, *min_ps;   // per row, or null
    const int32_t *top_ks;
    const float *uniforms;
    int32_t *tokens;
    float *logprobs;
};

// Order of the logits as unsigned numbers: -inf and NaN 0 (never drawn), zeros alike.
__device__ __forceinline__ uint32_t draw_key(float x)
{
    if (!(x > -INFINITY)) return 0u;
    const uint32_t b = __float_as_uint(x + 0.f);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float draw_logit(uint32_t key) { return __uint_as_float(key & 0x80000000u ? key & 0x7fffffffu : ~key); }

// Eight neighbouring logits from id i on, a multiple of 8; 0 past the end.
template <typename T>
__device__ __forceinline__ void draw_load8(const T *row, int i, int vocab, bool wide, float (&x)[8])
{
    if (wide && i + 8 <= vocab) {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int j = 0; j < 8; j += 4) *reinterpret_cast<float4 *>(x + j) = __ldg(reinterpret_cast<const float4 *>(row + i + j));
        } else {
            const uint4 w = __ldg(reinterpret_cast<const uint4 *>(row + i));
            const uint32_t p[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) *reinterpret_cast<float2 *>(x + 2 * j) = unpack2<T>(p[j]);
        }
    } else if (i >= 8 && i + 16 <= vocab) {
        // from the 16-byte pieces around them, shifted by what the row is off (a multiple of the type's size)
        constexpr int WORDS = sizeof(T) == 4 ? 12 : 8;
        const uintptr_t at = (uintptr_t)(row + i);
        const uint4 *p = reinterpret_cast<const uint4 *>(at & ~(uintptr_t)15);
        uint32_t w[WORDS];
#pragma unroll
        for (int j = 0; j < WORDS; j += 4) {
            const uint4 v = __ldg(p + j / 4);
            w[j] = v.x; w[j + 1] = v.y; w[j + 2] = v.z; w[j + 3] = v.w;
        }
        const unsigned off = (unsigned)(at & 15);
#pragma unroll
        for (int j = 0; j + 2 < WORDS; ++j) w[j] = off & 8 ? w[j + 2] : w[j];
#pragma unroll
        for (int j = 0; j + 1 < WORDS; ++j) w[j] = off & 4 ? w[j + 1] : w[j];
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int j = 0; j < 8; ++j) x[j] = __uint_as_float(w[j]);
        } else {
#pragma unroll
            for (int j = 0; j < 4; ++j) *reinterpret_cast<float2 *>(x + 2 * j) = unpack2<T>(off & 2 ? __funnelshift_r(w[j], w[j + 1], 16) : w[j]);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = i + j < vocab ? to_f32(row[i + j]) : 0.f;
    }
}
// ... as keys, mixed with the other row's if there is one; 0 past the end
template <typename T>
__device__ __forceinline__ void draw_keys(const DrawArgs &a, int r, int i, uint32_t (&k)[8])
{
    alignas(16) float x[8], u[8];
    draw_load8((const T *)a.logits + (size_t)r * a.row, i, a.vocab, a.wide, x);
    if (a.uncond) {
        draw_load8((const T *)a.uncond + (size_t)r * a.uncond_row, i, a.vocab, a.wide, u);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[j] = __fadd_rn(u[j], __fmul_rn(a.guidance, __fsub_rn(x[j], u[j])));
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) k[j] = i + j < a.vocab ? draw_key(x[j]) : 0u;
}

struct DrawShared {
    unsigned long long mass[kDrawBins];     // of the steps
    unsigned long long list[kDrawList];
    unsigned count[kDrawBins];
    uint32_t key[kDrawList], id[kDrawList]; // what can be kept, in order of ids
    double power[64];                       // 2^(j / 64)
    unsigned long long warp_mass[kDrawWarps];
    unsigned warp_count[kDrawWarps];
    uint32_t warp_key[kDrawWarps], warp_low[kDrawWarps];
    double largest, per_64th;               // the largest logit; 64 log2(e) / temperature
    unsigned long long before;
    uint32_t top, min_key;
    unsigned bin, n, bin_count;
    int pick;
};

// Functions that are not inlined: every phase runs once, and what bounds a small call is fetching its code.

// exp((x - largest) / temperature) in 64 bits, off by about 2^-51: the 64ths of the power of two from a table, the rest (up to 1/128 of a
// doubling) by the exponential series (table-driven, after Tang 1989).  Below 2^-1000: 0.
__device__ __forceinline__ double draw_share(uint32_t key, const DrawShared &s)
{
    const double x = (draw_logit(key) - s.largest) * s.per_64th, magic = 6755399441055744.0;
    const double k = x + magic, r = (x - (k - magic)) * 0.010830424696249145;   // ln 2 / 64
    double p = fma(r, 1.0 / 120, 1.0 / 24);
    p = fma(p, r, 1.0 / 6);
    p = fma(p, r, 0.5);
    p = fma(p, r, 1.0);
    p = fma(p, r, 1.0);
    const int n = __double2loint(k);                               // (two's complement in the low bits of the sum)
    const double y = p * s.power[n & 63];
    const double w = __hiloint2double(__double2hiint(y) + ((n >> 6) << 20), __double2loint(y));
    return key == s.top ? 1.0 : x > -64000.0 ? w : 0.0;            // (chosen, not branched over: neighbours' chains run side by side)
}
__device__ __forceinline__ float draw_exp2(float x)
{
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// ... as a whole multiple of 2^-42
__device__ __forceinline__ unsigned long long draw_weight(uint32_t key, const DrawShared &s)
{
    return (unsigned long long)__double_as_longlong(fma(draw_share(key, s), kDrawOne, 4503599627370496.0)) & 0xfffffffffffffULL;   // 2^52 + the multiple
}
__device__ __noinline__ unsigned long long draw_weight_of(uint32_t key, const DrawShared &s) { return draw_weight(key, s); }
__device__ __noinline__ bool draw_enough(uint32_t key, double min_p, const DrawShared &s) { return draw_share(key, s) >= min_p; }

// *sum += x in shared memory, by its two words: the low one's overflow is carried by whoever makes it.
__device__ __forceinline__ void draw_add(unsigned long long *sum, unsigned long long x)
{
    unsigned *const word = reinterpret_cast<unsigned *>(sum);
    const unsigned low = (unsigned)x;
    unsigned high = (unsigned)(x >> 32);
    if (low) high += atomicAdd(word, low) > ~low;
    if (high) atomicAdd(word + 1, high);
}
// Sum of x over the block, for all threads; before: what threads before this one have of it.
__device__ __noinline__ unsigned long long draw_scan(unsigned long long x, unsigned long long *before, DrawShared &s)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    unsigned long long incl = x;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const unsigned long long t = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += t; }
    __syncthreads();
    if (lane == 31) s.warp_mass[warp] = incl;
    __syncthreads();
    unsigned long long w = s.warp_mass[lane];
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const unsigned long long t = __shfl_up_sync(0xffffffffu, w, o); if (lane >= o) w += t; }
    const unsigned long long own = __shfl_sync(0xffffffffu, w, (warp + 31) & 31);
    *before = incl - x + (warp ? own : 0);
    return __shfl_sync(0xffffffffu, w, 31);
}
// The list's n entries, largest first (room for a power of two).
__device__ __noinline__ void draw_sort(DrawShared &s, unsigned n)
{
    if (n <= 64) {                                                 // a warp's registers hold them: entries lane, lane + 32
        if (threadIdx.x < 32) {
            const unsigned lane = threadIdx.x;
            unsigned long long x[2] = {lane < n ? s.list[lane] : 0, lane + 32 < n ? s.list[lane + 32] : 0};
#pragma unroll 1
            for (unsigned k = 2; k <= 64; k *= 2) {
#pragma unroll 1
                for (unsigned j = k / 2; j; j /= 2) {
                    const unsigned long long y0 = j == 32 ? x[1] : __shfl_xor_sync(0xffffffffu, x[0], j & 31), y1 = j == 32 ? x[0] : __shfl_xor_sync(0xffffffffu, x[1], j & 31);
                    // the lower of a pair keeps the larger, where larger ones come first
                    const bool low0 = j == 32 || !(lane & j), low1 = j != 32 && !(lane & j);
                    x[0] = (x[0] > y0) == (low0 == ((lane & k) == 0)) ? x[0] : y0;
                    x[1] = (x[1] > y1) == (low1 == (((lane + 32) & k) == 0)) ? x[1] : y1;
                }
            }
            s.list[lane] = x[0];
            s.list[lane + 32] = x[1];
        }
        __syncthreads();
        return;
    }
    unsigned size = 128;
    while (size < n) size *= 2;
    for (unsigned i = n + threadIdx.x; i < size; i += kDrawThreads) s.list[i] = 0;
    for (unsigned k = 2; k <= size; k *= 2) {
        for (unsigned j = k / 2; j; j /= 2) {
            // pairs within a warp's 64 entries need the warp alone
            if (j >= 32 || k == 2) __syncthreads();
            else __syncwarp();
            const unsigned t = threadIdx.x, i = 2 * t - (t & (j - 1)), o = i + j;
            if (t < size / 2) {
                const unsigned long long x = s.list[i], y = s.list[o];
                if ((x < y) == ((i & k) == 0)) { s.list[i] = y; s.list[o] = x; }
            }
        }
    }
    __syncthreads();
}
// Largest and lowest of the block's keys.
__device__ __noinline__ uint2 draw_ends(uint32_t most, uint32_t fewest, DrawShared &s)
{
    most = __reduce_max_sync(0xffffffffu, most);
    fewest = __reduce_min_sync(0xffffffffu, fewest);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) { s.warp_key[threadIdx.x >> 5] = most; s.warp_low[threadIdx.x >> 5] = fewest; }
    __syncthreads();
    return make_uint2(__reduce_max_sync(0xffffffffu, s.warp_key[threadIdx.x & 31]), __reduce_min_sync(0xffffffffu, s.warp_low[threadIdx.x & 31]));
}

// The row's keys, eight at a time: shared memory up to `stashed` (a multiple of 8), the rest read again.
template <typename T>
struct DrawRow {
    const uint32_t *stash;
    int r, stashed;
    __device__ __forceinline__ void at(const DrawArgs &a, int i, uint32_t (&k)[8]) const
    {
        if (i < stashed) {
            *reinterpret_cast<uint4 *>(k) = *reinterpret_cast<const uint4 *>(stash + i);
            *reinterpret_cast<uint4 *>(k + 4) = *reinterpret_cast<const uint4 *>(stash + i + 4);
        } else {
            draw_keys<T>(a, r, i, k);
        }
    }
};
constexpr int kDrawStride = 8 * kDrawThreads;

// Steps between the logits of two keys, even in the logits; or, where their distance is none or infinite, in the keys.  The two
// ends are in different steps.
struct DrawSteps {
    uint32_t top, low;
    float high, scale;
    bool by_key;
    __device__ __forceinline__ DrawSteps(uint32_t top_, uint32_t low_) : top(top_), low(low_), high(0.5f * draw_logit(top_))
    {
        scale = (kDrawBins - 1) / (high - 0.5f * draw_logit(low));   // (halves: the distance of finite logits is finite)
        by_key = !(scale > 0.f && scale <= FLT_MAX);
        if (by_key) scale = (float)(kDrawBins - 1) / (float)max(top - low, 1u);
    }
    // descending: 0 for the larger end
    __device__ __forceinline__ unsigned operator()(uint32_t key) const
    {
        const float x = by_key ? (float)(top - key) : high - 0.5f * draw_logit(key);
        return min((unsigned)max((int)(x * scale), 0), (unsigned)kDrawBins - 1u);
    }
    __device__ __forceinline__ bool has(uint32_t key) const { return key <= top && key >= low; }
};

// A range of keys around those of the steps first .. last, a step or more too wide at both ends: from .. from + more.  What lies outside
// needs no step of its own.  (The slack is well above what rounding moves: 2^-24 of the distance, and of the larger end.)
__device__ __forceinline__ uint2 draw_range(const DrawSteps &t, unsigned first, unsigned last)
{
    const float wide = 1.f / t.scale, down = (float)(last + 2u) * wide, up = first > 1u ? (float)(first - 1u) * wide : 0.f, slack = fabsf(t.high) * 4e-7f;
    uint32_t from, to;
    if (t.by_key) {
        from = down + 1.f < (float)(t.top - t.low) ? t.top - (uint32_t)(down + 1.f) : t.low;
        to = up > 1.f ? t.top - (uint32_t)(up - 1.f) : t.top;
    } else {
        from = max(draw_key(2.f * (t.high - down - slack)), t.low);
        to = first > 1u ? min(draw_key(2.f * (t.high - up + slack)), t.top) : t.top;
    }
    return make_uint2(from, max(to, from) - from);
}

// How many of the row's keys lie in each step, and with `masses` their weights.
template <typename T>
__device__ __noinline__ void draw_histogram(const DrawArgs &a, DrawRow<T> row, DrawSteps steps, bool masses, DrawShared &s)
{
    __syncthreads();
    for (int i = threadIdx.x; i < kDrawBins; i += kDrawThreads) { s.count[i] = 0; s.mass[i] = 0; }
    __syncthreads();
    for (int i = 8 * threadIdx.x; i < a.vocab; i += kDrawStride) {
        alignas(16) uint32_t k[8];
        row.at(a, i, k);
#pragma unroll
        for (int j = 0; j < 8; j += 2) {
            const bool in0 = steps.has(k[j]), in1 = steps.has(k[j + 1]);
            if (!in0 && !in1) continue;
            const unsigned b0 = steps(k[j]), b1 = steps(k[j + 1]);
            if (in0) atomicAdd(&s.count[b0], 1u);
            if (in1) atomicAdd(&s.count[b1], 1u);
            if (masses) {
                const unsigned long long w0 = draw_weight(k[j], s), w1 = draw_weight(k[j + 1], s);
                if (in0) draw_add(&s.mass[b0], w0);
                if (in1) draw_add(&s.mass[b1], w1);
            }
        }
    }
    __syncthreads();
}
// The ids with keys of the steps from `first` to `last` into the list, as key and id, sorted: larger keys first, of equal ones lower ids.  s.n: how
// many there are; more than the list holds are not sorted.
template <typename T>
__device__ __noinline__ void draw_gather(const DrawArgs &a, DrawRow<T> row, DrawSteps steps, unsigned first, unsigned last, DrawShared &s)
{
    const uint2 range = draw_range(steps, first, last);            // (a step for every id: 8 us of a pass over 131072)
    __syncthreads();
    if (threadIdx.x == 0) s.n = 0;
    __syncthreads();
    for (int i = 8 * threadIdx.x; i < a.vocab; i += kDrawStride) {
        alignas(16) uint32_t k[8];
        row.at(a, i, k);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (k[j] - range.x > range.y) continue;
            const unsigned b = steps(k[j]);
            if (b < first || b > last) continue;
            const unsigned at = atomicAdd(&s.n, 1u);
            if (at < kDrawList) s.list[at] = (unsigned long long)k[j] << 32 | (0xffffffffu - (unsigned)(i + j));
        }
    }
    __syncthreads();
    if (s.n <= kDrawList) draw_sort(s, s.n);
}
// The ids that can be kept into s.key and s.id in their order: keys above thr, and the first `ties` with just that key; a warp per segment of ids,
// 256 at a time.
template <typename T>
__device__ __noinline__ unsigned draw_list(const DrawArgs &a, DrawRow<T> row, uint32_t thr, unsigned ties, DrawShared &s)
{
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, per = ((a.vocab + kDrawWarps - 1) / kDrawWarps + 255) & ~255, i0 = warp * per, i1 = min(i0 + per, a.vocab);
    unsigned both = 0;                                             // keys above thr, 2^16 times keys of thr (ids of a lane: below 2^16)
    for (int i = i0 + 8 * lane; i < i1; i += 256) {
        alignas(16) uint32_t k[8];
        row.at(a, i, k);
#pragma unroll
        for (int j = 0; j < 8; ++j) both += (k[j] > thr ? 1u : 0u) + (k[j] == thr ? 0x10000u : 0u);
    }
    const unsigned above = __reduce_add_sync(0xffffffffu, both & 0xffffu), equal = __reduce_add_sync(0xffffffffu, both >> 16);
    __syncthreads();
    if (lane == 0) { s.warp_count[warp] = above; s.warp_key[warp] = equal; }
    __syncthreads();
    // entries and equals of the warps before this one
    const unsigned c = s.warp_count[lane], e = s.warp_key[lane];
    unsigned eq = __reduce_add_sync(0xffffffffu, lane < warp ? e : 0u), at = __reduce_add_sync(0xffffffffu, lane < warp ? c : 0u) + min(eq, ties);
    const unsigned n = __reduce_add_sync(0xffffffffu, c) + min(__reduce_add_sync(0xffffffffu, e), ties);
    if (above + equal) {
        for (int i = i0 + 8 * lane; i - 8 * lane < i1; i += 256) {
            alignas(16) uint32_t k[8] = {0, 0, 0, 0, 0, 0, 0, 0};
            if (i < i1) row.at(a, i, k);
            unsigned mine = 0, same = 0;                           // bits: kept for sure; of the border
#pragma unroll
            for (int j = 0; j < 8; ++j) { mine |= (k[j] > thr) << j; same |= (k[j] == thr) << j; }
            if (!__any_sync(0xffffffffu, mine | same)) continue;
            unsigned before = __popc(same) << 16, all = before;    // (sums of both counts)
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const unsigned t = __shfl_up_sync(0xffffffffu, before, o); if (lane >= o) before += t; }
            all = __shfl_sync(0xffffffffu, before, 31) >> 16;
            unsigned rank = eq + (before >> 16) - __popc(same);    // of this lane's first at the border
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (same >> j & 1u) mine |= (rank++ < ties) << j;
            before = __popc(mine);
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const unsigned t = __shfl_up_sync(0xffffffffu, before, o); if (lane >= o) before += t; }
            unsigned to = at + before - __popc(mine);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                if (mine >> j & 1u) {
                    s.key[to] = k[j];
                    s.id[to++] = (uint32_t)(i + j);
                }
            }
            at += __shfl_sync(0xffffffffu, before, 31);
            eq += all;
        }
    }
    __syncthreads();
    return n;
}
// Largest and lowest key of a step.
template <typename T>
__device__ __noinline__ uint2 draw_step_ends(const DrawArgs &a, DrawRow<T> row, DrawSteps steps, unsigned bin, DrawShared &s)
{
    const uint2 range = draw_range(steps, bin, bin);
    uint32_t most = 0, fewest = 0xffffffffu;
    for (int i = 8 * threadIdx.x; i < a.vocab; i += kDrawStride) {
        alignas(16) uint32_t k[8];
        row.at(a, i, k);
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if (k[j] - range.x <= range.y && steps(k[j]) == bin) { most = max(most, k[j]); fewest = min(fewest, k[j]); }
    }
    return draw_ends(most, fewest, s);
}
// The last step with ids in it of which the count (masses: the mass) before is below the goal, or else the first: s.bin, s.bin_count, s.before.
// start: what is before the first step.
__device__ __noinline__ void draw_find(bool masses, double goal, unsigned long long start, DrawShared &s)
{
    const int tid = threadIdx.x;
    if (tid == 0) s.pick = -1;
    unsigned long long before;
    const unsigned long long c0 = s.count[2 * tid], c1 = s.count[2 * tid + 1], m0 = masses ? s.mass[2 * tid] : c0, m1 = masses ? s.mass[2 * tid + 1] : c1;
    draw_scan(m0 + m1, &before, s);
    before += start;
    const bool g0 = c0 && ((double)before < goal || before == start), g1 = c1 && ((double)(before + m0) < goal || before + m0 == start);
    if (g0 || g1) atomicMax(&s.pick, 2 * tid + (g1 ? 1 : 0));
    __syncthreads();
    if (s.pick >> 1 == tid) {
        s.bin = (unsigned)s.pick;
        s.before = s.pick & 1 ? before + m0 : before;
        s.bin_count = (unsigned)(s.pick & 1 ? c1 : c0);
    }
    __syncthreads();
}
// Of the sorted list: the first entry with the same key as entry `at`.
__device__ __noinline__ unsigned draw_first_equal(const DrawShared &s, unsigned at)
{
    const uint32_t key = (uint32_t)(s.list[at] >> 32);
    unsigned first = 0;
    while (first < at) {
        const unsigned mid = (first + at) / 2;
        if ((uint32_t)(s.list[mid] >> 32) == key) at = mid;
        else first = mid + 1;
    }
    return first;
}

template <typename T>
__global__ void __launch_bounds__(kDrawThreads)
draw_kernel(const __grid_constant__ DrawArgs a, int stashed)
{
    extern __shared__ __align__(16) unsigned char draw_smem[];
    DrawShared &s = *reinterpret_cast<DrawShared *>(draw_smem);
    uint32_t *const draw_stash = reinterpret_cast<uint32_t *>(draw_smem + sizeof(DrawShared));
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, V = a.vocab;
    const DrawRow<T> row{draw_stash, r, stashed};
    if (tid < 64) s.power[tid] = exp2(tid / 64.0);
    pdl_wait();
    pdl_launch();
    // the largest and the lowest
    uint32_t top = 0, low = 0xffffffffu;
    unsigned able = 0;                                             // ids that can be drawn
#pragma unroll 2
    for (int i = 8 * tid; i < V; i += kDrawStride) {
        alignas(16) uint32_t k[8];
        draw_keys<T>(a, r, i, k);
        if (i < stashed) {
            *reinterpret_cast<uint4 *>(draw_stash + i) = *reinterpret_cast<const uint4 *>(k);
            *reinterpret_cast<uint4 *>(draw_stash + i + 4) = *reinterpret_cast<const uint4 *>(k + 4);
        }
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            top = max(top, k[j]);
            low = min(low, k[j] - 1u);                             // (a key of 0 becomes the largest number)
            able += k[j] != 0u;
        }
    }
    const uint32_t mine = top;
    const uint2 ends = draw_ends(top, low, s);
    top = ends.x;
    low = ends.y + 1u;
    unsigned long long unused;
    able = (unsigned)draw_scan(able, &unused, s);
    if (top == 0) {                                                // nothing to draw
        if (tid == 0) {
            a.tokens[r] = -1;
            if (a.logprobs) a.logprobs[r] = -INFINITY;
        }
        return;
    }
    const float temperature = a.temperatures ? a.temperatures[r] : a.temperature;
    int top_k = a.top_ks ? a.top_ks[r] : a.top_k;
    const float top_p = a.top_ps ? a.top_ps[r] : a.top_p;
    const float least = a.min_ps ? a.min_ps[r] : a.min_p;
    const double largest = draw_logit(top);
    const double min_p = largest == INFINITY ? 1.0 : least > 0.f ? fmin((double)least, 1.0) : 0.0;   // (infinite ones alone, where there are any)
    const double goal_u = fmin(fmax((double)a.uniforms[r], 0.0), 1.0);
    if (!(temperature > 0.f)) top_k = 1;
    const bool by_count = top_k > 0 && (unsigned)top_k < able, by_mass = top_p < 1.f && top_k != 1;
    if (!by_count) top_k = (int)able;
    if (tid == 0) {
        s.largest = largest;
        s.per_64th = 92.33248261893469 / (double)temperature;      // 64 / ln 2
        s.top = top;
    }
    __syncthreads();
    // the lowest key with a weight of min_p at least: 32 borders at a time
    if (warp == 0) {
        uint32_t lo = low, hi = top;                               // hi has it; what is below lo does not
        while (min_p > 0.0 && lo < hi) {
            const uint32_t step = (hi - lo) / 32u + 1u, at = min(hi - lo, step * lane) + lo;
            const unsigned has = __ballot_sync(0xffffffffu, draw_enough(at, min_p, s));
            const int first = has ? __ffs(has) - 1 : 32;           // (weights rise with keys)
            const uint32_t base = lo;
            if (first < 32) hi = min(hi, base + min(hi - base, step * first));
            if (first > 0) lo = min(hi, base + min(hi - base, step * (first - 1)) + 1u);
        }
        if (lane == 0) s.min_key = min_p > 0.0 ? hi : low;
    }
    __syncthreads();
    const uint32_t min_key = s.min_key;

    uint32_t thr = low;                                            // the border: keys above thr, and the first `ties` ids with just that key
    unsigned ties = 0xffffffffu;
    bool few = able <= kDrawList, cut = false;                     // at most 2048 ids can be kept; top_p cuts nothing more
    // The short way: what can be kept lies in the list, sorted, `n` of it by top_k.
    bool listed = false;
    unsigned n = 0;
    if (able <= kDrawThreads) {
        draw_gather(a, row, DrawSteps(top, low), 0u, kDrawBins - 1u, s);
        listed = true;
        n = (unsigned)top_k;
    } else if (by_count && top_k <= kDrawShort) {
        // The threads' largest keys: the top_k-th of them is not above the top_k-th of all, and few others are above it.
        for (int i = tid; i < kDrawBins; i += kDrawThreads) s.count[i] = 0;
        __syncthreads();
        const DrawSteps steps(top, low);
        if (mine) atomicAdd(&s.count[steps(mine)], 1u);
        __syncthreads();
        draw_find(false, (double)top_k, 0, s);
        const unsigned bin = s.bin;
        if (s.before + s.bin_count >= (unsigned)top_k) {           // (else fewer threads than that have a key)
            draw_gather(a, row, steps, 0u, bin, s);
            listed = s.n <= kDrawThreads;
            n = (unsigned)top_k;
        }
    }
    if (!listed && by_count) {
        few = few || top_k <= kDrawList;
        DrawSteps steps(top, low);
        unsigned long long start = 0;
        for (;;) {
            draw_histogram(a, row, steps, false, s);
            draw_find(false, (double)top_k, start, s);
            const unsigned bin = s.bin, in_bin = s.bin_count;
            const unsigned long long before = s.before;
            if (in_bin <= kDrawList) {
                draw_gather(a, row, steps, bin, bin, s);
                const unsigned last = (unsigned)(top_k - before) - 1u;   // that is kept
                thr = (uint32_t)(s.list[last] >> 32);
                ties = last + 1u - draw_first_equal(s, last);
                break;
            }
            // too many in one step: between its own largest and lowest
            const uint2 e = draw_step_ends(a, row, steps, bin, s);
            if (e.x == e.y) {
                thr = e.x;
                ties = (unsigned)(top_k - before);
                break;
            }
            steps = DrawSteps(e.x, e.y);
            start = before;
        }
    }
    if (!listed && !few && min_key > thr && largest != INFINITY) {
        // Few by min_p, whose mass is well below top_p of all, by weights in 32 bits (sums of a thread's ids, off by 2^-12 at most): then top_p
        // cuts nothing more.
        float sum = 0.f, part = 0.f;
        unsigned many = 0;
        const float high = draw_logit(top), scale = 1.44269504f / temperature;
        for (int i = 8 * tid; i < V; i += kDrawStride) {
            alignas(16) uint32_t k[8];
            row.at(a, i, k);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float w = k[j] >= thr && by_mass ? draw_exp2((draw_logit(k[j]) - high) * scale) : 0.f;   // (with ties that top_k leaves out: more)
                sum += k[j] > thr ? w : 0.f;
                part += k[j] >= min_key ? w : 0.f;
                many += k[j] >= min_key;
            }
        }
        many = (unsigned)draw_scan(many, &unused, s);
        cut = !by_mass;
        if (by_mass) {
            const unsigned long long all = draw_scan((unsigned long long)(sum * 1048576.f), &unused, s), kept = draw_scan((unsigned long long)(part * 1048576.f) + 1u, &unused, s);
            cut = (double)kept * 1.001 < (double)top_p * (double)all * 0.999;
        }
        if (cut) {
            thr = min_key;
            ties = 0xffffffffu;
            few = many <= kDrawList;
            // (a pass and a sort by logit and one by id, against two passes)
            if (many <= 256u || (many <= kDrawThreads && V >= 65536)) {
                draw_gather(a, row, DrawSteps(top, thr), 0u, kDrawBins - 1u, s);
                listed = true;
                n = many;
            }
        }
    }
    if (listed) {
        // an entry a thread
        unsigned long long e = s.list[tid], before;
        uint32_t key = (uint32_t)(e >> 32);
        unsigned long long w = tid < n ? draw_weight_of(key, s) : 0, total = draw_scan(w, &before, s);
        const double goal = by_mass && !cut ? fmax((double)top_p, 0.0) * (double)total : INFINITY;
        n = (unsigned)draw_scan(tid < n && (tid == 0 || ((double)before < goal && key >= min_key)) ? 1u : 0u, &before, s);   // (a head of the list)
        if (tid < n) s.list[tid] = e << 32 | e >> 32;              // by id
        if (tid == 0) s.pick = (int)n - 1;
        __syncthreads();
        draw_sort(s, n);
        e = s.list[tid];
        key = (uint32_t)e;
        w = tid < n ? draw_weight_of(key, s) : 0;
        total = draw_scan(w, &before, s);
        if (tid < n && (double)(before + w) >= goal_u * (double)total) atomicMin(&s.pick, tid);
        __syncthreads();
        if (tid == s.pick) {
            a.tokens[r] = (int)(0xffffffffu - (uint32_t)(e >> 32));
            if (a.logprobs) a.logprobs[r] = (float)((key == top ? 0.0 : (draw_logit(key) - largest) / (double)temperature) - log((double)total / kDrawOne));
        }
        return;
    }
    if (few) {
        n = draw_list(a, row, thr, ties, s);
        // two entries a thread
        const uint32_t k0 = s.key[2 * tid], k1 = s.key[2 * tid + 1];
        const bool has0 = 2u * tid < n, has1 = 2u * tid + 1u < n;
        const unsigned long long w0 = has0 ? draw_weight_of(k0, s) : 0, w1 = has1 ? draw_weight_of(k1, s) : 0;
        unsigned long long before;
        unsigned long long total = draw_scan(w0 + w1, &before, s);
        bool in0 = has0 && k0 >= min_key, in1 = has1 && k1 >= min_key;
        if (by_mass && !cut) {
            // the border by mass among them
            const double goal = fmax((double)top_p, 0.0) * (double)total;
            DrawSteps steps(top, thr);
            unsigned long long start = 0;
            for (;;) {
                for (int i = tid; i < kDrawBins; i += kDrawThreads) { s.count[i] = 0; s.mass[i] = 0; }
                if (tid == 0) s.n = 0;
                __syncthreads();
                const unsigned b0 = has0 && steps.has(k0) ? steps(k0) : kDrawBins, b1 = has1 && steps.has(k1) ? steps(k1) : kDrawBins;
                if (b0 < kDrawBins) { atomicAdd(&s.count[b0], 1u); draw_add(&s.mass[b0], w0); }
                if (b1 < kDrawBins) { atomicAdd(&s.count[b1], 1u); draw_add(&s.mass[b1], w1); }
                __syncthreads();
                draw_find(true, goal, start, s);
                const unsigned bin = s.bin;
                start = s.before;
                if (s.bin_count <= 64u) break;
                const uint2 e = draw_ends(max(b0 == bin ? k0 : 0u, b1 == bin ? k1 : 0u), min(b0 == bin ? k0 : 0xffffffffu, b1 == bin ? k1 : 0xffffffffu), s);
                if (e.x == e.y) break;
                steps = DrawSteps(e.x, e.y);
            }
            // (of one step; or of equal keys, more than are sorted quickly)
            const unsigned bin = s.bin;
            if (has0 && steps.has(k0) && steps(k0) == bin) s.list[atomicAdd(&s.n, 1u)] = (unsigned long long)k0 << 32 | (0xffffffffu - 2u * tid);
            if (has1 && steps.has(k1) && steps(k1) == bin) s.list[atomicAdd(&s.n, 1u)] = (unsigned long long)k1 << 32 | (0xfffffffeu - 2u * tid);
            __syncthreads();
            const unsigned in_bin = s.n;
            draw_sort(s, in_bin);
            const unsigned long long x0 = 2u * tid < in_bin ? draw_weight_of((uint32_t)(s.list[2 * tid] >> 32), s) : 0,
                                     x1 = 2u * tid + 1u < in_bin ? draw_weight_of((uint32_t)(s.list[2 * tid + 1] >> 32), s) : 0;
            unsigned long long at;
            draw_scan(x0 + x1, &at, s);
            at += start;
            const unsigned kept = (unsigned)draw_scan((2u * tid < in_bin && (tid == 0 || (double)at < goal)) + (2u * tid + 1u < in_bin && (double)(at + x0) < goal), &unused, s);
            const unsigned long long last = s.list[kept - 1u];     // as key and place in the list
            in0 = in0 && ((unsigned long long)k0 << 32 | (0xffffffffu - 2u * tid)) >= last;
            in1 = in1 && ((unsigned long long)k1 << 32 | (0xfffffffeu - 2u * tid)) >= last;
        }
        if (tid == 0) s.pick = 0x7fffffff;
        total = draw_scan((in0 ? w0 : 0) + (in1 ? w1 : 0), &before, s);
        if (in0) before += w0;
        const double goal = goal_u * (double)total;
        if (in0 && (double)before >= goal) atomicMin(&s.pick, 2 * tid);
        else if (in1 && (double)(before + w1) >= goal) atomicMin(&s.pick, 2 * tid + 1);
        __syncthreads();
        if (s.pick == 0x7fffffff) {                                // (rounding, u = 1: the last that is kept)
            const uint2 e = draw_ends(in1 ? 2u * tid + 2u : in0 ? 2u * tid + 1u : 0u, 0u, s);
            if (tid == 0) s.pick = (int)e.x - 1;
            __syncthreads();
        }
        if (tid == 0) {
            const uint32_t key = s.key[s.pick];
            a.tokens[r] = (int)s.id[s.pick];
            if (a.logprobs) a.logprobs[r] = (float)((key == top ? 0.0 : (draw_logit(key) - largest) / (double)temperature) - log((double)total / kDrawOne));
        }
        return;
    }
    if (by_mass && !cut) {
        // of the ids at top_k's border, the first `ties` count
        const uint32_t k_thr = thr;
        unsigned equal = 0;
        if (ties != 0xffffffffu) {
            for (int i = 8 * tid; i < V; i += kDrawStride) {
                alignas(16) uint32_t k[8];
                row.at(a, i, k);
#pragma unroll
                for (int j = 0; j < 8; ++j) equal += k[j] == thr;
            }
            equal = (unsigned)draw_scan(equal, &unused, s);
        }
        const unsigned drop = equal - min(equal, ties);
        DrawSteps steps(top, thr);
        unsigned long long start = 0;
        double goal = -1.0;
        for (;;) {
            draw_histogram(a, row, steps, true, s);
            if (tid == 0 && drop && steps.low == k_thr) {          // (they are the last of the last step that holds any)
                s.mass[steps(k_thr)] -= drop * draw_weight_of(k_thr, s);
                s.count[steps(k_thr)] -= drop;
            }
            __syncthreads();
            if (goal < 0.0) goal = fmax((double)top_p, 0.0) * (double)draw_scan(s.mass[2 * tid] + s.mass[2 * tid + 1], &unused, s);
            draw_find(true, goal, start, s);
            const unsigned bin = s.bin, less = steps.low == k_thr && bin == steps(k_thr) ? drop : 0u, in_bin = s.bin_count;
            const unsigned long long before = s.before;
            if (in_bin + less <= kDrawList) {
                draw_gather(a, row, steps, bin, bin, s);
                const unsigned long long w0 = 2u * tid < in_bin ? draw_weight_of((uint32_t)(s.list[2 * tid] >> 32), s) : 0,
                                         w1 = 2u * tid + 1u < in_bin ? draw_weight_of((uint32_t)(s.list[2 * tid + 1] >> 32), s) : 0;
                unsigned long long at;
                draw_scan(w0 + w1, &at, s);
                at += before;
                const unsigned in0 = 2u * tid < in_bin && (tid == 0 || (double)at < goal), in1 = 2u * tid + 1u < in_bin && (double)(at + w0) < goal;
                const unsigned kept = (unsigned)draw_scan(in0 + in1, &unused, s);
                thr = (uint32_t)(s.list[kept - 1u] >> 32);
                ties = kept - draw_first_equal(s, kept - 1u);
                break;
            }
            const uint2 e = draw_step_ends(a, row, steps, bin, s);
            if (e.x == e.y) {
                // equal keys: those with less than the goal before them, one at least
                const unsigned long long w = draw_weight_of(e.x, s);
                unsigned high = in_bin, at = 1;
                while (at < high) {
                    const unsigned mid = (at + high + 1) / 2;      // is the mid-th kept?
                    if ((double)(before + (mid - 1) * w) < goal) at = mid;
                    else high = mid - 1;
                }
                thr = e.x;
                ties = at;
                break;
            }
            steps = DrawSteps(e.x, e.y);
            start = before;
        }
        __syncthreads();
    }
    if (!cut && min_key > thr) {
        thr = min_key;
        ties = 0xffffffffu;
    }
    // Mass of what is kept, by segments of ids in order, one per warp; then the segment in which the running sum reaches its goal is cut
    // into one per warp again.  (Ids at the border count in order.)
    unsigned long long total = 0, before = 0;
    unsigned equal_before = 0;
    int begin = 0, end = V;
    double goal = 0.0;
    for (int level = 0;; ++level) {
        const int per = ((end - begin + kDrawWarps - 1) / kDrawWarps + 7) & ~7, i0 = begin + warp * per, i1 = min(i0 + per, end);   // (begin: a multiple of 8)
        unsigned long long sum = 0;
        unsigned equal = 0, kept = 0;
        for (int i = i0 + 8 * lane; i < i1; i += 256) {
            alignas(16) uint32_t k[8];
            row.at(a, i, k);
#pragma unroll
            for (int j = 0; j < 8; j += 2) {                       // (segments end at multiples of 8, or with the row)
                const bool in0 = k[j] > thr, in1 = k[j + 1] > thr;
                equal += (k[j] == thr) + (k[j + 1] == thr);
                kept += in0 + in1;
                if (!in0 && !in1) continue;
                const unsigned long long w0 = draw_weight(k[j], s), w1 = draw_weight(k[j + 1], s);
                sum += (in0 ? w0 : 0) + (in1 ? w1 : 0);
            }
        }
#pragma unroll
        for (int o = 16; o; o >>= 1) {
            sum += __shfl_xor_sync(0xffffffffu, sum, o);
            equal += __shfl_xor_sync(0xffffffffu, equal, o);
            kept += __shfl_xor_sync(0xffffffffu, kept, o);
        }
        __syncthreads();
        if (lane == 0) { s.warp_mass[warp] = sum; s.warp_count[warp] = equal; s.warp_key[warp] = kept; }
        __syncthreads();
        const unsigned long long w = draw_weight_of(thr, s);
        if (level == 0) {
            unsigned e = 0;
#pragma unroll 1
            for (int x = 0; x < kDrawWarps; ++x) { total += s.warp_mass[x]; e += s.warp_count[x]; }
            total += min(e, ties) * w;
            goal = goal_u * (double)total;
        }
        // the first segment with a kept id at which the sum reaches the goal; none (rounding, u = 1): the last with a kept id
        int pick = -1;
        unsigned long long pick_before = before;
        unsigned pick_equal = equal_before;
        {
            unsigned long long run = before;
            unsigned eq = equal_before;
#pragma unroll 1
            for (int x = 0; x < kDrawWarps; ++x) {
                const unsigned e = min(eq + s.warp_count[x], ties) - min(eq, ties);
                const unsigned long long after = run + s.warp_mass[x] + e * w;
                if (e || s.warp_key[x]) {
                    pick = x;
                    pick_before = run;
                    pick_equal = eq;
                    if ((double)after >= goal) break;
                }
                run = after;
                eq += s.warp_count[x];
            }
        }
        before = pick_before;
        equal_before = pick_equal;
        begin = begin + pick * per;
        end = min(begin + per, end);
        if (per <= 32) break;
    }
    // up to 32 ids: a lane each
    if (warp == 0) {
        const int i = begin + lane;
        alignas(16) uint32_t k8[8] = {0, 0, 0, 0, 0, 0, 0, 0};
        if ((i & ~7) < end) row.at(a, i & ~7, k8);
        uint32_t k = 0;
#pragma unroll
        for (int j = 0; j < 8; ++j)
            if ((i & 7) == j && i < end) k = k8[j];
        bool kept = i < end && k >= thr;
        const unsigned equal = __ballot_sync(0xffffffffu, kept && k == thr);
        if (kept && k == thr) kept = equal_before + __popc(equal & ((1u << lane) - 1u)) < ties;
        unsigned long long run = kept ? draw_weight_of(k, s) : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const unsigned long long x = __shfl_up_sync(0xffffffffu, run, o); if (lane >= o) run += x; }
        const unsigned all = __ballot_sync(0xffffffffu, kept), reached = __ballot_sync(0xffffffffu, kept && (double)(before + run) >= goal);
        const int pick = reached ? __ffs(reached) - 1 : 31 - __clz(all);
        if (lane == pick) {
            a.tokens[r] = i;
            if (a.logprobs) a.logprobs[r] = (float)((k == top ? 0.0 : (draw_logit(k) - largest) / (double)temperature) - log((double)total / kDrawOne));
        }
    }
}

namespace {

template <typename T>
cudaError_t launch_draw(const DrawArgs &a, dim3 grid, cudaStream_t st)
{
    constexpr int most = (227 * 1024 - (int)sizeof(DrawShared)) / 4;   // keys that fit
    static_assert(sizeof(DrawShared) % 16 == 0, "keys behind it");
    static int told[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const bool known = dev >= 0 && dev < 64;
    if (!known || !__atomic_load_n(&told[dev], __ATOMIC_ACQUIRE)) {
        e = cudaFuncSetAttribute((const void *)draw_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024);
        if (e != cudaSuccess) return e;
        if (known) __atomic_store_n(&told[dev], 1, __ATOMIC_RELEASE);
    }
    const int stashed = a.vocab <= (most & ~7) ? (a.vocab + 7) & ~7 : most & ~7;
    return launch_pdl(draw_kernel<T>, grid, kDrawThreads, sizeof(DrawShared) + (size_t)stashed * 4, st, a, stashed);
}

}  // namespace
}  // namespace adsa

using namespace adsa;

extern "C" int adsa_sample(const adsa_sampling *how, int dtype, const void *logits, long long row, const void *uncond, long long uncond_row, int rows,
                           int vocab, const float *uniforms, int32_t *tokens, float *logprobs, adsa_stream_t stream)
{
    if (!how || rows < 0 || vocab < 1 || vocab > kDrawMaxVocab) return ADSA_EINVAL;
    if (dtype != ADSA_BF16 && dtype != ADSA_F16 && dtype != ADSA_F32) return ADSA_EINVAL;
    if (rows == 0) return ADSA_OK;
    if (!logits || !uniforms || !tokens) return ADSA_EINVAL;
    const uintptr_t align = dtype == ADSA_F32 ? 3 : 1;
    if (((uintptr_t)logits | (uintptr_t)uncond) & align) return ADSA_EINVAL;
    if (((uintptr_t)uniforms | (uintptr_t)tokens | (uintptr_t)logprobs | (uintptr_t)how->temperatures | (uintptr_t)how->top_ks | (uintptr_t)how->top_ps |
         (uintptr_t)how->min_ps) & 3)
        return ADSA_EINVAL;
    if (how->temperature != how->temperature || how->top_p != how->top_p || how->min_p != how->min_p || !isfinite(how->guidance)) return ADSA_EINVAL;
    DrawArgs a = {};
    a.logits = logits; a.uncond = uncond; a.row = row; a.uncond_row = uncond_row;
    a.rows = rows; a.vocab = vocab;
    const long long pitch = dtype == ADSA_F32 ? 4 : 8;             // elements of 16 bytes
    a.wide = (((uintptr_t)logits | (uintptr_t)uncond) & 15) == 0 && row % pitch == 0 && (!uncond || uncond_row % pitch == 0);
    a.guidance = how->guidance; a.temperature = how->temperature; a.top_p = how->top_p; a.min_p = how->min_p; a.top_k = how->top_k;
    a.temperatures = how->temperatures; a.top_ps = how->top_ps; a.min_ps = how->min_ps; a.top_ks = how->top_ks;
    a.uniforms = uniforms; a.tokens = tokens; a.logprobs = logprobs;
    const cudaStream_t st = (cudaStream_t)stream;
    const dim3 grid((unsigned)rows);
    const cudaError_t e = dtype == ADSA_BF16 ? launch_draw<__nv_bfloat16>(a, grid, st) : dtype == ADSA_F16 ? launch_draw<__half>(a, grid, st) : launch_draw<float>(a, grid, st);
    return e == cudaSuccess ? ADSA_OK : ADSA_ECUDA;
}
