// The draw of the next token: temperature, the top_k largest logits, the smallest head of them that holds top_p of their mass,
// weights of min_p of the largest at least, and one of what is left by a given uniform number.
//
// All three rules keep a head of the ids in the order (logit descending, id ascending), so what is kept is one border: a key and how
// many of the ids with just that logit.  Keys are the logits' bits in an order that integers have; borders are found by the key's bytes,
// most significant first, from counts (top_k) or masses (top_p) per byte.  Weights are made in 64 bits and added up as whole
// multiples of 2^-42 of the largest: sums do not depend on their order, and an id is kept or drawn as the real numbers say.
//
// A block per row; keys lie in shared memory, as many as fit.  Where up to 2048 ids can be kept (by top_k, or the vocabulary has no more),
// these are sorted, cut, sorted again by id and summed: three passes over the row and two sorts.  Else the borders are found by histograms
// of 2048 steps between the largest and the lowest logit, of counts or of masses, and a sort of the step that holds the border (or again, where
// one step holds too many), and the sum is followed over the row itself.
#include <math.h>

#include "adsa_half.cuh"

namespace adsa {

constexpr int kDrawThreads = 1024, kDrawWarps = kDrawThreads / 32;
constexpr int kDrawBins = 2048, kDrawList = 2048;   // steps of a histogram; entries that are sorted
constexpr int kDrawMaxVocab = 1 << 20;       // so that 2^20 weights of 2^42 fit 63 bits
constexpr double kDrawOne = 4398046511104.0;   // 2^42

struct DrawArgs {
    const void *logits, *uncond;
    long long row, uncond_row;              // element strides
    int rows, vocab;
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

template <typename T>
__device__ __forceinline__ uint32_t draw_load(const DrawArgs &a, int r, int i)
{
    float x = to_f32(((const T *)a.logits)[(size_t)r * a.row + i]);
    if (a.uncond) {
        const float u = to_f32(((const T *)a.uncond)[(size_t)r * a.uncond_row + i]);
        x = __fadd_rn(u, __fmul_rn(a.guidance, __fsub_rn(x, u)));
    }
    return draw_key(x);
}

struct DrawShared {
    unsigned long long mass[kDrawBins];     // of the steps
    unsigned long long list[kDrawList];
    unsigned count[kDrawBins];
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
    if (key == s.top) return 1.0;
    if (!(x > -64000.0)) return 0.0;
    const double k = x + magic, r = (x - (k - magic)) * 0.010830424696249145;   // ln 2 / 64
    double p = fma(r, 1.0 / 120, 1.0 / 24);
    p = fma(p, r, 1.0 / 6);
    p = fma(p, r, 0.5);
    p = fma(p, r, 1.0);
    p = fma(p, r, 1.0);
    const int n = __double2loint(k);                               // (two's complement in the low bits of the sum)
    const double y = p * s.power[n & 63];
    return __hiloint2double(__double2hiint(y) + ((n >> 6) << 20), __double2loint(y));
}
// ... as a whole multiple of 2^-42
__device__ __forceinline__ unsigned long long draw_weight(uint32_t key, const DrawShared &s)
{
    return (unsigned long long)__double_as_longlong(fma(draw_share(key, s), kDrawOne, 4503599627370496.0)) & 0xfffffffffffffULL;   // 2^52 + the multiple
}
__device__ __noinline__ unsigned long long draw_weight_of(uint32_t key, const DrawShared &s) { return draw_weight(key, s); }
__device__ __noinline__ bool draw_enough(uint32_t key, double min_p, const DrawShared &s) { return draw_share(key, s) >= min_p; }

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
    unsigned size = 2;
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

// The row's keys: shared memory up to `stashed`, the rest read again.
template <typename T>
struct DrawRow {
    const uint32_t *stash;
    int r, stashed;
    __device__ __forceinline__ uint32_t at(const DrawArgs &a, int i) const { return i < stashed ? stash[i] : draw_load<T>(a, r, i); }
};

// Steps between the logits of two keys.
struct DrawSteps {
    uint32_t top, low;
    float high, scale;
    __device__ __forceinline__ DrawSteps(uint32_t top_, uint32_t low_) : top(top_), low(low_), high(0.5f * draw_logit(top_))
    {
        scale = (kDrawBins - 1) / (high - 0.5f * draw_logit(low));   // (halves: their difference is finite; it may round to 0)
    }
    // descending in x; 0 for the larger end, the last for the lower (0 x infinity is NaN, which converts to 0)
    __device__ __forceinline__ unsigned operator()(uint32_t key) const
    {
        return min((unsigned)max((int)((high - 0.5f * draw_logit(key)) * scale), 0), (unsigned)kDrawBins - 1u);
    }
    __device__ __forceinline__ bool has(uint32_t key) const { return key <= top && key >= low; }
};

// How many of the row's keys lie in each step, and with `masses` their weights.
template <typename T>
__device__ __noinline__ void draw_histogram(const DrawArgs &a, DrawRow<T> row, DrawSteps steps, bool masses, DrawShared &s)
{
    __syncthreads();
    for (int i = threadIdx.x; i < kDrawBins; i += kDrawThreads) { s.count[i] = 0; s.mass[i] = 0; }
    __syncthreads();
#pragma unroll 2
    for (int i = threadIdx.x; i < a.vocab; i += kDrawThreads) {
        const uint32_t k = row.at(a, i);
        if (!steps.has(k)) continue;
        const unsigned b = steps(k);
        atomicAdd(&s.count[b], 1u);
        if (masses) atomicAdd(&s.mass[b], draw_weight(k, s));
    }
    __syncthreads();
}
// The ids with keys in the steps from `first` to `last` into the list, as key and id, sorted: larger keys first, of equal ones lower ids.
template <typename T>
__device__ __noinline__ void draw_gather(const DrawArgs &a, DrawRow<T> row, DrawSteps steps, unsigned first, unsigned last, DrawShared &s)
{
    __syncthreads();
    if (threadIdx.x == 0) s.n = 0;
    __syncthreads();
#pragma unroll 2
    for (int i = threadIdx.x; i < a.vocab; i += kDrawThreads) {
        const uint32_t k = row.at(a, i);
        if (!steps.has(k)) continue;
        const unsigned b = steps(k);
        if (b >= first && b <= last) s.list[atomicAdd(&s.n, 1u)] = (unsigned long long)k << 32 | (0xffffffffu - (unsigned)i);
    }
    __syncthreads();
    draw_sort(s, s.n);
}
// Largest and lowest key of a step.
template <typename T>
__device__ __noinline__ uint2 draw_step_ends(const DrawArgs &a, DrawRow<T> row, DrawSteps steps, unsigned bin, DrawShared &s)
{
    uint32_t most = 0, fewest = 0xffffffffu;
    for (int i = threadIdx.x; i < a.vocab; i += kDrawThreads) {
        const uint32_t k = row.at(a, i);
        if (steps.has(k) && steps(k) == bin) { most = max(most, k); fewest = min(fewest, k); }
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
    __shared__ DrawShared s;
    extern __shared__ uint32_t draw_stash[];
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, V = a.vocab;
    const DrawRow<T> row{draw_stash, r, stashed};
    if (tid < 64) s.power[tid] = exp2(tid / 64.0);
    pdl_wait();
    pdl_launch();
    // the largest and the lowest
    uint32_t top = 0, low = 0xffffffffu;
    unsigned able = 0;                                             // ids that can be drawn
#pragma unroll 4
    for (int i = tid; i < V; i += kDrawThreads) {
        const uint32_t k = draw_load<T>(a, r, i);
        if (i < stashed) draw_stash[i] = k;
        top = max(top, k);
        low = min(low, k - 1u);                                    // (a key of 0 becomes the largest number)
        able += k != 0u;
    }
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
    unsigned ties = 0xffffffffu, n = 0;
    bool listed = able <= kDrawList, cut = false;                  // all that can be kept is in the list, sorted; what is in the list's first n is kept
    if (listed) {
        draw_gather(a, row, DrawSteps(top, low), 0u, kDrawBins - 1u, s);
    } else if (by_count) {
        DrawSteps steps(top, low);
        unsigned long long start = 0;
        for (bool first = true;; first = false) {
            draw_histogram(a, row, steps, false, s);
            draw_find(false, (double)top_k, start, s);
            const unsigned bin = s.bin, in_bin = s.bin_count;
            const unsigned long long before = s.before;
            listed = first && before + in_bin <= kDrawList;
            if (listed || in_bin <= kDrawList) {
                draw_gather(a, row, steps, listed ? 0u : bin, bin, s);
                if (!listed) {
                    const unsigned last = (unsigned)(top_k - before) - 1u;   // that is kept
                    thr = (uint32_t)(s.list[last] >> 32);
                    ties = last + 1u - draw_first_equal(s, last);
                }
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
    if (!listed && min_key > thr && min_p > 0.0) {
        // few by min_p, whose mass is below top_p of all: then top_p cuts nothing more
        unsigned long long sum = 0, few = 0;
        unsigned many = 0, equal = 0;
#pragma unroll 2
        for (int i = tid; i < V; i += kDrawThreads) {
            const uint32_t k = row.at(a, i);
            if (k < thr) continue;
            const unsigned long long w = by_mass && k > thr ? draw_weight(k, s) : 0;
            sum += w;
            equal += k == thr;
            if (k >= min_key) { few += w; ++many; }
        }
        many = (unsigned)draw_scan(many, &unused, s);
        bool first = !by_mass;
        if (by_mass) {
            const unsigned long long border = min(draw_scan(equal, &unused, s), (unsigned long long)ties) * draw_weight_of(thr, s);
            const double goal = fmax((double)top_p, 0.0) * (double)(draw_scan(sum, &unused, s) + border);
            first = (double)draw_scan(few, &unused, s) < goal;
        }
        if (first) {
            thr = min_key;
            ties = 0xffffffffu;
            if (many <= kDrawList) {
                draw_gather(a, row, DrawSteps(top, min_key), 0u, kDrawBins - 1u, s);
                listed = cut = true;
                n = many;
            }
        }
        if (first && !listed) cut = true;
    }
    if (listed && !cut) {
        n = min((unsigned)top_k, s.n);
        // two entries a thread: their weights, the mass before them
        const uint32_t k0 = (uint32_t)(s.list[2 * tid] >> 32), k1 = (uint32_t)(s.list[2 * tid + 1] >> 32);
        const unsigned long long w0 = 2u * tid < n ? draw_weight_of(k0, s) : 0, w1 = 2u * tid + 1u < n ? draw_weight_of(k1, s) : 0;
        unsigned long long before;
        const unsigned long long total = draw_scan(w0 + w1, &before, s);
        const double goal = by_mass ? fmax((double)top_p, 0.0) * (double)total : INFINITY;
        const unsigned in0 = 2u * tid < n && (tid == 0 || ((double)before < goal && k0 >= min_key)),
                       in1 = 2u * tid + 1u < n && (double)(before + w0) < goal && k1 >= min_key;
        n = (unsigned)draw_scan(in0 + in1, &unused, s);            // (a head of the list)
    }
    if (listed) {
        // by id
        unsigned long long e0 = s.list[2 * tid], e1 = s.list[2 * tid + 1], before;
        __syncthreads();
        s.list[2 * tid] = e0 << 32 | e0 >> 32;
        s.list[2 * tid + 1] = e1 << 32 | e1 >> 32;
        if (tid == 0) s.pick = (int)n - 1;
        __syncthreads();
        draw_sort(s, n);
        const unsigned long long v0 = 2u * tid < n ? draw_weight_of((uint32_t)s.list[2 * tid], s) : 0,
                                 v1 = 2u * tid + 1u < n ? draw_weight_of((uint32_t)s.list[2 * tid + 1], s) : 0;
        const unsigned long long total = draw_scan(v0 + v1, &before, s);
        const double at = goal_u * (double)total;
        if (2u * tid < n && (double)(before + v0) >= at) atomicMin(&s.pick, 2 * tid);
        else if (2u * tid + 1u < n && (double)(before + v0 + v1) >= at) atomicMin(&s.pick, 2 * tid + 1);
        __syncthreads();
        if (tid == 0) {
            const uint32_t key = (uint32_t)s.list[s.pick];
            a.tokens[r] = (int)(0xffffffffu - (uint32_t)(s.list[s.pick] >> 32));
            if (a.logprobs) a.logprobs[r] = (float)((key == top ? 0.0 : (draw_logit(key) - largest) / (double)temperature) - log((double)total / kDrawOne));
        }
        return;
    }
    if (by_mass && !cut) {
        // of the ids at top_k's border, the first `ties` count
        const uint32_t k_thr = thr;
        unsigned equal = 0;
        if (ties != 0xffffffffu) {
            for (int i = tid; i < V; i += kDrawThreads) equal += row.at(a, i) == thr;
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
    if (min_key > thr) {
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
        const int per = ((end - begin) + kDrawWarps - 1) / kDrawWarps, i0 = begin + warp * per, i1 = min(i0 + per, end);
        unsigned long long sum = 0;
        unsigned equal = 0, kept = 0;
        for (int i = i0 + lane; i < i1; i += 32) {
            const uint32_t k = row.at(a, i);
            if (k < thr) continue;
            if (k == thr) ++equal;
            else { sum += draw_weight(k, s); ++kept; }
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
        const uint32_t k = i < end ? row.at(a, i) : 0u;
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
    constexpr int most = (227 * 1024 - (int)sizeof(DrawShared) - 1024) / 4;
    static int told[64];
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const bool known = dev >= 0 && dev < 64;
    if (!known || !__atomic_load_n(&told[dev], __ATOMIC_ACQUIRE)) {
        e = cudaFuncSetAttribute((const void *)draw_kernel<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, most * 4);
        if (e != cudaSuccess) return e;
        if (known) __atomic_store_n(&told[dev], 1, __ATOMIC_RELEASE);
    }
    const int stashed = a.vocab < most ? a.vocab : most;
    return launch_pdl(draw_kernel<T>, grid, kDrawThreads, (size_t)stashed * 4, st, a, stashed);
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
    a.guidance = how->guidance; a.temperature = how->temperature; a.top_p = how->top_p; a.min_p = how->min_p; a.top_k = how->top_k;
    a.temperatures = how->temperatures; a.top_ps = how->top_ps; a.min_ps = how->min_ps; a.top_ks = how->top_ks;
    a.uniforms = uniforms; a.tokens = tokens; a.logprobs = logprobs;
    const cudaStream_t st = (cudaStream_t)stream;
    const dim3 grid((unsigned)rows);
    const cudaError_t e = dtype == ADSA_BF16 ? launch_draw<__nv_bfloat16>(a, grid, st) : dtype == ADSA_F16 ? launch_draw<__half>(a, grid, st) : launch_draw<float>(a, grid, st);
    return e == cudaSuccess ? ADSA_OK : ADSA_ECUDA;
}
