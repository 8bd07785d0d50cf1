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
    unsigned long long mass[kDrawBins];     // of the steps; of sorted entries
    unsigned long long list[kDrawList];
    unsigned count[kDrawBins];
    unsigned long long warp_mass[kDrawWarps];
    unsigned warp_count[kDrawWarps];
    uint32_t warp_key[kDrawWarps], warp_low[kDrawWarps];
    unsigned long long before, at;
    unsigned bin, n, bin_count;
    int pick;
};

// Sums over the block, for all threads: x, and the sum of what threads before this one have.
__device__ __forceinline__ unsigned long long draw_scan(unsigned long long x, unsigned long long &before, DrawShared &s)
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
    before = incl - x + (warp ? __shfl_sync(0xffffffffu, w, (warp + 31) & 31) : 0);
    return __shfl_sync(0xffffffffu, w, 31);
}
// The list's n entries, largest first (room for a power of two).
__device__ __forceinline__ void draw_sort(DrawShared &s, unsigned n)
{
    unsigned size = 2;
    while (size < n) size *= 2;
    for (unsigned i = n + threadIdx.x; i < size; i += kDrawThreads) s.list[i] = 0;
    for (unsigned k = 2; k <= size; k *= 2) {
        for (unsigned j = k / 2; j; j /= 2) {
            // pairs within a warp's 64 entries need the warp alone
            if (j >= 32 || j == k / 2) __syncthreads();
            else __syncwarp();
            for (unsigned t = threadIdx.x; t < size / 2; t += kDrawThreads) {
                const unsigned i = 2 * t - (t & (j - 1)), o = i + j;
                const unsigned long long x = s.list[i], y = s.list[o];
                if ((x < y) == ((i & k) == 0)) { s.list[i] = y; s.list[o] = x; }
            }
        }
    }
    __syncthreads();
}

// The row's keys: shared memory up to `stashed`, the rest read again.
template <typename T>
struct DrawRow {
    const DrawArgs &a;
    const uint32_t *stash;
    int r, stashed;
    __device__ __forceinline__ uint32_t operator[](int i) const { return i < stashed ? stash[i] : draw_load<T>(a, r, i); }
};

// Steps between the logits of two keys, the larger one's first.
struct DrawSteps {
    float high, scale;
    __device__ __forceinline__ DrawSteps(uint32_t top, uint32_t low) : high(0.5f * draw_logit(top))
    {
        scale = (kDrawBins - 1) / (high - 0.5f * draw_logit(low));   // (halves: their difference is finite; infinite for neighbours, see below)
    }
    // descending in x; 0 for the larger end, the last for the lower (0 x infinity is NaN, which converts to 0)
    __device__ __forceinline__ unsigned operator()(uint32_t key) const
    {
        return min((unsigned)max((int)((high - 0.5f * draw_logit(key)) * scale), 0), (unsigned)kDrawBins - 1u);
    }
};

template <typename T>
__global__ void __launch_bounds__(kDrawThreads)
draw_kernel(const __grid_constant__ DrawArgs a, int stashed)
{
    __shared__ DrawShared s;
    extern __shared__ uint32_t draw_stash[];
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, V = a.vocab;
    const DrawRow<T> row{a, draw_stash, r, stashed};
    pdl_wait();
    pdl_launch();
    // the largest and the lowest
    uint32_t top = 0, low = 0xffffffffu;
    unsigned able = 0;                                             // ids that can be drawn
    for (int i = tid; i < V; i += kDrawThreads) {
        const uint32_t k = draw_load<T>(a, r, i);
        if (i < stashed) draw_stash[i] = k;
        top = max(top, k);
        if (k) { low = min(low, k); ++able; }
    }
    top = __reduce_max_sync(0xffffffffu, top);
    low = __reduce_min_sync(0xffffffffu, low);
    able = __reduce_add_sync(0xffffffffu, able);
    if (lane == 0) { s.warp_key[warp] = top; s.warp_low[warp] = low; s.warp_count[warp] = able; }
    __syncthreads();
    top = __reduce_max_sync(0xffffffffu, s.warp_key[lane]);
    low = __reduce_min_sync(0xffffffffu, s.warp_low[lane]);
    able = __reduce_add_sync(0xffffffffu, s.warp_count[lane]);
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
    const double largest = draw_logit(top), t = temperature;
    const double min_p = largest == INFINITY ? 1.0 : least > 0.f ? fmin((double)least, 1.0) : 0.0;   // (infinite ones alone, where there are any)
    const double goal_u = fmin(fmax((double)a.uniforms[r], 0.0), 1.0);
    if (!(temperature > 0.f)) top_k = 1;
    const bool by_count = top_k > 0 && (unsigned)top_k < able, by_mass = top_p < 1.f && top_k != 1;
    if (!by_count) top_k = (int)able;
    const auto share_of = [&](uint32_t key) { return key == top ? 1.0 : exp((draw_logit(key) - largest) / t); };
    const auto weight_of = [&](uint32_t key) { return (unsigned long long)(share_of(key) * kDrawOne + 0.5); };
    const auto enough = [&](uint32_t key) { return key == top || !(min_p > 0.0) || share_of(key) >= min_p; };
    const auto answer = [&](int id, uint32_t key, unsigned long long total) {
        a.tokens[r] = id;
        if (a.logprobs) a.logprobs[r] = (float)((key == top ? 0.0 : (draw_logit(key) - largest) / t) - log((double)total / kDrawOne));
    };

    // Histogram of the keys between high and low (both among them) above `above`: of counts, or of the masses of those that count.
    const auto histogram = [&](uint32_t high, uint32_t lowest, const DrawSteps &steps, bool masses) {
        for (int i = tid; i < kDrawBins; i += kDrawThreads) { s.count[i] = 0; s.mass[i] = 0; }
        __syncthreads();
        for (int i = tid; i < V; i += kDrawThreads) {
            const uint32_t k = row[i];
            if (k > high || k < lowest || k == 0) continue;
            const unsigned b = steps(k);
            atomicAdd(&s.count[b], 1u);
            if (masses) atomicAdd(&s.mass[b], weight_of(k));
        }
        __syncthreads();
    };
    // The ids with keys from high to lowest in steps up to `last` (from `first` on) into the list, as key and id, so that larger ones come first.
    const auto gather = [&](uint32_t high, uint32_t lowest, const DrawSteps &steps, unsigned first, unsigned last) {
        if (tid == 0) s.n = 0;
        __syncthreads();
        for (int i = tid; i < V; i += kDrawThreads) {
            const uint32_t k = row[i];
            if (k > high || k < lowest || k == 0) continue;
            const unsigned b = steps(k);
            if (b < first || b > last) continue;
            s.list[atomicAdd(&s.n, 1u)] = (unsigned long long)k << 32 | (0xffffffffu - (unsigned)i);
        }
        __syncthreads();
        draw_sort(s, s.n);
    };
    // The step in which the running count passes need - 1, or the last whose masses before it are below the goal: s.bin, s.bin_count, s.before
    const auto find_step = [&](bool masses, unsigned long long need, double goal, unsigned long long start) {
        if (tid == 0) s.pick = -1;
        __syncthreads();
        unsigned long long before;
        const unsigned long long c0 = s.count[2 * tid], c1 = s.count[2 * tid + 1], m0 = masses ? s.mass[2 * tid] : c0, m1 = masses ? s.mass[2 * tid + 1] : c1;
        draw_scan(m0 + m1, before, s);
        before += start;
        const auto good = [&](unsigned long long c, unsigned long long at) { return c && (masses ? (double)at < goal || at == start : at < need); };
        const bool g0 = good(c0, before), g1 = good(c1, before + m0);
        if (g0 || g1) atomicMax(&s.pick, 2 * tid + (g1 ? 1 : 0));
        __syncthreads();
        if (s.pick >> 1 == tid) {
            s.bin = (unsigned)s.pick;
            s.before = s.pick & 1 ? before + m0 : before;
            s.bin_count = (unsigned)(s.pick & 1 ? c1 : c0);
        }
        __syncthreads();
    };

    uint32_t thr = low;                                            // the border: keys above thr, and the first `ties` ids with just that key
    unsigned ties = 0xffffffffu;
    bool listed = able <= kDrawList;                               // all that can be kept is in the list, sorted
    if (listed) {
        gather(top, low, DrawSteps(top, low), 0u, kDrawBins - 1u);
    } else if (by_count) {
        uint32_t high = top, lowest = low;
        unsigned long long start = 0;
        for (int level = 0;; ++level) {
            const DrawSteps steps(high, lowest);
            histogram(high, lowest, steps, false);
            find_step(false, (unsigned)top_k, 0.0, start);
            const unsigned bin = s.bin, in_bin = s.bin_count;
            const unsigned long long before = s.before;
            if (level == 0 && before + in_bin <= kDrawList) {
                gather(high, lowest, steps, 0u, bin);
                listed = true;
                break;
            }
            if (in_bin <= kDrawList) {
                gather(high, lowest, steps, bin, bin);
                const unsigned at = (unsigned)(top_k - before) - 1u;   // the last that is kept
                thr = (uint32_t)(s.list[at] >> 32);
                unsigned first = 0, last = at;                     // its first equal
                while (first < last) {
                    const unsigned mid = (first + last) / 2;
                    if ((uint32_t)(s.list[mid] >> 32) == thr) last = mid;
                    else first = mid + 1;
                }
                ties = at - first + 1u;
                break;
            }
            // too many in one step: between its own largest and lowest
            uint32_t most = 0, fewest = 0xffffffffu;
            for (int i = tid; i < V; i += kDrawThreads) {
                const uint32_t k = row[i];
                if (k <= high && k >= lowest && k && steps(k) == bin) { most = max(most, k); fewest = min(fewest, k); }
            }
            most = __reduce_max_sync(0xffffffffu, most);
            fewest = __reduce_min_sync(0xffffffffu, fewest);
            if (lane == 0) { s.warp_key[warp] = most; s.warp_low[warp] = fewest; }
            __syncthreads();
            high = __reduce_max_sync(0xffffffffu, s.warp_key[lane]);
            lowest = __reduce_min_sync(0xffffffffu, s.warp_low[lane]);
            __syncthreads();
            start = before;
            if (high == lowest) { thr = high; ties = (unsigned)(top_k - before); break; }
        }
    }
    if (listed) {
        unsigned n = min((unsigned)top_k, s.n);
        // two entries a thread: their weights, the mass before them
        const auto key_at = [&](unsigned i) { return (uint32_t)(s.list[i] >> 32); };
        const unsigned long long w0 = 2u * tid < n ? weight_of(key_at(2 * tid)) : 0, w1 = 2u * tid + 1u < n ? weight_of(key_at(2 * tid + 1)) : 0;
        unsigned long long before;
        unsigned long long total = draw_scan(w0 + w1, before, s);
        const double goal = by_mass ? fmax((double)top_p, 0.0) * (double)total : INFINITY;
        const bool in0 = 2u * tid < n && (tid == 0 || ((double)before < goal && enough(key_at(2 * tid)))),
                   in1 = 2u * tid + 1u < n && (double)(before + w0) < goal && enough(key_at(2 * tid + 1));
        unsigned long long none;
        n = (unsigned)draw_scan((unsigned)in0 + (unsigned)in1, none, s);   // (a head of the list)
        // by id
        unsigned long long e0 = 0, e1 = 0;
        if (in0) e0 = (s.list[2 * tid] << 32) | (s.list[2 * tid] >> 32);
        if (in1) e1 = (s.list[2 * tid + 1] << 32) | (s.list[2 * tid + 1] >> 32);
        __syncthreads();
        s.list[2 * tid] = e0;
        s.list[2 * tid + 1] = e1;
        __syncthreads();
        draw_sort(s, n);
        const auto low_key = [&](unsigned i) { return (uint32_t)s.list[i]; };
        const unsigned long long v0 = 2u * tid < n ? weight_of(low_key(2 * tid)) : 0, v1 = 2u * tid + 1u < n ? weight_of(low_key(2 * tid + 1)) : 0;
        if (tid == 0) s.pick = (int)n - 1;
        total = draw_scan(v0 + v1, before, s);
        const double at = goal_u * (double)total;
        if (2u * tid < n && (double)(before + v0) >= at) atomicMin(&s.pick, 2 * tid);
        else if (2u * tid + 1u < n && (double)(before + v0 + v1) >= at) atomicMin(&s.pick, 2 * tid + 1);
        __syncthreads();
        if (tid == 0) answer((int)(0xffffffffu - (uint32_t)(s.list[s.pick] >> 32)), low_key(s.pick), total);
        return;
    }
    if (by_mass) {
        // mass of what top_k keeps: of the ids at its border, the first `ties`
        unsigned long long sum = 0, none;
        unsigned equal = 0;
        uint32_t high = top, lowest = thr;
        DrawSteps steps(high, lowest);
        histogram(high, lowest, steps, true);
        for (int i = tid; i < V; i += kDrawThreads) equal += row[i] == thr;
        const unsigned n_equal = (unsigned)draw_scan(equal, none, s), drop = n_equal - min(n_equal, ties);
        if (tid == 0 && drop) {                                    // (they are in the last step that holds any)
            s.mass[steps(thr)] -= drop * weight_of(thr);
            s.count[steps(thr)] -= drop;
        }
        __syncthreads();
        sum = s.mass[2 * tid] + s.mass[2 * tid + 1];
        const double goal = fmax((double)top_p, 0.0) * (double)draw_scan(sum, none, s);
        unsigned long long start = 0;
        const uint32_t k_thr = thr;
        for (;;) {
            find_step(true, 0, goal, start);
            const unsigned bin = s.bin, in_bin = s.bin_count + (bin == steps(k_thr) && lowest == k_thr ? drop : 0u);
            const unsigned long long before = s.before;
            uint32_t most = 0, fewest = 0xffffffffu;
            if (in_bin <= kDrawList) {
                gather(high, lowest, steps, bin, bin);
                const unsigned n = s.n - (bin == steps(k_thr) && lowest == k_thr ? drop : 0u);
                const unsigned long long w0 = 2u * tid < n ? weight_of((uint32_t)(s.list[2 * tid] >> 32)) : 0,
                                         w1 = 2u * tid + 1u < n ? weight_of((uint32_t)(s.list[2 * tid + 1] >> 32)) : 0;
                unsigned long long at;
                draw_scan(w0 + w1, at, s);
                at += before;
                const unsigned kept = (unsigned)draw_scan((unsigned)(2u * tid < n && ((double)at < goal || tid == 0)) + (unsigned)(2u * tid + 1u < n && (double)(at + w0) < goal), none, s);
                thr = (uint32_t)(s.list[kept - 1u] >> 32);
                unsigned first = 0, last = kept - 1u;
                while (first < last) {
                    const unsigned mid = (first + last) / 2;
                    if ((uint32_t)(s.list[mid] >> 32) == thr) last = mid;
                    else first = mid + 1;
                }
                ties = kept - first;
                break;
            }
            for (int i = tid; i < V; i += kDrawThreads) {
                const uint32_t k = row[i];
                if (k <= high && k >= lowest && k && steps(k) == bin) { most = max(most, k); fewest = min(fewest, k); }
            }
            most = __reduce_max_sync(0xffffffffu, most);
            fewest = __reduce_min_sync(0xffffffffu, fewest);
            if (lane == 0) { s.warp_key[warp] = most; s.warp_low[warp] = fewest; }
            __syncthreads();
            high = __reduce_max_sync(0xffffffffu, s.warp_key[lane]);
            lowest = __reduce_min_sync(0xffffffffu, s.warp_low[lane]);
            __syncthreads();
            start = before;
            if (high == lowest) {
                // equal keys: those with less than the goal before them, one at least
                const unsigned long long w = weight_of(high);
                unsigned n = in_bin - (high == k_thr ? drop : 0u), at = 1;
                while (at < n) {
                    const unsigned mid = (at + n + 1) / 2;         // is the mid-th kept?
                    if ((double)(before + (mid - 1) * w) < goal) at = mid;
                    else n = mid - 1;
                }
                thr = high;
                ties = at;
                break;
            }
            steps = DrawSteps(high, lowest);
            histogram(high, lowest, steps, true);
            if (tid == 0 && drop && lowest == k_thr) {
                s.mass[steps(k_thr)] -= drop * weight_of(k_thr);
                s.count[steps(k_thr)] -= drop;
            }
            __syncthreads();
        }
        __syncthreads();
    }
    const auto kept_key = [&](uint32_t k) { return k >= thr && k && enough(k); };   // (min_p is a border of keys too)
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
            const uint32_t k = row[i];
            if (!kept_key(k)) continue;
            if (k == thr) ++equal;
            else { sum += weight_of(k); ++kept; }
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
        const unsigned long long w = weight_of(thr);
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
        const uint32_t k = i < end ? row[i] : 0u;
        bool kept = i < end && kept_key(k);
        const unsigned equal = __ballot_sync(0xffffffffu, kept && k == thr);
        if (kept && k == thr) kept = equal_before + __popc(equal & ((1u << lane) - 1u)) < ties;
        unsigned long long run = kept ? weight_of(k) : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const unsigned long long x = __shfl_up_sync(0xffffffffu, run, o); if (lane >= o) run += x; }
        const unsigned all = __ballot_sync(0xffffffffu, kept), reached = __ballot_sync(0xffffffffu, kept && (double)(before + run) >= goal);
        const int pick = reached ? __ffs(reached) - 1 : 31 - __clz(all);
        if (lane == pick) {
            answer(i, k, total);
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
