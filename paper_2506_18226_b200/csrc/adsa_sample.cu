// The draw of the next token: temperature, the top_k largest logits, the smallest head of them that holds top_p of their mass,
// weights of min_p of the largest at least, and one of what is left by a given uniform number.
//
// All three rules keep a head of the ids in the order (logit descending, id ascending), so what is kept is one border: a key and how
// many of the ids with just that logit.  Keys are the logits' bits in an order that integers have; borders are found by the key's bytes,
// most significant first, from counts (top_k) or masses (top_p) per byte.  Weights are made in 64 bits and added up as whole
// multiples of 2^-42 of the largest: sums do not depend on their order, and an id is kept or drawn as the real numbers say.
//
// A block per row.
#include <math.h>

#include "adsa_half.cuh"

namespace adsa {

constexpr int kDrawThreads = 1024, kDrawWarps = kDrawThreads / 32;
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
    unsigned long long mass[256];
    unsigned count[256];
    unsigned long long warp_mass[kDrawWarps];
    unsigned warp_count[kDrawWarps];
    uint32_t warp_key[kDrawWarps];
    unsigned long long before;              // mass above the border's key so far
    uint32_t prefix;
    unsigned need, first;
};

__device__ __forceinline__ unsigned long long sum_of(unsigned long long x, DrawShared &s)
{
#pragma unroll
    for (int o = 16; o; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    __syncthreads();
    if ((threadIdx.x & 31) == 0) s.warp_mass[threadIdx.x >> 5] = x;
    __syncthreads();
    x = 0;
    for (int w = 0; w < kDrawWarps; ++w) x += s.warp_mass[w];
    return x;
}

template <typename T>
__global__ void __launch_bounds__(kDrawThreads)
draw_kernel(const __grid_constant__ DrawArgs a)
{
    __shared__ DrawShared s;
    const int r = blockIdx.x, tid = threadIdx.x, lane = tid & 31, warp = tid >> 5, V = a.vocab;
    pdl_wait();
    pdl_launch();
    // the largest
    uint32_t top = 0;
    for (int i = tid; i < V; i += kDrawThreads) top = max(top, draw_load<T>(a, r, i));
    top = __reduce_max_sync(0xffffffffu, top);
    if (lane == 0) s.warp_key[warp] = top;
    __syncthreads();
    for (int w = 0; w < kDrawWarps; ++w) top = max(top, s.warp_key[w]);
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
    if (!(temperature > 0.f)) top_k = 1;
    const auto weight_of = [&](uint32_t key) -> unsigned long long {   // of the largest's, 2^42; of infinite largest ones: they alone
        const double x = draw_logit(key);
        return key == top ? (unsigned long long)kDrawOne : (unsigned long long)(exp((x - largest) / t) * kDrawOne + 0.5);
    };
    // the border: keys above thr, and the first `ties` ids with just that key
    uint32_t thr = 1;
    unsigned ties = 0xffffffffu;
    if (top_k > 0 && top_k < V) {
        if (tid == 0) { s.prefix = 0u; s.need = (unsigned)top_k; }
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (tid < 256) s.count[tid] = 0u;
            __syncthreads();
            const uint32_t prefix = s.prefix, mask = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
            for (int i = tid; i < V; i += kDrawThreads) {
                const uint32_t k = draw_load<T>(a, r, i);
                if ((k & mask) == prefix) atomicAdd(&s.count[(k >> shift) & 255u], 1u);
            }
            __syncthreads();
            if (tid == 0) {
                unsigned need = s.need, b = 255u;
                for (;; --b) {
                    if (s.count[b] >= need || b == 0u) break;
                    need -= s.count[b];
                }
                s.prefix = prefix | (b << shift);
                s.need = need;
            }
            __syncthreads();
        }
        if (s.prefix > 0u) { thr = s.prefix; ties = s.need; }       // (key 0: fewer than top_k can be drawn at all)
    }
    if (top_p < 1.f && top_k != 1) {
        // mass of what top_k keeps (of the ids at its border, the first `ties`)
        unsigned long long sum = 0;
        unsigned equal = 0;
        for (int i = tid; i < V; i += kDrawThreads) {
            const uint32_t k = draw_load<T>(a, r, i);
            if (k > thr) sum += weight_of(k);
            equal += k == thr;
        }
        const unsigned n_equal = (unsigned)min(sum_of(equal, s), (unsigned long long)ties);
        const unsigned long long total = sum_of(sum, s) + n_equal * weight_of(thr);
        const double goal = fmax((double)top_p, 0.0) * (double)total;
        if (tid == 0) { s.prefix = 0u; s.before = 0; }
        for (int shift = 24; shift >= 0; shift -= 8) {
            if (tid < 256) { s.mass[tid] = 0; s.count[tid] = 0; }
            __syncthreads();
            const uint32_t prefix = s.prefix, mask = shift == 24 ? 0u : 0xffffffffu << (shift + 8);
            for (int i = tid; i < V; i += kDrawThreads) {
                const uint32_t k = draw_load<T>(a, r, i);
                if ((k & mask) == prefix && k > thr) {
                    atomicAdd(&s.mass[(k >> shift) & 255u], weight_of(k));
                    atomicAdd(&s.count[(k >> shift) & 255u], 1u);
                }
            }
            if (tid == 0 && (thr & mask) == prefix) {
                atomicAdd(&s.mass[(thr >> shift) & 255u], n_equal * weight_of(thr));
                atomicAdd(&s.count[(thr >> shift) & 255u], n_equal);
            }
            __syncthreads();
            if (tid == 0) {
                // the last byte with ids whose mass before it is below the goal
                unsigned long long before = s.before, at = before;
                unsigned b = 255u, found = 255u;
                bool any = false;
                for (;; --b) {
                    if (s.count[b]) {
                        if (any && !((double)before < goal)) break;
                        found = b;
                        at = before;
                        any = true;
                        before += s.mass[b];
                    }
                    if (b == 0u) break;
                }
                s.prefix = prefix | (found << shift);
                s.before = at;
                s.need = s.count[found];
            }
            __syncthreads();
        }
        // of the ids at the border, those with less than the goal before them: one at least
        const unsigned long long w = weight_of(s.prefix), before = s.before;
        unsigned n = s.need, lo = 1;
        while (lo < n) {
            const unsigned mid = (lo + n + 1) / 2;                 // is the mid-th kept?
            if ((double)(before + (mid - 1) * w) < goal) lo = mid;
            else n = mid - 1;
        }
        thr = s.prefix;
        ties = lo;
        __syncthreads();
    }
    // min_p is a border of keys too
    const auto kept_key = [&](uint32_t k) {
        return k >= thr && (k == top || !(min_p > 0.0) || exp((draw_logit(k) - largest) / t) >= min_p);
    };
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
            const uint32_t k = draw_load<T>(a, r, i);
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
            goal = fmin(fmax((double)a.uniforms[r], 0.0), 1.0) * (double)total;
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
        const uint32_t k = i < end ? draw_load<T>(a, r, i) : 0u;
        bool kept = i < end && kept_key(k);
        const unsigned equal = __ballot_sync(0xffffffffu, kept && k == thr);
        if (kept && k == thr) kept = equal_before + __popc(equal & ((1u << lane) - 1u)) < ties;
        unsigned long long run = kept ? weight_of(k) : 0;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const unsigned long long x = __shfl_up_sync(0xffffffffu, run, o); if (lane >= o) run += x; }
        const unsigned all = __ballot_sync(0xffffffffu, kept), reached = __ballot_sync(0xffffffffu, kept && (double)(before + run) >= goal);
        const int pick = reached ? __ffs(reached) - 1 : 31 - __clz(all);
        if (lane == pick) {
            a.tokens[r] = i;
            if (a.logprobs) a.logprobs[r] = (float)((k == top ? 0.0 : (draw_logit(k) - largest) / t) - log((double)total / kDrawOne));
        }
    }
}

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
    const cudaError_t e = dtype == ADSA_BF16 ? launch_pdl(draw_kernel<__nv_bfloat16>, grid, kDrawThreads, 0, st, a)
                          : dtype == ADSA_F16 ? launch_pdl(draw_kernel<__half>, grid, kDrawThreads, 0, st, a)
                                              : launch_pdl(draw_kernel<float>, grid, kDrawThreads, 0, st, a);
    return e == cudaSuccess ? ADSA_OK : ADSA_ECUDA;
}
