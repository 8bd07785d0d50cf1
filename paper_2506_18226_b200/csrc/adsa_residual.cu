// The norms around a block, fused with its gate and residual scale:
//   z  = y / sqrt(mean y^2 + eps) * w_post      (or z = y)
//   x' = x + scale * gate * z
//   h  = x' / sqrt(mean x'^2 + eps) * w_pre
// One pass: y and x are read once and stay in registers over both sums, x' and h are written once.  h is made from x'
// before x' is rounded, so a 16-bit residual stream rounds once, on its way out.  HBM bounds it.
#include "adsa_half.cuh"

namespace adsa {

constexpr int kResMaxThreads = 1024;

// Sum over the `warps` warps of a row (warps 0 .. warps-1 of its part of the block); every thread of the block calls it.
__device__ __forceinline__ float row_sum(float x, float *slots, int warps, int warp, int lane)
{
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    if (warps == 1) return x;                 // (uniform over the block)
    if (lane == 0) slots[warp] = x;
    __syncthreads();
    x = lane < warps ? slots[lane] : 0.f;     // every warp adds the parts in the same order
#pragma unroll
    for (int o = 16; o > 0; o >>= 1) x += __shfl_xor_sync(0xffffffffu, x, o);
    return x;
}

// A row belongs to row_threads threads (whole warps), each with up to NP pieces of eight elements; a block holds
// blockDim / row_threads rows.
template <typename T, typename X, int NP>
__global__ void __launch_bounds__(kResMaxThreads)
norm_residual_kernel(const T *y, const X *x, const T *w_post, const T *gate, const T *w_pre, X *x_out, T *h, long long rows, int dim,
                     long long rows_per_gate, int row_threads, float scale, float eps)
{
    typedef Pack<T, 8> PT;
    typedef Pack<X, 8> PX;
    __shared__ float slots[2][32];
    pdl_wait();
    pdl_launch();
    const int part = threadIdx.x / row_threads, tid = threadIdx.x - part * row_threads, lane = threadIdx.x & 31, warp = tid >> 5;
    const int warps = row_threads >> 5, parts = blockDim.x / row_threads, first = part * warps;
    const long long row = (long long)blockIdx.x * parts + part;
    const bool live = row < rows;
    const int pieces = dim / 8;
    PT py[NP];
    PX px[NP];
    if (live) {
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            const int i = tid + p * row_threads;
            if (i < pieces) {
                py[p] = reinterpret_cast<const PT *>(y + row * dim)[i];
                px[p] = reinterpret_cast<const PX *>(x + row * dim)[i];
            }
        }
    }
    float inv = 1.f;
    if (w_post) {
        float ss = 0.f;
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            if (live && tid + p * row_threads < pieces) {
#pragma unroll
                for (int e = 0; e < 8; ++e) { const float f = to_f32(py[p].e[e]); ss = fmaf(f, f, ss); }
            }
        }
        ss = row_sum(ss, slots[0] + first, warps, warp, lane);
        inv = rsqrtf(ss / (float)dim + eps);
    }
    float v[NP][8], ss = 0.f;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        const int i = tid + p * row_threads;
        if (live && i < pieces) {
            PT wp, g;
            if (w_post) wp = reinterpret_cast<const PT *>(w_post)[i];
            if (gate) g = reinterpret_cast<const PT *>(gate + row / rows_per_gate * dim)[i];
            PX o;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                float z = to_f32(py[p].e[e]);
                if (w_post) z *= inv * to_f32(wp.e[e]);
                if (gate) z *= to_f32(g.e[e]);
                v[p][e] = fmaf(scale, z, to_f32(px[p].e[e]));
                o.e[e] = from_f32<X>(v[p][e]);
                ss = fmaf(v[p][e], v[p][e], ss);
            }
            reinterpret_cast<PX *>(x_out + row * dim)[i] = o;
        }
    }
    if (!h) return;                            // (uniform)
    ss = row_sum(ss, slots[1] + first, warps, warp, lane);
    inv = rsqrtf(ss / (float)dim + eps);
    if (!live) return;
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        const int i = tid + p * row_threads;
        if (i < pieces) {
            const PT wp = reinterpret_cast<const PT *>(w_pre)[i];
            PT o;
#pragma unroll
            for (int e = 0; e < 8; ++e) o.e[e] = from_f32<T>(v[p][e] * inv * to_f32(wp.e[e]));
            reinterpret_cast<PT *>(h + row * dim)[i] = o;
        }
    }
}

namespace {

template <typename T, typename X>
cudaError_t launch_norm_residual(const void *y, const void *x, const void *w_post, const void *gate, const void *w_pre, void *x_out,
                                 void *h, long long rows, int dim, long long rows_per_gate, float scale, float eps, cudaStream_t st)
{
    const int pieces = dim / 8;
    int np = 1;
    while (np < 2 && pieces > kResMaxThreads * np) np *= 2;
    const int row_threads = ((pieces + np - 1) / np + 31) / 32 * 32;
    const int parts = row_threads >= 256 ? 1 : 256 / row_threads;
    const long long blocks = (rows + parts - 1) / parts;
    if (blocks > 0x7fffffffLL) return cudaErrorInvalidValue;
    const dim3 grid((unsigned)blocks);
    const unsigned threads = (unsigned)(parts * row_threads);
#define ADSA_RES(N) \
    return launch_pdl(norm_residual_kernel<T, X, N>, grid, threads, 0, st, (const T *)y, (const X *)x, (const T *)w_post, (const T *)gate, \
                      (const T *)w_pre, (X *)x_out, (T *)h, rows, dim, rows_per_gate, row_threads, scale, eps)
    if (np == 1) ADSA_RES(1);
    ADSA_RES(2);
#undef ADSA_RES
}

}  // namespace
}  // namespace adsa

using namespace adsa;

extern "C" int adsa_norm_residual(int dtype, int x_dtype, const void *y, const void *x, const void *w_post, const void *gate,
                                  long long n_gates, const void *w_pre, void *x_out, void *h, long long rows, int dim, float scale, float eps,
                                  adsa_stream_t stream)
{
    if ((dtype != ADSA_BF16 && dtype != ADSA_F16) || (x_dtype != dtype && x_dtype != ADSA_F32)) return ADSA_EINVAL;
    if (rows < 0 || dim < 8 || dim % 8 || dim > ADSA_MAX_NORM_DIM || !(eps >= 0.f)) return ADSA_EINVAL;
    if (rows == 0) return ADSA_OK;
    if (!y || !x || !x_out || (h != nullptr) != (w_pre != nullptr)) return ADSA_EINVAL;
    if (gate && (n_gates < 1 || rows % n_gates)) return ADSA_EINVAL;
    if (((uintptr_t)y | (uintptr_t)x | (uintptr_t)w_post | (uintptr_t)gate | (uintptr_t)w_pre | (uintptr_t)x_out | (uintptr_t)h) & 15)
        return ADSA_EINVAL;
    const long long per_gate = gate ? rows / n_gates : 1;
    cudaStream_t st = (cudaStream_t)stream;
    cudaError_t e;
    if (dtype == ADSA_BF16)
        e = x_dtype == ADSA_F32 ? launch_norm_residual<__nv_bfloat16, float>(y, x, w_post, gate, w_pre, x_out, h, rows, dim, per_gate, scale, eps, st)
                                : launch_norm_residual<__nv_bfloat16, __nv_bfloat16>(y, x, w_post, gate, w_pre, x_out, h, rows, dim, per_gate, scale, eps, st);
    else
        e = x_dtype == ADSA_F32 ? launch_norm_residual<__half, float>(y, x, w_post, gate, w_pre, x_out, h, rows, dim, per_gate, scale, eps, st)
                                : launch_norm_residual<__half, __half>(y, x, w_post, gate, w_pre, x_out, h, rows, dim, per_gate, scale, eps, st);
    return e == cudaSuccess ? ADSA_OK : ADSA_ECUDA;
}
