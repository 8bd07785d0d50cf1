// The norms around a block, fused with its gate and residual scale:
//   z  = y / sqrt(mean y^2 + eps) * w_post      (or z = y)
//   x' = x + scale * gate * z
//   h  = x' / sqrt(mean x'^2 + eps) * w_pre
// y and x are read once and stay in registers over both sums, x' and h are written once.  h is made from x' before x' is
// rounded, so a 16-bit residual stream rounds once, on its way out.  HBM bounds it.
#include "adsa_half.cuh"

namespace adsa {

constexpr int kResMaxThreads = 1024;
constexpr int kResDeepRows = 148 * 16;        // rows from which threads hold two pieces: 16 blocks an SM of a B200

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

// eight elements as they lie in memory, and as four pairs of floats
template <typename T> struct Eight { uint4 w; };
template <> struct Eight<float> { float4 a, b; };
template <typename T>
__device__ __forceinline__ void spread(const Eight<T> &r, float2 (&f)[4])
{
    f[0] = unpack2<T>(r.w.x); f[1] = unpack2<T>(r.w.y); f[2] = unpack2<T>(r.w.z); f[3] = unpack2<T>(r.w.w);
}
__device__ __forceinline__ void spread(const Eight<float> &r, float2 (&f)[4])
{
    f[0] = make_float2(r.a.x, r.a.y); f[1] = make_float2(r.a.z, r.a.w); f[2] = make_float2(r.b.x, r.b.y); f[3] = make_float2(r.b.z, r.b.w);
}
template <typename T>
__device__ __forceinline__ void put_eight(T *p, const float2 (&f)[4])
{
    *reinterpret_cast<uint4 *>(p) = make_uint4(pack2<T>(f[0].x, f[0].y), pack2<T>(f[1].x, f[1].y), pack2<T>(f[2].x, f[2].y), pack2<T>(f[3].x, f[3].y));
}
template <>
__device__ __forceinline__ void put_eight<float>(float *p, const float2 (&f)[4])
{
    reinterpret_cast<float4 *>(p)[0] = make_float4(f[0].x, f[0].y, f[1].x, f[1].y);
    reinterpret_cast<float4 *>(p)[1] = make_float4(f[2].x, f[2].y, f[3].x, f[3].y);
}

// A row belongs to row_threads threads (whole warps), each with up to NP pieces of eight elements; a block holds
// blockDim / row_threads rows.
template <typename T, typename X, int NP>
__global__ void __launch_bounds__(kResMaxThreads)
norm_residual_kernel(const T *y, const X *x, const T *w_post, const T *gate, const T *w_pre, X *x_out, T *h, long long rows, int dim,
                     long long rows_per_gate, int row_threads, float scale, float eps)
{
    __shared__ float slots[2][32];
    pdl_wait();
    pdl_launch();
    const int part = threadIdx.x / row_threads, tid = threadIdx.x - part * row_threads, lane = threadIdx.x & 31, warp = tid >> 5;
    const int warps = row_threads >> 5, parts = blockDim.x / row_threads, first = part * warps;
    const long long row = (long long)blockIdx.x * parts + part;
    const int pieces = row < rows ? dim / 8 : 0;
    Eight<T> py[NP];
    Eight<X> px[NP];
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        const int i = tid + p * row_threads;
        if (i < pieces) {
            py[p] = reinterpret_cast<const Eight<T> *>(y + row * dim)[i];
            px[p] = reinterpret_cast<const Eight<X> *>(x + row * dim)[i];
        }
    }
    const float inv_dim = 1.f / (float)dim;
    float2 f2 = make_float2(1.f, 1.f);
    if (w_post) {
        float2 s2 = make_float2(0.f, 0.f);
#pragma unroll
        for (int p = 0; p < NP; ++p) {
            if (tid + p * row_threads < pieces) {
                float2 f[4];
                spread(py[p], f);
#pragma unroll
                for (int e = 0; e < 4; ++e) s2 = fma2(f[e], f[e], s2);
            }
        }
        const float inv = rsqrtf(row_sum(s2.x + s2.y, slots[0] + first, warps, warp, lane) * inv_dim + eps);
        f2 = make_float2(inv, inv);
    }
    const T *gr = gate ? gate + row / rows_per_gate * dim : nullptr;
    float2 v[NP][4], s2 = make_float2(0.f, 0.f);
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        const int i = tid + p * row_threads;
        if (i < pieces) {
            float2 z[4], w[4];
            spread(py[p], z);
            spread(px[p], v[p]);
            if (w_post) {
                spread(reinterpret_cast<const Eight<T> *>(w_post)[i], w);
#pragma unroll
                for (int e = 0; e < 4; ++e) z[e] = mul2(mul2(z[e], f2), w[e]);
            }
            if (gate) {
                spread(reinterpret_cast<const Eight<T> *>(gr)[i], w);
#pragma unroll
                for (int e = 0; e < 4; ++e) z[e] = mul2(z[e], w[e]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                v[p][e] = fma2(z[e], make_float2(scale, scale), v[p][e]);
                s2 = fma2(v[p][e], v[p][e], s2);
            }
            put_eight<X>(x_out + row * dim + i * 8, v[p]);
        }
    }
    if (!h) return;                            // (uniform)
    const float inv = rsqrtf(row_sum(s2.x + s2.y, slots[1] + first, warps, warp, lane) * inv_dim + eps);
    const float2 i2 = make_float2(inv, inv);
#pragma unroll
    for (int p = 0; p < NP; ++p) {
        const int i = tid + p * row_threads;
        if (i < pieces) {
            float2 w[4];
            spread(reinterpret_cast<const Eight<T> *>(w_pre)[i], w);
#pragma unroll
            for (int e = 0; e < 4; ++e) v[p][e] = mul2(mul2(v[p][e], i2), w[e]);
            put_eight<T>(h + row * dim + i * 8, v[p]);
        }
    }
}

namespace {

template <typename T, typename X>
cudaError_t launch_norm_residual(const void *y, const void *x, const void *w_post, const void *gate, const void *w_pre, void *x_out,
                                 void *h, long long rows, int dim, long long rows_per_gate, float scale, float eps, cudaStream_t st)
{
    const int pieces = dim / 8;
    // Few rows: one piece a thread, so that a row is one load deep (32 x 1280: 2.2 us).  Many: two.  A block per row, unless
    // a warp or less does: 36608 x 1280 with a 32-bit residual takes 96.9 us that way (5.8 TB/s), 98.6 with one piece a
    // thread, 100 with two rows a block, 109 with four and with a row per warp and five pieces a thread.
    const int want = rows >= kResDeepRows || pieces > kResMaxThreads ? 2 : 1;
    const int row_threads = ((pieces + want - 1) / want + 31) / 32 * 32, np = (pieces + row_threads - 1) / row_threads;
    const int parts = row_threads > 32 ? 1 : 4;
    const long long blocks = (rows + parts - 1) / parts;
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
    if (rows < 0 || rows > 0x7fffffffLL || dim < 8 || dim % 8 || dim > ADSA_MAX_NORM_DIM || !(eps >= 0.f)) return ADSA_EINVAL;
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
