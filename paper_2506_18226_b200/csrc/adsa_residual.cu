// The norms around a block, fused with its gate and residual scale:
//   z  = y / sqrt(mean y^2 + eps) * w_post      (or z = y)
//   x' = x + scale * gate * z
//   h  = x' / sqrt(mean x'^2 + eps) * w_pre
// y and x are read once, x' and h written once.  h is made from x' before x' is rounded, so a 16-bit residual stream
// rounds once, on its way out.  HBM bounds it.  Two kernels: for few rows (a decode step) a block per row with everything
// in registers, one load deep; for many rows persistent warps that copy whole rows ahead into shared memory (bulk copies,
// several rows in flight at all times) and make x' twice from there rather than hold it.
#include "adsa_async.cuh"
#include "adsa_half.cuh"

namespace adsa {

constexpr int kResMaxThreads = 1024;
constexpr int kRingThreads = 256, kRingSmem = 200 * 1024, kRingMaxStages = 4;
constexpr int kRingRows = 148 * 16;            // rows from which the ring kernel is used

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

// eight elements of a 16-bit row or of a residual row, as four pairs of floats
template <typename T>
__device__ __forceinline__ void eight(const T *p, float2 (&f)[4])
{
    const uint4 w = *reinterpret_cast<const uint4 *>(p);
    f[0] = unpack2<T>(w.x); f[1] = unpack2<T>(w.y); f[2] = unpack2<T>(w.z); f[3] = unpack2<T>(w.w);
}
template <>
__device__ __forceinline__ void eight<float>(const float *p, float2 (&f)[4])
{
    const float4 a = reinterpret_cast<const float4 *>(p)[0], b = reinterpret_cast<const float4 *>(p)[1];
    f[0] = make_float2(a.x, a.y); f[1] = make_float2(a.z, a.w); f[2] = make_float2(b.x, b.y); f[3] = make_float2(b.z, b.w);
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

// A group of `warps` warps (1, 2, 4 or 8) owns a row at a time; its ring holds `stages` rows of y and x.
template <typename T, typename X>
__global__ void __launch_bounds__(kRingThreads, 1)
norm_residual_ring_kernel(const T *y, const X *x, const T *w_post, const T *gate, const T *w_pre, X *x_out, T *h, long long rows, int dim,
                          long long rows_per_gate, int warps, int stages, float scale, float eps)
{
    extern __shared__ __align__(128) unsigned char ring_smem[];
    __shared__ uint64_t bars[8 * kRingMaxStages];
    __shared__ float slots[2][8];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, group = warp / warps, groups = 8 / warps;
    const int in = threadIdx.x - group * warps * 32, threads = warps * 32, pieces = dim / 8;
    const uint32_t y_bytes = (uint32_t)dim * sizeof(T), x_bytes = (uint32_t)dim * sizeof(X), row_bytes = y_bytes + x_bytes;
    unsigned char *ring = ring_smem + (size_t)group * stages * row_bytes;
    const uint32_t full = smem_u32(bars + group * kRingMaxStages);
    if (threadIdx.x == 0) {
        for (int i = 0; i < 8 * kRingMaxStages; ++i) mbar_init(smem_u32(bars + i), 1);
        mbar_init_fence();
    }
    __syncthreads();
    pdl_wait();
    pdl_launch();
    const long long stride = (long long)gridDim.x * groups, first = (long long)blockIdx.x * groups + group;
    // one thread of the group copies; a stage is free once the whole group has read it
    const auto copy = [&](long long row, int stage) {
        if (row >= rows) return;
        const uint32_t dst = smem_u32(ring + (size_t)stage * row_bytes);
        mbar_expect_tx(full + 8 * stage, row_bytes);
        bulk_g2s(dst, y + row * dim, y_bytes, full + 8 * stage);
        bulk_g2s(dst + y_bytes, x + row * dim, x_bytes, full + 8 * stage);
    };
    if (in == 0)
        for (int i = 0; i < stages; ++i) copy(first + i * stride, i);
    const auto meet = [&]() {
        if (warps == 1) __syncwarp();
        else asm volatile("bar.sync %0, %1;" ::"r"(1 + group), "r"(threads) : "memory");
    };
    const auto sum = [&](float v, int which) {                     // over the group's threads; all add in the same order
#pragma unroll
        for (int o = 16; o > 0; o >>= 1) v += __shfl_xor_sync(0xffffffffu, v, o);
        if (warps == 1) return v;
        if (lane == 0) slots[which][warp] = v;
        meet();
        v = 0.f;
        for (int w = 0; w < warps; ++w) v += slots[which][group * warps + w];
        return v;
    };
    const float inv_dim = 1.f / (float)dim;
    int stage = 0, limit = kCopySpinLimit;
    uint32_t phase = 0;
    for (long long row = first; row < rows; row += stride) {
        if (!mbar_wait_bounded(full + 8 * stage, phase, limit)) limit = kCopySpinAfterTimeout;
        const T *ys = reinterpret_cast<const T *>(ring + (size_t)stage * row_bytes);
        const X *xs = reinterpret_cast<const X *>(ring + (size_t)stage * row_bytes + y_bytes);
        const T *gr = gate ? gate + row / rows_per_gate * dim : nullptr;
        float inv = 1.f;
        if (w_post) {
            float2 s2 = make_float2(0.f, 0.f);
            for (int p = in; p < pieces; p += threads) {
                float2 f[4];
                eight<T>(ys + p * 8, f);
#pragma unroll
                for (int e = 0; e < 4; ++e) s2 = fma2(f[e], f[e], s2);
            }
            inv = rsqrtf(sum(s2.x + s2.y, 0) * inv_dim + eps);
        }
        const float2 k2 = make_float2(scale, scale), inv2 = make_float2(inv, inv);
        const auto made = [&](int p, float2 (&v)[4]) {             // x' of eight elements
            float2 z[4], w[4];
            eight<T>(ys + p * 8, z);
            eight<X>(xs + p * 8, v);
            if (w_post) {
                eight<T>(w_post + p * 8, w);
#pragma unroll
                for (int e = 0; e < 4; ++e) z[e] = mul2(mul2(z[e], inv2), w[e]);
            }
            if (gr) {
                eight<T>(gr + p * 8, w);
#pragma unroll
                for (int e = 0; e < 4; ++e) z[e] = mul2(z[e], w[e]);
            }
#pragma unroll
            for (int e = 0; e < 4; ++e) v[e] = fma2(z[e], k2, v[e]);
        };
        float2 s2 = make_float2(0.f, 0.f);
#pragma unroll 2
        for (int p = in; p < pieces; p += threads) {
            float2 v[4];
            made(p, v);
            put_eight<X>(x_out + row * dim + p * 8, v);
#pragma unroll
            for (int e = 0; e < 4; ++e) s2 = fma2(v[e], v[e], s2);
        }
        if (h) {
            inv = rsqrtf(sum(s2.x + s2.y, 1) * inv_dim + eps);
            const float2 out2 = make_float2(inv, inv);
#pragma unroll 2
            for (int p = in; p < pieces; p += threads) {
                float2 v[4], w[4];
                made(p, v);
                eight<T>(w_pre + p * 8, w);
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = mul2(mul2(v[e], out2), w[e]);
                put_eight<T>(h + row * dim + p * 8, v);
            }
        }
        meet();
        if (in == 0) copy(row + stages * stride, stage);
        if (++stage == stages) { stage = 0; phase ^= 1u; }
    }
}

namespace {

template <typename T, typename X>
cudaError_t launch_norm_residual(const void *y, const void *x, const void *w_post, const void *gate, const void *w_pre, void *x_out,
                                 void *h, long long rows, int dim, long long rows_per_gate, float scale, float eps, cudaStream_t st)
{
    const int pieces = dim / 8;
    const size_t row_bytes = (size_t)dim * (sizeof(T) + sizeof(X));
    if (rows >= kRingRows && 2 * row_bytes <= kRingSmem) {
        int warps = 1;                       // of a row: as few as leave eight pieces a lane and two rows in flight
        while (warps < 8 && (pieces > 256 * warps || 2 * row_bytes * (8 / warps) > kRingSmem)) warps *= 2;
        int stages = (int)(kRingSmem / (row_bytes * (8 / warps)));
        stages = stages > kRingMaxStages ? kRingMaxStages : stages;
        const size_t smem = row_bytes * (8 / warps) * stages;
        const auto kern = norm_residual_ring_kernel<T, X>;
        const cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingSmem);
        if (e != cudaSuccess) return e;
        const int per_sm = smem * 2 <= kRingSmem ? 2 : 1;
        return launch_pdl(kern, dim3(148u * per_sm), kRingThreads, smem, st, (const T *)y, (const X *)x, (const T *)w_post, (const T *)gate,
                          (const T *)w_pre, (X *)x_out, (T *)h, rows, dim, rows_per_gate, warps, stages, scale, eps);
    }
    const int np = pieces > kResMaxThreads ? 2 : 1;
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
