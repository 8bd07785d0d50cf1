// What the stateless decoder operators share: the two 16-bit element types, wide accesses, and the launch that lets a
// kernel's set-up overlap the tail of the kernel ahead of it in the stream.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/adsa.h"

namespace adsa {

template <typename T> __device__ __forceinline__ float to_f32(T x);
template <> __device__ __forceinline__ float to_f32<__nv_bfloat16>(__nv_bfloat16 x) { return __bfloat162float(x); }
template <> __device__ __forceinline__ float to_f32<__half>(__half x) { return __half2float(x); }
template <> __device__ __forceinline__ float to_f32<float>(float x) { return x; }

template <typename T> __device__ __forceinline__ T from_f32(float x);   // round to nearest even
template <> __device__ __forceinline__ __nv_bfloat16 from_f32<__nv_bfloat16>(float x) { return __float2bfloat16_rn(x); }
template <> __device__ __forceinline__ __half from_f32<__half>(float x) { return __float2half_rn(x); }
template <> __device__ __forceinline__ float from_f32<float>(float x) { return x; }

template <typename T> __device__ __forceinline__ uint32_t pack2(float lo, float hi);
template <> __device__ __forceinline__ uint32_t pack2<__nv_bfloat16>(float lo, float hi)
{
    __nv_bfloat162 p = __floats2bfloat162_rn(lo, hi);
    return *reinterpret_cast<uint32_t *>(&p);
}
template <> __device__ __forceinline__ uint32_t pack2<__half>(float lo, float hi)
{
    __half2 p = __floats2half2_rn(lo, hi);
    return *reinterpret_cast<uint32_t *>(&p);
}

// two neighbouring elements as floats
template <typename T> __device__ __forceinline__ float2 unpack2(uint32_t w);
template <> __device__ __forceinline__ float2 unpack2<__nv_bfloat16>(uint32_t w) { return make_float2(__uint_as_float(w << 16), __uint_as_float(w & 0xffff0000u)); }
template <> __device__ __forceinline__ float2 unpack2<__half>(uint32_t w) { return __half22float2(*reinterpret_cast<const __half2 *>(&w)); }

// two 32-bit operations in one instruction
__device__ __forceinline__ float2 fma2(float2 a, float2 b, float2 c)
{
    float2 d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;"
        : "=l"(reinterpret_cast<uint64_t &>(d))
        : "l"(reinterpret_cast<uint64_t &>(a)), "l"(reinterpret_cast<uint64_t &>(b)), "l"(reinterpret_cast<uint64_t &>(c)));
    return d;
}
__device__ __forceinline__ float2 mul2(float2 a, float2 b)
{
    float2 d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<uint64_t &>(d)) : "l"(reinterpret_cast<uint64_t &>(a)), "l"(reinterpret_cast<uint64_t &>(b)));
    return d;
}
__device__ __forceinline__ float2 add2(float2 a, float2 b)
{
    float2 d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(reinterpret_cast<uint64_t &>(d)) : "l"(reinterpret_cast<uint64_t &>(a)), "l"(reinterpret_cast<uint64_t &>(b)));
    return d;
}

// N elements moved by one access (N * sizeof(T) = 2 .. 32 bytes)
template <typename T, int N>
struct alignas(sizeof(T) * N < 16 ? sizeof(T) * N : 16) Pack {
    T e[N];
};

// Kernels launched through here call pdl_wait() before they touch global memory: the kernel ahead has then completed
// and its writes are visible.  pdl_launch() after it lets the next such kernel begin its own set-up.  (One exception: the sweep of a
// shared-prefix call behind that call's wide kernel, which has waited for both, in that order; the sweep waits before it ends.)
__device__ __forceinline__ void pdl_wait() { asm volatile("griddepcontrol.wait;" ::: "memory"); }
__device__ __forceinline__ void pdl_launch() { asm volatile("griddepcontrol.launch_dependents;" ::: "memory"); }

// a pool a call can work on: sizes in range, 16-byte aligned
inline bool paged_kv_ok(const adsa_paged_kv *kv)
{
    if (!kv || !kv->k_pool || !kv->v_pool || (((uintptr_t)kv->k_pool | (uintptr_t)kv->v_pool) & 15)) return false;
    if (kv->dtype != ADSA_BF16 && kv->dtype != ADSA_F16) return false;
    if (kv->head_dim < 2 || kv->head_dim > ADSA_MAX_HEAD_DIM || kv->head_dim % 2) return false;
    if (kv->row_stride < kv->head_dim || kv->row_stride > ADSA_MAX_HEAD_DIM || kv->row_stride % 8) return false;
    if (kv->n_kv_heads < 1 || kv->n_pages < 1 || kv->page_rows < 1 || kv->page_rows > 4096) return false;
    return (long long)kv->n_pages * kv->n_kv_heads <= 0x7fffffffLL / kv->page_rows;   // rows are addressed by 32-bit coordinates
}

// Lets a kernel (with at most 512 bytes of static shared memory) use all of an SM's 227 KB on the current device; asks the
// driver once per device.  told: one word per device, zero at first.
inline cudaError_t allow_smem(const void *kernel, int (&told)[64])
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const bool known = dev >= 0 && dev < 64;
    if (known && __atomic_load_n(&told[dev], __ATOMIC_ACQUIRE)) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, 227 * 1024 - 512);
    if (e == cudaSuccess && known) __atomic_store_n(&told[dev], 1, __ATOMIC_RELEASE);
    return e;
}

// cluster: blocks of a thread block cluster, which divides the grid
template <typename... P, typename... A>
inline cudaError_t launch_pdl_cluster(void (*kernel)(P...), dim3 grid, unsigned cluster, unsigned threads, size_t smem, cudaStream_t st, A... args)
{
    cudaLaunchAttribute attr[2];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    attr[1].id = cudaLaunchAttributeClusterDimension;
    attr[1].val.clusterDim.x = cluster;
    attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3(threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = cluster > 1 ? 2 : 1;
    return cudaLaunchKernelEx(&cfg, kernel, static_cast<P>(args)...);
}
template <typename... P, typename... A>
inline cudaError_t launch_pdl(void (*kernel)(P...), dim3 grid, unsigned threads, size_t smem, cudaStream_t st, A... args)
{
    return launch_pdl_cluster(kernel, grid, 1u, threads, smem, st, args...);
}

}  // namespace adsa
