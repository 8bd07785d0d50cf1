// What the kernels of adsa_shared_prefix_attn share: their arguments, lengths and groups as the device finds them, copies.
#pragma once

#include <cuda.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "adsa_async.cuh"
#include "adsa_half.cuh"

namespace adsa {

constexpr int kWideQueries = 128;           // query rows of an item of the wide kernel
constexpr int kWideTile = 128;              // cached rows of a unit of the wide kernel

struct PrefixArgs {
    const void *q;
    long long q_row, q_head;                // element strides of q
    const int32_t *table, *n_rows;          // [batch][max_pages], [batch]
    const int32_t *p_table, *p_rows, *start;   // [groups][max_p_pages], [groups], [groups + 1]
    uint32_t *status;
    int batch, groups, kv_heads, per_kv;    // per_kv: query heads of a key head
    int max_pages, max_p_pages, page_rows, n_pages, box_rows;
    int d;
    float scale_log2e;
    // workspace
    uint32_t *plan;                         // [entries + 1] first unit of every entry (groups, then batch rows)
    float *p_state, *p_ml, *o_state, *o_ml; // prefix slots, own-row slots: rows of d_pad floats, (m, l) pairs
    int n_p_slots, n_o_slots;
    // groups with more query rows per key head than this go to the wide kernel, with a plan and slots of its own
    int wide_above;
    uint32_t *w_plan;                       // [groups + 1]
    float *w_state, *w_ml;                  // slots of kWideQueries rows
    int n_w_slots, w_runs;
    int runs;                               // blocks of the sweep kernel's grid
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

// P is rounded to 16 bits for the second product.  It lies in 0 .. 1 relative to the running maximum; 16-bit floats of
// the half type lose precision below 2^-14, so there P is scaled by 2^8 (it cancels in o / l; the states carry it in m).
template <typename T> struct WeightBias { static constexpr float value = 0.f; };
template <> struct WeightBias<__half> { static constexpr float value = 8.f; };

cudaError_t launch_prefix_wide(int dtype, int nsub, const PrefixArgs &a, const CUtensorMap &km, const CUtensorMap &vm, cudaStream_t st);

}  // namespace adsa
