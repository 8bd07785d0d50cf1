// Decode attention for a batch whose groups share a long prefix (adsa_shared_prefix_attn).
//
// For query head j of batch row b:  o = sum_i softmax_i(scale q.k_i) v_i over the rows of the prefix of b's group and b's
// own rows.  A softmax over a union of sets is the merge of the sets' own states (maximum m, sum l, weighted rows o):
//   m = max m_s,  l = sum l_s 2^(m_s - m),  o = sum o_s 2^(m_s - m) / l
// so the prefix is swept ONCE per group and key head, by all of the group's queries together (a real matrix product:
// members x query heads per key head rows against the prefix), and each batch row's own rows by its queries alone.
//
// Work split.  The unit is a tile of 64 cached rows of one key head.  All units of a call (of every prefix, 64 query
// rows at a time, then of every batch row) form one list; block c of C takes units c U / C .. (c + 1) U / C, whatever
// they belong to, so long and short rows, prefixes and single rows balance without the host knowing a length.  Where a block's
// range changes from one item to the next it leaves the item's partial state in the workspace; a second small kernel
// merges the states of each output row.  Lengths, tables and group boundaries are read on the device: a captured graph follows them.
//
// What a warp does per 16 cached rows: S = Q K^T and O += P V on mma.sync tiles of 16 query rows.  Where 16 query rows
// or fewer share a key head the four warps of a block split the cached rows of a tile, with up to 64 they split the query rows.
// One query row per cached row is 1 flop per byte: HBM bounds it, and the products run on the tensor cores only
// because that takes the fewest instructions per byte.
#include <cuda.h>
#include <float.h>
#include <math.h>
#include <type_traits>

#include "adsa_async.cuh"
#include "adsa_half.cuh"

namespace adsa {

constexpr int kPaTile = 64;                 // cached rows of a unit
constexpr int kPaWarps = 4;                 // warps that compute; one more warp copies
constexpr int kPaThreads = (kPaWarps + 1) * 32;
constexpr int kPaMaxEntries = 8192;         // groups + batch rows of a call
constexpr int kPaMergeThreads = 128;

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
    int blocks;                             // of the sweep kernel
};

// how many warps share the query rows of an item with m of them (the rest share its cached rows)
__host__ __device__ __forceinline__ int query_warps(int m) { return m <= 16 ? 1 : m <= 32 ? 2 : 4; }

__device__ __forceinline__ int clamp_rows(int n, int max_pages, int page_rows)
{
    const long long most = (long long)max_pages * page_rows;
    return n < 0 ? 0 : n > most ? (int)most : n;
}
__device__ __forceinline__ int group_begin(const PrefixArgs &a, int g) { return min(max(a.start[g], 0), a.batch); }
__device__ __forceinline__ int group_members(const PrefixArgs &a, int g) { return max(group_begin(a, g + 1) - group_begin(a, g), 0); }

// units of an entry: groups first, then batch rows
__device__ __forceinline__ uint32_t entry_units(const PrefixArgs &a, int e)
{
    if (e < a.groups) {
        const int m = group_members(a, e) * a.per_kv;
        const int n = clamp_rows(a.p_rows[e], a.max_p_pages, a.page_rows);
        return (uint32_t)((m + 63) / 64) * (uint32_t)a.kv_heads * (uint32_t)((n + kPaTile - 1) / kPaTile);
    }
    const int n = clamp_rows(a.n_rows[e - a.groups], a.max_pages, a.page_rows);
    return (uint32_t)a.kv_heads * (uint32_t)((n + kPaTile - 1) / kPaTile);
}

// Every one of these blocks has a unit, so every state between an item's first and last block exists.
__device__ __forceinline__ uint32_t working_blocks(const PrefixArgs &a, uint32_t total) { return min((uint32_t)a.blocks, total); }

// A run of units of one item inside a block's range.
struct Segment {
    const int32_t *pages;                   // page table of the cached rows
    int n;                                  // cached rows of the item
    int head;                               // key head
    int tile0, tiles;                       // the run
    int row0, rows;                         // packed query rows (batch row * per_kv + head in the key head): first, count
    int slot;                               // of the partial state
    bool prefix;
};

struct Walk {
    const uint32_t *plan;                   // shared copy
    uint32_t u, end;
    int e, entries, block;
    __device__ void begin(const PrefixArgs &a, const uint32_t *plan_, int block_)
    {
        plan = plan_;
        entries = a.groups + a.batch;
        block = block_;
        const uint32_t total = plan[entries], blocks = working_blocks(a, total);
        u = end = 0;
        if ((uint32_t)block < blocks) {
            u = (uint32_t)((unsigned long long)block * total / blocks);
            end = (uint32_t)((unsigned long long)(block + 1) * total / blocks);
        }
        int lo = 0, hi = entries;           // the last entry whose first unit is <= u
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (plan[mid] <= u) lo = mid;
            else hi = mid - 1;
        }
        e = lo;
    }
    __device__ bool next(const PrefixArgs &a, Segment &s)
    {
        if (u >= end) return false;
        while (u >= plan[e + 1]) ++e;
        const uint32_t at = u - plan[e];
        uint32_t tiles;
        if (e < a.groups) {
            const int members = group_members(a, e), m = members * a.per_kv, mt = (m + 63) / 64;
            s.n = clamp_rows(a.p_rows[e], a.max_p_pages, a.page_rows);
            tiles = (uint32_t)((s.n + kPaTile - 1) / kPaTile);
            const int item = (int)(at / tiles), b0 = group_begin(a, e);
            s.head = item / mt;
            const int q = item - s.head * mt;
            s.row0 = b0 * a.per_kv + q * 64;
            s.rows = min(m - q * 64, 64);
            s.pages = a.p_table + (size_t)e * a.max_p_pages;
            s.slot = (int)(((long long)b0 * a.per_kv / 64 + e) * a.kv_heads) + item + block;
            s.prefix = true;
            s.tile0 = (int)(at - (uint32_t)item * tiles);
        } else {
            const int b = e - a.groups;
            s.n = clamp_rows(a.n_rows[b], a.max_pages, a.page_rows);
            tiles = (uint32_t)((s.n + kPaTile - 1) / kPaTile);
            s.head = (int)(at / tiles);
            s.row0 = b * a.per_kv;
            s.rows = a.per_kv;
            s.pages = a.table + (size_t)b * a.max_pages;
            s.slot = b * a.kv_heads + s.head + block;
            s.prefix = false;
            s.tile0 = (int)(at - (uint32_t)s.head * tiles);
        }
        s.tiles = (int)min(tiles - (uint32_t)s.tile0, end - u);
        u += (uint32_t)s.tiles;
        return true;
    }
};

__device__ __forceinline__ void pa_ldsm(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void pa_ldsm_t(uint32_t addr, uint32_t (&r)[4])
{
    asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <typename T>
__device__ __forceinline__ void pa_mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if constexpr (std::is_same<T, __nv_bfloat16>::value)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
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

// NSUB: 64-element sub-tiles of a row (head elements / 64, rounded up).  STAGES: tiles in flight per block.
template <typename T, int NSUB, int STAGES>
__global__ void __launch_bounds__(kPaThreads, NSUB <= 2 ? 2 : 1)
prefix_sweep_kernel(const __grid_constant__ PrefixArgs a, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map)
{
    constexpr int KS = 4 * NSUB;                                   // 16-element steps over a row
    constexpr uint32_t kSub = kPaTile * 128, kHalf = NSUB * kSub;  // bytes: a sub-tile; K (or V) of a tile
    constexpr int DP = 64 * NSUB;                                  // floats of a state row
    constexpr float kBias = WeightBias<T>::value;
    extern __shared__ unsigned char pa_smem[];
    __shared__ uint64_t bars[2 * STAGES];
    __shared__ uint32_t warp_sums[kPaThreads / 32];
    const uint32_t ring = (smem_u32(pa_smem) + 1023u) & ~1023u;
    uint32_t *plan = reinterpret_cast<uint32_t *>(pa_smem + (ring - smem_u32(pa_smem)) + (size_t)STAGES * 2 * kHalf);
    const uint32_t full = smem_u32(bars), empty = full + 8 * STAGES;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int entries = a.groups + a.batch;

    if (tid == 0) {
        for (int i = 0; i < STAGES; ++i) { mbar_init(full + 8 * i, 1); mbar_init(empty + 8 * i, kPaWarps); }
        mbar_init_fence();
        asm volatile("prefetch.tensormap [%0];" ::"l"(&k_map) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&v_map) : "memory");
    }
    pdl_wait();
    pdl_launch();

    // ---- first unit of every entry: each thread sums a run of entries, the runs are scanned over the block ----
    const int run = (entries + kPaThreads - 1) / kPaThreads, e0 = min(tid * run, entries), e1 = min(e0 + run, entries);
    uint32_t mine = 0;
    for (int e = e0; e < e1; ++e) { const uint32_t w = entry_units(a, e); plan[e] = mine; mine += w; }
    uint32_t incl = mine;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) { const uint32_t t = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += t; }
    if (lane == 31) warp_sums[warp] = incl;
    __syncthreads();
    uint32_t before = incl - mine;
    for (int w = 0; w < warp; ++w) before += warp_sums[w];
    for (int e = e0; e < e1; ++e) plan[e] += before;
    if (tid == kPaThreads - 1) plan[entries] = before + mine;
    __syncthreads();
    if (blockIdx.x == 0)
        for (int e = tid; e <= entries; e += kPaThreads) a.plan[e] = plan[e];

    Walk walk;
    walk.begin(a, plan, blockIdx.x);
    Segment s;

    if (warp == kPaWarps) {                                        // ---- the copying warp ----
        int stage = 0, limit = kCopySpinLimit;
        uint32_t phase = 0;
        while (walk.next(a, s)) {
            for (int t = s.tile0; t < s.tile0 + s.tiles; ++t) {
                if (!mbar_wait_bounded(empty + 8 * stage, phase ^ 1u, limit)) {
                    limit = kCopySpinAfterTimeout;
                    if (a.status && lane == 0) atomicOr(a.status, ADSA_DEV_COPY_TIMEOUT);
                }
                const int rows = min(kPaTile, s.n - t * kPaTile), boxes = (rows + a.box_rows - 1) / a.box_rows;
                if (lane == 0) mbar_expect_tx(full + 8 * stage, (uint32_t)(boxes * a.box_rows) * 128u * 2u * NSUB);
                __syncwarp();
                const uint32_t k_dst = ring + stage * 2 * kHalf;
                for (int i = lane; i < boxes; i += 32) {
                    const int row = t * kPaTile + i * a.box_rows, pg = row / a.page_rows;
                    int page = s.pages[pg];
                    if (page < 0 || page >= a.n_pages) {           // (the row's result is then unspecified)
                        page = 0;
                        if (a.status) atomicOr(a.status, ADSA_DEV_BAD_PAGE);
                    }
                    const int y = (page * a.kv_heads + s.head) * a.page_rows + row - pg * a.page_rows;
                    const uint32_t dst = k_dst + (uint32_t)(i * a.box_rows) * 128u;
#pragma unroll
                    for (int c = 0; c < NSUB; ++c) {
                        pa_tma(dst + c * kSub, &k_map, c * 64, y, full + 8 * stage);
                        pa_tma(dst + kHalf + c * kSub, &v_map, c * 64, y, full + 8 * stage);
                    }
                }
                if (++stage == STAGES) { stage = 0; phase ^= 1u; }
            }
        }
        return;
    }

    // ---- the computing warps ----
    const int g = lane >> 2, t4 = lane & 3, mi = lane >> 3, lr = lane & 7;
    int stage = 0, limit = kCopySpinLimit;
    uint32_t phase = 0;
    while (walk.next(a, s)) {
        const int wq = query_warps(s.rows), wk = kPaWarps / wq;     // warps over query rows, warps over cached rows
        const int qb = warp & (wq - 1), kb = warp / wq;
        // Q as the A operand: rows g and g + 8 of this warp's sixteen, elements 16 ks + 2 t4, + 1 and + 8, + 9
        uint32_t qa[KS][4];
        {
            const T *qp[2];
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = qb * 16 + g + 8 * h, packed = s.row0 + r, b = packed / a.per_kv, j = packed - b * a.per_kv;
                qp[h] = r < s.rows ? (const T *)a.q + b * a.q_row + (s.head * a.per_kv + j) * a.q_head : nullptr;
            }
#pragma unroll
            for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const int col = 16 * ks + 2 * t4 + (i >> 1) * 8;
                    qa[ks][i] = qp[i & 1] && col < a.d ? *reinterpret_cast<const uint32_t *>(qp[i & 1] + col) : 0u;
                }
            }
        }
        float o[2 * KS][4], m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f};
#pragma unroll
        for (int nb = 0; nb < 2 * KS; ++nb) { o[nb][0] = o[nb][1] = o[nb][2] = o[nb][3] = 0.f; }

        for (int t = s.tile0; t < s.tile0 + s.tiles; ++t) {
            if (!mbar_wait_bounded(full + 8 * stage, phase, limit)) {
                limit = kCopySpinAfterTimeout;
                if (a.status && lane == 0) atomicOr(a.status, ADSA_DEV_COPY_TIMEOUT);
            }
            const uint32_t ks_u32 = ring + stage * 2 * kHalf, vs_u32 = ks_u32 + kHalf;
            const int valid = min(kPaTile, s.n - t * kPaTile);
            for (int c0 = kb * 16; c0 < valid; c0 += wk * 16) {     // sixteen cached rows
                if (c0 + 16 > valid) {
                    // rows behind the end hold anything; a weight of zero does not silence an infinity or a NaN of V
                    for (int i = lane; i < 16 * 8 * NSUB; i += 32) {
                        const int r = c0 + i / (8 * NSUB), ch = i % (8 * NSUB);
                        if (r >= valid)
                            asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};"
                                         ::"r"(vs_u32 + (ch >> 3) * kSub + r * 128 + (ch & 7) * 16), "r"(0u) : "memory");
                    }
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // before the next copy into these bytes
                    __syncwarp();
                }
                float sc[2][4];
#pragma unroll
                for (int nb = 0; nb < 2; ++nb) sc[nb][0] = sc[nb][1] = sc[nb][2] = sc[nb][3] = 0.f;
#pragma unroll
                for (int ks = 0; ks < KS; ++ks) {
                    uint32_t kf[4];
                    const int row = c0 + (mi >> 1) * 8 + lr, ch = (2 * ks + (mi & 1)) & 7;
                    pa_ldsm(ks_u32 + (ks >> 2) * kSub + row * 128 + ((ch ^ lr) << 4), kf);
                    pa_mma<T>(sc[0], qa[ks], kf[0], kf[1]);
                    pa_mma<T>(sc[1], qa[ks], kf[2], kf[3]);
                }
                float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
                for (int nb = 0; nb < 2; ++nb) {
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int col = c0 + nb * 8 + 2 * t4 + (i & 1);
                        sc[nb][i] = col < valid ? sc[nb][i] * a.scale_log2e : -INFINITY;
                        mx[i >> 1] = fmaxf(mx[i >> 1], sc[nb][i]);
                    }
                }
                // a new maximum anywhere in the warp: find it over the four lanes of a row, rescale what was summed
                if (__any_sync(0xffffffffu, mx[0] > m_run[0] || mx[1] > m_run[1])) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 1));
                        mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], 2));
                        const float m_new = fmaxf(m_run[h], mx[h]);
                        const float corr = m_new == -INFINITY ? 1.f : pa_exp2(m_run[h] - m_new);
                        m_run[h] = m_new;
                        l_run[h] *= corr;
#pragma unroll
                        for (int nb = 0; nb < 2 * KS; ++nb) { o[nb][2 * h] *= corr; o[nb][2 * h + 1] *= corr; }
                    }
                }
                uint32_t pa[4];
                {
                    float p[2][4];
#pragma unroll
                    for (int nb = 0; nb < 2; ++nb) {
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const float m = m_run[i >> 1];
                            p[nb][i] = pa_exp2(sc[nb][i] - (m == -INFINITY ? 0.f : m) + kBias);
                            l_run[i >> 1] += p[nb][i];              // the sum takes the weights before they are rounded
                        }
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) pa[i] = pack2<T>(p[i >> 1][(i & 1) * 2], p[i >> 1][(i & 1) * 2 + 1]);
                }
#pragma unroll
                for (int dp = 0; dp < KS; ++dp) {
                    uint32_t vf[4];
                    const int row = c0 + (mi & 1) * 8 + lr, ch = (2 * dp + (mi >> 1)) & 7;
                    pa_ldsm_t(vs_u32 + (dp >> 2) * kSub + row * 128 + ((ch ^ lr) << 4), vf);
                    pa_mma<T>(o[2 * dp], pa, vf[0], vf[1]);
                    pa_mma<T>(o[2 * dp + 1], pa, vf[2], vf[3]);
                }
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(empty + 8 * stage);
            if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        }
        // ---- the partial state ----
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            l_run[h] += __shfl_xor_sync(0xffffffffu, l_run[h], 1);
            l_run[h] += __shfl_xor_sync(0xffffffffu, l_run[h], 2);
        }
        // a slot holds wk states of s.rows rows
        const bool fits = s.slot < (s.prefix ? a.n_p_slots : a.n_o_slots);
        if (!fits && a.status && lane == 0) atomicOr(a.status, ADSA_DEV_BAD_GROUPS);
        if (fits) {
            const size_t slot_rows = s.prefix ? 64 : (size_t)(kPaWarps / query_warps(a.per_kv)) * a.per_kv;
            const size_t first = (size_t)s.slot * slot_rows + (size_t)kb * s.rows;
            float *st = s.prefix ? a.p_state : a.o_state, *ml = s.prefix ? a.p_ml : a.o_ml;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = qb * 16 + g + 8 * h;
                if (r < s.rows) {
                    if (t4 == 0) *reinterpret_cast<float2 *>(ml + 2 * (first + r)) = make_float2(m_run[h] - kBias, l_run[h]);
#pragma unroll
                    for (int nb = 0; nb < 2 * KS; ++nb) {
                        const int col = nb * 8 + 2 * t4;
                        if (col < a.d) *reinterpret_cast<float2 *>(st + (first + r) * DP + col) = make_float2(o[nb][2 * h], o[nb][2 * h + 1]);
                    }
                }
            }
        }
    }
}

// One block per output row (batch row, query head): the states of the prefix units and of the row's own units.
template <typename T, int NSUB>
__global__ void __launch_bounds__(kPaMergeThreads)
prefix_merge_kernel(const __grid_constant__ PrefixArgs a, T *out, float *out_f32, float *lse)
{
    constexpr int DP = 64 * NSUB, WARPS = kPaMergeThreads / 32, PER = 2 * NSUB;   // PER floats per lane
    __shared__ float s_m[WARPS], s_l[WARPS], s_o[WARPS][DP];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int heads = a.kv_heads * a.per_kv;
    const int b = blockIdx.x / heads, qh = blockIdx.x - b * heads, head = qh / a.per_kv, j = qh - head * a.per_kv;
    pdl_wait();
    pdl_launch();
    const uint32_t total = a.plan[a.groups + a.batch], blocks = working_blocks(a, total);
    // the block that holds unit u: the last c with floor(c total / blocks) <= u
    const auto block_of = [&](uint32_t u) { return (int)((((unsigned long long)u + 1) * blocks - 1) / total); };

    // the group of the batch row: the last one that begins at or before it
    int grp = -1;
    {
        int lo = -1, hi = a.groups - 1;
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (group_begin(a, mid) <= b) lo = mid;
            else hi = mid - 1;
        }
        if (lo >= 0 && b < group_begin(a, lo + 1)) grp = lo;
    }
    // runs of states: prefix, then own rows
    size_t p_first = 0, o_first;
    int p_segs = 0, p_step = 0, p_subs = 0, o_segs = 0;
    const int o_subs = kPaWarps / query_warps(a.per_kv), o_step = o_subs * a.per_kv;
    if (grp >= 0) {
        const int b0 = group_begin(a, grp), m = group_members(a, grp) * a.per_kv, mt = (m + 63) / 64;
        const int packed = (b - b0) * a.per_kv + j, q = packed / 64, rows = min(m - q * 64, 64);
        const int n = clamp_rows(a.p_rows[grp], a.max_p_pages, a.page_rows), tiles = (n + kPaTile - 1) / kPaTile;
        if (tiles > 0) {
            const int item = head * mt + q;
            const uint32_t u = a.plan[grp] + (uint32_t)item * (uint32_t)tiles;
            const int c0 = block_of(u), c1 = block_of(u + tiles - 1);
            const long long slot = ((long long)b0 * a.per_kv / 64 + grp) * a.kv_heads + item + c0;
            p_segs = (int)min((long long)(c1 - c0 + 1), max(0LL, a.n_p_slots - slot));
            p_subs = kPaWarps / query_warps(rows);
            p_step = rows;
            p_first = (size_t)slot * 64 + (packed - q * 64);
        }
    }
    {
        const int n = clamp_rows(a.n_rows[b], a.max_pages, a.page_rows), tiles = (n + kPaTile - 1) / kPaTile;
        o_first = 0;
        if (tiles > 0) {
            const uint32_t u = a.plan[a.groups + b] + (uint32_t)head * (uint32_t)tiles;
            const int c0 = block_of(u), c1 = block_of(u + tiles - 1);
            o_segs = c1 - c0 + 1;
            o_first = (size_t)(b * a.kv_heads + head + c0) * o_step + j;
        }
    }
    const int n_p = p_segs * p_subs, n_states = n_p + o_segs * o_subs;
    float m = -INFINITY, l = 0.f, o[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) o[e] = 0.f;
    for (int i = warp; i < n_states; i += WARPS) {
        const float *st, *ml;
        if (i < n_p) {
            const int seg = i / p_subs, sub = i - seg * p_subs;
            const size_t row = p_first + (size_t)seg * 64 + (size_t)sub * p_step;
            st = a.p_state + row * DP; ml = a.p_ml + 2 * row;
        } else {
            const int k = i - n_p, seg = k / o_subs, sub = k - seg * o_subs;
            const size_t row = o_first + (size_t)seg * o_step + (size_t)sub * a.per_kv;
            st = a.o_state + row * DP; ml = a.o_ml + 2 * row;
        }
        const float2 s = *reinterpret_cast<const float2 *>(ml);
        float x[PER];
#pragma unroll
        for (int e = 0; e < PER; e += 2) *reinterpret_cast<float2 *>(x + e) = *reinterpret_cast<const float2 *>(st + e * 32 + 2 * lane);
        if (s.y == 0.f && s.x == -INFINITY) continue;               // an empty state
        const float M = fmaxf(m, s.x), w1 = m == -INFINITY ? 0.f : pa_exp2(m - M), w2 = s.x == -INFINITY ? 0.f : pa_exp2(s.x - M);
        l = l * w1 + s.y * w2;
#pragma unroll
        for (int e = 0; e < PER; ++e) o[e] = o[e] * w1 + x[e] * w2;
        m = M;
    }
    if (lane == 0) { s_m[warp] = m; s_l[warp] = l; }
#pragma unroll
    for (int e = 0; e < PER; e += 2) *reinterpret_cast<float2 *>(&s_o[warp][e * 32 + 2 * lane]) = make_float2(o[e], o[e + 1]);
    __syncthreads();
    float M = -INFINITY;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) M = fmaxf(M, s_m[w]);
    float wgt[WARPS], L = 0.f;
#pragma unroll
    for (int w = 0; w < WARPS; ++w) {
        wgt[w] = s_m[w] == -INFINITY ? 0.f : pa_exp2(s_m[w] - M);
        L += s_l[w] * wgt[w];
    }
    const bool empty = n_states == 0;
    const float inv = empty ? 0.f : 1.f / L;
    const size_t row = (size_t)b * heads + qh;
    for (int e = threadIdx.x; e < a.d; e += kPaMergeThreads) {
        float x = 0.f;
#pragma unroll
        for (int w = 0; w < WARPS; ++w) x += s_o[w][e] * wgt[w];
        x = empty ? 0.f : x * inv;
        if (out) out[row * a.d + e] = from_f32<T>(x);
        if (out_f32) out_f32[row * a.d + e] = x;
    }
    if (lse && threadIdx.x == 0) lse[row] = empty ? -INFINITY : (M + log2f(L)) * 0.693147180559945309f;
}

namespace {

struct PrefixLayout {
    size_t plan, p_state, p_ml, o_state, o_ml, bytes;
    long long p_slots, o_slots;
    int nsub, blocks;
};

int sm_count()
{
    int dev = 0, n = 0;
    if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&n, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess) {
        cudaGetLastError();
        return 148;
    }
    return n;
}

bool layout_of(int batch, int groups, int n_heads, int kv_heads, int head_dim, PrefixLayout *o)
{
    if (batch < 1 || groups < 0 || batch + (long long)groups > kPaMaxEntries || kv_heads < 1 || n_heads < kv_heads || n_heads % kv_heads ||
        n_heads / kv_heads > 64 || head_dim < 2 || head_dim % 2 || head_dim > ADSA_MAX_HEAD_DIM)
        return false;
    const int per_kv = n_heads / kv_heads;
    o->nsub = (head_dim + 63) / 64;
    o->blocks = sm_count() * (o->nsub <= 2 ? 2 : 1);
    const auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
    o->p_slots = groups ? ((long long)batch * per_kv / 64 + groups) * kv_heads + o->blocks : 0;
    o->o_slots = (long long)batch * kv_heads + o->blocks;
    const size_t dp = 64 * o->nsub, p_rows = (size_t)o->p_slots * 64, o_rows = (size_t)o->o_slots * (kPaWarps / query_warps(per_kv)) * per_kv;
    if (o->p_slots > 0x7fffffffLL || o->o_slots > 0x7fffffffLL || (long long)batch * n_heads > 0x7fffffffLL) return false;
    o->plan = 0;
    o->p_state = up((size_t)(batch + groups + 1) * 4);
    o->p_ml = o->p_state + up(p_rows * dp * 4);
    o->o_state = o->p_ml + up(p_rows * 8);
    o->o_ml = o->o_state + up(o_rows * dp * 4);
    o->bytes = o->o_ml + up(o_rows * 8);
    return true;
}

typedef CUresult (*encode_t)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                             const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                             CUtensorMapFloatOOBfill);
encode_t encoder()
{
    static encode_t fn = [] {
        void *f = nullptr;
        cudaDriverEntryPointQueryResult r;
        if (cudaGetDriverEntryPoint("cuTensorMapEncodeTiled", &f, cudaEnableDefault, &r) != cudaSuccess || r != cudaDriverEntryPointSuccess) {
            cudaGetLastError();
            f = nullptr;
        }
        return (encode_t)f;
    }();
    return fn;
}

// A pool as a table of rows of head_dim elements: boxes of box_rows rows x 64 elements in the 128-byte swizzle; what lies
// beyond head_dim arrives as zero, whatever the padding holds.
bool pool_map(CUtensorMap *m, const adsa_paged_kv &kv, void *pool, int box_rows)
{
    const encode_t encode = encoder();
    if (!encode) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)kv.head_dim, (cuuint64_t)kv.n_pages * kv.n_kv_heads * kv.page_rows};
    const cuuint64_t strides[1] = {(cuuint64_t)kv.row_stride * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)box_rows}, estr[2] = {1, 1};
    return encode(m, kv.dtype == ADSA_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, 2, pool, dims, strides, box, estr,
                  CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                  CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

template <typename T, int NSUB, int STAGES>
cudaError_t launch_prefix(const PrefixArgs &a, const CUtensorMap &km, const CUtensorMap &vm, void *out, float *out_f32, float *lse, cudaStream_t st)
{
    const size_t smem = 1024 + (size_t)STAGES * 2 * NSUB * kPaTile * 128 + (size_t)(a.batch + a.groups + 1) * 4;
    const auto kern = prefix_sweep_kernel<T, NSUB, STAGES>;
    cudaError_t e = cudaFuncSetAttribute(kern, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem);
    if (e != cudaSuccess) return e;
    e = launch_pdl(kern, dim3((unsigned)a.blocks), kPaThreads, smem, st, a, km, vm);
    if (e != cudaSuccess) return e;
    return launch_pdl(prefix_merge_kernel<T, NSUB>, dim3((unsigned)(a.batch * a.kv_heads * a.per_kv)), kPaMergeThreads, 0, st, a, (T *)out, out_f32, lse);
}

template <typename T>
cudaError_t launch_prefix_type(int nsub, const PrefixArgs &a, const CUtensorMap &km, const CUtensorMap &vm, void *out, float *out_f32,
                               float *lse, cudaStream_t st)
{
    switch (nsub) {                          // 96 KB of tiles in flight per block, two blocks per SM; wide rows: one block
    case 1: return launch_prefix<T, 1, 6>(a, km, vm, out, out_f32, lse, st);
    case 2: return launch_prefix<T, 2, 3>(a, km, vm, out, out_f32, lse, st);
    case 3: return launch_prefix<T, 3, 4>(a, km, vm, out, out_f32, lse, st);
    default: return launch_prefix<T, 4, 3>(a, km, vm, out, out_f32, lse, st);
    }
}

}  // namespace
}  // namespace adsa

using namespace adsa;

extern "C" {

int adsa_shared_prefix_workspace_bytes(int batch, int n_groups, int n_heads, int n_kv_heads, int head_dim, size_t *out_bytes)
{
    PrefixLayout l;
    if (!out_bytes || !layout_of(batch, n_groups, n_heads, n_kv_heads, head_dim, &l)) return ADSA_EINVAL;
    *out_bytes = l.bytes;
    return ADSA_OK;
}

int adsa_shared_prefix_attn(const adsa_paged_kv *kv, const void *q, long long q_row, long long q_head, int batch, int n_heads,
                            const int32_t *page_table, int max_pages, const int32_t *n_rows, const int32_t *prefix_table, int max_prefix_pages,
                            const int32_t *prefix_rows, const int32_t *group_start, int n_groups, float softmax_scale, void *out,
                            float *out_f32, float *lse, void *workspace, size_t workspace_bytes, uint32_t *status, adsa_stream_t stream)
{
    PrefixLayout l;
    if (!paged_kv_ok(kv) || batch < 0 || max_pages < 1 || n_groups < 0) return ADSA_EINVAL;
    if (batch == 0) return ADSA_OK;
    if (!layout_of(batch, n_groups, n_heads, kv->n_kv_heads, kv->head_dim, &l)) return ADSA_EINVAL;
    if (!q || !page_table || !n_rows || (!out && !out_f32) || !workspace || !(softmax_scale >= 0.f)) return ADSA_EINVAL;
    if (n_groups && (!prefix_table || !prefix_rows || !group_start || max_prefix_pages < 1)) return ADSA_EINVAL;
    if (((uintptr_t)q & 3) || q_row % 2 || q_head % 2 || ((uintptr_t)workspace & 255) || ((uintptr_t)out & 1)) return ADSA_EINVAL;
    if (((uintptr_t)page_table | (uintptr_t)n_rows | (uintptr_t)prefix_table | (uintptr_t)prefix_rows | (uintptr_t)group_start |
         (uintptr_t)out_f32 | (uintptr_t)lse | (uintptr_t)status) & 3)
        return ADSA_EINVAL;
    if ((long long)max_pages * kv->page_rows > 0x7fffffc0LL || (long long)max_prefix_pages * kv->page_rows > 0x7fffffc0LL) return ADSA_EINVAL;
    // the units of a call are counted in 32 bits
    const double own_units = (double)batch * kv->n_kv_heads * ((double)max_pages * kv->page_rows / kPaTile + 1);
    const double p_units = ((double)batch * (n_heads / kv->n_kv_heads) / 64 + n_groups) * kv->n_kv_heads *
                           ((double)max_prefix_pages * kv->page_rows / kPaTile + 1);
    if (own_units + (n_groups ? p_units : 0) > 4e9) return ADSA_EINVAL;
    if (workspace_bytes < l.bytes) return ADSA_ENOMEM;
    int box = 64;
    while (kv->page_rows % box) box /= 2;    // boxes of the largest power of two that divides a page never straddle two pages
    CUtensorMap km, vm;
    if (!pool_map(&km, *kv, kv->k_pool, box) || !pool_map(&vm, *kv, kv->v_pool, box)) return ADSA_ECUDA;
    unsigned char *ws = (unsigned char *)workspace;
    PrefixArgs a = {};
    a.q = q; a.q_row = q_row; a.q_head = q_head;
    a.table = page_table; a.n_rows = n_rows; a.p_table = prefix_table; a.p_rows = prefix_rows; a.start = group_start;
    a.status = status;
    a.batch = batch; a.groups = n_groups; a.kv_heads = kv->n_kv_heads; a.per_kv = n_heads / kv->n_kv_heads;
    a.max_pages = max_pages; a.max_p_pages = max_prefix_pages; a.page_rows = kv->page_rows; a.n_pages = kv->n_pages; a.box_rows = box;
    a.d = kv->head_dim;
    const float scale = softmax_scale == 0.f ? 1.0f / sqrtf((float)kv->head_dim) : softmax_scale;
    a.scale_log2e = scale * 1.44269504088896341f;
    a.plan = (uint32_t *)(ws + l.plan);
    a.p_state = (float *)(ws + l.p_state); a.p_ml = (float *)(ws + l.p_ml);
    a.o_state = (float *)(ws + l.o_state); a.o_ml = (float *)(ws + l.o_ml);
    a.n_p_slots = (int)l.p_slots; a.n_o_slots = (int)l.o_slots; a.blocks = l.blocks;
    cudaStream_t st = (cudaStream_t)stream;
    const cudaError_t e = kv->dtype == ADSA_BF16 ? launch_prefix_type<__nv_bfloat16>(l.nsub, a, km, vm, out, out_f32, lse, st)
                                                  : launch_prefix_type<__half>(l.nsub, a, km, vm, out, out_f32, lse, st);
    return e == cudaSuccess ? ADSA_OK : ADSA_ECUDA;
}

}  // extern "C"
