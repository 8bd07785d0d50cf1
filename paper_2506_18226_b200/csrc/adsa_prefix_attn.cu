// Decode attention for a batch whose groups share a long prefix (adsa_shared_prefix_attn).
//
// For query head j of batch row b:  o = sum_i softmax_i(scale q.k_i) v_i over the rows of the prefix of b's group and b's
// own rows.  A softmax over a union of sets is the merge of the sets' own states (maximum m, sum l, weighted rows o):
//   m = max m_s,  l = sum l_s 2^(m_s - m),  o = sum o_s 2^(m_s - m) / l
// so the prefix is swept ONCE per group and key head, by all of the group's queries together (a real matrix product:
// members x query heads per key head rows against the prefix), and each batch row's own rows by its queries alone.  Long
// prefixes of large groups go to a kernel of their own (adsa_prefix_wide.cu); everything else is swept here.
//
// Work split.  The unit is a tile of 128 (wider rows: 64) cached rows of one key head.  All units of a call (of every
// prefix, 32 query rows at a time, then of every batch row) form one list that is cut into runs, whatever they belong to
// (Cut), so long and short rows, prefixes and single rows mix without the host knowing a length.  Where a run changes from
// one item to the next it leaves the item's partial state in the workspace; a small kernel merges the states of each output
// row.  Lengths, tables and group boundaries are read on the device: a captured graph follows them.  A run is a block of the
// grid, and a grid may have five times as many blocks as fit the GPU; a resident block that has finished its run takes
// over one that has not started (cluster launch control), without refilling its pipeline.  SMs differ in the bandwidth
// they get and items in their cost per tile: with one run per block the slowest block took 279 us where the median took
// 225 (64 rows of 2304 x 32 heads x 100 elements).  Where the tables are short this is not worth its fixed cost: a block takes
// all cached rows of one batch row and key head, prefix first, and writes the output itself (DIRECT; direct_pays has the rule).
// With few batch rows a cluster of up to 8 blocks shares them and merges its states through shared memory.
//
// What a warp does per 16 cached rows: S^T = K Q^T and O^T += V^T P^T on mma.sync tiles with the cached rows as M and
// eight query rows as N (the fewest that the instruction takes).  Up to 8 query rows of a key head: the four warps of a
// block split the cached rows of a tile; up to 16: two and two; up to 32: each warp has its own eight query rows.  One
// query row per cached row is 1 flop per byte: HBM bounds it, and the products run on the tensor cores only because that
// takes the fewest instructions per byte.
//
// Measured in a captured graph: 64 rows x 32 heads of 100 elements over 2424 shared (four groups) and up to 2304 own rows,
// 1.19 GB: 203 us, 5.8 TB/s; 2 us of it go by until the lengths are read and cut, 1.5 until the first tile, 4 in the merge.
// 32 rows x 20 heads of 64 over 120 shared and 1024 own rows, 169 MB: 39.7 us, of which 27 stream.  DIRECT: two rows x 12 heads over
// 120 shared and 100 own rows: 5.2 us, a chain of three dependent reads; two rows x 8 heads of 128 over 128 shared and 4096 own
// rows, 35 MB, clusters of 8: 11.9 us (list: 23.5).
#include <math.h>
#include <type_traits>

#include "adsa_prefix.cuh"

namespace adsa {

// cached rows of a unit: 32 KB of K and V for rows of up to 128 elements
__host__ __device__ constexpr int tile_rows(int nsub) { return nsub == 1 ? 128 : 64; }
constexpr int kPaQueries = 32;              // query rows of an item at most
constexpr int kPaWarps = 4;                 // warps that compute; one more warp copies
constexpr int kPaThreads = (kPaWarps + 1) * 32;
constexpr int kPaMaxEntries = 4096;         // batch rows + twice the groups of a call: 8 bytes of shared memory each beside the tiles
constexpr int kPaMergeThreads = 128;
constexpr int kPaSplit = 8;                 // blocks of a cluster at most
// how prefix_sweep_kernel gets its work: runs of one list; a batch row and key head to a block; .. to a cluster of blocks
enum { kModeList, kModeBlocks, kModeClusters };
constexpr long long kPaMaxRows = 0x7fffff00LL;   // a sequence: row numbers stay in 32 bits past the last tile
// A group's prefix goes to the wide kernel if the group has more query rows of a key head than fit one item here, where the
// mean group has and the prefix tables hold at least 8192 rows of up to 64 elements (4096 of up to 128).  Two groups of 33
// rows, 8 key heads of 128 (us, here / wide): 512 rows 20 / 21, 4096 40 / 31, 32768 144 / 71; of 128 rows: 36 / 42,
// 68 / 59, 267 / 98; heads of 64, 33 rows: 18 / 20, 26 / 28, 82 / 62.  20 rows: 17 / 20, 26 / 30, 89 / 70.
constexpr int kWideAbove = 32;
constexpr long long kWideRows = 8192;

// Blocks of a cluster that share the cached rows of one item: as many as the GPU holds at once (the eighth is what clusters of 8
// leave of a group of SMs; in two turns they are slow: 14 rows x 20 heads of 64, 32 KB, 1 / 2 / 4 blocks 6.1 / 12.6 / 23.9 us),
// while there are tiles for them.  2 rows x 8 heads
// of 64, 1 / 2 / 4 / 8 blocks in us: 64 KB 5.7 / 6.5 / 6.4 / 6.6, 128 KB 7.0 / 7.1 / 6.5 / 6.7, 288 KB 10.2 / 8.9 / 7.7 / 7.4,
// 1 MB 25.5 / 16.1 / 11.5 / 9.4.
inline int direct_split(long long items, long long blocks, double most)
{
    int n = 1;
    while (n < kPaSplit && items * 2 * n <= blocks * 7 / 8 && most >= fmax(128.0, 64.0 * n) * 1024) n *= 2;
    return n;
}

// A block (or cluster) per batch row and key head, by the bytes of K and V that the tables hold for one of them (most) and how many
// of these the list would not read, as the other rows of a group have (again).  It does not balance, and saves the list, the second
// kernel and the states, of which every query head has its own.  Measured, list / direct in us.  While all are resident at once: 2
// rows x 12 heads of 64, 32 KB 8.4 / 5.6, 1 MB (8 blocks) 19.5 / 9.9; 8 x 20 of 128, 576 KB 24.1 / 18.0, 1 MB 29.5 / 28.7; longer
// rows beside short ones leave too much to one block.  In two turns: 20 rows x 20 heads of 64, 32 KB 14.6 / 10.4, 192 KB 24.5 /
// 16.6, 256 KB of which half prefix 20.4 / 19.0, 528 KB of which 512 prefix 18.6 / 30.6.  In more, heads of 64: 256 rows x 32 heads
// on 8, 48 KB of which a third prefix 46.0 / 35.8, 192 KB of which a third 81.1 / 70.2, 288 KB of which 32 prefix 141 / 99.9; 128
// x 32 on 32, 96 KB of which a third 77.4 / 90.5, 288 KB of which 32 213 / 173; 32 x 20 of 128, 2.2 turns, 576 KB 63.3 / 67.9.
// (Lengths are on the device, so what the tables could hold decides; the header tells the caller.)
inline bool direct_pays(long long items, long long blocks, int per_kv, double most, double again)
{
    if (items <= blocks) return most <= direct_split(items, blocks, most) * 640.0 * 1024;
    const bool two_turns = items <= 2 * blocks;
    if (two_turns && most <= 256 * 1024) return true;
    if (most > 600 * 1024) return false;
    return two_turns || per_kv > 1 ? most >= 3 * again : items >= 4 * blocks && most >= 9 * again;
}

// how many warps share the query rows of an item with m <= kPaQueries of them (the rest share its cached rows)
__host__ __device__ __forceinline__ int query_warps(int m) { return m <= 8 ? 1 : m <= 16 ? 2 : 4; }
// items of a key head with m query rows, and the query rows a slot of a batch row's own items must hold
__host__ __device__ __forceinline__ int query_items(int m) { return (m + kPaQueries - 1) / kPaQueries; }
__host__ __device__ __forceinline__ int own_slot_rows(int per_kv)
{
    return per_kv >= kPaQueries ? kPaQueries : kPaWarps / query_warps(per_kv) * per_kv;
}

// Lengths and boundaries as read (and clamped) once per block; entries are groups, then batch rows.
struct Shared {
    uint32_t *plan;                         // [entries + 1] first unit of every entry
    int *len;                               // [entries] cached rows
    int *begin;                             // [groups + 1]
    uint32_t *wide;                         // [groups] first unit of every group in the wide kernel's list
};
__device__ __forceinline__ int members(const Shared &c, int g) { return max(c.begin[g + 1] - c.begin[g], 0); }

// Neighbouring units of one item inside a run.
struct Segment {
    const int32_t *pages;                   // page table of the cached rows
    int n;                                  // cached rows of the item
    int head;                               // key head
    int tile0, tiles;                       // the units
    int row0, rows;                         // packed query rows (batch row * per_kv + head in the key head): first, count
    int slot;                               // of the partial state
    bool prefix;
};

template <int TILE>
struct Walk {
    uint32_t u, end;
    int e, run;
    bool empty;                             // the run has no units at all
    __device__ void begin(const PrefixArgs &a, const Shared &c, const Cut &cut, int run_)
    {
        run = run_;
        const int entries = a.groups + a.batch;
        u = end = 0;
        if ((uint32_t)run < cut.runs) { u = cut.begin_of(run); end = cut.begin_of(run + 1); }
        empty = u >= end;
        int lo = 0, hi = entries;           // the last entry whose first unit is <= u
        while (lo < hi) {
            const int mid = (lo + hi + 1) >> 1;
            if (c.plan[mid] <= u) lo = mid;
            else hi = mid - 1;
        }
        e = lo;
    }
    __device__ bool next(const PrefixArgs &a, const Shared &c, Segment &s)
    {
        if (u >= end) return false;
        while (u >= c.plan[e + 1]) ++e;
        const uint32_t at = u - c.plan[e];
        const bool pre = e < a.groups;
        const int b0 = pre ? c.begin[e] : e - a.groups, m = (pre ? members(c, e) : 1) * a.per_kv, mt = query_items(m);
        s.n = c.len[e];
        const uint32_t tiles = (uint32_t)((s.n + TILE - 1) / TILE), item = at / tiles;   // (key head, then query rows)
        s.head = mt == 1 ? (int)item : (int)item / mt;
        const int q = (int)item - s.head * mt;
        s.row0 = b0 * a.per_kv + q * kPaQueries;
        s.rows = min(m - q * kPaQueries, kPaQueries);
        s.pages = pre ? a.p_table + (size_t)e * a.max_p_pages : a.table + (size_t)b0 * a.max_pages;
        s.slot = (pre ? first_group_item(a, e, b0, kPaQueries) : b0 * a.kv_heads * mt) + (int)item + run;
        s.prefix = pre;
        s.tile0 = (int)(at - item * tiles);
        s.tiles = (int)min(tiles - (uint32_t)s.tile0, end - u);
        u += (uint32_t)s.tiles;
        return true;
    }
};

// Every thread of every block of the cluster takes part; what was written to shared memory before is seen after
__device__ __forceinline__ void pa_cluster_sync()
{
    asm volatile("barrier.cluster.arrive.release;\nbarrier.cluster.wait.acquire;" ::: "memory");
}
// the address of block `rank`'s copy of what lies at `addr` in this block's shared memory
__device__ __forceinline__ uint32_t pa_of_rank(uint32_t addr, uint32_t rank)
{
    uint32_t r;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(r) : "r"(addr), "r"(rank));
    return r;
}
__device__ __forceinline__ float2 pa_ld_cluster(uint32_t addr)
{
    float2 v;
    asm volatile("ld.shared::cluster.v2.f32 {%0, %1}, [%2];" : "=f"(v.x), "=f"(v.y) : "r"(addr) : "memory");
    return v;
}

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
// the transpose of an 8 x 8 matrix of 16-bit elements held by a warp (row lane / 4, columns 2 (lane % 4), + 1)
__device__ __forceinline__ uint32_t pa_transpose(uint32_t x)
{
    uint32_t y;
    asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
    return y;
}

// A block that has not started: asked for with pa_ask_block, its index (or -1: every block has started) read from the
// 16-byte answer once the barrier has counted it.
__device__ __forceinline__ void pa_ask_block(uint32_t answer, uint32_t bar)
{
    asm volatile("clusterlaunchcontrol.try_cancel.async.shared::cta.mbarrier::complete_tx::bytes.b128 [%0], [%1];" ::"r"(answer), "r"(bar) : "memory");
}
__device__ __forceinline__ int pa_answer(uint32_t answer)
{
    uint32_t ok, x;
    asm volatile("{\n\t.reg .b128 r;\n\t.reg .pred p;\n\tld.shared.b128 r, [%2];\n\t"
                 "clusterlaunchcontrol.query_cancel.is_canceled.pred.b128 p, r;\n\tselp.u32 %0, 1, 0, p;\n\tmov.u32 %1, 0;\n\t"
                 "@p clusterlaunchcontrol.query_cancel.get_first_ctaid::x.b32.b128 %1, r;\n\t}"
                 : "=r"(ok), "=r"(x) : "r"(answer) : "memory");
    return ok ? (int)x : -1;
}

// NSUB: 64-element sub-tiles of a row (head elements / 64, rounded up).  STAGES: tiles in flight per block.
// PACKED: the rows of a page are copied as they lie, one bulk copy per page, instead of 64-element columns in the
// 128-byte swizzle.  Rows whose 16-byte pieces are odd in number put the eight rows of an ldmatrix on eight different
// banks without a swizzle, and such rows straddle memory sectors when they are fetched column by column: with 208-byte rows
// the columns ran at 4.4 TB/s where 256-byte rows run at 6.2.
// DIRECT: no list and no merge: a block sweeps all that one batch row's queries of one key head attend, prefix and own rows, and
// writes the output.  For calls so small that reading and cutting the lengths and the second kernel would cost more than
// the sweep (direct_pays).
template <typename T, int NSUB, int STAGES, bool PACKED, int MODE>
__global__ void __launch_bounds__(kPaThreads, NSUB <= 2 ? 2 : 1)
prefix_sweep_kernel(const __grid_constant__ PrefixArgs a, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map)
{
    constexpr bool DIRECT = MODE != kModeList;
    constexpr int KS = 4 * NSUB;                                   // 16-element steps over a row
    constexpr int TILE = tile_rows(NSUB), NB = TILE / 64;          // blocks of 16 cached rows that a warp has in hand at a time
    constexpr uint32_t kSub = TILE * 128, kHalf = NSUB * kSub;  // bytes: a sub-tile; K (or V) of a tile
    constexpr int DP = 64 * NSUB;                                  // floats of a state row
    constexpr float kBias = WeightBias<T>::value;
    extern __shared__ unsigned char pa_smem[];
    __shared__ uint64_t bars[2 * STAGES + 4];
    __shared__ __align__(16) uint4 answers[2];
    __shared__ uint2 warp_sums[kPaThreads / 32];
    const uint32_t ring = (smem_u32(pa_smem) + 1023u) & ~1023u, pitch = PACKED ? (uint32_t)a.row_stride * 2u : 128u;
    Shared c;
    c.plan = reinterpret_cast<uint32_t *>(pa_smem + (ring - smem_u32(pa_smem)) + (size_t)STAGES * 2 * kHalf);
    c.len = reinterpret_cast<int *>(c.plan + a.groups + a.batch + 1);
    c.begin = c.len + a.groups + a.batch;
    c.wide = reinterpret_cast<uint32_t *>(c.begin + a.groups + 1);
    const uint32_t full = smem_u32(bars), empty = full + 8 * STAGES, asked = empty + 8 * STAGES, heard = asked + 16, answer = smem_u32(answers);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int entries = a.groups + a.batch, split = MODE == kModeClusters ? a.split : 1;

    if (tid == 0) {
        for (int i = 0; i < STAGES; ++i) { mbar_init(full + 8 * i, 1); mbar_init(empty + 8 * i, kPaWarps); }
        for (int i = 0; i < 2; ++i) { mbar_init(asked + 8 * i, 1); mbar_init(heard + 8 * i, kPaWarps + 1); }
        mbar_init_fence();
        asm volatile("prefetch.tensormap [%0];" ::"l"(&k_map) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&v_map) : "memory");
    }
    // DIRECT: the batch row, its query item, rows of prefix and own rows, and which of their tiles are this block's
    int part = 0, own_b = 0, own_q = 0, item = 0, rank = 0, parts_n[2] = {0, 0}, from[2] = {0, 0}, to[2] = {0, 0}, group = -1;
    uint32_t total = 0, wide_total = 0;
    Walk<TILE> walk = {};
    const bool behind_wide = !DIRECT && a.w_resident > 0;
    if constexpr (DIRECT) {
        item = (int)blockIdx.x / split;
        rank = (int)blockIdx.x - item * split;
        const int qi = query_items(a.per_kv), rest = item / qi;
        own_q = item - rest * qi;
        own_b = rest / a.kv_heads;
        pdl_wait();
        pdl_launch();
        parts_n[1] = clamp_rows(a.n_rows[own_b], a.max_pages, a.page_rows);
        for (int g0 = 0; g0 < a.groups && group < 0; g0 += 128) {   // the first group that holds the batch row
            uint32_t first = 0xffffffffu;
#pragma unroll
            for (int j = 3; j >= 0; --j) {
                const int g = g0 + 32 * j + lane;
                if (g < a.groups && group_begin(a, g) <= own_b && own_b < group_begin(a, g + 1)) first = (uint32_t)g;
            }
            group = (int)__reduce_min_sync(0xffffffffu, first);
        }
        if (group >= 0) parts_n[0] = clamp_rows(a.p_rows[group], a.max_p_pages, a.page_rows);
        if (blockIdx.x == 0 && a.status)
            for (int g = tid; g < a.groups; g += kPaThreads)
                if (a.start[g] > a.start[g + 1]) atomicOr(a.status, ADSA_DEV_BAD_GROUPS);
        const int pre = (parts_n[0] + TILE - 1) / TILE, all = pre + (parts_n[1] + TILE - 1) / TILE;
        const int lo = (int)((long long)all * rank / split), hi = (int)((long long)all * (rank + 1) / split);
        from[0] = min(lo, pre);
        to[0] = min(hi, pre);
        from[1] = max(lo - pre, 0);
        to[1] = max(hi - pre, 0);
        __syncthreads();                                           // (the barriers are set up)
    }
    if constexpr (!DIRECT) {
        // The small tables into L2 while the kernel ahead still runs (hints; they are read after the wait)
        {
            const auto hint = [&](const int32_t *p, long long n) {
                for (long long i = ((long long)blockIdx.x * kPaThreads + tid) * 32; i < min(n, 65536LL); i += (long long)gridDim.x * kPaThreads * 32)
                    asm volatile("prefetch.global.L2 [%0];" ::"l"(p + i));
            };
            hint(a.table, (long long)a.batch * a.max_pages);
            hint(a.n_rows, a.batch);
            hint(a.p_table, (long long)a.groups * a.max_p_pages);
            hint(a.p_rows, a.groups);
            hint(a.start, a.groups > 0 ? a.groups + 1 : 0);
        }
        // Behind the wide kernel of the same call (which has waited for what was ahead of it before this one could begin) there
        // is nothing to wait for here; each block waits before it ends, so that the merge finds both kernels' states.
        if (!behind_wide) pdl_wait();
        pdl_launch();

        // ---- lengths, boundaries, first unit of every entry: each thread sums a few entries, the sums are scanned over the block ----
        const int per = (entries + kPaThreads - 1) / kPaThreads, e0 = min(tid * per, entries), e1 = min(e0 + per, entries);
        bool falls = false;
        for (int g = tid; g <= a.groups && a.groups > 0; g += kPaThreads) {
            c.begin[g] = group_begin(a, g);
            falls = falls || (g > 0 && a.start[g - 1] > a.start[g]);
        }
        for (int e = e0; e < e1; ++e)
            c.len[e] = e < a.groups ? clamp_rows(a.p_rows[e], a.max_p_pages, a.page_rows) : clamp_rows(a.n_rows[e - a.groups], a.max_pages, a.page_rows);
        if (__syncthreads_or(falls)) {                             // groups that overlap could be more units than are counted in 32 bits
            for (int g = tid; g <= a.groups; g += kPaThreads) c.begin[g] = 0;
            if (a.status && tid == 0) atomicOr(a.status, ADSA_DEV_BAD_GROUPS);
            __syncthreads();
        }
        uint2 mine = make_uint2(0u, 0u);                               // units of this list, of the wide kernel's
        for (int e = e0; e < e1; ++e) {
            const int m = (e < a.groups ? members(c, e) : 1) * a.per_kv;
            c.plan[e] = mine.x;
            if (e < a.groups) c.wide[e] = mine.y;
            if (e < a.groups && m > a.wide_above) mine.y += WideItems(m, c.len[e]).head_units * (uint32_t)a.kv_heads;
            else mine.x += (uint32_t)query_items(m) * (uint32_t)a.kv_heads * (uint32_t)((c.len[e] + TILE - 1) / TILE);
        }
        uint2 incl = mine;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) {
            const uint32_t x = __shfl_up_sync(0xffffffffu, incl.x, o), y = __shfl_up_sync(0xffffffffu, incl.y, o);
            if (lane >= o) { incl.x += x; incl.y += y; }
        }
        if (lane == 31) warp_sums[warp] = incl;
        __syncthreads();
        uint2 before = make_uint2(incl.x - mine.x, incl.y - mine.y);
        for (int w = 0; w < kPaThreads / 32; ++w) {
            const uint2 s = warp_sums[w];
            if (w < warp) { before.x += s.x; before.y += s.y; }
            total += s.x;
            wide_total += s.y;
        }
        for (int e = e0; e < e1; ++e) {
            c.plan[e] += before.x;
            if (e < a.groups) c.wide[e] += before.y;
        }
        if (tid == 0) c.plan[entries] = total;
        __syncthreads();
    }
    const Cut cut(total, (uint32_t)max(a.resident, 1));
    if constexpr (!DIRECT) walk.begin(a, c, cut, blockIdx.x);
    Segment s;
    // The next segment of this block's runs.  Each warp follows the runs by itself; the copying warp asks for the next
    // run when it begins one, into the answer slot that all warps have read the last time; warp 0 leaves the run's share
    // of the plan for the merge (that goes by run, as any block may be taken over before it starts).
    int limit = kCopySpinLimit;
    uint32_t turns = 0;                                            // runs finished by this warp
    const auto ask = [&]() {
        if (lane == 0) {
            const uint32_t i = turns & 1u;
            if (!mbar_wait_bounded(heard + 8 * i, ((turns >> 1) & 1u) ^ 1u, limit)) limit = kCopySpinAfterTimeout;
            mbar_expect_tx(asked + 8 * i, 16);
            pa_ask_block(answer + 16 * i, asked + 8 * i);
        }
        __syncwarp();                                              // the other lanes must not spin for the answer before it is asked for
    };
    const auto leave_plan = [&](int run) {
        const uint32_t share = max(cut.runs, 1u);
        for (int b = (uint32_t)run < share ? run + lane * (int)share : a.batch; b < a.batch; b += 32 * (int)share) {
            // the batch row's own units, and its group's: the last group that begins at or before it.  Everything a merging
            // warp needs is in the row's own three words of four: one line that all of them read would hold them up.
            uint4 group = make_uint4(0u, 0u, 0u, 0u);
            uint32_t slot = 0u;
            int lo = -1, hi = a.groups - 1;
            while (lo < hi) {
                const int mid = (lo + hi + 1) >> 1;
                if (c.begin[mid] <= b) lo = mid;
                else hi = mid - 1;
            }
            if (lo >= 0 && b < c.begin[lo + 1]) {
                const int m = members(c, lo) * a.per_kv;
                const bool wide = m > a.wide_above;
                const int tile = wide ? kWideTile : TILE;
                group = make_uint4(wide ? c.wide[lo] : c.plan[lo], (uint32_t)(c.len[lo] + tile - 1) / tile, (uint32_t)c.begin[lo], (uint32_t)m);
                slot = (uint32_t)first_group_item(a, lo, c.begin[lo], wide ? kWideQueries : kPaQueries);
            }
            a.plan[3 * b] = make_uint4(c.plan[a.groups + b], (uint32_t)(c.len[a.groups + b] + TILE - 1) / TILE, total, slot);
            a.plan[3 * b + 1] = group;
            a.plan[3 * b + 2] = make_uint4(wide_total, 0u, 0u, 0u);
        }
        __syncwarp();
    };
    // patient: wait for whatever comes.  Otherwise only go as far as an answer that is already asked for: behind an empty run the
    // next answer is asked for when the copying warp gets there, which may first need tiles of the segment in hand to be freed.
    enum { kEnd, kSegment, kLater };
    const auto advance = [&](Segment &n, bool patient) {
        if constexpr (DIRECT) {
            while (part < 2 && from[part] == to[part]) ++part;
            if (part == 2) return kEnd;
            const int rest = item / query_items(a.per_kv);
            n.pages = part == 0 ? a.p_table + (size_t)group * a.max_p_pages : a.table + (size_t)own_b * a.max_pages;
            n.n = parts_n[part];
            n.head = rest - own_b * a.kv_heads;
            n.tile0 = from[part];
            n.tiles = to[part] - from[part];
            n.row0 = own_b * a.per_kv + own_q * kPaQueries;
            n.rows = min(a.per_kv - own_q * kPaQueries, kPaQueries);
            ++part;
            return kSegment;
        } else {
            while (!walk.next(a, c, n)) {
                if (!patient && walk.empty) return kLater;
                const uint32_t i = turns & 1u;
                int run = -1;
                if (mbar_wait_bounded(asked + 8 * i, (turns >> 1) & 1u, limit)) run = pa_answer(answer + 16 * i);
                else {
                    limit = kCopySpinAfterTimeout;
                    if (a.status && lane == 0) atomicOr(a.status, ADSA_DEV_COPY_TIMEOUT);
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");   // the answer is read before the slot is asked into again
                __syncwarp();
                if (lane == 0) mbar_arrive(heard + 8 * i);
                ++turns;
                if (run < 0) return kEnd;
                if (warp == kPaWarps) ask();
                if (warp == 0) leave_plan(run);
                walk.begin(a, c, cut, run);
            }
            return kSegment;
        }
    };

    if (warp == kPaWarps) {                                        // ---- the copying warp ----
        int stage = 0;
        uint32_t phase = 0;
        const int page_shift = (a.page_rows & (a.page_rows - 1)) == 0 ? 31 - __clz(a.page_rows) : -1;
        const auto page_of = [&](int row) { return page_shift >= 0 ? row >> page_shift : row / a.page_rows; };
        if (!DIRECT) ask();
        while (advance(s, true) == kSegment) {
            // page ids are read 32 at a time, a lane each
            const int last_page = page_of(s.n - 1);
            int window = -64, ids = 0;
            for (int t = s.tile0; t < s.tile0 + s.tiles; ++t) {
                const int rows = min(TILE, s.n - t * TILE), page0 = page_of(t * TILE), page1 = page_of(t * TILE + rows - 1);
                const int pieces = PACKED ? page1 - page0 + 1 : (rows + a.box_rows - 1) / a.box_rows;
                if (page1 >= window + 32) {
                    window = page0;
                    ids = window + lane <= last_page ? s.pages[window + lane] : 0;
                }
                const uint32_t k_dst = ring + stage * 2 * kHalf;
                bool waited = false;
                for (int i0 = 0; i0 < pieces; i0 += 32) {
                    const int i = min(i0 + lane, pieces - 1), row = PACKED ? max(t * TILE, (page0 + i) * a.page_rows) : t * TILE + i * a.box_rows;
                    const int pg = PACKED ? page0 + i : page_of(row);
                    int page = __shfl_sync(0xffffffffu, ids, (pg - window) & 31);
                    if (pg - window >= 32) page = s.pages[pg];     // a tile of more than 32 pages
                    if (page < 0 || page >= a.n_pages) {           // (the row's result is then unspecified)
                        page = 0;
                        if (a.status) atomicOr(a.status, ADSA_DEV_BAD_PAGE);
                    }
                    const int y = (page * a.kv_heads + s.head) * a.page_rows + row - pg * a.page_rows;
                    const uint32_t dst = k_dst + (uint32_t)(row - t * TILE) * (PACKED ? pitch : 128u);
                    if (!waited) {                                 // the addresses are ready when the stage is
                        waited = true;
                        if (!mbar_wait_bounded(empty + 8 * stage, phase ^ 1u, limit)) {
                            limit = kCopySpinAfterTimeout;
                            if (a.status && lane == 0) atomicOr(a.status, ADSA_DEV_COPY_TIMEOUT);
                        }
                        if (lane == 0) mbar_expect_tx(full + 8 * stage, PACKED ? (uint32_t)rows * pitch * 2u : (uint32_t)(pieces * a.box_rows) * 128u * 2u * NSUB);
                        __syncwarp();
                    }
                    if (i0 + lane < pieces) {
                        if constexpr (PACKED) {
                            const uint32_t bytes = (uint32_t)(min((pg + 1) * a.page_rows, t * TILE + rows) - row) * pitch;
                            bulk_g2s(dst, (const unsigned char *)a.k_pool + (size_t)y * pitch, bytes, full + 8 * stage);
                            bulk_g2s(dst + kHalf, (const unsigned char *)a.v_pool + (size_t)y * pitch, bytes, full + 8 * stage);
                        } else {
#pragma unroll
                            for (int c = 0; c < NSUB; ++c) {
                                pa_tma(dst + c * kSub, &k_map, c * 64, y, full + 8 * stage);
                                pa_tma(dst + kHalf + c * kSub, &v_map, c * 64, y, full + 8 * stage);
                            }
                        }
                    }
                }
                if (++stage == STAGES) { stage = 0; phase ^= 1u; }
            }
        }
        if (behind_wide) pdl_wait();
        if constexpr (MODE == kModeClusters) {
            pa_cluster_sync();
            pa_cluster_sync();
        }
        return;
    }

    // ---- the computing warps ----
    const int g = lane >> 2, t4 = lane & 3, mi = lane >> 3, lr = lane & 7;
    // lane's row address in a 16-row block for K (as A: cached rows x elements) and V (transposed: elements x cached rows)
    const uint32_t k_row = (uint32_t)((mi & 1) * 8 + lr) * pitch, v_row = (uint32_t)((mi >> 1) * 8 + lr) * pitch;
    const int k_ch = mi >> 1, v_ch = mi & 1;
    // byte offset of 16-byte piece 2 step + half of a row
    const auto piece_at = [&](int step, int half) {
        return PACKED ? (uint32_t)(32 * step + 16 * half) : (uint32_t)(step >> 2) * kSub + (uint32_t)((((2 * step + half) & 7) ^ lr) << 4);
    };
    int stage = 0;
    uint32_t phase = 0;
    // Q^T as the B operand: query row g of this warp's eight, elements 16 ks + 2 t4, + 1 and + 8, + 9; asked for one segment ahead.
    // Up to four query rows are there twice: columns 0 .. 3 of the products carry the weights' hi parts on, columns 4 .. 7 the lo parts.
    uint32_t qn[KS][2];
    const auto ask_q = [&](const Segment &n) {
        const int qb = warp & (query_warps(n.rows) - 1), r = n.rows <= 4 ? g & 3 : qb * 8 + g, packed = n.row0 + r, b = packed / a.per_kv, j = packed - b * a.per_kv;
        const T *qp = (const T *)a.q + b * a.q_row + (n.head * a.per_kv + j) * a.q_head;
        const bool there = r < n.rows;
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int col = 16 * ks + 2 * t4 + i * 8;
                qn[ks][i] = there && col < a.d ? __ldg(reinterpret_cast<const uint32_t *>(qp + col)) : 0u;
            }
        }
    };
    Segment nxt;
    auto more = advance(nxt, true);
    if (more == kSegment) ask_q(nxt);
    if (!DIRECT && warp == 0) leave_plan(blockIdx.x);              // while the first tile is on its way
    // state of query rows 2 t4 and 2 t4 + 1: maximum (alike in the eight lanes of a t4), this lane's share of the sum, O^T
    float o[KS][4], m_run[2] = {-INFINITY, -INFINITY}, l_run[2] = {0.f, 0.f};
#pragma unroll
    for (int dp = 0; dp < KS; ++dp) { o[dp][0] = o[dp][1] = o[dp][2] = o[dp][3] = 0.f; }
    const float lo_whole = t4 >= 2 ? WeightSplit<T>::one : 0.f;
    const uint32_t lo_sign = t4 >= 2 ? 0x80000000u : 0u;
    const auto add_lo_columns = [&]() {
#pragma unroll
        for (int dp = 0; dp < KS; ++dp) {
#pragma unroll
            for (int i = 0; i < 4; ++i) o[dp][i] += __shfl_xor_sync(0xffffffffu, o[dp][i], 2);
        }
    };
    while (more == kSegment) {
        s = nxt;
        uint32_t qa[KS][2];
#pragma unroll
        for (int ks = 0; ks < KS; ++ks) { qa[ks][0] = qn[ks][0]; qa[ks][1] = qn[ks][1]; }
        more = advance(nxt, false);
        if (more == kSegment) ask_q(nxt);
        const int wq = query_warps(s.rows), wk = kPaWarps / wq;     // warps over query rows, warps over cached rows
        const int qb = warp & (wq - 1), kb = warp / wq;
        const bool apart = s.rows > 4;                              // the lo parts are a product of their own
        for (int t = s.tile0; t < s.tile0 + s.tiles; ++t) {
            if (!mbar_wait_bounded(full + 8 * stage, phase, limit)) {
                limit = kCopySpinAfterTimeout;
                if (a.status && lane == 0) atomicOr(a.status, ADSA_DEV_COPY_TIMEOUT);
            }
            const uint32_t ks_u32 = ring + stage * 2 * kHalf, vs_u32 = ks_u32 + kHalf;
            const int valid = min(TILE, s.n - t * TILE);
            for (int c0 = kb * 16 * NB; c0 < valid; c0 += wk * 16 * NB) {   // NB times sixteen cached rows
                const bool tail = c0 + 16 * NB > valid;
                const uint32_t v_at = vs_u32 + (uint32_t)c0 * pitch + v_row;
                float sc[NB][4];
#pragma unroll
                for (int n = 0; n < NB; ++n) {
                    float s2[4] = {0.f, 0.f, 0.f, 0.f};              // two chains of products
                    sc[n][0] = sc[n][1] = sc[n][2] = sc[n][3] = 0.f;
#pragma unroll
                    for (int ks = 0; ks < KS; ++ks) {
                        if (PACKED && ks >= KS - 4 && 16 * ks >= a.d) break;
                        uint32_t kf[4];
                        pa_ldsm(ks_u32 + (uint32_t)(c0 + 16 * n) * pitch + k_row + piece_at(ks, k_ch), kf);
                        if (PACKED && ks >= KS - 4 && 16 * ks + 16 > a.d) {   // padding and the next row: not part of this one
                            if (16 * ks + 2 * t4 >= a.d) kf[0] = kf[1] = 0u;
                            if (16 * ks + 8 + 2 * t4 >= a.d) kf[2] = kf[3] = 0u;
                        }
                        if (ks & 1) pa_mma<T>(s2, kf, qa[ks][0], qa[ks][1]);
                        else pa_mma<T>(sc[n], kf, qa[ks][0], qa[ks][1]);
                    }
#pragma unroll
                    for (int i = 0; i < 4; ++i) sc[n][i] += s2[i];
                }
                float mx[2] = {-INFINITY, -INFINITY};
#pragma unroll
                for (int n = 0; n < NB; ++n) {
                    if (tail) {
                        if (c0 + 16 * n + g >= valid) sc[n][0] = sc[n][1] = -INFINITY;
                        if (c0 + 16 * n + g + 8 >= valid) sc[n][2] = sc[n][3] = -INFINITY;
                    }
                    mx[0] = fmaxf(mx[0], fmaxf(sc[n][0], sc[n][2]));
                    mx[1] = fmaxf(mx[1], fmaxf(sc[n][1], sc[n][3]));
                }
                // a new maximum anywhere in the warp: find it over the rows of the block, rescale what was summed
                if (__any_sync(0xffffffffu, mx[0] > m_run[0] || mx[1] > m_run[1])) {
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
#pragma unroll
                        for (int x = 4; x < 32; x <<= 1) mx[h] = fmaxf(mx[h], __shfl_xor_sync(0xffffffffu, mx[h], x));
                        const float m_new = fmaxf(m_run[h], mx[h]);
                        const float corr = m_new == -INFINITY ? 1.f : pa_exp2((m_run[h] - m_new) * a.scale_log2e);
                        m_run[h] = m_new;
                        l_run[h] *= corr;
#pragma unroll
                        for (int dp = 0; dp < KS; ++dp) { o[dp][h] *= corr; o[dp][h + 2] *= corr; }
                    }
                }
                float shift[2];
#pragma unroll
                for (int h = 0; h < 2; ++h) shift[h] = kBias - (m_run[h] == -INFINITY ? 0.f : m_run[h]) * a.scale_log2e;
                // weights, then O += P V; kApart: a branch around each of the second products would stand between the loads of V
                const auto weigh = [&](auto kApart) {
                    constexpr bool APART = decltype(kApart)::value;
                    uint32_t pb[NB][2], pl[APART ? NB : 1][2];
#pragma unroll
                    for (int n = 0; n < NB; ++n) {
                        float p[4];
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            p[i] = pa_exp2(fmaf(sc[n][i], a.scale_log2e, shift[i & 1]));
                            l_run[i & 1] += p[i];                   // the sum takes the weights before they are rounded
                        }
#pragma unroll
                        for (int i = 0; i < 2; ++i) {
                            const float2 w = make_float2(p[2 * i], p[2 * i + 1]);
                            if constexpr (APART) {
                                uint32_t hi, lo;
                                split_weights<T>(w, hi, lo);
                                pb[n][i] = pa_transpose(hi);
                                pl[n][i] = pa_transpose(lo);
                            } else {
                                pb[n][i] = pa_transpose(weights_of_lane<T>(w, lo_whole, lo_sign));
                            }
                        }
                    }
                    // rows behind the end hold anything, and a weight of zero does not silence an infinity or a NaN of V
                    if (!tail) {
#pragma unroll
                        for (int n = 0; n < NB; ++n) {
#pragma unroll
                            for (int dp = 0; dp < KS; ++dp) {
                                if (PACKED && dp >= KS - 4 && 16 * dp >= a.d) break;   // (rows of O past the head elements are not kept)
                                uint32_t vf[4];
                                pa_ldsm_t(v_at + n * 16u * pitch + piece_at(dp, v_ch), vf);
                                pa_mma<T>(o[dp], vf, pb[n][0], pb[n][1]);
                                if constexpr (APART) pa_mma<T>(o[dp], vf, pl[n][0], pl[n][1]);
                            }
                        }
                    } else {
#pragma unroll
                        for (int n = 0; n < NB; ++n) {
                            const int left = valid - c0 - 16 * n - 2 * t4;   // of the cached rows 2 t4, + 1 and + 8, + 9
                            const uint32_t lo = left >= 2 ? 0xffffffffu : left == 1 ? 0xffffu : 0u, hi = left >= 10 ? 0xffffffffu : left == 9 ? 0xffffu : 0u;
#pragma unroll
                            for (int dp = 0; dp < KS; ++dp) {
                                if (PACKED && dp >= KS - 4 && 16 * dp >= a.d) break;   // (rows of O past the head elements are not kept)
                                uint32_t vf[4];
                                pa_ldsm_t(v_at + n * 16u * pitch + piece_at(dp, v_ch), vf);
                                vf[0] &= lo; vf[1] &= lo; vf[2] &= hi; vf[3] &= hi;
                                pa_mma<T>(o[dp], vf, pb[n][0], pb[n][1]);
                                if constexpr (APART) pa_mma<T>(o[dp], vf, pl[n][0], pl[n][1]);
                            }
                        }
                    }
                };
                if (apart) weigh(std::true_type{});
                else weigh(std::false_type{});
            }
            __syncwarp();
            if (lane == 0) mbar_arrive(empty + 8 * stage);
            if (++stage == STAGES) { stage = 0; phase ^= 1u; }
        }
        if constexpr (!DIRECT) {                                   // (else the own rows carry the state of the prefix on)
            // ---- the partial state: a slot holds wk states of s.rows rows ----
            if (!apart) add_lo_columns();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
#pragma unroll
                for (int x = 4; x < 32; x <<= 1) l_run[h] += __shfl_xor_sync(0xffffffffu, l_run[h], x);
            }
            const bool fits = s.slot < (s.prefix ? a.n_p_slots : a.n_o_slots);
            if (!fits && a.status && lane == 0) atomicOr(a.status, ADSA_DEV_BAD_GROUPS);
            const size_t first = (size_t)s.slot * (s.prefix ? kPaQueries : own_slot_rows(a.per_kv)) + (size_t)kb * s.rows;
            float *st = s.prefix ? a.p_state : a.o_state, *ml = s.prefix ? a.p_ml : a.o_ml;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int r = qb * 8 + 2 * t4 + h;
                if (fits && r < s.rows) {
                    if (g == 0) *reinterpret_cast<float2 *>(ml + 2 * (first + r)) = make_float2(m_run[h] * a.scale_log2e - kBias, l_run[h]);
#pragma unroll
                    for (int dp = 0; dp < KS; ++dp) {
                        if (dp * 16 + g < a.d) st[(first + r) * DP + dp * 16 + g] = o[dp][h];
                        if (dp * 16 + g + 8 < a.d) st[(first + r) * DP + dp * 16 + g + 8] = o[dp][h + 2];
                    }
                }
                m_run[h] = -INFINITY;
                l_run[h] = 0.f;
            }
#pragma unroll
            for (int dp = 0; dp < KS; ++dp) { o[dp][0] = o[dp][1] = o[dp][2] = o[dp][3] = 0.f; }
            if (more == kLater) {
                more = advance(nxt, true);
                if (more == kSegment) ask_q(nxt);
            }
        }
    }
    if constexpr (DIRECT) {
        // ---- the warps' states to shared memory (the tiles have been read), then the outputs ----
        const int rows = min(a.per_kv - own_q * kPaQueries, kPaQueries), wq = query_warps(rows), wk = kPaWarps / wq, qb = warp & (wq - 1), kb = warp / wq;
        float *states = reinterpret_cast<float *>(pa_smem + (ring - smem_u32(pa_smem))), *mls = states + kPaQueries * DP;
        if (rows <= 4) add_lo_columns();
        asm volatile("bar.sync 1, 128;" ::: "memory");
#pragma unroll
        for (int h = 0; h < 2; ++h) {
#pragma unroll
            for (int x = 4; x < 32; x <<= 1) l_run[h] += __shfl_xor_sync(0xffffffffu, l_run[h], x);
            const int r = qb * 8 + 2 * t4 + h;
            if (r < rows) {
                if (g == 0) { mls[2 * (kb * rows + r)] = m_run[h] * a.scale_log2e - kBias; mls[2 * (kb * rows + r) + 1] = l_run[h]; }
#pragma unroll
                for (int dp = 0; dp < KS; ++dp) {
                    states[(kb * rows + r) * DP + dp * 16 + g] = o[dp][h];
                    states[(kb * rows + r) * DP + dp * 16 + g + 8] = o[dp][h + 2];
                }
            }
        }
        asm volatile("bar.sync 1, 128;" ::: "memory");
        const bool empty = parts_n[0] + parts_n[1] == 0;
        const int head = item / query_items(a.per_kv) - own_b * a.kv_heads, half = a.d / 2;
        const size_t out_row = ((size_t)own_b * a.kv_heads + head) * a.per_kv + own_q * kPaQueries;
        const auto leave = [&](int r, int e, float M, float L, float x, float y) {
            const float inv = empty ? 0.f : 1.f / L;
            x = empty ? 0.f : x * inv;
            y = empty ? 0.f : y * inv;
            const size_t at = (out_row + r) * a.d + e;
            if (a.out) *reinterpret_cast<uint32_t *>((T *)a.out + at) = pack2<T>(x, y);
            if (a.out_f32) *reinterpret_cast<float2 *>(a.out_f32 + at) = make_float2(x, y);
            if (a.lse && e == 0) a.lse[out_row + r] = empty ? -INFINITY : (M + log2f(L)) * 0.693147180559945309f;
        };
        // one state per query row and block, behind the warps' states
        float *merged = mls + 2 * kPaQueries, *merged_ml = merged + kPaQueries * DP;
        for (int i = tid; i < rows * half; i += kPaWarps * 32) {
            const int r = i / half, e = 2 * (i - r * half);
            float M = -INFINITY, L = 0.f, x = 0.f, y = 0.f;
            for (int k = 0; k < wk; ++k) M = fmaxf(M, mls[2 * (k * rows + r)]);
            for (int k = 0; k < wk; ++k) {
                const float m = mls[2 * (k * rows + r)], w = m == -INFINITY ? 0.f : pa_exp2(m - M);
                if (m == -INFINITY && mls[2 * (k * rows + r) + 1] == 0.f) continue;   // an empty state
                L += mls[2 * (k * rows + r) + 1] * w;
                x += states[(k * rows + r) * DP + e] * w;
                y += states[(k * rows + r) * DP + e + 1] * w;
            }
            if constexpr (MODE != kModeClusters) leave(r, e, M, L, x, y);
            else {
                *reinterpret_cast<float2 *>(merged + r * DP + e) = make_float2(x, y);
                if (e == 0) *reinterpret_cast<float2 *>(merged_ml + 2 * r) = make_float2(M, L);
            }
        }
        if constexpr (MODE == kModeClusters) {
            // the blocks of the cluster merge their states the same way, each a part of the outputs
            pa_cluster_sync();
            const uint32_t at = smem_u32(merged), at_ml = smem_u32(merged_ml);
            for (int i = rank * kPaWarps * 32 + tid; i < rows * half; i += split * kPaWarps * 32) {
                const int r = i / half, e = 2 * (i - r * half);
                float2 ml[kPaSplit], v[kPaSplit];
#pragma unroll
                for (int k = 0; k < kPaSplit; ++k) {
                    ml[k] = make_float2(-INFINITY, 0.f);
                    v[k] = make_float2(0.f, 0.f);
                    if (k < split) {
                        ml[k] = pa_ld_cluster(pa_of_rank(at_ml + 8 * r, k));
                        v[k] = pa_ld_cluster(pa_of_rank(at + 4 * (r * DP + e), k));
                    }
                }
                float M = -INFINITY, L = 0.f, x = 0.f, y = 0.f;
#pragma unroll
                for (int k = 0; k < kPaSplit; ++k) M = fmaxf(M, ml[k].x);
#pragma unroll
                for (int k = 0; k < kPaSplit; ++k) {
                    if (ml[k].x == -INFINITY && ml[k].y == 0.f) continue;   // an empty state
                    const float w = ml[k].x == -INFINITY ? 0.f : pa_exp2(ml[k].x - M);
                    L += ml[k].y * w;
                    x += v[k].x * w;
                    y += v[k].y * w;
                }
                leave(r, e, M, L, x, y);
            }
            pa_cluster_sync();                                     // no block ends while another reads its shared memory
        }
    }
}

// An output row (batch row, query head) is merged by a block: the states of the prefix units and of the row's own units,
// dealt to four warps.  (A warp per row instead: 109.8 us against 97.8 for 2048 rows of about 23 states.)
template <typename T, int NSUB>
__global__ void __launch_bounds__(kPaMergeThreads)
prefix_merge_kernel(const __grid_constant__ PrefixArgs a)
{
    constexpr int DP = 64 * NSUB, WARPS = kPaMergeThreads / 32, PER = 2 * NSUB;   // PER floats per lane
    __shared__ float s_m[WARPS], s_l[WARPS], s_o[WARPS][DP];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int heads = a.kv_heads * a.per_kv;
    const int b = (int)blockIdx.x / heads, qh = (int)blockIdx.x - b * heads, head = qh / a.per_kv, j = qh - head * a.per_kv;
    const size_t row = blockIdx.x;
    pdl_wait();
    pdl_launch();
    const uint4 own_part = a.plan[3 * (size_t)b], group = a.plan[3 * (size_t)b + 1];
    const uint32_t wide_total = a.plan[3 * (size_t)b + 2].x;
    // the prefix's states, then the row's own
    const int b0 = (int)group.z, m = (int)group.w;
    const bool pre = group.y > 0, own = own_part.y > 0, wide = pre && m > a.wide_above;   // (y: tiles)
    const int queries = wide ? kWideQueries : kPaQueries, mt = (m + queries - 1) / queries;
    const int packed = (b - b0) * a.per_kv + j, q = packed / queries, p_rows = min(m - q * queries, queries), p_item = head * mt + q;
    const int own_mt = query_items(a.per_kv), own_q = j / kPaQueries, own_rows = min(a.per_kv - own_q * kPaQueries, kPaQueries);
    const int own_item = head * own_mt + own_q;
    // first and last run of both, one division chain for all four: lanes 0, 1 the prefix's, 2, 3 the own rows'
    const bool of_prefix = (lane & 2) == 0, of_wide = of_prefix && wide;
    uint32_t unit, units;                    // first unit of the item, and from there to the first unit of its last tile
    if (of_wide) {
        const uint32_t cost = p_rows > 128 ? 2u : 1u;
        unit = group.x + (uint32_t)head * ((uint32_t)(m + 127) / 128u * group.y) + (uint32_t)q * 2u * group.y;
        units = cost * (group.y - 1u);
    } else {
        unit = of_prefix ? group.x + (uint32_t)p_item * group.y : own_part.x + (uint32_t)own_item * own_part.y;
        units = (of_prefix ? group.y : own_part.y) - 1u;
    }
    if (lane & 1) unit += units;
    uint32_t run = 0u;
    if (of_wide) run = WideCut(wide_total, (uint32_t)a.w_resident).run_of(unit);
    else if (of_prefix ? pre : own) run = Cut(own_part.z, (uint32_t)a.resident).run_of(unit);
    const uint32_t p0 = __shfl_sync(0xffffffffu, run, 0), p1 = __shfl_sync(0xffffffffu, run, 1), o0 = __shfl_sync(0xffffffffu, run, 2),
                   o1 = __shfl_sync(0xffffffffu, run, 3);
    const float *p_state = wide ? a.w_state : a.p_state, *p_ml = wide ? a.w_ml : a.p_ml;
    const int p_subs = wide ? (p_rows > 128 ? 1 : 2) : kPaWarps / query_warps(p_rows), p_step = wide ? 128 : p_rows, o_subs = kPaWarps / query_warps(own_rows), o_step = own_slot_rows(a.per_kv);
    const long long p_slot0 = (long long)own_part.w + p_item + p0, o_slot0 = (long long)b * a.kv_heads * own_mt + own_item + o0;
    const int p_segs = pre ? (int)min((long long)(p1 - p0 + 1), max(0LL, (wide ? a.n_w_slots : a.n_p_slots) - p_slot0)) : 0;
    const int o_segs = own ? (int)min((long long)(o1 - o0 + 1), max(0LL, a.n_o_slots - o_slot0)) : 0;
    const size_t p_slot = queries, p_first = (size_t)p_slot0 * p_slot + (packed - q * queries);
    const size_t o_first = (size_t)o_slot0 * o_step + (j - own_q * kPaQueries);
    const int n_p = p_segs * p_subs, n_states = n_p + o_segs * o_subs;
    float m_run = -INFINITY, l = 0.f, o[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) o[e] = 0.f;
    constexpr int AHEAD = 4;                // states in flight per warp
    for (int i0 = warp; i0 < n_states; i0 += AHEAD * WARPS) {
        float2 ml[AHEAD];
        float x[AHEAD][PER];
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            const int i = i0 + k * WARPS;
            ml[k] = make_float2(-INFINITY, 0.f);
            if (i < n_states) {
                const bool first = i < n_p;
                const int at = first ? i : i - n_p, subs = first ? p_subs : o_subs, seg = at / subs, sub = at - seg * subs;
                const size_t at_row = first ? p_first + (size_t)seg * p_slot + (size_t)sub * p_step : o_first + (size_t)seg * o_step + (size_t)sub * own_rows;
                ml[k] = *reinterpret_cast<const float2 *>((first ? p_ml : a.o_ml) + 2 * at_row);
                const float *st = (first ? p_state : a.o_state) + at_row * DP;
#pragma unroll
                for (int e = 0; e < PER; e += 2) *reinterpret_cast<float2 *>(&x[k][e]) = *reinterpret_cast<const float2 *>(st + e * 32 + 2 * lane);
            }
        }
#pragma unroll
        for (int k = 0; k < AHEAD; ++k) {
            if (ml[k].y == 0.f && ml[k].x == -INFINITY) continue;   // an empty state
            const float M = fmaxf(m_run, ml[k].x), w1 = m_run == -INFINITY ? 0.f : pa_exp2(m_run - M), w2 = ml[k].x == -INFINITY ? 0.f : pa_exp2(ml[k].x - M);
            l = l * w1 + ml[k].y * w2;
#pragma unroll
            for (int e = 0; e < PER; ++e) o[e] = o[e] * w1 + x[k][e] * w2;
            m_run = M;
        }
    }
    const bool empty = n_states == 0;
    if (lane == 0) { s_m[warp] = m_run; s_l[warp] = l; }
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
    const float inv = empty ? 0.f : 1.f / L;
    for (int e = 2 * threadIdx.x; e < a.d; e += 2 * kPaMergeThreads) {
        float2 x = make_float2(0.f, 0.f);
#pragma unroll
        for (int w = 0; w < WARPS; ++w) { x.x += s_o[w][e] * wgt[w]; x.y += s_o[w][e + 1] * wgt[w]; }
        x = empty ? make_float2(0.f, 0.f) : make_float2(x.x * inv, x.y * inv);
        if (a.out) *reinterpret_cast<uint32_t *>((T *)a.out + row * a.d + e) = pack2<T>(x.x, x.y);
        if (a.out_f32) *reinterpret_cast<float2 *>(a.out_f32 + row * a.d + e) = x;
    }
    if (a.lse && threadIdx.x == 0) a.lse[row] = empty ? -INFINITY : (M + log2f(L)) * 0.693147180559945309f;
}

namespace {

struct PrefixLayout {
    size_t plan, p_state, p_ml, o_state, o_ml, w_state, w_ml, bytes;
    long long p_slots, o_slots, w_slots;
    int wide_blocks;                         // of the wide kernel; 0: the mean group is too small for it
    int nsub, blocks, max_runs;              // blocks that fit the GPU; runs of the largest call
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
    if (batch < 1 || groups < 0 || batch + 2LL * groups > kPaMaxEntries || kv_heads < 1 || n_heads < kv_heads || n_heads % kv_heads ||
        n_heads / kv_heads > 64 || head_dim < 2 || head_dim % 2 || head_dim > ADSA_MAX_HEAD_DIM)
        return false;
    const int per_kv = n_heads / kv_heads;
    o->nsub = (head_dim + 63) / 64;
    o->blocks = sm_count() * (o->nsub <= 2 ? 2 : 1);
    o->max_runs = 5 * o->blocks;
    o->wide_blocks = groups && o->nsub <= 2 && (long long)batch * per_kv > (long long)kWideAbove * groups ? sm_count() : 0;
    o->w_slots = o->wide_blocks ? ((long long)batch * per_kv / kWideQueries + groups) * kv_heads + o->wide_blocks : 0;
    const auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
    o->p_slots = groups ? ((long long)batch * per_kv / kPaQueries + groups) * kv_heads + o->max_runs : 0;
    o->o_slots = (long long)batch * kv_heads * query_items(per_kv) + o->max_runs;
    const size_t dp = 64 * o->nsub, p_rows = (size_t)o->p_slots * kPaQueries, o_rows = (size_t)o->o_slots * own_slot_rows(per_kv);
    if (o->p_slots > 0x7fffffffLL || o->o_slots > 0x7fffffffLL || (long long)batch * n_heads > 0x7fffffffLL) return false;
    o->plan = 0;
    o->p_state = o->plan + up((size_t)batch * 48);
    o->p_ml = o->p_state + up(p_rows * dp * 4);
    o->o_state = o->p_ml + up(p_rows * 8);
    o->o_ml = o->o_state + up(o_rows * dp * 4);
    o->w_state = o->o_ml + up(o_rows * 8);
    o->w_ml = o->w_state + up((size_t)o->w_slots * kWideQueries * dp * 4);
    o->bytes = o->w_ml + up((size_t)o->w_slots * kWideQueries * 8);
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

template <typename T, int NSUB, int STAGES, bool PACKED>
cudaError_t launch_prefix(const PrefixArgs &a, unsigned runs, bool direct, const CUtensorMap &km, const CUtensorMap &vm, cudaStream_t st)
{
    const size_t tiles = 1024 + (size_t)STAGES * 2 * NSUB * tile_rows(NSUB) * 128, plan = (size_t)(2 * a.batch + 4 * a.groups + 2) * 4;
    static int told[3][64];
    if (direct) {
        const auto blocks = prefix_sweep_kernel<T, NSUB, STAGES, PACKED, kModeBlocks>, clusters = prefix_sweep_kernel<T, NSUB, STAGES, PACKED, kModeClusters>;
        const auto kern = a.split > 1 ? clusters : blocks;
        const cudaError_t e = allow_smem((const void *)kern, told[a.split > 1 ? 1 : 0]);
        const unsigned grid = (unsigned)(a.batch * a.kv_heads * query_items(a.per_kv) * a.split);
        return e != cudaSuccess ? e : launch_pdl_cluster(kern, dim3(grid), (unsigned)a.split, kPaThreads, tiles, st, a, km, vm);
    }
    const auto kern = prefix_sweep_kernel<T, NSUB, STAGES, PACKED, kModeList>;
    cudaError_t e = allow_smem((const void *)kern, told[2]);
    if (e != cudaSuccess) return e;
    e = launch_pdl(kern, dim3(runs), kPaThreads, tiles + plan, st, a, km, vm);
    if (e != cudaSuccess) return e;
    return launch_pdl(prefix_merge_kernel<T, NSUB>, dim3((unsigned)(a.batch * a.kv_heads * a.per_kv)), kPaMergeThreads, 0, st, a);
}

template <typename T>
cudaError_t launch_prefix_type(int nsub, const PrefixArgs &a, unsigned runs, bool direct, const CUtensorMap &km, const CUtensorMap &vm, cudaStream_t st)
{
    // 96 KB of tiles in flight per block and two blocks per SM; wide rows: 192 KB and one block
    const bool packed = a.row_stride / 8 % 2 != 0 && a.row_stride <= 64 * nsub;   // (a stage holds rows of 64 nsub elements)
#define ADSA_PREFIX(NSUB, STAGES) \
    return packed ? launch_prefix<T, NSUB, STAGES, true>(a, runs, direct, km, vm, st) : launch_prefix<T, NSUB, STAGES, false>(a, runs, direct, km, vm, st)
    switch (nsub) {
    case 1: ADSA_PREFIX(1, 3);
    case 2: ADSA_PREFIX(2, 3);
    case 3: ADSA_PREFIX(3, 4);
    default: ADSA_PREFIX(4, 3);
    }
#undef ADSA_PREFIX
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
    if (((uintptr_t)q & 3) || q_row % 2 || q_head % 2 || ((uintptr_t)workspace & 255) || ((uintptr_t)out & 3) || ((uintptr_t)out_f32 & 7)) return ADSA_EINVAL;
    if (((uintptr_t)page_table | (uintptr_t)n_rows | (uintptr_t)prefix_table | (uintptr_t)prefix_rows | (uintptr_t)group_start |
         (uintptr_t)lse | (uintptr_t)status) & 3)
        return ADSA_EINVAL;
    if ((long long)max_pages * kv->page_rows > kPaMaxRows || (long long)max_prefix_pages * kv->page_rows > kPaMaxRows) return ADSA_EINVAL;
    // the units of a call are counted in 32 bits
    const double own_units = (double)batch * kv->n_kv_heads * 2 * ((double)max_pages * kv->page_rows / tile_rows(l.nsub) + 1);
    const double p_units = ((double)batch * (n_heads / kv->n_kv_heads) / kPaQueries + n_groups) * kv->n_kv_heads *
                           ((double)max_prefix_pages * kv->page_rows / tile_rows(l.nsub) + 1);
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
    a.d = kv->head_dim; a.row_stride = kv->row_stride; a.k_pool = kv->k_pool; a.v_pool = kv->v_pool;
    const float scale = softmax_scale == 0.f ? 1.0f / sqrtf((float)kv->head_dim) : softmax_scale;
    a.scale_log2e = scale * 1.44269504088896341f;
    a.out = out; a.out_f32 = out_f32; a.lse = lse;
    a.plan = (uint4 *)(ws + l.plan);
    a.p_state = (float *)(ws + l.p_state); a.p_ml = (float *)(ws + l.p_ml);
    a.o_state = (float *)(ws + l.o_state); a.o_ml = (float *)(ws + l.o_ml);
    a.n_p_slots = (int)l.p_slots; a.n_o_slots = (int)l.o_slots;
    const double row_bytes = (double)kv->page_rows * l.nsub * 256;
    const double prefix_bytes = n_groups ? max_prefix_pages * row_bytes : 0.0;
    const long long items = (long long)batch * kv->n_kv_heads * query_items(a.per_kv);
    const double most = max_pages * row_bytes + prefix_bytes;
    const bool direct = direct_pays(items, l.blocks, a.per_kv, most, prefix_bytes * (1.0 - fmin(1.0, (double)n_groups / batch)));
    a.split = direct ? direct_split(items, l.blocks, most) : 1;
    const bool wide = !direct && l.wide_blocks && (long long)max_prefix_pages * kv->page_rows * l.nsub >= kWideRows;
    a.wide_above = wide ? kWideAbove : 0x7fffffff;
    a.w_state = (float *)(ws + l.w_state); a.w_ml = (float *)(ws + l.w_ml);
    a.n_w_slots = (int)l.w_slots; a.w_resident = wide ? l.wide_blocks : 0; a.resident = l.blocks;

    // as many blocks as there can be runs, and no more than there can be units
    const double units = own_units + (n_groups ? p_units : 0);
    const unsigned runs = units < l.max_runs ? (unsigned)units : (unsigned)l.max_runs;
    cudaStream_t st = (cudaStream_t)stream;
    if (a.w_resident && launch_prefix_wide(kv->dtype, l.nsub, a, km, vm, st) != cudaSuccess) return ADSA_ECUDA;
    const cudaError_t e = kv->dtype == ADSA_BF16 ? launch_prefix_type<__nv_bfloat16>(l.nsub, a, runs, direct, km, vm, st)
                                                  : launch_prefix_type<__half>(l.nsub, a, runs, direct, km, vm, st);
    return e == cudaSuccess ? ADSA_OK : ADSA_ECUDA;
}

}  // extern "C"
