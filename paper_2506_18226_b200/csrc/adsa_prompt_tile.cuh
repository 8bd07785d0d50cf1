// What the tile kernels of the prompt attention share: the list of items cut into one run per block, the warp that walks a run, waits
// and copies.
#pragma once

#include "adsa_prompt.cuh"
#include "adsa_tc.cuh"

namespace adsa {

constexpr int kTileThreads = 384;           // warps 0 .. 3, 4 .. 7: two groups; 8 copies K and V; 9 issues the products; 10 copies Q; 11 walks
constexpr int kTileColumns = 512;           // all of tensor memory: S (and P) of the groups at 0 and 128, O at 256 and 384
constexpr float kTileSlack = 8.f;
constexpr int kTileRing = 4;                // items ahead
constexpr int kTileSeqs = 64;                // sequences that are kept in shared memory, read once
constexpr int kFewRows = 32;                // query rows of an item of the kernel for few rows
constexpr unsigned kTileMinRun = 12;        // units of a run, at least, where items may be cut

struct TileDesc {                           // an item of a run, as the walking warp finds it
    PromptSeq s;
    int b, head, q;
    int t0, t1;                             // tiles of this run; t1 < 0: no more items
    int slot;                               // of the partial state; -1: the whole item
};
struct TilePos {
    int b, head, q, tile;
    __device__ __forceinline__ bool before(const TilePos &o) const
    {
        if (b != o.b) return b < o.b;
        if (head != o.head) return head < o.head;
        return q != o.q ? q < o.q : tile < o.tile;
    }
};
template <bool WIDE>
__device__ __forceinline__ TilePos next_pos(const PromptArgs &a, const PromptSeq &s, TilePos pos)
{
    pos.tile = 0;
    if (++pos.q * item_tokens<WIDE>(a) < s.m) return pos;
    pos.q = 0;
    if (s.m == 0 || ++pos.head >= a.kv_heads) { pos.head = 0; ++pos.b; }
    return pos;
}
__device__ __forceinline__ void tile_tma3(uint32_t dst, const CUtensorMap *map, int x, int y, int z, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.3d.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];"
                 ::"r"(dst), "l"(map), "r"(x), "r"(y), "r"(z), "r"(bar) : "memory");
}

// Bounded waits of a block.  One that runs out says so in gave_up, and the block's later ones run out at their first poll.  What the block does from then on
// stays inside its buffers, but works on what happens to be there: no copy begins without its slot, no item is taken, nothing is written to the outputs or
// the states, the merge leaves out items with a part of this block, and the status says so.
struct TileWaits {
    int limit, gave_up;                     // polls; 0 or 1
};
__device__ __forceinline__ bool tile_wait(TileWaits &w, uint32_t bar, uint32_t parity)
{
    for (int polls = 0; !mbar_try_wait(bar, parity); ++polls) {
        if (polls < *(volatile int *)&w.limit) continue;
        *(volatile int *)&w.gave_up = 1;
        *(volatile int *)&w.limit = 0;
        return false;
    }
    return true;
}
// the same for a whole warp, which goes on as one
__device__ __forceinline__ bool tile_wait_warp(TileWaits &w, uint32_t bar, uint32_t parity)
{
    for (int polls = 0; !__all_sync(0xffffffffu, mbar_try_wait(bar, parity)); ++polls) {
        if (__all_sync(0xffffffffu, polls < *(volatile int *)&w.limit)) continue;
        *(volatile int *)&w.gave_up = 1;
        *(volatile int *)&w.limit = 0;
        return false;
    }
    return true;
}
__device__ __forceinline__ bool tile_gave_up(const TileWaits &w) { return *(const volatile int *)&w.gave_up != 0; }
// What is in flight when a block gives up has to land before it ends: n barriers, bit i of `flight` the parity that the last copy to barrier i
// completes; products: those of this warp, by barrier `bar`.  (Not inlined: no sound block runs it.)
static __device__ __noinline__ void tile_land(uint32_t bar, int n, uint32_t flight, bool products)
{
    if (products) {
        if (tc_elect()) tc_commit(bar);
        __syncwarp();
    }
    for (int i = 0; i < n; ++i) mbar_wait_bounded(bar + 8 * i, flight >> i & 1u, 1 << 12);   // (16 ms)
    __syncwarp();
}

template <int BYTES>
__device__ __forceinline__ void tile_copy(uint32_t dst, const void *src)
{
    if constexpr (BYTES == 16) asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
    else asm volatile("cp.async.ca.shared.global [%0], [%1], %2;" ::"r"(dst), "l"(src), "n"(BYTES) : "memory");
}
// where byte x of a row lies in a tile of 128-byte columns in the 128-byte swizzle
__device__ __forceinline__ uint32_t tile_at(int row, int x, uint32_t sub)
{
    return (uint32_t)(x >> 7) * sub + (uint32_t)row * 128u + (uint32_t)((((x >> 4) & 7) ^ (row & 7)) << 4) + (uint32_t)(x & 15);
}
__device__ __forceinline__ float tile_max3(float x, float y, float z)
{
    float m;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(x), "f"(y), "f"(z));
    return m;
}
// largest magnitude, or NaN if one of them is
__device__ __forceinline__ float tile_magnitude(float x, float y, float z)
{
    float m;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(m) : "f"(x), "f"(y), "f"(z));
    return m;
}
// largest of 16, 8, 4 bytes that divides all of these
__device__ __forceinline__ int piece_of(const void *p, long long token, long long head, int d)
{
    const unsigned long long x = (unsigned long long)(uintptr_t)p | (unsigned long long)(token * 2) | (unsigned long long)(head * 2) | (unsigned)(d * 2);
    return x & 7 ? 4 : x & 15 ? 8 : 16;
}

// The item that unit u of the list (of 2^shift units each) lies in, and the tile that a run beginning there takes first; by a whole warp.
template <bool WIDE>
__device__ TilePos tile_locate(const PromptArgs &a, const unsigned *plan, const PromptSeq *seqs, unsigned u, int shift, unsigned tol, int lane)
{
    if (u >= plan[a.batch]) return {a.batch, 0, 0, 0};
    int b = 0;
    for (int b0 = 0;; b0 += 32) {
        const int done = __popc(__ballot_sync(0xffffffffu, b0 + lane < a.batch && plan[b0 + lane + 1] <= u));
        b = b0 + done;
        if (done < 32) break;
    }
    const PromptSeq s = seqs ? seqs[b] : prompt_seq(a, b);
    // (bounded: where boundaries do not ascend, sums may stop inside this sequence, at the largest number)
    const unsigned per_head = max((plan[b + 1] - plan[b]) / (unsigned)a.kv_heads, 1u);
    unsigned rem = u - plan[b];
    const int head = (int)min(rem / per_head, (unsigned)a.kv_heads - 1u);
    rem = min(rem - head * per_head, per_head - 1u);
    for (int q0 = 0;; q0 += 32) {
        const bool in = (q0 + lane) * item_tokens<WIDE>(a) < s.m;
        const TileItem<WIDE> mine(a, s, in ? q0 + lane : 0);
        const unsigned cost = in ? mine.cost(shift) : 0u;
        unsigned incl = cost;
#pragma unroll
        for (int o = 1; o < 32; o <<= 1) { const unsigned t = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += t; }
        const unsigned past = __ballot_sync(0xffffffffu, incl > rem);
        if (!past && (q0 + 32) * item_tokens<WIDE>(a) < s.m) {
            rem -= __shfl_sync(0xffffffffu, incl, 31);
            continue;
        }
        const int at = past ? __ffs(past) - 1 : 31;         // (past is never empty here: the plan counted the same items)
        const unsigned item_cost = __shfl_sync(0xffffffffu, cost, at), off = rem - (__shfl_sync(0xffffffffu, incl, at) - item_cost);
        const int tiles = __shfl_sync(0xffffffffu, mine.tiles, at);
        const bool two = __shfl_sync(0xffffffffu, mine.tile_cost(), at) == 2u;
        const unsigned left = item_cost - off;
        const bool near = min(off, left) <= tol;
        const unsigned inside = off << shift;
        int q = q0 + at, tile = near || inside <= kTileOver ? 0 : (int)(two ? (inside - kTileOver + 1u) / 2u : inside - kTileOver);
        if (near ? off <= left : tile < tiles || tiles == 0) return {b, head, q, tile};
        if (++q * item_tokens<WIDE>(a) < s.m) return {b, head, q, 0};
        return head + 1 < a.kv_heads ? TilePos{b, head + 1, 0, 0} : TilePos{b + 1, 0, 0, 0};
    }
}

// x + y, or the largest number
__device__ __forceinline__ unsigned tile_sum(unsigned x, unsigned y) { return x > ~y ? 0xffffffffu : x + y; }

// The list of the call's work, plan[b] units before sequence b, and where this block's run begins and ends; by all threads.  Units are counted in 32
// bits (the list lies in shared memory beside the tiles); a call of more, some half a minute's work, is counted again in units of 2^9, 2^18, 2^27, in
// which an item has one at least: a call has fewer than 2^31 items, but for sequences whose boundaries do not ascend and overlap (sums then stop at
// the largest number, and which rows are made is not specified).
template <bool WIDE>
__device__ __forceinline__ void tile_plan(const PromptArgs &a, unsigned *plan, PromptSeq *seqs, TilePos *ends, int warp, int lane)
{
    int shift = 0;
#pragma unroll 1
    for (;; shift += 9) {
        // units of every sequence: short ones by a lane each, long ones by their warp; then their running sum
        for (int b0 = warp * 32; b0 < a.batch; b0 += kTileThreads) {
            const int b = b0 + lane;
            PromptSeq s = {};
            if (b < a.batch) {
                s = prompt_seq(a, b);
                if (seqs) seqs[b] = s;
            }
            const bool many = s.m > 32 * item_tokens<WIDE>(a);
            unsigned units = 0;
            if (!many) {
                for (int q = 0; q * item_tokens<WIDE>(a) < s.m; ++q) units = tile_sum(units, TileItem<WIDE>(a, s, q).cost(shift));
            }
            for (unsigned todo = __ballot_sync(0xffffffffu, many); todo; todo &= todo - 1) {
                const int src = __ffs(todo) - 1;
                PromptSeq t = {};
                t.m = __shfl_sync(0xffffffffu, s.m, src);
                t.n = __shfl_sync(0xffffffffu, s.n, src);
                t.p = __shfl_sync(0xffffffffu, s.p, src);
                unsigned sum = 0;
                for (int q = lane; q * item_tokens<WIDE>(a) < t.m; q += 32) sum = tile_sum(sum, TileItem<WIDE>(a, t, q).cost(shift));
                const unsigned high = __reduce_add_sync(0xffffffffu, sum >> 16), low = __reduce_add_sync(0xffffffffu, sum & 0xffffu);
                sum = high > 0xffffu ? 0xffffffffu : tile_sum(high << 16, low);
                if (lane == src) units = sum;
            }
            if (b < a.batch) plan[b + 1] = __umulhi(units, (unsigned)a.kv_heads) ? 0xffffffffu : units * (unsigned)a.kv_heads;
        }
        __syncthreads();
        if (warp == 11) {
            if (lane == 0) plan[0] = 0;
            unsigned before = 0;
            for (int b0 = 0; b0 < a.batch; b0 += 32) {
                unsigned incl = b0 + lane < a.batch ? plan[b0 + lane + 1] : 0;
#pragma unroll
                for (int o = 1; o < 32; o <<= 1) { const unsigned t = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl = tile_sum(incl, t); }
                if (b0 + lane < a.batch) plan[b0 + lane + 1] = tile_sum(before, incl);
                before = tile_sum(before, __shfl_sync(0xffffffffu, incl, 31));
            }
        }
        __syncthreads();
        if (plan[a.batch] != 0xffffffffu || shift == 27) break;
        __syncthreads();                                               // (all have read it)
    }
    const unsigned total = plan[a.batch], runs = min(max(a.split ? total / kTileMinRun : total, 1u), gridDim.x);
    if (warp == 10 || warp == 11) {                                // where this block's run begins and ends
        const unsigned run = blockIdx.x + (warp - 10);
        const unsigned u = run > runs ? total : (unsigned)((unsigned long long)run * total / runs);
        const TilePos at = tile_locate<WIDE>(a, plan, seqs, u, shift, a.split ? total / runs / 32u : 0xffffffffu, lane);
        if (lane == 0) ends[warp - 10] = at;
    }
}

// The warp that walks a block's run and names its items to the others, a few ahead of them, unless the block has given up; desc: what the run leaves for the
// merge.
template <bool WIDE>
__device__ __forceinline__ void tile_walk(const PromptArgs &a, const PromptSeq *seqs, const TilePos *ends, TileDesc *ring, uint32_t d_full, uint32_t d_empty, int lane, TileWaits &waits,
                                          int4 *desc)
{
    int at = 0;
    uint32_t d_phase = 0;
    const unsigned run = blockIdx.x;
    int4 left = make_int4(-1, 0, 0, 0);                         // {sequence of the item that this run begins and leaves unfinished, key
                                                               // head, item; whether an item cut before ends here}
    int4 of = left;                                            // that sequence's first token, tokens, own rows, rows of the prefix
    const TilePos end = ends[1];
    TilePos pos = ends[0];
    int have = -1;
    bool going = true;
    PromptSeq s = {};
    const auto go_on = [&](uint32_t bar, uint32_t parity) { return tile_wait_warp(waits, bar, parity) && __all_sync(0xffffffffu, !tile_gave_up(waits)); };
    while (pos.before(end)) {
        if (pos.b != have) { s = seqs ? seqs[pos.b] : prompt_seq(a, pos.b); have = pos.b; }
        if (s.m == 0) { pos = next_pos<WIDE>(a, s, pos); continue; }
        const TileItem<WIDE> item(a, s, pos.q);
        const bool last = pos.b == end.b && pos.head == end.head && pos.q == end.q;
        const int t1 = last ? end.tile : item.tiles;
        const bool whole = pos.tile == 0 && t1 == item.tiles;
        if (!whole) {
            if (pos.tile > 0) left.w = t1 == item.tiles;
            else {
                left = make_int4(pos.b, pos.head, pos.q, left.w);
                of = make_int4((int)s.q0, s.m, s.n, s.p);
            }
        }
        going = go_on(d_empty + 8 * at, d_phase ^ 1u);
        if (!going) break;
        if (lane == 0) {
            ring[at] = {s, pos.b, pos.head, pos.q, pos.tile, t1, whole ? -1 : (int)(2 * run) + (pos.tile > 0 ? 0 : 1)};
            mbar_arrive(d_full + 8 * at);
        }
        if (++at == kTileRing) { at = 0; d_phase ^= 1u; }
        if (last) break;
        pos = next_pos<WIDE>(a, s, pos);
    }
    if (going && go_on(d_empty + 8 * at, d_phase ^ 1u) && lane == 0) {
        ring[at].t1 = -1;
        mbar_arrive(d_full + 8 * at);
    }
    if (lane == 0) {
        desc[0] = left;
        desc[1] = of;
    }
}

// One item's tiles of a paged cache or of packed rows, as the copying warp needs them, in registers.
struct TileSource {
    const int32_t *own, *pre;               // page tables
    int p, n, before, head, tok;            // rows of the prefix, own rows; tiles of the prefix; packed: token of the first own row
    __device__ __forceinline__ TileSource(const PromptArgs &a, const TileDesc &it)
        : own(a.table ? a.table + (size_t)it.b * a.max_pages : nullptr), pre(it.s.p ? a.p_table + (size_t)it.s.group * a.max_p_pages : nullptr), p(it.s.p),
          n(it.s.n), before((it.s.p + kTileRows - 1) / kTileRows), head(it.head), tok((int)it.s.k0) {}
    __device__ __forceinline__ int valid(int t) const { return min(t < before ? p - t * kTileRows : n - (t - before) * kTileRows, kTileRows); }
    __device__ __forceinline__ int row0(int t) const { return (t < before ? t : t - before) * kTileRows; }
    // row of the pool where box `box` of tile t begins; -1: the tile has no such box
    __device__ __forceinline__ int pool_row(const PromptArgs &a, int t, int box) const
    {
        if (!a.table || box << a.box_shift >= valid(t)) return -1;
        const int row = row0(t) + (box << a.box_shift), at = a.by_page(row);
        return (prompt_page(a, (t < before ? pre : own)[at]) * a.kv_heads + head) * a.page_rows + row - at * a.page_rows;
    }
    __device__ __forceinline__ uint32_t bytes(const PromptArgs &a, int t, uint32_t full) const   // that the boxes of tile t bring, of a tile's `full`
    {
        return a.table ? (uint32_t)((valid(t) + a.box_rows - 1) >> a.box_shift << a.box_shift) * (full / kTileRows) : full;
    }
};
// the list of the call's work: units before each sequence; the sequences, of few
inline size_t tile_list_bytes(int batch) { return (size_t)((batch + 2) & ~1) * 4 + (batch <= kTileSeqs ? (size_t)batch * sizeof(PromptSeq) : 0); }
// lets a kernel use `most` bytes of an SM's shared memory on the current device; asks the driver once per device
inline cudaError_t tile_allow_smem(const void *kernel, int (&told)[64], size_t most)
{
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const bool known = dev >= 0 && dev < 64;
    if (known && __atomic_load_n(&told[dev], __ATOMIC_ACQUIRE)) return cudaSuccess;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)most);
    if (e == cudaSuccess && known) __atomic_store_n(&told[dev], 1, __ATOMIC_RELEASE);
    return e;
}

cudaError_t launch_prompt_few(int dtype, const PromptArgs &a, unsigned blocks, const CUtensorMap &km, const CUtensorMap &vm, cudaStream_t st);

}  // namespace adsa
