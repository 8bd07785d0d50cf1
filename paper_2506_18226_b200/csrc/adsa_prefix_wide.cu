// The prefix of a large group: many query rows per key head against one long run of cached rows, which is a real matrix
// product, on the fifth-generation tensor cores.
//
// A block (one per SM) has two groups of four warps, a query row per thread, with a 128-row tile of Q, 128 tensor-memory
// columns of scores and up to 128 of O each.  Per tile of 128 cached rows and group: S = Q K^T (tcgen05, 128 x 128, operands
// in shared memory), softmax weights by the group's threads (row maxima and sums need no exchange between threads), P
// written back over S in tensor memory as 16-bit values, a hi and a lo part (split_weights) over 64 columns each, O += P V for both
// (tcgen05, P as the tensor-memory operand, V as it lies: rows of K, elements contiguous).  One warp copies (TMA) and one thread
// issues all products, so that one group's products run under the other's softmax.  An item is 256 query rows of a key head: both
// groups take every tile of K and V, each with its own 128 rows, so a tile is fetched once for 256 rows; the last 128 or fewer
// rows of a group are an item whose tiles the two groups take in turns.
//
// 256 rows x 8 key heads of 128: every further 32768 cached rows (34 GFLOP, 52 with the lo parts' products) take 38 us, 1.4
// PFLOP/s of products done; the launch for 32768 rows takes 52 us by itself, first tiles and the states at the end included.  What
// bounds an iteration (128 cached rows, both groups: 2.7 us, of which the products keep the tensor cores busy for 1.7) is a
// group's own chain: its softmax, of which 0.5 us are exponentials, then its products and what wakes them.  (Weights of one
// 16-bit value: 27 us, 46 for the launch; of the difference the lo parts' products are half, making and storing them the rest.)
// Descriptors have to stay in uniform registers: built by `lane == 0` in ordinary ones, an iteration took a third longer.
//
// The running maximum of a row only moves when a tile exceeds it by more than 8 (in log2 units); until then weights up to
// 2^8 are allowed, sums and products stay exact multiples, and O in tensor memory is rarely rescaled.
#include <type_traits>

#include "adsa_prefix.cuh"

namespace adsa {

constexpr int kWideThreads = 320;           // warps 0 .. 3, 4 .. 7: the groups; warp 8 copies; warp 9 issues the products
constexpr int kWideColumns = 512;           // all of tensor memory: S (and P) of the groups at 0 and 128, O at 256 and 384
constexpr float kWideSlack = 8.f;

// ---- tcgen05 ----------------------------------------------------------------------------------------------------------
__device__ __forceinline__ void tc_alloc(uint32_t slot, uint32_t columns)
{
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(slot), "r"(columns) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
}
__device__ __forceinline__ void tc_dealloc(uint32_t at, uint32_t columns)
{
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(at), "r"(columns) : "memory");
}
__device__ __forceinline__ void tc_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void tc_commit(uint32_t bar)
{
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}
// both operands in shared memory
__device__ __forceinline__ void tc_mma_ss(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n\t}"
                 ::"r"(d), "l"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// A in tensor memory
__device__ __forceinline__ void tc_mma_ts(uint32_t d, uint32_t a, uint64_t b, uint32_t idesc, uint32_t accumulate)
{
    asm volatile("{\n\t.reg .pred p;\n\tsetp.ne.u32 p, %4, 0;\n\ttcgen05.mma.cta_group::1.kind::f16 [%0], [%1], %2, %3, p;\n\t}"
                 ::"r"(d), "r"(a), "l"(b), "r"(idesc), "r"(accumulate) : "memory");
}
// 32 columns of the warp's 32 rows: one row per lane
__device__ __forceinline__ void tc_load32(uint32_t at, float (&v)[32])
{
    uint32_t *r = reinterpret_cast<uint32_t *>(v);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16,%17,%18,%19,%20,%21,%22,%23,"
                 "%24,%25,%26,%27,%28,%29,%30,%31}, [%32];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]),
                   "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]),
                   "=r"(r[31])
                 : "r"(at) : "memory");
}
__device__ __forceinline__ void tc_load_wait() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_store_wait() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tc_store16(uint32_t at, const uint32_t (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]),
                 "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
__device__ __forceinline__ void tc_store8(uint32_t at, const uint32_t (&r)[8])
{
    asm volatile("tcgen05.st.sync.aligned.32x32b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                 ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
}
__device__ __forceinline__ void tc_load16(uint32_t at, float (&v)[16])
{
    uint32_t *r = reinterpret_cast<uint32_t *>(v);
    asm volatile("tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(at) : "memory");
}
__device__ __forceinline__ void tc_store16f(uint32_t at, const float (&v)[16])
{
    tc_store16(at, *reinterpret_cast<const uint32_t (*)[16]>(v));
}

// one lane of the warp, in a form that leaves what it computes in uniform registers
__device__ __forceinline__ bool tc_elect()
{
    uint32_t one;
    asm volatile("{\n\t.reg .pred p;\n\telect.sync _|p, 0xffffffff;\n\tselp.u32 %0, 1, 0, p;\n\t}" : "=r"(one));
    return one != 0;
}

// Shared-memory operand of rows of 128 bytes in the 128-byte swizzle: start, stride between 64-element columns of the
// operand where it has several (only a transposed operand uses it), 1024 bytes between groups of eight rows.
__device__ __forceinline__ uint64_t tc_operand(uint32_t at, uint32_t column_stride)
{
    return (uint64_t)((at & 0x3ffffu) >> 4) | ((uint64_t)(column_stride >> 4) << 16) | ((uint64_t)(1024u >> 4) << 32) | (1ull << 46) | (2ull << 61);
}
// fp32 accumulator, 16-bit A and B of one type, M = 128; transposed: B's elements lie contiguous along N
template <typename T>
__device__ __forceinline__ uint32_t tc_shape(int n, bool transposed)
{
    const uint32_t type = std::is_same<T, __nv_bfloat16>::value ? 1u : 0u;
    return (1u << 4) | (type << 7) | (type << 10) | (transposed ? 1u << 16 : 0u) | ((uint32_t)(n >> 3) << 17) | ((uint32_t)(128 >> 4) << 24);
}

// Half-type weights carry a factor of 2^6 (up to 2^14 with the slack), so that small ones keep their precision.
template <typename T> struct WideBias { static constexpr float value = 0.f; };
template <> struct WideBias<__half> { static constexpr float value = 6.f; };

struct WideSegment {
    const int32_t *pages;
    int n, head, tile0, tiles, row0, rows, slot;
};

// Follows a run of units as the sweep of the smaller items does; entries are groups.  A tile of an item of more than 128
// query rows counts two units and belongs to the run that has its first.
struct WideWalk {
    const uint32_t *plan;
    uint32_t u, end;
    int e, run;
    __device__ void begin(const PrefixArgs &a, const uint32_t *plan_, int run_)
    {
        plan = plan_;
        run = run_;
        const WideCut cut(plan[a.groups], (uint32_t)a.w_resident);
        u = end = 0;
        if ((uint32_t)run < cut.runs) { u = cut.begin_of(run); end = cut.begin_of(run + 1); }
        e = 0;
    }
    __device__ bool next(const PrefixArgs &a, WideSegment &s)
    {
        while (u < end) {
            while (u >= plan[e + 1]) ++e;
            const uint32_t at = u - plan[e];
            const int b0 = group_begin(a, e), m = group_members(a, e) * a.per_kv;
            s.n = clamp_rows(a.p_rows[e], a.max_p_pages, a.page_rows);
            const WideItems w(m, s.n);
            s.head = (int)(at / w.head_units);
            const uint32_t in = at - (uint32_t)s.head * w.head_units, q = min(in / (2u * w.tiles), (uint32_t)w.items - 1u);
            s.row0 = b0 * a.per_kv + (int)q * kWideQueries;
            s.rows = min(m - (int)q * kWideQueries, kWideQueries);
            s.pages = a.p_table + (size_t)e * a.max_p_pages;
            s.slot = first_group_item(a, e, b0, kWideQueries) + s.head * w.items + (int)q + run;
            const uint32_t cost = s.rows > 128 ? 2u : 1u, first = in - q * 2u * w.tiles;   // units of a tile; first unit in the item
            const uint32_t last = min(first + (end - u), cost * w.tiles);
            s.tile0 = (int)((first + cost - 1u) / cost);
            s.tiles = (int)((last + cost - 1u) / cost) - s.tile0;
            u += last - first;
            if (s.tiles > 0) return true;
        }
        return false;
    }
};

// SLOTS: K or V tiles in shared memory
template <typename T, int NSUB, int SLOTS>
__global__ void __launch_bounds__(kWideThreads, 1)
prefix_wide_kernel(const __grid_constant__ PrefixArgs a, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map)
{
    constexpr int DP = 64 * NSUB;
    constexpr uint32_t kSub = kWideTile * 128, kTile = NSUB * kSub;   // bytes of a 64-element column of a tile, of a tile
    constexpr float kBias = WideBias<T>::value;
    extern __shared__ unsigned char wide_smem[];
    __shared__ uint64_t bars[2 * SLOTS + 8];
    __shared__ uint32_t s_tmem;
    const uint32_t base = (smem_u32(wide_smem) + 1023u) & ~1023u;
    const uint32_t q_at = base, ring = base + 2 * kTile;
    uint32_t *plan = reinterpret_cast<uint32_t *>(wide_smem + (base - smem_u32(wide_smem)) + (size_t)(2 + SLOTS) * kTile);
    const uint32_t full = smem_u32(bars), empty = full + 8 * SLOTS, q_full = empty + 8 * SLOTS, s_full = q_full + 16, p_full = s_full + 16;
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);   // (known to be uniform)

    if (tid == 0) {
        for (int i = 0; i < SLOTS; ++i) { mbar_init(full + 8 * i, 1); mbar_init(empty + 8 * i, 1); }
        for (int g = 0; g < 2; ++g) { mbar_init(q_full + 8 * g, 4); mbar_init(s_full + 8 * g, 1); mbar_init(p_full + 16 * g, 4); mbar_init(p_full + 16 * g + 8, 4); }
        mbar_init_fence();
        asm volatile("prefetch.tensormap [%0];" ::"l"(&k_map) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&v_map) : "memory");
    }
    // The order of these two carries the sweep behind this kernel: it begins as soon as every block here has passed them, and reads
    // tables, queries and rows and writes its states without a wait of its own, on the strength of this one.
    pdl_wait();
    pdl_launch();
    if (warp == 9) tc_alloc(smem_u32(&s_tmem), kWideColumns);
    // first unit of every group: one warp, 32 groups at a time
    if (warp == 8) {
        uint32_t before = 0;
        bool falls = false;
        for (int g0 = 0; g0 < a.groups; g0 += 32) {
            const int g = g0 + lane;
            uint32_t w = 0;
            if (g < a.groups) {
                falls = falls || a.start[g] > a.start[g + 1];
                const int m = group_members(a, g) * a.per_kv;
                if (m > a.wide_above) w = WideItems(m, clamp_rows(a.p_rows[g], a.max_p_pages, a.page_rows)).head_units * (uint32_t)a.kv_heads;
            }
            uint32_t incl = w;
#pragma unroll
            for (int o = 1; o < 32; o <<= 1) { const uint32_t t = __shfl_up_sync(0xffffffffu, incl, o); if (lane >= o) incl += t; }
            if (g < a.groups) plan[g] = before + incl - w;
            before += __shfl_sync(0xffffffffu, incl, 31);
        }
        if (lane == 0) plan[a.groups] = before;
        if (__any_sync(0xffffffffu, falls)) {                      // (boundaries that do not ascend: no groups, as in the sweep)
            __syncwarp();
            for (int g = lane; g <= a.groups; g += 32) plan[g] = 0;
        }
    }
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, s_tmem, 0);

    WideWalk walk;
    walk.begin(a, plan, blockIdx.x);
    WideSegment s = {};
    int limit = kCopySpinLimit;
    const auto wait = [&](uint32_t bar, uint32_t parity) {
        if (!mbar_wait_bounded(bar, parity, limit)) {
            limit = kCopySpinAfterTimeout;
            if (a.status && lane == 0) atomicOr(a.status, ADSA_DEV_COPY_TIMEOUT);
        }
    };

    if (warp == 8) {                                               // ---- copies ----
        int slot = 0;
        uint32_t phase = 0;
        const auto copy = [&](int t, bool value) {                 // K or V of tile t into the next slot
            const int rows = min(kWideTile, s.n - t * kWideTile), boxes = (rows + a.box_rows - 1) / a.box_rows;
            wait(empty + 8 * slot, phase ^ 1u);
            if (lane == 0) mbar_expect_tx(full + 8 * slot, (uint32_t)(boxes * a.box_rows) * 128u * NSUB);
            __syncwarp();
            for (int i = lane; i < boxes; i += 32) {
                const int row = t * kWideTile + i * a.box_rows, pg = row / a.page_rows;
                int page = s.pages[pg];
                if (page < 0 || page >= a.n_pages) {               // (the group's result is then unspecified)
                    page = 0;
                    if (a.status) atomicOr(a.status, ADSA_DEV_BAD_PAGE);
                }
                const int y = (page * a.kv_heads + s.head) * a.page_rows + row - pg * a.page_rows;
                const uint32_t dst = ring + (uint32_t)slot * kTile + (uint32_t)(i * a.box_rows) * 128u;
#pragma unroll
                for (int c = 0; c < NSUB; ++c) pa_tma(dst + c * kSub, value ? &v_map : &k_map, c * 64, y, full + 8 * slot);
            }
            if (++slot == SLOTS) { slot = 0; phase ^= 1u; }
        };
        // in the order the products take them: K0 V0 K1 V1 .. where both groups share a tile, else K0 K1 V0 K2 V1 K3 ..
        while (walk.next(a, s)) {
            const int ahead = s.rows > 128 ? 1 : 2, end = s.tile0 + s.tiles;
            for (int t = s.tile0; t < min(s.tile0 + ahead, end); ++t) copy(t, false);
            for (int t = s.tile0; t < end; ++t) {
                copy(t, true);
                if (t + ahead < end) copy(t + ahead, false);
            }
        }
    } else if (warp == 9) {                                        // ---- products ----
        const int k_steps = (a.d + 15) / 16, d_cols = k_steps * 16;
        const uint32_t s_shape = tc_shape<T>(kWideTile, false), o_shape = tc_shape<T>(d_cols, true);
        int slot = 0, valid = 0;
        uint32_t phase = 0, q_phase[2] = {0, 0}, p_phase[2] = {0, 0};
        const auto take = [&]() {                                  // the next slot, once its tile is there
            wait(full + 8 * slot, phase);
            const int taken = slot;
            if (++slot == SLOTS) { slot = 0; phase ^= 1u; }
            return taken;
        };
        const auto score = [&](int g, int k_slot, uint32_t q) {    // S = Q K^T
            const uint64_t qd = tc_operand(q, 16), kd = tc_operand(ring + (uint32_t)k_slot * kTile, 16);
            if (tc_elect()) {
#pragma unroll
                for (int ks = 0; ks < 4 * NSUB; ++ks) {
                    const uint64_t off = ((uint32_t)(ks >> 2) * kSub + (uint32_t)(ks & 3) * 32u) >> 4;
                    if (ks < k_steps) tc_mma_ss(tmem + g * 128, qd + off, kd + off, s_shape, ks > 0);
                }
            }
        };
        const auto take_v = [&](int t) {                           // V of tile t
            const int taken = take();
            valid = s.n - t * kWideTile;
            if (valid < kWideTile) {
                // rows behind the end hold anything, and a weight of zero does not silence an infinity or a NaN
                const uint32_t v_at = ring + (uint32_t)taken * kTile;
                for (int i = lane; i < (kWideTile - valid) * 8 * NSUB; i += 32) {
                    const int r = valid + i / (8 * NSUB), ch = i % (8 * NSUB);
                    asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(v_at + (ch >> 3) * kSub + r * 128 + (ch & 7) * 16), "r"(0u) : "memory");
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
            }
            return taken;
        };
        const auto weigh = [&](int g, int v_slot, bool first) {    // O += P V, once the group has left P
            const uint64_t vd = tc_operand(ring + (uint32_t)v_slot * kTile, kSub);
#pragma unroll
            for (int half = 0; half < 2; ++half) {                 // P comes in two halves: the first is used while the second is made
                wait(p_full + 16 * g + 8 * half, p_phase[g]);
                tc_after();
                if (tc_elect()) {
#pragma unroll
                    for (int k = 0; k < kWideTile / 32; ++k) {
                        const int ks = half * (kWideTile / 32) + k;
                        tc_mma_ts(tmem + 256 + g * 128, tmem + g * 128 + ks * 8, vd + (uint64_t)(ks * 128), o_shape, !first || ks > 0);
                        tc_mma_ts(tmem + 256 + g * 128, tmem + g * 128 + 64 + ks * 8, vd + (uint64_t)(ks * 128), o_shape, 1u);
                    }
                }
                __syncwarp();
            }
            p_phase[g] ^= 1u;
        };
        const auto done = [&](uint32_t bar) {                      // counted when everything issued so far is complete
            if (tc_elect()) tc_commit(bar);
            __syncwarp();
        };
        while (walk.next(a, s)) {
            wait(q_full, q_phase[0]);
            q_phase[0] ^= 1u;
            if (s.rows > 128) {
                wait(q_full + 8, q_phase[1]);
                q_phase[1] ^= 1u;
            }
            tc_after();
            const int T_ = s.tiles;
            if (s.rows > 128) {
                int k = take();
                score(0, k, q_at);
                done(s_full);
                score(1, k, q_at + kTile);
                done(empty + 8 * k);
                done(s_full + 8);
                for (int i = 0; i < T_; ++i) {
                    const int v = take_v(s.tile0 + i);
                    const bool more = i + 1 < T_;
                    weigh(0, v, i == 0);
                    if (more) { k = take(); score(0, k, q_at); }
                    done(s_full);                                  // the next scores, or O is whole
                    weigh(1, v, i == 0);
                    done(empty + 8 * v);
                    if (more) { score(1, k, q_at + kTile); done(empty + 8 * k); }
                    done(s_full + 8);
                }
            } else {
                for (int g = 0; g < min(2, T_); ++g) {
                    const int k = take();
                    score(g, k, q_at);
                    done(empty + 8 * k);
                    done(s_full + 8 * g);
                }
                for (int i = 0; i < T_; ++i) {
                    const int g = i & 1, v = take_v(s.tile0 + i);
                    weigh(g, v, i < 2);
                    done(empty + 8 * v);
                    if (i + 2 < T_) {
                        const int k = take();
                        score(g, k, q_at);
                        done(empty + 8 * k);
                    }
                    done(s_full + 8 * g);
                }
            }
        }
    } else {                                                       // ---- a query row per thread ----
        const int g = warp >> 2, row = tid & 127;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, s_col = tmem + g * 128 + lanes, o_col = tmem + 256 + g * 128 + lanes;
        const uint32_t my_s = s_full + 8 * g, my_p = p_full + 16 * g;
        const bool wide_q = a.d % 8 == 0 && (((uintptr_t)a.q | (uintptr_t)(a.q_row * 2) | (uintptr_t)(a.q_head * 2)) & 15) == 0;
        uint32_t s_phase = 0;
        while (walk.next(a, s)) {
            const bool both = s.rows > 128;                        // both groups take every tile, else in turns
            const int r = both ? g * 128 + row : row;              // query row of the item
            const bool there = r < s.rows;
            const int step = both ? 1 : 2, t0 = s.tile0 + (both ? 0 : g), tiles = both ? s.tiles : (s.tiles + 1 - g) / 2;
            if (both || g == 0) {
                // the row of Q into shared memory, zero beyond the head elements and the group's rows; asked for at once
                const int packed = s.row0 + r, b = packed / a.per_kv, j = packed - b * a.per_kv;
                const T *qp = (const T *)a.q + b * a.q_row + (s.head * a.per_kv + j) * a.q_head;
                const uint32_t at = q_at + g * kTile;
                uint4 w[8 * NSUB];
                if (wide_q) {
#pragma unroll
                    for (int ch = 0; ch < 8 * NSUB; ++ch)
                        w[ch] = there && ch * 8 < a.d ? __ldg(reinterpret_cast<const uint4 *>(qp + ch * 8)) : make_uint4(0u, 0u, 0u, 0u);
                } else {
#pragma unroll
                    for (int ch = 0; ch < 8 * NSUB; ++ch) {
                        uint32_t *p = reinterpret_cast<uint32_t *>(&w[ch]);
#pragma unroll
                        for (int i = 0; i < 4; ++i) {
                            const int e = ch * 8 + 2 * i;
                            p[i] = there && e < a.d ? __ldg(reinterpret_cast<const uint32_t *>(qp + e)) : 0u;
                        }
                    }
                }
#pragma unroll
                for (int ch = 0; ch < 8 * NSUB; ++ch)
                    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};"
                                 ::"r"(at + (uint32_t)(ch >> 3) * kSub + (uint32_t)row * 128u + (uint32_t)(((ch & 7) ^ (row & 7)) << 4)),
                                 "r"(w[ch].x), "r"(w[ch].y), "r"(w[ch].z), "r"(w[ch].w) : "memory");
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                tc_before();
                __syncwarp();
                // (a group that has no Q to load must not arrive: with no tile either it may be an item ahead)
                if (lane == 0) mbar_arrive(q_full + 8 * g);
            }
            float m = -INFINITY;                                   // raw units; the row's weights are relative to it
            float2 l2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
            for (int i = 0; i < tiles; ++i) {
                const int valid = s.n - (t0 + i * step) * kWideTile;   // cached rows of the tile
                wait(my_s, s_phase);
                s_phase ^= 1u;
                tc_after();
                float v[kWideTile];
#pragma unroll
                for (int c = 0; c < kWideTile; c += 32) tc_load32(s_col + c, *reinterpret_cast<float (*)[32]>(v + c));
                tc_load_wait();
                if (valid < kWideTile) {
#pragma unroll
                    for (int c = 0; c < kWideTile; ++c) v[c] = c < valid ? v[c] : -INFINITY;
                }
                float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int c = 0; c < kWideTile; ++c) mx4[c & 3] = fmaxf(mx4[c & 3], v[c]);
                const float mx = fmaxf(fmaxf(mx4[0], mx4[1]), fmaxf(mx4[2], mx4[3]));
                const bool move = (mx - m) * a.scale_log2e > kWideSlack || m == -INFINITY;
                if (__any_sync(0xffffffffu, move)) {
                    const float m_new = move ? fmaxf(m, mx) : m;
                    const float corr = m_new == -INFINITY || m == -INFINITY ? (m == m_new ? 1.f : 0.f) : pa_exp2((m - m_new) * a.scale_log2e);
                    m = m_new;
#pragma unroll
                    for (int k = 0; k < 2; ++k) { l2[k].x *= corr; l2[k].y *= corr; }
                    if (i > 0) {                                   // the products before this tile's are complete: their S is
#pragma unroll 1
                        for (int c = 0; c < DP; c += 16) {
                            float x[16];
                            tc_load16(o_col + c, x);
                            tc_load_wait();
#pragma unroll
                            for (int k = 0; k < 16; ++k) x[k] *= corr;
                            tc_store16f(o_col + c, x);
                        }
                    }
                }
                const float shift = kBias - (m == -INFINITY ? 0.f : m) * a.scale_log2e;
                const float2 scale2 = make_float2(a.scale_log2e, a.scale_log2e), shift2 = make_float2(shift, shift);
#pragma unroll
                for (int c = 0; c < kWideTile; c += 16) {
                    uint32_t p[8], p_lo[8];
#pragma unroll
                    for (int k = 0; k < 8; ++k) {
                        float2 x = fma2(make_float2(v[c + 2 * k], v[c + 2 * k + 1]), scale2, shift2);
                        x.x = pa_exp2(x.x);
                        x.y = pa_exp2(x.y);
                        l2[k & 1] = add2(l2[k & 1], x);            // the sum takes the weights before they are rounded
                        split_weights<T>(x, p[k], p_lo[k]);
                    }
                    tc_store8(s_col + c / 2, p);                   // over scores that are in registers by now
                    tc_store8(s_col + 64 + c / 2, p_lo);
                    if (c % 64 == 48) {
                        tc_store_wait();
                        tc_before();
                        __syncwarp();
                        if (lane == 0) mbar_arrive(my_p + 8 * (c / 64));
                    }
                }
            }
            if (tiles > 0) {
                wait(my_s, s_phase);
                s_phase ^= 1u;
                tc_after();
            }
            const bool fits = s.slot < a.n_w_slots;
            if (!fits && a.status && lane == 0) atomicOr(a.status, ADSA_DEV_BAD_GROUPS);
            const size_t at = (size_t)s.slot * kWideQueries + (both ? r : g * 128 + row);
            if (fits && there)                                     // (no tile: an empty state)
                *reinterpret_cast<float2 *>(a.w_ml + 2 * at) = make_float2(m * a.scale_log2e - kBias, l2[0].x + l2[0].y + l2[1].x + l2[1].y);
            if (tiles > 0) {
#pragma unroll 1
                for (int c = 0; c < DP; c += 32) {
                    float v[32];
                    tc_load32(o_col + c, v);
                    tc_load_wait();
                    if (fits && there) {
#pragma unroll
                        for (int i = 0; i < 32; i += 8)            // whole 32-byte sectors: a lane's neighbours write other rows
                            asm volatile("st.global.v8.f32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                                         ::"l"(a.w_state + at * DP + c + i), "f"(v[i]), "f"(v[i + 1]), "f"(v[i + 2]), "f"(v[i + 3]), "f"(v[i + 4]),
                                         "f"(v[i + 5]), "f"(v[i + 6]), "f"(v[i + 7]) : "memory");
                    }
                }
            }
            tc_before();                                           // read before the next item's products write O
        }
    }
    tc_before();
    __syncthreads();
    if (warp == 9) {
        tc_after();
        tc_dealloc(tmem, kWideColumns);
    }
}

namespace {

template <typename T, int NSUB, int SLOTS>
cudaError_t launch_wide(const PrefixArgs &a, const CUtensorMap &km, const CUtensorMap &vm, cudaStream_t st)
{
    const size_t smem = 1024 + (size_t)(2 + SLOTS) * NSUB * kWideTile * 128 + (size_t)(a.groups + 1) * 4;
    const auto kern = prefix_wide_kernel<T, NSUB, SLOTS>;
    static int told[64];
    const cudaError_t e = allow_smem((const void *)kern, told);
    if (e != cudaSuccess) return e;
    return launch_pdl(kern, dim3((unsigned)a.w_resident), kWideThreads, smem, st, a, km, vm);
}

template <typename T>
cudaError_t launch_wide_type(int nsub, const PrefixArgs &a, const CUtensorMap &km, const CUtensorMap &vm, cudaStream_t st)
{
    if (nsub == 1) return launch_wide<T, 1, 8>(a, km, vm, st);
    // 224 KB of Q and tiles leave room for the plan of some 400 groups
    return a.groups <= 256 ? launch_wide<T, 2, 5>(a, km, vm, st) : launch_wide<T, 2, 4>(a, km, vm, st);
}

}  // namespace

cudaError_t launch_prefix_wide(int dtype, int nsub, const PrefixArgs &a, const CUtensorMap &km, const CUtensorMap &vm, cudaStream_t st)
{
    return dtype == ADSA_BF16 ? launch_wide_type<__nv_bfloat16>(nsub, a, km, vm, st) : launch_wide_type<__half>(nsub, a, km, vm, st);
}

}  // namespace adsa
