// Attention of few query rows per sequence (single tokens, guesses to be checked, a row of a grid) over packed rows or a paged
// cache: what the tile kernel does, laid out for calls whose time is that of reading the cache.
//
// An item has up to 32 query rows of a key head.  They are spread over a 128-row tile of Q so that each of a group's four warps has
// 8 of them, and a warp takes its scores from tensor memory four lanes to a row: 32 exponentials a thread and tile for all 128 cached
// rows, on all four parts of an SM, where a row per thread takes 128 on as many parts as have rows.  The two groups
// take the tiles in turns, so that one's products run under the other's softmax, and join their states at the end.  Q takes half of what
// two halves take and outputs go straight to memory: the ring of tiles has the rest, 160 to 192 KB.
//
// 32 sequences of one token over 1144 rows of 20 heads of 64 (188 MB): 41 .. 45 us, 4.2 .. 4.6 TB/s of 6.5 measured; 8 x 5 tokens over up to 16384 rows of 8 key
// heads of 128 (302 MB): 61 .. 62 us, 4.9 TB/s.  Weights are rounded as the tile kernel rounds them.  What bounds: for long rows the memory; for short ones an item's fixed part, some 5000 clocks of first copies,
// joining and outputs, most of them waiting for instructions that run once per item (so this code is kept short).

#include "adsa_prompt_tile.cuh"

namespace adsa {

constexpr int kFewThreads = kTileThreads + 32;   // warp 8 copies K, warp 12 V: one warp for both, at 700 clocks a copy, was what bounded

struct FewControl {
    uint64_t bars[48];
    TileDesc ring[kTileRing];
    TilePos ends[2];                        // of this block's run
    int4 desc[2];                           // what it leaves for the merge
    float2 ml[kFewRows];                    // (m, l) of group 1
    TileWaits waits;
    uint32_t turn[16];                      // of the last copy into each slot, K's or V's: what is in flight, when the block gives up
    uint32_t tmem;
};

// 16 rows of the warp's part of tensor memory x 8 N columns, four lanes to a row: register 4 i + 2 h + e of lane t has row t / 4 + 8 h,
// column 8 i + 2 (t % 4) + e
__device__ __forceinline__ void few_load4(uint32_t at, float (&v)[16])
{
    uint32_t *r = reinterpret_cast<uint32_t *>(v);
    asm volatile("tcgen05.ld.sync.aligned.16x256b.x4.b32 {%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];"
                 : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]), "=r"(r[9]), "=r"(r[10]),
                   "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
                 : "r"(at) : "memory");
}
__device__ __forceinline__ void few_store4(uint32_t at, const float (&v)[16])
{
    const uint32_t *r = reinterpret_cast<const uint32_t *>(v);
    asm volatile("tcgen05.st.sync.aligned.16x256b.x4.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
                 "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}
// the same with 4 N columns of two 16-bit values: register 2 i + h of lane t has row t / 4 + 8 h, values 8 i + 2 (t % 4) and the next
__device__ __forceinline__ void few_store_pairs(uint32_t at, const uint32_t (&r)[16])
{
    asm volatile("tcgen05.st.sync.aligned.16x128b.x8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15,%16};"
                 ::"r"(at), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]), "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]),
                 "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}

template <typename T, int NSUB, int SLOTS>
__global__ void __launch_bounds__(kFewThreads, 1)
prompt_few_kernel(const __grid_constant__ PromptArgs a, const __grid_constant__ CUtensorMap k_map, const __grid_constant__ CUtensorMap v_map)
{
    constexpr int DO = 64 * NSUB;
    constexpr uint32_t kSub = kTileRows * 128, kSlot = NSUB * kSub;
    constexpr float kBias = WideBias<T>::value;
    extern __shared__ unsigned char few_smem[];
    const uint32_t base = (smem_u32(few_smem) + 1023u) & ~1023u;
    const uint32_t q_at = base, ring = base + kSlot;
    unsigned char *const ctl = few_smem + (base - smem_u32(few_smem)) + (size_t)(SLOTS + 1) * kSlot;
    FewControl &c = *reinterpret_cast<FewControl *>(ctl);
    unsigned *const plan = reinterpret_cast<unsigned *>(ctl + sizeof(FewControl));
    const uint32_t full = smem_u32(c.bars), empty = full + 8 * SLOTS, q_full = empty + 8 * SLOTS, q_empty = q_full + 8, s_full = q_empty + 8, p_full = s_full + 16,
                   o_full = p_full + 16, m_full = o_full + 16, m_empty = m_full + 8, d_full = m_empty + 8, d_empty = d_full + 8 * kTileRing, last = d_empty + 8 * kTileRing;
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);   // (known to be uniform)

    if (tid == 0) {
        for (int i = 0; i < SLOTS; ++i) { mbar_init(full + 8 * i, 1); mbar_init(empty + 8 * i, 1); }
        mbar_init(q_full, 1);
        mbar_init(q_empty, 1);
        for (int g = 0; g < 2; ++g) { mbar_init(s_full + 8 * g, 1); mbar_init(p_full + 8 * g, 4); mbar_init(o_full + 8 * g, 1); }
        mbar_init(m_full, 4);
        mbar_init(m_empty, 4);
        for (int i = 0; i < kTileRing; ++i) { mbar_init(d_full + 8 * i, 1); mbar_init(d_empty + 8 * i, 12); }
        mbar_init(last, 1);
        c.waits = {a.polls, 0};
        for (int i = 0; i < SLOTS; ++i) c.turn[i] = 1u;            // (none: as if a phase before the first)
        mbar_init_fence();
        asm volatile("prefetch.tensormap [%0];" ::"l"(&k_map) : "memory");
        asm volatile("prefetch.tensormap [%0];" ::"l"(&v_map) : "memory");
    }
    // what the copies of Q leave of a row's last 16 elements is zero from the start
    if (a.d % 16) {
        for (uint32_t i = tid; i < kSlot / 16; i += kFewThreads)
            asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(q_at + 16 * i), "r"(0u) : "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 9) tc_alloc(smem_u32(&c.tmem), kTileColumns);
    pdl_wait();
    pdl_launch();
    PromptSeq *const seqs = a.batch <= kTileSeqs ? reinterpret_cast<PromptSeq *>(plan + ((a.batch + 2) & ~1)) : nullptr;
    tile_plan<true>(a, plan, seqs, c.ends, warp, lane);
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, c.tmem, 0);

    const auto wait = [&](uint32_t bar, uint32_t parity) { tile_wait(c.waits, bar, parity); };
    int at = 0;                                                    // the next item of the ring
    uint32_t d_phase = 0;
    const auto next_item = [&]() {                                 // leaves the one before to be written over
        __syncwarp();
        if (lane == 0) mbar_arrive(d_empty + 8 * at);
        if (++at == kTileRing) { at = 0; d_phase ^= 1u; }
    };
    const auto go_on = [&](uint32_t bar, uint32_t parity) { return tile_wait_warp(c.waits, bar, parity); };   // for a whole warp
    const auto have_item = [&]() { return go_on(d_full + 8 * at, d_phase) && c.ring[at].t1 >= 0; };   // c.ring[at] is one
    if (warp == 11) {                                              // ---- the list of items ----
        tile_walk<true>(a, seqs, c.ends, c.ring, d_full, d_empty, lane, c.waits, c.desc);
    } else if (warp == 8 || warp == 12) {                          // ---- copies of K, of V ----
        const bool value = warp == 12;
        const CUtensorMap *map = value ? &v_map : &k_map;
        uint32_t base = 0;                                         // copies of both before this item (but for whole pairs of turns)
        bool going = true;
        for (; have_item(); next_item()) {
            const TileDesc &it = c.ring[at];
            const TileSource src(a, it);
            const int t0 = it.t0, n = it.t1 - t0;
#pragma unroll 1
            for (int i = 0; going && i < n; ++i) {
                // K0 K1 V0 K2 V1 K3 .., in the order the products take them
                const uint32_t place = base + (uint32_t)(value ? min(2 * i + 2, 2 * n - 1) : max(2 * i - 1, 0)), turn = place / SLOTS, slot = place - turn * SLOTS;
                const uint32_t dst = ring + slot * kSlot, bar = full + 8 * slot;
                const int t = t0 + i;
                int y = src.pool_row(a, t, lane);
                going = go_on(empty + 8 * slot, (turn & 1u) ^ 1u);
                if (!going) break;
                if (tc_elect()) {
                    c.turn[slot] = turn;
                    mbar_expect_tx(bar, src.bytes(a, t, kSlot));
                }
                __syncwarp();
                if (a.table) {
                    // one lane issues for all: a copy by several lanes at a time is issued lane by lane too, with more ado
#pragma unroll 1
                    for (int b = 0; b << a.box_shift < src.valid(t); ++b) {
                        if (b && (b & 31) == 0) y = src.pool_row(a, t, b + lane);
                        const int row = __shfl_sync(0xffffffffu, y, b & 31);
                        if (tc_elect()) {
#pragma unroll
                            for (int s = 0; s < NSUB; ++s) pa_tma(dst + (uint32_t)(b << a.box_shift) * 128u + s * kSub, map, s * 64, row, bar);
                        }
                    }
                } else if (tc_elect()) {
                    const int tok = src.tok + src.row0(t);
                    const bool tf = a.tokens_first >> (value ? 2 : 1) & 1;
#pragma unroll
                    for (int s = 0; s < NSUB; ++s) tile_tma3(dst + s * kSub, map, s * 64, tf ? tok : src.head, tf ? src.head : tok, bar);
                }
                __syncwarp();
            }
            if (!going) break;
            base = (base + 2u * (uint32_t)n) % (2u * SLOTS);
        }
    } else if (warp == 10) {                                       // ---- copies of Q ----
        uint32_t phase = 0;
        const int piece = piece_of(a.q, a.q_token, a.q_head, a.d);
        for (; have_item(); next_item()) {
            const TileDesc &it = c.ring[at];
            if (it.t1 == it.t0) continue;
            const TileItem<true> item(a, it.s, it.q);
            const int rows = item.count * a.per_kv;
            const unsigned char *src = (const unsigned char *)a.q + 2 * ((it.s.q0 + item.first) * a.q_token + (long long)it.head * a.per_kv * a.q_head);
            if (!go_on(q_empty, phase ^ 1u)) break;
            phase ^= 1u;
#pragma unroll 1
            for (int r0 = 0; r0 < rows; r0 += 4) {
                const int r = r0 + (lane >> 3), t = a.by_per_kv(r), m = (r >> 3) * 32 + (r & 7);
                const unsigned char *from = src + 2 * (t * a.q_token + (r - t * a.per_kv) * a.q_head);
                if (r < rows) {
#pragma unroll 1
                    for (int x = (lane & 7) * piece; x < 2 * a.d; x += 8 * piece) {
                        const uint32_t to = q_at + tile_at(m, x, kSub);
                        if (piece == 16) tile_copy<16>(to, from + x);
                        else if (piece == 8) tile_copy<8>(to, from + x);
                        else tile_copy<4>(to, from + x);
                    }
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0) mbar_arrive(q_full);
        }
    } else if (warp == 9) {                                        // ---- products ----
        const int k_steps = (a.d + 15) / 16;
        const uint32_t s_shape = tc_shape<T>(kTileRows, false), o_shape = tc_shape<T>(k_steps * 16, true);
        int slot = 0;
        uint32_t phase = 0, q_phase = 0, p_phase = 0;               // (p_phase: bit g of group g)
        bool going = true;                                         // what did not come is neither used nor told to be free
        const auto take = [&]() {                                  // the next slot, once its tile is there
            going = go_on(full + 8 * slot, phase);
            const int taken = slot;
            if (++slot == SLOTS) { slot = 0; phase ^= 1u; }
            return taken;
        };
        const auto done = [&](uint32_t bar) {                      // counted when everything issued so far is complete
            if (tc_elect()) tc_commit(bar);
            __syncwarp();
        };
        for (; have_item(); next_item()) {
            const TileDesc &it = c.ring[at];
            // (shuffled, so that the compiler knows them to be uniform)
            const int t0 = __shfl_sync(0xffffffffu, it.t0, 0), n = __shfl_sync(0xffffffffu, it.t1, 0) - t0, p_rows = __shfl_sync(0xffffffffu, it.s.p, 0),
                      own_rows = __shfl_sync(0xffffffffu, it.s.n, 0), before = (p_rows + kTileRows - 1) / kTileRows;
            if (n == 0) continue;
            if (!go_on(q_full, q_phase)) break;
            q_phase ^= 1u;
            tc_after();
#pragma unroll 1
            for (int step = 0; step < n + 2; ++step) {
                const int g = step & 1, j = step - 2;              // O of tile j, then the scores of tile `step`, for the same group
                if (j >= 0) {
                    const int v = take(), t = t0 + j, valid = t < before ? p_rows - t * kTileRows : own_rows - (t - before) * kTileRows;
                    if (!going) break;
                    if (valid < kTileRows) {
                        // rows behind the end hold anything, and a weight of zero does not silence an infinity or a NaN
                        const uint32_t v_at = ring + (uint32_t)v * kSlot;
                        for (int i = lane; i < (kTileRows - valid) * 8 * NSUB; i += 32) {
                            const int r = valid + i / (8 * NSUB), ch = i % (8 * NSUB);
                            asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(v_at + (ch >> 3) * kSub + r * 128 + (ch & 7) * 16), "r"(0u) : "memory");
                        }
                        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                        __syncwarp();
                    }
                    wait(p_full + 8 * g, p_phase >> g & 1u);
                    p_phase ^= 1u << g;
                    tc_after();
                    const uint64_t vd = tc_operand(ring + (uint32_t)v * kSlot, kSub);
                    if (tc_elect()) {
#pragma unroll
                        for (int ks = 0; ks < kTileRows / 16; ++ks)
                            tc_mma_ts(tmem + 256 + g * 128, tmem + g * 128 + ks * 8, vd + (uint64_t)(ks * 128), o_shape, j >= 2 || ks > 0);
                    }
                    __syncwarp();
                    done(empty + 8 * v);
                    if (j + 2 >= n) done(o_full + 8 * g);          // that was the group's last
                }
                if (step < n) {
                    const int k = take();
                    if (!going) break;
                    const uint64_t qd = tc_operand(q_at, 16), kd = tc_operand(ring + (uint32_t)k * kSlot, 16);
                    if (tc_elect()) {
#pragma unroll
                        for (int ks = 0; ks < 4 * NSUB; ++ks) {
                            const uint64_t off = ((uint32_t)(ks >> 2) * kSub + (uint32_t)(ks & 3) * 32u) >> 4;
                            if (ks < k_steps) tc_mma_ss(tmem + g * 128, qd + off, kd + off, s_shape, ks > 0);
                        }
                    }
                    __syncwarp();
                    done(s_full + 8 * g);
                    done(empty + 8 * k);
                    if (step + 1 == n) done(q_empty);
                }
            }
            if (!going) break;
        }
    } else if (warp < 8) {                                         // ---- four lanes to a query row ----
        const int g = warp >> 2, col = 2 * (lane & 3), row = (warp & 3) * 8 + (lane >> 2);
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, s_col = tmem + g * 128 + lanes, o_col = tmem + 256 + g * 128 + lanes;
        const int in = a.by_per_kv(row), in_head = row - in * a.per_kv;   // token in the item, head in the key head's
        uint32_t s_phase = 0, o_phase = 0, m_phase = 0;
        bool again = false;                                        // a row came out too large for its type, or NaN where its weights are fine
        for (; have_item(); next_item()) {
            const TileDesc &it = c.ring[at];
            const TileItem<true> item(a, it.s, it.q);
            const bool warp_there = (warp & 3) * 8 < item.count * a.per_kv;
            const int own = it.s.seen(min(item.first + in, it.s.m - 1), a.causal);
            const int p_rows = it.s.p, before = (p_rows + kTileRows - 1) / kTileRows, t0 = it.t0, n = it.t1 - t0, tiles = (n + 1 - g) / 2;
            float m = -INFINITY, l = 0.f;                          // (l: this lane's part of the row's sum)
#pragma unroll 1
            for (int i = 0; i < tiles; ++i) {
                const int t = t0 + 2 * i + g;
                wait(s_full + 8 * g, s_phase);
                s_phase ^= 1u;
                tc_after();
                if (warp_there) {
                    float v[4][16];                                // (of 16 rows, 8 of them the item's: v[.][4 x], v[.][4 x + 1])
#pragma unroll
                    for (int x = 0; x < 4; ++x) few_load4(s_col + 32 * x, v[x]);
                    tc_load_wait();
                    const int valid = (t < before ? p_rows - t * kTileRows : own - (t - before) * kTileRows) - col;   // from this lane's first column on
                    if (__any_sync(0xffffffffu, valid < kTileRows)) {
#pragma unroll
                        for (int x = 0; x < 16; ++x) {
                            float *w = &v[x / 4][4 * (x % 4)];
                            w[0] = 8 * x < valid ? w[0] : -INFINITY;
                            w[1] = 8 * x + 1 < valid ? w[1] : -INFINITY;
                        }
                    }
                    float mx2[2] = {-INFINITY, -INFINITY};
#pragma unroll
                    for (int x = 0; x < 16; ++x) mx2[x & 1] = tile_max3(mx2[x & 1], v[x / 4][4 * (x % 4)], v[x / 4][4 * (x % 4) + 1]);
                    float mx = fmaxf(mx2[0], mx2[1]);
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1));
                    mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 2));
                    const bool move = (mx - m) * a.scale_log2e > kTileSlack || m == -INFINITY;
                    if (__any_sync(0xffffffffu, move)) {
                        const float m_new = move ? fmaxf(m, mx) : m;
                        const float corr = m_new == -INFINITY || m == -INFINITY ? (m == m_new ? 1.f : 0.f) : pa_exp2((m - m_new) * a.scale_log2e);
                        m = m_new;
                        l *= corr;
                        if (i > 0) {                               // the products before this tile's are complete: their S is
#pragma unroll 1
                            for (int x = 0; x < DO; x += 32) {
                                float o[16];
                                few_load4(o_col + x, o);
                                tc_load_wait();
#pragma unroll
                                for (int k = 0; k < 16; k += 4) { o[k] *= corr; o[k + 1] *= corr; }
                                few_store4(o_col + x, o);
                            }
                        }
                    }
                    const float shift = kBias - (m == -INFINITY ? 0.f : m) * a.scale_log2e;
                    const float2 scale2 = make_float2(a.scale_log2e, a.scale_log2e), shift2 = make_float2(shift, shift);
                    float2 sum[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
                    uint32_t p[2][16];
#pragma unroll
                    for (int x = 0; x < 16; ++x) {
                        float2 w = fma2(make_float2(v[x / 4][4 * (x % 4)], v[x / 4][4 * (x % 4) + 1]), scale2, shift2);
                        w.x = pa_exp2(w.x);
                        w.y = pa_exp2(w.y);
                        sum[x & 1] = add2(sum[x & 1], w);          // the sum takes the weights before they are rounded
                        p[x / 8][2 * (x % 8)] = pack2<T>(w.x, w.y);
                        p[x / 8][2 * (x % 8) + 1] = 0u;
                    }
                    l += sum[0].x + sum[0].y + sum[1].x + sum[1].y;
                    few_store_pairs(s_col, p[0]);                  // over scores that are in registers by now
                    few_store_pairs(s_col + 32, p[1]);
                    tc_store_wait();
                }
                tc_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(p_full + 8 * g);
            }
            if (tiles > 0) {
                wait(o_full + 8 * g, o_phase);
                o_phase ^= 1u;
                tc_after();
            }
            // the row's state: O (in tensor memory) and l relative to 2^m2
            l += __shfl_xor_sync(0xffffffffu, l, 1);
            l += __shfl_xor_sync(0xffffffffu, l, 2);
            float m2 = m == -INFINITY ? -INFINITY : m * a.scale_log2e - kBias;
            if (g == 1) {
                if ((lane & 3) == 0) c.ml[row] = make_float2(m2, l);
                tc_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(m_full);
                wait(m_empty, m_phase);                            // (group 0 has read this group's O)
                m_phase ^= 1u;
                tc_after();
                continue;
            }
            wait(m_full, m_phase);
            m_phase ^= 1u;
            tc_after();
            const bool partial = it.slot >= 0, none = p_rows + own == 0, two = n > 1;
            const bool there = row < item.count * a.per_kv && !tile_gave_up(c.waits);   // (what a block makes after it gave up is not written)
            float w0 = 1.f, w1 = 0.f;
            if (two) {
                const float2 other = c.ml[row];
                const float M = fmaxf(m2, other.x);
                w0 = m2 == -INFINITY ? 0.f : pa_exp2(m2 - M);
                w1 = other.x == -INFINITY ? 0.f : pa_exp2(other.x - M);
                l = l * w0 + other.y * w1;
                m2 = M;
            }
            if (!partial) {
                const float inv = 1.f / l;
                w0 *= inv;
                w1 *= inv;
            }
            const size_t to = (size_t)(it.s.q0 + item.first + in) * (a.kv_heads * a.per_kv) + it.head * a.per_kv + in_head;
            if (there && (lane & 3) == 0) {
                if (partial) *reinterpret_cast<float2 *>(a.state_ml + 2 * ((size_t)it.slot * 256 + row)) = make_float2(m2, l);
                else if (a.lse) a.lse[to] = none ? -INFINITY : (m2 + log2f(l)) * 0.693147180559945309f;
            }
            if (warp_there) {
                bool fits = true;
#pragma unroll 1
                for (int x0 = 0; x0 < a.d; x0 += 32) {
                    float o[16], o1[16];
#pragma unroll
                    for (int k = 0; k < 16; ++k) o[k] = o1[k] = 0.f;
                    if (tiles > 0) few_load4(o_col + x0, o);
                    if (two) few_load4(o_col + 128 + x0, o1);
                    tc_load_wait();
#pragma unroll
                    for (int i = 0; i < 4; ++i) {
                        const int x = x0 + 8 * i + col;
                        float2 y = make_float2(o[4 * i] * w0, o[4 * i + 1] * w0);
                        if (two) y = make_float2(fmaf(o1[4 * i], w1, y.x), fmaf(o1[4 * i + 1], w1, y.y));
                        if (none) y = make_float2(0.f, 0.f);
                        if (there && x < a.d) {
                            if (partial) {
                                *reinterpret_cast<float2 *>(a.state + ((size_t)it.slot * (DO / 4) + x / 4) * 1024 + row * 4 + x % 4) = y;
                            } else {
                                fits = fits && prompt_fits<T>(y.x) && prompt_fits<T>(y.y);
                                if (a.out) *reinterpret_cast<uint32_t *>((T *)a.out + to * a.d + x) = pack2<T>(y.x, y.y);
                                if (a.out_f32) *reinterpret_cast<float2 *>(a.out_f32 + to * a.d + x) = y;
                            }
                        }
                    }
                    __syncwarp();
                }
                if (!fits) {
                    if (!prompt_lost(a, l)) again = true;
                    else if ((lane & 3) == 0) prompt_mark_lost(a, to * a.d);
                }
            }
            tc_before();                                           // read before the next item's products write O
            __syncwarp();
            if (lane == 0) mbar_arrive(m_empty);
        }
        // rows that came out too large or NaN, by what they attend alone: the run once more, in whole items
        if (__any_sync(0xffffffffu, again)) {
            const TilePos end = c.ends[1];
            PromptOdd odd;
            odd.reset(-1, 0);
            odd.whole = tile_gave_up(c.waits);
            for (TilePos pos = c.ends[0]; pos.before(end);) {
                const PromptSeq s = prompt_seq(a, pos.b);
                if (s.m > 0) {
                    const TileItem<true> item(a, s, pos.q);
                    const bool last = pos.b == end.b && pos.head == end.head && pos.q == end.q;
                    const int rows = item.count * a.per_kv;
                    if (pos.tile == 0 && (!last || end.tile == item.tiles)) {
                        for (int r = warp * 8; r < min((warp + 1) * 8, rows); ++r) {
                            const int i = a.by_per_kv(r), tok = item.first + i, head = pos.head * a.per_kv + r - i * a.per_kv;
                            const size_t first = ((size_t)(s.q0 + tok) * (a.kv_heads * a.per_kv) + head) * a.d;
                            bool bad = false;
                            if (prompt_marked_lost(a, first)) continue;
                            for (int e = lane; e < a.d; e += 32) bad = bad || prompt_odd<T>(a, first + e);
                            if (__any_sync(0xffffffffu, bad)) prompt_mend_row<T>(a, s, pos.b, tok, head, lane, 0, a.d, odd);
                        }
                    }
                }
                pos = next_pos<true>(a, s, pos);
            }
        }
    }
    tc_before();
    __syncthreads();
    const bool gave_up = tile_gave_up(c.waits);
    if (warp == 9) {
        if (gave_up) tile_land(last, 1, 0u, true);
        tc_after();
        tc_dealloc(tmem, kTileColumns);
    }
    if (tid == 0 && a.split) {
        const int4 d = c.desc[0];
        a.run_desc[2 * blockIdx.x] = make_int4(d.x, d.y, d.z, d.w | (gave_up ? 2 : 0));
        a.run_desc[2 * blockIdx.x + 1] = c.desc[1];
    }
    if (gave_up) {
        if (tid == 0 && a.status) atomicOr(a.status, ADSA_DEV_COPY_TIMEOUT);
        if (warp == 8) {
            uint32_t flight = 0;
            for (int i = 0; i < SLOTS; ++i) flight |= (c.turn[i] & 1u) << i;
            tile_land(full, SLOTS, flight, false);
        }
    }
}

namespace {

template <typename T, int NSUB, int SLOTS>
cudaError_t launch_few(const PromptArgs &a, unsigned blocks, const CUtensorMap &km, const CUtensorMap &vm, cudaStream_t st)
{
    constexpr size_t most = 227 * 1024, fixed = 1024 + (size_t)(SLOTS + 1) * NSUB * kTileRows * 128 + sizeof(FewControl);
    static_assert(2 * SLOTS + 19 <= 48 && SLOTS <= 16, "barriers, turns");
    const size_t smem = fixed + tile_list_bytes(a.batch);
    if (smem > most) return cudaErrorInvalidValue;                 // (not with the batches that the calls take)
    const auto kern = prompt_few_kernel<T, NSUB, SLOTS>;
    static int told[64];
    const cudaError_t e = tile_allow_smem((const void *)kern, told, most);
    return e != cudaSuccess ? e : launch_pdl(kern, dim3(blocks), kFewThreads, smem, st, a, km, vm);
}

}  // namespace

cudaError_t launch_prompt_few(int dtype, const PromptArgs &a, unsigned blocks, const CUtensorMap &km, const CUtensorMap &vm, cudaStream_t st)
{
    if (dtype == ADSA_BF16) return a.d <= 64 ? launch_few<__nv_bfloat16, 1, 11>(a, blocks, km, vm, st) : launch_few<__nv_bfloat16, 2, 5>(a, blocks, km, vm, st);
    return a.d <= 64 ? launch_few<__half, 1, 11>(a, blocks, km, vm, st) : launch_few<__half, 2, 5>(a, blocks, km, vm, st);
}

}  // namespace adsa
