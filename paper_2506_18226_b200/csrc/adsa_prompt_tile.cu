// Attention of many query rows per sequence on the fifth-generation tensor cores, for packed prompts and for chunks of new
// tokens over a paged cache.
//
// A block (one per SM) has two groups of four warps, a query row per thread, with a 128-row tile of Q, 128 tensor-memory columns
// of scores and up to 128 of O each.  Per tile of 128 cached rows and group: S = Q K^T (operands in shared memory), softmax weights
// by the group's threads (row maxima and sums need no exchange between threads), P written back over S in tensor memory as 16-bit
// values, O += P V (P from tensor memory, V as it lies: rows of K, elements contiguous).  One warp copies K and V, one Q, one issues
// all products, one walks the list of items ahead of the others, so that one group's products run under the other's softmax and
// the next item's copies and first scores under the last one's outputs.
//
// An item is the query rows of a run of tokens for all query heads of one key head (row = token * heads + head): with more than 128 rows,
// both groups take every tile, each with its own half; up to 128, the groups take the tiles in turns, and join their states through
// tensor memory at the end.  Heads of more than 128 elements (WIDE): items of up to 128 rows, both groups make the same scores and
// weights, and each has 128 elements of O.
//
// The list of items in units (a tile of a half; eight for what an item costs beside them) is cut into one run per block.  A cut near the
// end of an item moves there; else the item's states go to the workspace, and a second kernel joins them.
//
// The running maximum of a row only moves when a tile exceeds it by more than 8 (in log2 units): until then weights up to 2^8
// are allowed, sums and products stay exact multiples, and O is rarely rescaled.  Weights are rounded once to the 16-bit type, their sum is taken before: a
// second value for what the rounding leaves would add half as many products again and as many conversions to the chain below; so the error of an output
// against 64 bits is 1.1 to 1.4 times that of rounding it alone (bfloat16 0.0016 -> 0.0018 .. 0.0023, half 0.00021 -> 0.00023 .. 0.00029).
// Rows of V behind the end are cleared in shared memory before they are used.  A weight of zero does not silence an infinity or NaN of a
// later token's V in the same tile: a row that comes out NaN or too large for its type is mended by one warp from the rows it attends.
//
// 16384 tokens x 16 heads on 4 of 128, causal (1.1 TFLOP): 0.99 .. 1.03 ms, 1.07 .. 1.11 PFLOP/s of 1.68 measured.  128 cached rows for both groups take 3200
// clocks at 1.7 GHz; the products alone are 2048, the exponentials too (both units 64% busy, issue slots 38%).  What bounds is a group's chain:
// scores out of tensor memory, their maximum, 128 exponentials a thread, the last quarter's product, the next scores.  Weights come in quarters, so
// that three of four products run under the softmax.  A third of the exponentials by polynomial on the multiply-add pipe:
// 1020 us where 960 went without, by the length of the code.  Code that does not run counts: with row copies, 32-bit outputs and the call that makes
// rows again in one loop, 144 KB of it, 48 prompts of 640 tokens took 277 us, 242 without.  An item's fixed part is 5000 clocks (its last product,
// outputs, next scores), which is what short prompts see: 48 of 143 to 1144 tokens, 26 items of three tiles a block, 316 .. 328 us.
#include <math.h>

#include "adsa_prompt_tile.cuh"

namespace adsa {

constexpr int kTileStage = 32;              // elements of an output row that a warp turns over in shared memory at a time: those of one load
constexpr int kFewMean = 32;                 // query rows per sequence and key head, on the mean, up to which the kernel for few rows runs
struct TileControl {
    uint64_t bars[44];
    TileDesc ring[kTileRing];
    TilePos ends[2];                        // of this block's run
    int4 desc[2];                           // what it leaves for the merge
    TileWaits waits;
    uint32_t tmem;
};

// PLAIN: what calls as a rule are: everything copied by boxes, outputs of 16 bits in 16-byte pieces.  What is left (row copies, other
// outputs) has a kernel of its own for its code's sake: it slowed this one by 10 to 15%, without being run.
template <typename T, int NSUB, int SLOTS, bool PLAIN>
__global__ void __launch_bounds__(kTileThreads, 1)
prompt_tile_kernel(const __grid_constant__ PromptArgs a, const __grid_constant__ CUtensorMap q_map, const __grid_constant__ CUtensorMap k_map,
                   const __grid_constant__ CUtensorMap v_map)
{
    constexpr bool WIDE = NSUB > 2;
    constexpr int PARTS = WIDE ? 2 : 1, PSUB = NSUB / PARTS;   // a tile of K or V lies in PARTS slots of PSUB columns of 64 elements
    constexpr int DO = 64 * PSUB;                             // elements of O of a group
    constexpr uint32_t kSub = kTileRows * 128, kSlot = PSUB * kSub, kQ = (WIDE ? 1 : 2) * NSUB * kSub, kStage = 32 * kTileStage * 2;
    constexpr float kBias = WideBias<T>::value;
    extern __shared__ unsigned char tile_smem[];
    const uint32_t base = (smem_u32(tile_smem) + 1023u) & ~1023u;
    const uint32_t q_at = base, ring = base + kQ;
    unsigned char *const stages = tile_smem + (base - smem_u32(tile_smem)) + kQ + (size_t)SLOTS * kSlot, *const ctl = stages + 8 * kStage;
    TileControl &c = *reinterpret_cast<TileControl *>(ctl);
    unsigned *const plan = reinterpret_cast<unsigned *>(ctl + sizeof(TileControl));
    const uint32_t full = smem_u32(c.bars), empty = full + 8 * SLOTS, q_full = empty + 8 * SLOTS, q_empty = q_full + 16, s_full = q_empty + 16,
                   p_full = s_full + 16, o_full = p_full + 64, m_full = o_full + 16, m_empty = m_full + 8, d_full = m_empty + 8,
                   d_empty = d_full + 8 * kTileRing, q_come = d_empty + 8 * kTileRing, last = q_come + 8;
    const int tid = threadIdx.x, lane = tid & 31, warp = __shfl_sync(0xffffffffu, tid >> 5, 0);   // (known to be uniform)

    if (tid == 0) {
        for (int i = 0; i < SLOTS; ++i) { mbar_init(full + 8 * i, 1); mbar_init(empty + 8 * i, 1); }
        for (int g = 0; g < 2; ++g) {
            mbar_init(q_full + 8 * g, 1); mbar_init(q_empty + 8 * g, 1); mbar_init(s_full + 8 * g, 1); mbar_init(o_full + 8 * g, 1);
            for (int i = 0; i < 4; ++i) mbar_init(p_full + 32 * g + 8 * i, 4);
        }
        mbar_init(q_come, 1);
        mbar_init(last, 1);
        c.waits = {a.polls, 0};
        mbar_init(m_full, 4);
        mbar_init(m_empty, 4);
        for (int i = 0; i < kTileRing; ++i) { mbar_init(d_full + 8 * i, 1); mbar_init(d_empty + 8 * i, 11); }
        mbar_init_fence();
        if (a.q_boxes || a.q_shifted) asm volatile("prefetch.tensormap [%0];" ::"l"(&q_map) : "memory");
        if (a.box_rows) {
            asm volatile("prefetch.tensormap [%0];" ::"l"(&k_map) : "memory");
            asm volatile("prefetch.tensormap [%0];" ::"l"(&v_map) : "memory");
        }
    }
    // what row copies leave of a row's last 16 elements is zero from the start
    if (!PLAIN && (!a.q_boxes || !a.box_rows) && a.d % 16) {
        for (uint32_t i = tid; i < (kQ + SLOTS * kSlot) / 16; i += kTileThreads)
            asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(base + 16 * i), "r"(0u) : "memory");
        asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
    }
    if (warp == 9) tc_alloc(smem_u32(&c.tmem), kTileColumns);
    pdl_wait();
    pdl_launch();
    PromptSeq *const seqs = a.batch <= kTileSeqs ? reinterpret_cast<PromptSeq *>(plan + ((a.batch + 2) & ~1)) : nullptr;
    tile_plan<WIDE>(a, plan, seqs, c.ends, warp, lane);
    tc_before();
    __syncthreads();
    tc_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, c.tmem, 0);

    const auto wait = [&](uint32_t bar, uint32_t parity) { tile_wait(c.waits, bar, parity); };
    uint32_t flight = 0xffffffffu;                                 // bit i: the parity that this warp's last copy to its barrier i completes
    int at = 0;                                                    // the next item of the ring
    uint32_t d_phase = 0;
    const auto next_item = [&]() {                                 // leaves the one before to be written over
        __syncwarp();
        if (lane == 0) mbar_arrive(d_empty + 8 * at);
        if (++at == kTileRing) { at = 0; d_phase ^= 1u; }
    };
    const auto go_on = [&](uint32_t bar, uint32_t parity) { return tile_wait_warp(c.waits, bar, parity); };   // for a whole warp
    const auto have_item = [&]() { return go_on(d_full + 8 * at, d_phase) && c.ring[at].t1 >= 0; };   // c.ring[at] is one
    // where the elements of a head's row begin in a tile of K or V
    const auto shift_of = [&](int head, bool value) { return !PLAIN && a.shifted ? (int)(head * (value ? a.v_head : a.k_head)) & 7 : 0; };

    // 168 registers a thread at the launch: the groups take what the other four warps leave
    if (warp >= 8) asm volatile("setmaxnreg.dec.sync.aligned.u32 72;");
    if (warp == 11) {                                              // ---- the list of items ----
        tile_walk<WIDE>(a, seqs, c.ends, c.ring, d_full, d_empty, lane, c.waits, c.desc);
    } else if (warp == 8) {                                        // ---- copies of K and V ----
        int slot = 0, waiting = 0;                                 // waiting: row copies in flight that nobody knows of yet
        uint32_t phase = 0;
        const int k_piece = piece_of(a.k, a.table ? a.row_stride : a.k_token, a.table ? 0 : a.k_head, a.d),
                  v_piece = piece_of(a.v, a.table ? a.row_stride : a.v_token, a.table ? 0 : a.v_head, a.d);
        // (by all lanes or none: a lane that flushed alone would not have waited for the others' copies, nor counted them)
        const auto ready = [&](uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, mbar_try_wait(bar, parity)) != 0; };
        const auto flush = [&]() {                                 // tell of all row copies
            asm volatile("cp.async.wait_all;" ::: "memory");
            asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
            __syncwarp();
            if (lane == 0)
                for (int i = waiting; i > 0; --i) mbar_arrive(full + 8 * (slot >= i ? slot - i : slot - i + SLOTS));
            waiting = 0;
        };
        // row by row: a lane knows one row of 32, eight lanes copy one
        const auto by_rows = [&](auto piece_, const TileDesc &it, bool pre, int row0, int x0, int valid, uint32_t dst, bool value) {
            constexpr int piece = decltype(piece_)::value;
            const unsigned char *src = (const unsigned char *)(value ? a.v : a.k);
            const int bytes = min(2 * a.d - 2 * x0, PSUB * 128);
#pragma unroll 1
            for (int r0 = 0; r0 < valid; r0 += 32) {
                unsigned long long off = 0;
                if (r0 + lane < valid) off = 2ULL * prompt_row(a, it.s, it.b, it.head, (pre ? 0 : it.s.p) + row0 + r0 + lane, value) + 2ULL * x0;
#pragma unroll
                for (int i = 0; i < 32; i += 4) {
                    const int r = r0 + i + (lane >> 3);
                    const unsigned char *from = src + __shfl_sync(0xffffffffu, off, i + (lane >> 3));
                    if (r < valid) {
#pragma unroll 4
                        for (int x = (lane & 7) * piece; x < bytes; x += 8 * piece) tile_copy<piece>(dst + tile_at(r, x, kSub), from + x);
                    }
                }
            }
        };
        // a part of K or V of tile t into the next slot; y: where the lane's box lies in the pool
        const auto copy = [&](const TileDesc &it, const TileSource &src, int t, int y, bool value, int part) {
            const int x0 = part * PSUB * 64;
            const uint32_t dst = ring + (uint32_t)slot * kSlot, bar = full + 8 * slot;
            const CUtensorMap *map = value ? &v_map : &k_map;
            if (!PLAIN && waiting && !ready(empty + 8 * slot, phase ^ 1u)) flush();
            if (!go_on(empty + 8 * slot, phase ^ 1u)) return false;
            if (PLAIN || a.box_rows) {
                if (tc_elect()) mbar_expect_tx(bar, src.bytes(a, t, kSlot));
                __syncwarp();
                if (a.table) {
                    // one lane issues for all: a copy by several lanes at a time is issued lane by lane too, with more ado
                    for (int i = 0; i << a.box_shift < src.valid(t); ++i) {
                        if (i && (i & 31) == 0) y = src.pool_row(a, t, i + lane);
                        const int row = __shfl_sync(0xffffffffu, y, i & 31);
                        if (tc_elect()) {
#pragma unroll
                            for (int s = 0; s < PSUB; ++s) pa_tma(dst + (uint32_t)(i << a.box_shift) * 128u + s * kSub, map, x0 + s * 64, row, bar);
                        }
                    }
                } else if (tc_elect()) {
                    const int tok = src.tok + src.row0(t);
                    const bool tf = a.tokens_first >> (value ? 2 : 1) & 1;
#pragma unroll
                    for (int s = 0; s < PSUB; ++s) {
                        if (!PLAIN && a.shifted) pa_tma(dst + s * kSub, map, (int)(src.head * (value ? a.v_head : a.k_head)) - shift_of(src.head, value) + s * 64, tok, bar);
                        else tile_tma3(dst + s * kSub, map, x0 + s * 64, tf ? tok : src.head, tf ? src.head : tok, bar);
                    }
                }
                __syncwarp();
            } else if constexpr (!PLAIN) {
                const int piece = value ? v_piece : k_piece, valid = src.valid(t), row0 = src.row0(t);
                const bool pre = t < src.before;
                if (piece == 16) by_rows(std::integral_constant<int, 16>(), it, pre, row0, x0, valid, dst, value);
                else if (piece == 8) by_rows(std::integral_constant<int, 8>(), it, pre, row0, x0, valid, dst, value);
                else by_rows(std::integral_constant<int, 4>(), it, pre, row0, x0, valid, dst, value);
                ++waiting;
            }
            if (++slot == SLOTS) { slot = 0; phase ^= 1u; }
            return true;
        };
        bool going = true;
        // in the order the products take them: K0 V0 K1 V1 .. where both groups share a tile, else K0 K1 V0 K2 V1 K3 ..
        for (;;) {
            if (!PLAIN && waiting && !ready(d_full + 8 * at, d_phase)) flush();
            if (!have_item()) break;
            const TileDesc &it = c.ring[at];
            const bool turns = !WIDE && it.s.m - it.q * item_tokens<WIDE>(a) <= a.half_tokens;
            const TileSource src(a, it);
            const int ahead = turns ? 2 : 1, t0 = it.t0, n = it.t1 - t0;
            int k_next = 0, v_next = 0, y_last = -1, y_before = -1;   // pool rows of this lane's box in the last K and the one before it
#pragma unroll 1
            for (int j = 0; going && j < 2 * n; ++j) {
                const bool value = k_next == n || k_next - v_next == ahead;
                const int t = t0 + (value ? v_next : k_next);
                int y = k_next - v_next == 2 ? y_before : y_last;  // V lies where K does
                if (!value) {
                    y = src.pool_row(a, t, lane);
                    y_before = y_last;
                    y_last = y;
                }
                (value ? v_next : k_next) += 1;
#pragma unroll 1
                for (int p = 0; going && p < PARTS; ++p) going = copy(it, src, t, y, value, p);
            }
            if (!going) break;
            next_item();
        }
        if (!PLAIN && waiting) flush();
        flight = (phase ? 0u : 0xffffffffu << slot) | (phase ? (1u << slot) - 1u : 0u);   // below `slot` this round's, above it the last one's
    } else if (warp == 10) {                                       // ---- copies of Q ----
        uint32_t phase = 0, come = 0;                              // (phase: bit h of half h)
        bool going = true;
        const int q_piece = piece_of(a.q, a.q_token, a.q_head, a.d), tph = a.half_tokens;
        for (; have_item(); next_item()) {
            const TileDesc &it = c.ring[at];
            if (it.t1 == it.t0) continue;
            const TileItem<WIDE> item(a, it.s, it.q);
#pragma unroll 1
            for (int h = 0; going && h < (item.pair ? 2 : 1); ++h) {
                const int tok = item.first + h * tph, tokens = min(item.count - h * tph, tph);
                const uint32_t dst = q_at + (uint32_t)h * NSUB * kSub, bar = q_full + 8 * h;
                going = go_on(q_empty + 8 * h, (phase >> h & 1u) ^ 1u);
                if (!going) break;
                phase ^= 1u << h;
                if (PLAIN || a.q_boxes) {
                    if (lane == 0) {
                        const int boxes = (a.d + 63) / 64, y = it.head * a.per_kv, z = (int)it.s.q0 + tok;
                        mbar_expect_tx(bar, (uint32_t)(boxes * tph * a.per_kv) * 128u);
                        for (int s = 0; s < boxes; ++s)
                            tile_tma3(dst + s * kSub, &q_map, s * 64, y, z, bar);
                    }
                    __syncwarp();
                } else if constexpr (!PLAIN) {
                    const unsigned char *src = (const unsigned char *)a.q + 2 * ((it.s.q0 + tok) * a.q_token + (long long)it.head * a.per_kv * a.q_head);
                    const int shift = shift_of(it.head, false), piece = shift ? min(q_piece, (2 * shift) & -(2 * shift)) : q_piece;
                    const auto by_rows = [&](auto piece_) {
                        constexpr int piece = decltype(piece_)::value;
#pragma unroll 2
                        for (int r0 = 0; r0 < tokens * a.per_kv; r0 += 4) {
                            const int r = r0 + (lane >> 3), t = a.by_per_kv(r);
                            const unsigned char *from = src + 2 * (t * a.q_token + (r - t * a.per_kv) * a.q_head);
                            if (r < tokens * a.per_kv)
#pragma unroll 4
                                for (int x = (lane & 7) * piece; x < 2 * a.d; x += 8 * piece) tile_copy<piece>(dst + tile_at(r, x + 2 * shift, kSub), from + x);
                        }
                    };
                    if (a.q_shifted) {                             // q's rows lie as K's do
                        if (lane == 0) {
                            const int boxes = (a.d + 63) / 64;
                            mbar_expect_tx(q_come, (uint32_t)boxes * kSub);
                            for (int s = 0; s < boxes; ++s) pa_tma(dst + s * kSub, &q_map, (int)(it.head * a.q_head) - shift + s * 64, (int)it.s.q0 + tok, q_come);
                        }
                        __syncwarp();
                        come ^= 1u;
                        going = go_on(q_come, come ^ 1u);
                        if (!going) break;
                    }
                    if (a.shifted) {                               // what K has beside the head's elements meets zeros
                        const int end = (a.d + shift + 15) / 16 * 16;
                        for (int r = lane; r < kTileRows; r += 32) {
                            for (int x = shift > 0 ? 0 : a.d; x < end; x = x + 2 == shift ? shift + a.d : x + 2)
                                asm volatile("st.shared.u32 [%0], %1;" ::"r"(dst + tile_at(r, 2 * x, kSub)), "r"(0u) : "memory");
                        }
                    }
                    if (!a.q_shifted) {
                        if (piece == 16) by_rows(std::integral_constant<int, 16>());
                        else if (piece == 8) by_rows(std::integral_constant<int, 8>());
                        else by_rows(std::integral_constant<int, 4>());
                    }
                    asm volatile("cp.async.wait_all;" ::: "memory");
                    asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar);
                }
            }
            if (!going) break;
        }
        flight = (phase ^ 3u) | (come ^ 1u) << 2;                  // (0, 1: the halves'; 2: q_come)
    } else if (warp == 9) {                                        // ---- products ----
        int k_steps = (a.d + 15) / 16, d_cols = k_steps * 16;       // (of this head's place in K; in V)
        const uint32_t s_shape = tc_shape<T>(kTileRows, false);
        int slot = 0;
        uint32_t phase = 0, q_phase = 0, p_phase = 0;               // (bit g: of group or half g)
        bool going = true;                                         // what did not come is neither used nor told to be free
        const auto take = [&]() {                                  // the next slot, once its tile is there
            going = go_on(full + 8 * slot, phase);
            const int taken = slot;
            if (++slot == SLOTS) { slot = 0; phase ^= 1u; }
            return taken;
        };
        const auto score = [&](int g, const int (&k_slot)[PARTS], uint32_t q) {   // S = Q K^T
            const uint64_t qd = tc_operand(q, 16), kd0 = tc_operand(ring + (uint32_t)k_slot[0] * kSlot, 16),
                           kd1 = tc_operand(ring + (uint32_t)k_slot[PARTS - 1] * kSlot, 16);
            if (tc_elect()) {
#pragma unroll
                for (int ks = 0; ks < 4 * NSUB; ++ks) {
                    const uint64_t q_off = ((uint32_t)(ks >> 2) * kSub + (uint32_t)(ks & 3) * 32u) >> 4;
                    const uint64_t k_off = ((uint32_t)((ks >> 2) % PSUB) * kSub + (uint32_t)(ks & 3) * 32u) >> 4;
                    if (ks < k_steps) tc_mma_ss(tmem + g * 128, qd + q_off, (ks < 4 * PSUB ? kd0 : kd1) + k_off, s_shape, ks > 0);
                }
            }
        };
        const auto take_v = [&](int valid) {                           // V of tile t, or a part of it
            const int taken = take();
            if (valid < kTileRows) {
                // rows behind the end hold anything, and a weight of zero does not silence an infinity or a NaN
                const uint32_t v_at = ring + (uint32_t)taken * kSlot;
                for (int i = lane; i < (kTileRows - valid) * 8 * PSUB; i += 32) {
                    const int r = valid + i / (8 * PSUB), ch = i % (8 * PSUB);
                    asm volatile("st.shared.v4.u32 [%0], {%1,%1,%1,%1};" ::"r"(v_at + (ch >> 3) * kSub + r * 128 + (ch & 7) * 16), "r"(0u) : "memory");
                }
                asm volatile("fence.proxy.async.shared::cta;" ::: "memory");
                __syncwarp();
            }
            return taken;
        };
        const auto weigh = [&](int g, int v_slot, bool first) {    // O += P V, once the group has left P
            const uint64_t vd = tc_operand(ring + (uint32_t)v_slot * kSlot, kSub);
            const uint32_t o_shape = tc_shape<T>(WIDE ? min(d_cols - g * DO, DO) : d_cols, true);
#pragma unroll 1
            for (int part = 0; part < 4; ++part) {                 // P comes in quarters: one is used while the next is made
                wait(p_full + 32 * g + 8 * part, p_phase >> g & 1u);
                tc_after();
                if (tc_elect()) {
#pragma unroll
                    for (int k = 0; k < kTileRows / 64; ++k) {
                        const int ks = part * (kTileRows / 64) + k;
                        tc_mma_ts(tmem + 256 + g * 128, tmem + g * 128 + ks * 8, vd + (uint64_t)(ks * 128), o_shape, !first || ks > 0);
                    }
                }
                __syncwarp();
            }
            p_phase ^= 1u << g;
        };
        const auto done = [&](uint32_t bar) {                      // counted when everything issued so far is complete
            if (tc_elect()) tc_commit(bar);
            __syncwarp();
        };
        const auto queries = [&](int h) {
            going = go_on(q_full + 8 * h, q_phase >> h & 1u) && going;
            q_phase ^= 1u << h;
        };
        for (; have_item(); next_item()) {
            const TileDesc &it = c.ring[at];
            // (shuffled, so that the compiler knows them to be uniform)
            const int t0 = __shfl_sync(0xffffffffu, it.t0, 0), n = __shfl_sync(0xffffffffu, it.t1, 0) - t0, p_rows = __shfl_sync(0xffffffffu, it.s.p, 0),
                      own_rows = __shfl_sync(0xffffffffu, it.s.n, 0), before = (p_rows + kTileRows - 1) / kTileRows;
            if (n == 0) continue;
            const TileItem<WIDE> item(a, it.s, it.q);
            const bool pair = __shfl_sync(0xffffffffu, (int)item.pair, 0);
            if (!PLAIN && a.shifted) {
                k_steps = __shfl_sync(0xffffffffu, (a.d + shift_of(it.head, false) + 15) / 16, 0);
                d_cols = __shfl_sync(0xffffffffu, (a.d + shift_of(it.head, true) + 15) / 16, 0) * 16;
            }
            queries(0);
            if (pair) queries(1);
            if (!going) break;
            tc_after();
            // Steps of the two groups in turn.  Each: O of a tile, for the group whose weights are due, then the scores of its next tile.  Where
            // both groups take every tile, group 0 takes it and group 1 leaves it; else the group of the step does both.
            const bool turns = !WIDE && !pair;
            const int ahead = turns ? 2 : 1, steps = turns ? n + 2 : 2 * n + 2;
            // the first half's tokens attend no more tiles than the second's
            const int n0 = pair ? __shfl_sync(0xffffffffu, min(max(tiles_until(a, it.s, item.first + a.half_tokens - 1) - t0, 0), n), 0) : n;
            int k[PARTS], v[PARTS];
            if (n0 == 0) done(q_empty);
#pragma unroll 1
            for (int step = 0; step < steps; ++step) {
                const int g = step & 1, i = turns ? step : step >> 1, mine = g == 0 ? n0 : n, j = i - ahead;   // scores of tile i, O of tile j
                const bool takes = turns || g == 0, leaves = turns || g == 1;
                if (j >= 0) {
                    if (takes) {
                        const int t = t0 + j, valid = t < before ? p_rows - t * kTileRows : own_rows - (t - before) * kTileRows;
#pragma unroll
                        for (int p = 0; p < PARTS; ++p) { v[p] = take_v(valid); if (!going) break; }
                        if (!going) break;
                    }
                    if (j < mine) {
                        weigh(g, WIDE && g == 1 ? v[PARTS - 1] : v[0], j < ahead);
                        if (j + ahead >= mine) done(o_full + 8 * g);           // that was the group's last
                    }
                    if (WIDE) done(empty + 8 * (g == 1 ? v[PARTS - 1] : v[0]));
                    else if (leaves) done(empty + 8 * v[0]);
                }
                if (i < n) {
                    if (takes) {
#pragma unroll
                        for (int p = 0; p < PARTS; ++p) { k[p] = take(); if (!going) break; }
                        if (!going) break;
                    }
                    if (i < mine) {
                        score(g, k, pair && g == 1 ? q_at + NSUB * kSub : q_at);
                        done(s_full + 8 * g);
                        // the last scores that read this half of Q
                        if (pair ? i + 1 == mine : i + 1 == n && leaves) done(q_empty + (pair ? 8 * g : 0));
                    }
                    if (leaves) {
#pragma unroll
                        for (int p = 0; p < PARTS; ++p) done(empty + 8 * k[p]);
                    }
                }
            }
            if (!going) break;
        }
    } else {                                                       // ---- a query row per thread ----
        asm volatile("setmaxnreg.inc.sync.aligned.u32 216;");
        const int g = warp >> 2, row = tid & 127;
        const uint32_t lanes = (uint32_t)((warp & 3) * 32) << 16, s_col = tmem + g * 128 + lanes, o_col0 = tmem + 256 + g * 128 + lanes;
        const uint32_t my_s = s_full + 8 * g, my_p = p_full + 32 * g, my_o = o_full + 8 * g;
        const int tph = a.half_tokens, heads = a.kv_heads * a.per_kv;
        uint32_t s_phase = 0, o_phase = 0, m_phase = 0;
        bool again = false;                                        // a row of this lane came out too large for its type, or NaN where its weights are fine
        for (; have_item(); next_item()) {
            const TileDesc &it = c.ring[at];
            const TileItem<WIDE> item(a, it.s, it.q);
            const bool turns = !WIDE && !item.pair;                // the groups take the tiles in turns
            const int half = item.pair ? g : 0, in = a.by_per_kv(row), tok = item.first + half * tph + in, head = it.head * a.per_kv + row - in * a.per_kv;
            bool there = in < tph && in + half * tph < item.count;
            const int own = it.s.seen(min(tok, it.s.m - 1), a.causal), before = (it.s.p + kTileRows - 1) / kTileRows;
            const bool warp_there = __any_sync(0xffffffffu, there);
            const int p_rows = it.s.p, t0 = it.t0;
            int tiles = it.t1 - t0;
            if (turns) tiles = (tiles + 1 - g) / 2;
            else if (item.pair && g == 0) tiles = min(max(tiles_until(a, it.s, item.first + tph - 1) - it.t0, 0), tiles);
            float m = -INFINITY;                                   // raw units; the row's weights are relative to it
            float2 l2[2] = {make_float2(0.f, 0.f), make_float2(0.f, 0.f)};
            for (int i = 0; i < tiles; ++i) {
                const int t = t0 + (turns ? 2 * i + g : i);
                const int valid = t < before ? p_rows - t * kTileRows : own - (t - before) * kTileRows;   // rows of the tile that this row attends
                wait(my_s, s_phase);
                s_phase ^= 1u;
                tc_after();
                if (!warp_there) {
                    tc_before();
                    if (lane < 4) mbar_arrive(my_p + 8 * lane);
                    continue;
                }
                alignas(8) float v[kTileRows];
#pragma unroll
                for (int x = 0; x < kTileRows; x += 32) tc_load32(s_col + x, *reinterpret_cast<float (*)[32]>(v + x));
                tc_load_wait();
                if (__any_sync(0xffffffffu, valid < kTileRows)) {
#pragma unroll
                    for (int x = 0; x < kTileRows; ++x) v[x] = x < valid ? v[x] : -INFINITY;
                }
                float mx4[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
                for (int x = 0; x < kTileRows; x += 2) mx4[x / 2 & 3] = tile_max3(mx4[x / 2 & 3], v[x], v[x + 1]);
                const float mx = fmaxf(tile_max3(mx4[0], mx4[1], mx4[2]), mx4[3]);
                const bool move = (mx - m) * a.scale_log2e > kTileSlack || m == -INFINITY;
                if (__any_sync(0xffffffffu, move)) {
                    const float m_new = move ? fmaxf(m, mx) : m;
                    const float corr = m_new == -INFINITY || m == -INFINITY ? (m == m_new ? 1.f : 0.f) : pa_exp2((m - m_new) * a.scale_log2e);
                    m = m_new;
#pragma unroll
                    for (int k = 0; k < 2; ++k) { l2[k].x *= corr; l2[k].y *= corr; }
                    if (i > 0) {                                   // the products before this tile's are complete: their S is
#pragma unroll 1
                        for (int x = 0; x < DO; x += 16) {
                            float o[16];
                            tc_load16(o_col0 + x, o);
                            tc_load_wait();
#pragma unroll
                            for (int k = 0; k < 16; ++k) o[k] *= corr;
                            tc_store16f(o_col0 + x, o);
                        }
                    }
                }
                const float shift = kBias - (m == -INFINITY ? 0.f : m) * a.scale_log2e;
                const float2 scale2 = make_float2(a.scale_log2e, a.scale_log2e), shift2 = make_float2(shift, shift);
#pragma unroll
                for (int x = 0; x < kTileRows; x += 32) {
                    uint32_t p[16];
#pragma unroll
                    for (int k = 0; k < 16; ++k) {
                        float2 w = fma2(make_float2(v[x + 2 * k], v[x + 2 * k + 1]), scale2, shift2);
                        w.x = pa_exp2(w.x);
                        w.y = pa_exp2(w.y);
                        l2[k & 1] = add2(l2[k & 1], w);            // the sum takes the weights before they are rounded
                        p[k] = pack2<T>(w.x, w.y);
                    }
                    tc_store16(s_col + x / 2, p);                  // over scores that are in registers by now
                    tc_store_wait();
                    tc_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(my_p + 8 * (x / 32));
                }
            }
            if (tiles > 0) {
                wait(my_o, o_phase);
                o_phase ^= 1u;
                tc_after();
            }
            // the row's state: O (in tensor memory) and l relative to 2^m2
            float m2 = m == -INFINITY ? -INFINITY : m * a.scale_log2e - kBias, l = l2[0].x + l2[0].y + l2[1].x + l2[1].y, w0 = 1.f, w1 = 0.f;
            bool both = false;
            if (turns) {
                if (g == 1) {
                    reinterpret_cast<float2 *>(stages + warp * kStage)[lane] = make_float2(m2, l);
                    tc_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(m_full);
                    wait(m_empty, m_phase);                        // (group 0 has read this group's O)
                    m_phase ^= 1u;
                    tc_after();
                    continue;
                }
                wait(m_full, m_phase);
                m_phase ^= 1u;
                tc_after();
                both = it.t1 - it.t0 > 1;
                if (both) {
                    const float2 other = reinterpret_cast<const float2 *>(stages + (warp + 4) * kStage)[lane];
                    const float M = fmaxf(m2, other.x);
                    w0 = m2 == -INFINITY ? 0.f : pa_exp2(m2 - M);
                    w1 = other.x == -INFINITY ? 0.f : pa_exp2(other.x - M);
                    l = l * w0 + other.y * w1;
                    m2 = M;
                }
            }
            const int c0 = WIDE ? g * DO : 0, c1 = min(a.d, c0 + DO);   // elements of the output
            const bool none = it.s.p + own == 0, partial = it.slot >= 0;
            const float inv = 1.f / l;
            if (!partial && none) w0 = w1 = 0.f;
            else if (!partial) { w0 *= inv; w1 *= inv; }
            there = there && !tile_gave_up(c.waits);               // (what a block makes after it gave up is not written)
            const int at_row = there ? (int)((it.s.q0 + tok) * heads + head) : -1;   // (rows of a call are below 2^31)
            const size_t at_slot = (size_t)it.slot * 256 + (WIDE ? g * 128 : half * 128) + row;
            float most = 0.f;                                      // of the row's outputs
            if (warp_there) {
                const uint32_t shift = (uint32_t)shift_of(it.head, true), o_col = o_col0 + shift;
                // 32 elements of the row's output, or of its state; zeros where the 16 columns lie past the head's elements
                const auto load = [&](int x, float (&o)[32]) {
                    const bool second = x + 16 < c1 - c0;
#pragma unroll
                    for (int k = 0; k < 32; ++k) o[k] = 0.f;
                    if (tiles > 0) {
                        tc_load16(o_col + x, *reinterpret_cast<float (*)[16]>(o));
                        if (second) tc_load16(o_col + x + 16, *reinterpret_cast<float (*)[16]>(o + 16));
                        tc_load_wait();
#pragma unroll
                        for (int k = 0; k < 32; k += 2) *reinterpret_cast<float2 *>(o + k) = mul2(*reinterpret_cast<float2 *>(o + k), make_float2(w0, w0));
                    }
                    if (both) {
                        alignas(8) float o1[32];
#pragma unroll
                        for (int k = 16; k < 32; ++k) o1[k] = 0.f;
                        tc_load16(tmem + 384 + lanes + shift + x, *reinterpret_cast<float (*)[16]>(o1));
                        if (second) tc_load16(tmem + 384 + lanes + shift + x + 16, *reinterpret_cast<float (*)[16]>(o1 + 16));
                        tc_load_wait();
#pragma unroll
                        for (int k = 0; k < 32; k += 2)
                            *reinterpret_cast<float2 *>(o + k) = fma2(*reinterpret_cast<float2 *>(o1 + k), make_float2(w1, w1), *reinterpret_cast<float2 *>(o + k));
                    }
                };
                if (partial) {
#pragma unroll 1
                    for (int x = 0; x < c1 - c0; x += 32) {
                        alignas(8) float o[32];
                        load(x, o);
                        if (there) {
#pragma unroll
                            for (int k = 0; k < 32; k += 4)        // neighbouring rows lie next to each other
                                *reinterpret_cast<float4 *>(a.state + ((at_slot >> 8) * (DO / 4) + (x + k) / 4) * 1024 + (at_slot & 255) * 4) =
                                    make_float4(o[k], o[k + 1], o[k + 2], o[k + 3]);
                        }
                        __syncwarp();
                    }
                    if (there) *reinterpret_cast<float2 *>(a.state_ml + 2 * at_slot) = make_float2(m2, l);
                } else {
                    const auto outputs = [&](int x, float (&o)[32]) {   // 32 elements of the output
                        load(x, o);
                        if (__any_sync(0xffffffffu, none)) {
#pragma unroll
                            for (int k = 0; k < 32; ++k) o[k] = none ? 0.f : o[k];
                        }
                        if (!PLAIN && c1 - c0 - x < 32) {          // (what lies past the head's elements is not of its products)
#pragma unroll
                            for (int k = 0; k < 32; ++k) o[k] = k < c1 - c0 - x ? o[k] : 0.f;
                        }
#pragma unroll
                        for (int k = 0; k < 32; k += 2) most = tile_magnitude(most, o[k], o[k + 1]);
                    };
                    if constexpr (PLAIN) {
                        // a row per lane, in whole sectors of 32 bytes (through shared memory, so that lanes shared rows: 7% slower for
                        // items of three tiles)
#pragma unroll 1
                        for (int x = 0; x < c1 - c0; x += 32) {
                            alignas(8) float o[32];
                            outputs(x, o);
#pragma unroll
                            for (int k = 0; k < 32; k += 16)
                                if (there && x + k < c1 - c0)
                                    asm volatile("st.global.v8.b32 [%0], {%1,%2,%3,%4,%5,%6,%7,%8};"
                                                 ::"l"((T *)a.out + (size_t)at_row * a.d + c0 + x + k), "r"(pack2<T>(o[k], o[k + 1])), "r"(pack2<T>(o[k + 2], o[k + 3])),
                                                 "r"(pack2<T>(o[k + 4], o[k + 5])), "r"(pack2<T>(o[k + 6], o[k + 7])), "r"(pack2<T>(o[k + 8], o[k + 9])),
                                                 "r"(pack2<T>(o[k + 10], o[k + 11])), "r"(pack2<T>(o[k + 12], o[k + 13])), "r"(pack2<T>(o[k + 14], o[k + 15]))
                                                 : "memory");
                            __syncwarp();
                        }
                    } else {
                        const uint32_t stage = smem_u32(stages) + warp * kStage;
                        const bool wide_out = a.d % 8 == 0 && ((uintptr_t)a.out & 15) == 0, half_out = a.d % 4 == 0 && ((uintptr_t)a.out & 7) == 0;
#pragma unroll 1
                        for (int x0 = 0; x0 < c1 - c0; x0 += kTileStage) {
                            alignas(8) float o[32];
                            outputs(x0, o);
                            if (a.out_f32 && there) {
#pragma unroll
                                for (int k = 0; k < 32; k += 2)
                                    if (k < c1 - c0 - x0) *reinterpret_cast<float2 *>(a.out_f32 + (size_t)at_row * a.d + c0 + x0 + k) = make_float2(o[k], o[k + 1]);
                            }
#pragma unroll
                            for (int k = 0; k < 32; k += 8)
                                asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};"
                                             ::"r"(stage + (uint32_t)(lane * kTileStage * 2) + (uint32_t)(((k / 8) ^ (lane & (kTileStage / 8 - 1))) << 4)),
                                             "r"(pack2<T>(o[k], o[k + 1])), "r"(pack2<T>(o[k + 2], o[k + 3])), "r"(pack2<T>(o[k + 4], o[k + 5])),
                                             "r"(pack2<T>(o[k + 6], o[k + 7])) : "memory");
                            __syncwarp();
                            if (a.out && wide_out) {                   // 16 bytes a lane, kTileStage / 8 lanes a row
                                constexpr int LANES = kTileStage / 8;
                                uint4 w[LANES];
#pragma unroll
                                for (int i = 0; i < LANES; ++i) {
                                    const int r = i * (32 / LANES) + lane / LANES;
                                    w[i] = *reinterpret_cast<const uint4 *>(stages + warp * kStage + r * kTileStage * 2 + ((lane % LANES ^ (r & (LANES - 1))) << 4));
                                }
#pragma unroll
                                for (int i = 0; i < LANES; ++i) {
                                    const int to = __shfl_sync(0xffffffffu, at_row, i * (32 / LANES) + lane / LANES);
                                    if (to >= 0 && c0 + x0 + lane % LANES * 8 < c1) *reinterpret_cast<uint4 *>((T *)a.out + (size_t)to * a.d + c0 + x0 + lane % LANES * 8) = w[i];
                                }
                            } else if (a.out) {                        // 8 or 4 bytes a lane
                                const auto pieces = [&](auto words_) {
                                    constexpr int WORDS = decltype(words_)::value, LANES = kTileStage / 2 / WORDS;
#pragma unroll 4
                                    for (int i = 0; i < 32; i += 32 / LANES) {
                                        const int r = i + lane / LANES, e = 2 * WORDS * (lane % LANES), to = __shfl_sync(0xffffffffu, at_row, r);
                                        const uint32_t *from = reinterpret_cast<const uint32_t *>(
                                            stages + warp * kStage + r * kTileStage * 2 + (((e / 8) ^ (r & (kTileStage / 8 - 1))) << 4) + e % 8 * 2);
                                        uint32_t *out = reinterpret_cast<uint32_t *>((T *)a.out + (size_t)max(to, 0) * a.d + c0 + x0 + e);
                                        if (to >= 0 && c0 + x0 + e < c1) {
                                            if constexpr (WORDS == 2) *reinterpret_cast<uint2 *>(out) = *reinterpret_cast<const uint2 *>(from);
                                            else *out = *from;
                                        }
                                    }
                                };
                                if (half_out) pieces(std::integral_constant<int, 2>());
                                else pieces(std::integral_constant<int, 1>());
                            }
                            __syncwarp();
                        }
                    }
                    if (there && a.lse && c0 == 0) a.lse[at_row] = none ? -INFINITY : (m2 + log2f(l)) * 0.693147180559945309f;
                }
            }
            tc_before();                                           // read before the next item's products write O
            if (turns) {
                __syncwarp();
                if (lane == 0) mbar_arrive(m_empty);
            }
            if (there && !partial && !prompt_fits<T>(most)) {
                if (prompt_lost(a, l)) prompt_mark_lost(a, (size_t)at_row * a.d + c0);
                else again = true;
            }
        }
        // Rows that came out too large or NaN, by what they attend alone: the run once more, in whole items.  (A call in the loop above
        // cost it 8%.)
        if (__any_sync(0xffffffffu, again)) {
            const TilePos end = c.ends[1];
            PromptOdd odd;
            odd.reset(-1, 0);
            odd.whole = tile_gave_up(c.waits);
            for (TilePos pos = c.ends[0]; pos.before(end); pos.tile = 0) {
                const PromptSeq s = prompt_seq(a, pos.b);
                if (s.m > 0) {
                    const TileItem<WIDE> item(a, s, pos.q);
                    const bool last = pos.b == end.b && pos.head == end.head && pos.q == end.q;
                    if (pos.tile == 0 && (!last || end.tile == item.tiles) && (WIDE || item.pair || g == 0)) {
                        const int in = a.by_per_kv(row), at = in + (item.pair ? g * tph : 0), c0 = WIDE ? g * DO : 0, c1 = min(a.d, c0 + DO);
                        const int tok = item.first + at, head = pos.head * a.per_kv + row - in * a.per_kv;
                        bool bad = false;
                        if (in < tph && at < item.count) {
                            const size_t first = ((size_t)(s.q0 + tok) * heads + head) * a.d;
                            if (!prompt_marked_lost(a, first + c0))
                                for (int e = c0; e < c1 && !bad; ++e) bad = prompt_odd<T>(a, first + e);
                        }
                        for (unsigned todo = __ballot_sync(0xffffffffu, bad); todo; todo &= todo - 1) {
                            const int src = __ffs(todo) - 1;
                            prompt_mend_row<T>(a, s, pos.b, __shfl_sync(0xffffffffu, tok, src), __shfl_sync(0xffffffffu, head, src), lane, c0, c1, odd);
                        }
                    }
                }
                pos = next_pos<WIDE>(a, s, pos);
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
        if (warp == 8) tile_land(full, SLOTS, flight, false);
        if (warp == 10 && (PLAIN || a.q_boxes)) tile_land(q_full, 2, flight, false);
        if (!PLAIN && warp == 10 && a.q_shifted) tile_land(q_come, 1, flight >> 2, false);
    }
}

constexpr int kTileMergeThreads = 256;
// The rows `mend` (token, query head; token -1: none) of a cut item of sequence b and key head h, by a block: its warps look at a part of K and V each, and
// one mends the rows.
template <typename T>
__device__ __noinline__ void prompt_mend_block(const PromptArgs &a, const int2 *mend, int (*firsts)[32], int b, int h, int lane, int warp, int c0, int c1)
{
    for (int i = threadIdx.x; i < 13 * 32; i += kTileMergeThreads) firsts[i / 32][i % 32] = kOddNone;
    const PromptSeq whole = prompt_seq(a, b);
    int last = -1;                                                 // of the tokens
    for (int w = 0; w < kTileMergeThreads / 32; ++w) last = max(last, mend[w].x);
    const int n = whole.p + whole.seen(last, a.causal), part = (n + kTileMergeThreads / 32 - 1) / (kTileMergeThreads / 32), from = min(warp * part, n), to = min(from + part, n);
    PromptOdd odd;
    odd.reset(b, h);
    odd.whole = false;
    __syncthreads();
    {
        int first[4][3];
#pragma unroll
        for (int e = 0; e < 12; ++e) first[e / 3][e % 3] = kOddNone;
        if (!a.shifted) {
            prompt_look_v<T>(a, whole, b, h, 0, min(n, 32), lane, c0, c1, first);   // (every column may have its NaN there)
            prompt_look_v<T>(a, whole, b, h, from, to, lane, c0, c1, first);
        }
#pragma unroll
        for (int e = 0; e < 12; ++e)
            if (first[e / 3][e % 3] != kOddNone) atomicMin(&firsts[e][lane], first[e / 3][e % 3]);
    }
    __syncthreads();
    bool infinite = false;                                         // of a column: K decides
#pragma unroll
    for (int e = 0; e < 12; ++e) odd.first[e / 3][e % 3] = firsts[e][lane];
#pragma unroll
    for (int e = 0; e < 4; ++e) infinite = infinite || (odd.first[e][0] == kOddNone && min(odd.first[e][1], odd.first[e][2]) != kOddNone);
    if (a.shifted || __any_sync(0xffffffffu, infinite)) {          // (the same for all warps)
        const int k_first = a.shifted ? prompt_look_k<T, true>(a, whole, b, h, from, to, lane) : prompt_look_k<T, false>(a, whole, b, h, from, to, lane);
        if (k_first != kOddNone) atomicMin(&firsts[12][lane], k_first);
        __syncthreads();
        odd.k_first = firsts[12][lane];
        odd.k_rows = n;
    }
    if (warp) return;
    odd.rows = n;
    for (int w = 0; w < kTileMergeThreads / 32; ++w) {
        const int2 which = mend[w];
        if (which.x >= 0) prompt_mend_row<T>(a, whole, b, which.x, which.y, lane, c0, c1, odd);
    }
}

// Joins the states of items that runs have cut: a warp per row, blocks (cut, eight rows).  The run that began such an item
// names it; the runs behind it have one state each, up to the one that ended the item.  Rows of a block that are to be mended are so by one warp, after all
// have looked at a part of K and V for them.
template <typename T, int NSUB, bool FEW>
__global__ void __launch_bounds__(kTileMergeThreads, 4)
prompt_tile_merge_kernel(const __grid_constant__ PromptArgs a, int runs)
{
    constexpr bool WIDE = NSUB > 2;                                // (the kernel for few rows: items of one half of up to 64 rows)
    constexpr int DO = WIDE ? 128 : 64 * NSUB, PER = DO / 32, AHEAD = 4;
    __shared__ int2 mend[kTileMergeThreads / 32];                  // token, query head; token -1: nothing to mend
    __shared__ int firsts[13][32];                                 // (of prompt_mend_block)
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, r = (int)blockIdx.y * (kTileMergeThreads / 32) + warp;
    pdl_wait();
    pdl_launch();
    const int lead = blockIdx.x;
    const int4 d = a.run_desc[2 * lead];
    if (d.x < 0 || d.w & 2) return;
    const int4 d2 = a.run_desc[2 * lead + 1];
    PromptSeq s = {};
    s.q0 = d2.x;
    s.m = d2.y;
    s.n = d2.z;
    s.p = d2.w;
    const TileItem<WIDE || FEW> item(a, s, d.z);
    const int half = r >> 7, tph = a.half_tokens, in = a.by_per_kv(r & 127), in_item = in + (WIDE ? 0 : half * tph);   // (half: the same for a block)
    int pieces = 1;
    for (int w = 0; lead + pieces < runs && !w; ++pieces) {
        w = a.run_desc[2 * (lead + pieces)].w;
        if (w & 2) return;                                         // a block that gave up has left no state
    }
    const bool there = in < tph && in_item < item.count && !(half && !WIDE && !item.pair);
    const int c0 = WIDE ? half * DO : 0, c1 = min(a.d, c0 + DO);
    bool bad = false;
    if (there) {
        const int tok = item.first + in_item, head = d.y * a.per_kv + (r & 127) - in * a.per_kv;
        float m = -INFINITY, l = 0.f, o[PER];
#pragma unroll
        for (int e = 0; e < PER; ++e) o[e] = 0.f;
        for (int i0 = 0; i0 < pieces; i0 += AHEAD) {
            float2 ml[AHEAD];
            float x[AHEAD][PER];
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                const int i = i0 + k;
                ml[k] = make_float2(-INFINITY, 0.f);
                if (i < pieces) {
                    const size_t slot = (size_t)2 * (lead + i) + (i == 0 ? 1 : 0);
                    ml[k] = *reinterpret_cast<const float2 *>(a.state_ml + 2 * (slot * 256 + r));
                    // a lane has PER neighbouring elements
                    const float *from = a.state + (slot * (DO / 4) + lane * PER / 4) * 1024 + r * 4 + lane * PER % 4;
                    if constexpr (PER == 4) *reinterpret_cast<float4 *>(x[k]) = *reinterpret_cast<const float4 *>(from);
                    else *reinterpret_cast<float2 *>(x[k]) = *reinterpret_cast<const float2 *>(from);
                }
            }
#pragma unroll
            for (int k = 0; k < AHEAD; ++k) {
                if (i0 + k >= pieces) continue;
                const float M = fmaxf(m, ml[k].x), w1 = m == -INFINITY ? 0.f : pa_exp2(m - M), w2 = ml[k].x == -INFINITY ? 0.f : pa_exp2(ml[k].x - M);
                l = l * w1 + ml[k].y * w2;
#pragma unroll
                for (int e = 0; e < PER; ++e) o[e] = o[e] * w1 + x[k][e] * w2;
                m = M;
            }
        }
        const bool none = s.p + s.seen(tok, a.causal) == 0;
        const float inv = none ? 0.f : 1.f / l;
        const size_t row = ((size_t)s.q0 + tok) * a.kv_heads * a.per_kv + head;
#pragma unroll
        for (int e = 0; e < PER; e += 2) {
            const int at = c0 + lane * PER + e;
            if (at >= c1) continue;
            const float2 x = none ? make_float2(0.f, 0.f) : make_float2(o[e] * inv, o[e + 1] * inv);
            bad = bad || !prompt_fits<T>(x.x) || !prompt_fits<T>(x.y);
            if (a.out) *reinterpret_cast<uint32_t *>((T *)a.out + row * a.d + at) = pack2<T>(x.x, x.y);
            if (a.out_f32) *reinterpret_cast<float2 *>(a.out_f32 + row * a.d + at) = x;
        }
        if (a.lse && lane == 0 && c0 == 0) a.lse[row] = none ? -INFINITY : (m + log2f(l)) * 0.693147180559945309f;
        bad = __any_sync(0xffffffffu, bad) && !prompt_lost(a, l);
        if (lane == 0) mend[warp] = make_int2(bad ? tok : -1, head);
    } else if (lane == 0) {
        mend[warp] = make_int2(-1, 0);
    }
    // (lanes look at what others wrote)
    if (__syncthreads_or(bad)) prompt_mend_block<T>(a, mend, firsts, d.x, d.y, lane, warp, c0, c1);
}

size_t prompt_workspace(int head_dim, int sms, PromptArgs *a, void *workspace)
{
    const auto up = [](size_t x) { return (x + 255) & ~(size_t)255; };
    const size_t rows = (size_t)2 * sms * 256, desc = up((size_t)sms * 2 * sizeof(int4)), state = up(rows * (head_dim <= 64 ? 64 : 128) * 4);
    if (a) {
        unsigned char *const w = (unsigned char *)workspace;
        a->run_desc = (int4 *)w;
        a->state = (float *)(w + desc);
        a->state_ml = (float *)(w + desc + state);
    }
    return desc + state + up(rows * 8);
}

namespace {

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
bool encode(CUtensorMap *m, int dtype, int rank, const void *at, const cuuint64_t *dims, const cuuint64_t *strides, const cuuint32_t *box)
{
    const encode_t fn = encoder();
    const cuuint32_t estr[3] = {1, 1, 1};
    return fn && fn(m, dtype == ADSA_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, (cuuint32_t)rank, const_cast<void *>(at), dims,
                    strides, box, estr, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                    CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}
// Rows of heads and tokens as boxes of heads x tokens rows of 64 elements; heads before tokens, or (one head to a box) the other way
// round, where that makes strides ascend.  False: not aligned as a box has to be.
bool rows_map(CUtensorMap *m, int dtype, const void *at, int d, long long n_heads, long long head, long long n_tokens, long long token, int box_heads,
              int box_tokens, bool *tokens_first)
{
    if (((uintptr_t)at & 15) || head % 8 || token % 8 || head <= 0 || token <= 0 || n_tokens < 1) return false;
    const bool tf = box_heads == 1 && token < head;
    const cuuint64_t h = (cuuint64_t)n_heads, t = (cuuint64_t)n_tokens, hs = (cuuint64_t)head * 2, ts = (cuuint64_t)token * 2;
    const cuuint64_t dims[3] = {(cuuint64_t)d, tf ? t : h, tf ? h : t}, strides[2] = {tf ? ts : hs, tf ? hs : ts};
    const cuuint32_t box[3] = {64, (cuuint32_t)(tf ? box_tokens : box_heads), (cuuint32_t)(tf ? box_heads : box_tokens)};
    *tokens_first = tf;
    return encode(m, dtype, 3, at, dims, strides, box);
}
// Rows whose heads begin at any even element, out of 16-byte aligned tokens: boxes of 64 elements x 128 tokens of the whole row.
bool shifted_map(CUtensorMap *m, int dtype, const void *at, int d, long long n_heads, long long head, long long n_tokens, long long token)
{
    if (((uintptr_t)at & 15) || token % 8 || token > 0x7fffffff || head <= 0 || (n_heads - 1) * head + d > token || n_tokens < 1) return false;
    const cuuint64_t dims[2] = {(cuuint64_t)((n_heads - 1) * head + d), (cuuint64_t)n_tokens}, strides[1] = {(cuuint64_t)token * 2};
    const cuuint32_t box[2] = {64, kTileRows};
    return encode(m, dtype, 2, at, dims, strides, box);
}
bool page_map(CUtensorMap *m, int dtype, const PromptArgs &a, const void *pool, int box_rows)
{
    const cuuint64_t dims[2] = {(cuuint64_t)a.d, (cuuint64_t)a.n_pages * a.kv_heads * a.page_rows}, strides[1] = {(cuuint64_t)a.row_stride * 2};
    const cuuint32_t box[2] = {64, (cuuint32_t)box_rows};
    return encode(m, dtype, 2, pool, dims, strides, box);
}

template <typename T, int NSUB, bool FEW>
cudaError_t launch_merge(const PromptArgs &a, unsigned blocks, cudaStream_t st)
{
    return launch_pdl(prompt_tile_merge_kernel<T, NSUB, FEW>, dim3(blocks - 1, (FEW ? kFewRows : 256) / (kTileMergeThreads / 32)), kTileMergeThreads, 0, st, a, (int)blocks);
}

template <typename T, int NSUB, int SLOTS, bool PLAIN>
cudaError_t launch_tiles(const PromptArgs &a, unsigned blocks, const CUtensorMap &qm, const CUtensorMap &km, const CUtensorMap &vm, cudaStream_t st)
{
    constexpr size_t tile = (size_t)kTileRows * 128, q = (NSUB > 2 ? 1 : 2) * NSUB * tile, slot = (NSUB > 2 ? 2 : NSUB) * tile;
    constexpr size_t fixed = 1024 + q + SLOTS * slot + 8 * 32 * kTileStage * 2 + sizeof(TileControl), most = 227 * 1024;
    static_assert(2 * SLOTS + 28 <= 44, "barriers");
    const size_t smem = fixed + tile_list_bytes(a.batch);
    if (smem > most) return cudaErrorInvalidValue;                 // (not with the batches that the calls take)
    const auto kern = prompt_tile_kernel<T, NSUB, SLOTS, PLAIN>;
    static int told[64];
    cudaError_t e = tile_allow_smem((const void *)kern, told, most);
    if (e != cudaSuccess) return e;
    e = launch_pdl(kern, dim3(blocks), kTileThreads, smem, st, a, qm, km, vm);
    if (e != cudaSuccess || !a.split || blocks < 2) return e;
    return launch_merge<T, NSUB, false>(a, blocks, st);
}
template <typename T, bool PLAIN>
cudaError_t launch_tiles_type(const PromptArgs &a, unsigned blocks, const CUtensorMap &qm, const CUtensorMap &km, const CUtensorMap &vm, cudaStream_t st)
{
    if (a.d <= 64) return launch_tiles<T, 1, 8, PLAIN>(a, blocks, qm, km, vm, st);
    if (a.d <= 128) return launch_tiles<T, 2, 4, PLAIN>(a, blocks, qm, km, vm, st);
    return launch_tiles<T, 4, 4, PLAIN>(a, blocks, qm, km, vm, st);
}

}  // namespace

// Whether items are cut for an even share of each block.  Uncut, the blocks that have an item less than others wait for up to one item (half
// of one, where they have many); cut, a second kernel and the states take some 9 us.  By the items there are, sequences of mean length, and the
// tiles that tables (or the mean sequence) have room for, us a tile each.  Measured, uncut / cut in us: one token x 2 x 12 heads of 64 over 128
// rows 7.0 / 9.9, 1024 10.6 / 12.4, 2048 14.9 / 13.0; x 32 x 20 over 1144 42.9 / 49.0, 2048 60.6 / 61.8; 5 tokens x 8 x 8 key heads of 128 over up
// to 16384 94.7 / 59.5; prompts of 2 x 128 x 12 heads of 64 7.7 / 15.3, of 16 x 512 x 8 key heads of 128 62 / 69, of 16384 x 4 1036 / 948.
static bool cuts_pay(const PromptArgs &a, unsigned blocks, int item_tokens, double us_a_tile)
{
    const double mean = (double)a.n_q / a.batch, rows = a.table ? ((double)a.max_pages + (a.groups ? a.max_p_pages : 0)) * a.page_rows : (double)a.n_k / a.batch;
    const double share = a.batch * fmax(1.0, ceil(mean / item_tokens)) * a.kv_heads / blocks;   // items a block
    const double item = ceil(rows / kTileRows) * us_a_tile + 3.0;
    return item * (share <= 1.0 ? 1.0 - share : fmin(ceil(share) - share, 0.5)) > 9.0;
}

cudaError_t launch_prompt_tiles(int dtype, const PromptArgs &args, int sms, cudaStream_t st)
{
    PromptArgs a = args;
    a.half_tokens = kTileRows / a.per_kv;
    a.by_per_kv = FastDiv((uint32_t)a.per_kv);
    a.by_page = FastDiv((uint32_t)max(a.page_rows, 1));
    CUtensorMap qm = {}, km = {}, vm = {};
    const int heads = a.kv_heads * a.per_kv;
    bool tf = false;
    a.q_boxes = rows_map(&qm, dtype, a.q, a.d, heads, a.q_head, a.n_q, a.q_token, a.per_kv, kTileRows / a.per_kv, &tf) && !tf;
    a.tokens_first = 0;
    a.box_rows = 0;
    if (a.table) {
        int box = kTileRows;
        while (a.page_rows % box) box /= 2;                        // the largest power of two that divides a page: boxes never straddle two
        if (page_map(&km, dtype, a, a.k, box) && page_map(&vm, dtype, a, a.v, box)) a.box_rows = box;
        while (1 << a.box_shift < box) ++a.box_shift;
    } else {
        bool kt = false, vt = false;
        if (rows_map(&km, dtype, a.k, a.d, a.kv_heads, a.k_head, a.n_k, a.k_token, 1, kTileRows, &kt) &&
            rows_map(&vm, dtype, a.v, a.d, a.kv_heads, a.v_head, a.n_k, a.v_token, 1, kTileRows, &vt)) {
            a.box_rows = kTileRows;                                // (the shift is a pool's)
            a.tokens_first = (kt ? 2 : 0) | (vt ? 4 : 0);
        } else if ((a.d <= 58 || (a.d > 64 && a.d <= 112)) && shifted_map(&km, dtype, a.k, a.d, a.kv_heads, a.k_head, a.n_k, a.k_token) &&
                   shifted_map(&vm, dtype, a.v, a.d, a.kv_heads, a.v_head, a.n_k, a.v_token)) {
            a.box_rows = kTileRows;                                // (elements of a head and the 6 before it fit its columns, in steps of 16)
            a.shifted = 1;
            a.q_boxes = 0;                                         // (q has to lie where the head's elements do, between zeros)
            a.q_shifted = a.per_kv == 1 && (a.q_head - a.k_head) % 8 == 0 && shifted_map(&qm, dtype, a.q, a.d, heads, a.q_head, a.n_q, a.q_token);
        }
    }
    const unsigned blocks = (unsigned)sms;
    // Few rows a sequence, on the mean (lengths lie on the device: a long sequence among many single tokens goes by items of 32 rows, which read its cache
    // eight times as often as items of 256; 255 single tokens over 1000 rows beside 1024 over 4096: 342 us, 161 + 92 in two calls).  Measured, this kernel / the other in us: 32 sequences x 20 heads of 64 over 600 rows, 8 rows each 30.1 /
    // 42.4, 32 rows 32.3 / 42.3, 48 rows (by two items) 44.4 / 43.1; 8 x 8 key heads of 128 over 8000 rows, 8 rows 50.8 / 55.2, 32 rows 52.1 /
    // 57.0, 48 rows 68.3 / 58.1.
    if (a.box_rows && !a.shifted && a.d <= 128 && a.per_kv <= kFewRows && a.n_q * a.per_kv <= (long long)kFewMean * a.batch) {
        a.half_tokens = kFewRows / a.per_kv;
        a.split = cuts_pay(a, blocks, kFewRows / a.per_kv, a.d <= 64 ? 0.6 : 1.2);
        const cudaError_t e = launch_prompt_few(dtype, a, blocks, km, vm, st);
        if (e != cudaSuccess || !a.split || blocks < 2) return e;
        if (dtype == ADSA_BF16) return a.d <= 64 ? launch_merge<__nv_bfloat16, 1, true>(a, blocks, st) : launch_merge<__nv_bfloat16, 2, true>(a, blocks, st);
        return a.d <= 64 ? launch_merge<__half, 1, true>(a, blocks, st) : launch_merge<__half, 2, true>(a, blocks, st);
    }
    a.split = cuts_pay(a, blocks, (a.d > 128 ? 1 : 2) * a.half_tokens, a.d <= 64 ? 1.4 : 1.9);
    const bool plain = a.q_boxes && a.box_rows && !a.shifted && a.out && !a.out_f32 && a.d % 16 == 0 && ((uintptr_t)a.out & 31) == 0;
    if (dtype == ADSA_BF16) return plain ? launch_tiles_type<__nv_bfloat16, true>(a, blocks, qm, km, vm, st) : launch_tiles_type<__nv_bfloat16, false>(a, blocks, qm, km, vm, st);
    return plain ? launch_tiles_type<__half, true>(a, blocks, qm, km, vm, st) : launch_tiles_type<__half, false>(a, blocks, qm, km, vm, st);
}

}  // namespace adsa
