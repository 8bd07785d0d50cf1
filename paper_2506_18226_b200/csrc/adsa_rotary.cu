// Rotary positions with several axes, on their own (adsa_rope_axes) and on the way into a paged cache
// (adsa_paged_append).
//
// Pair i of a head turns by phi = pos[axis(i)] * theta_i: (a, b) -> (a cos - b sin, a sin + b cos).  The angle is
// taken as turns: pos * (theta_i / 2 pi) in 64 bits, the whole turns dropped, the rest (at most half a turn, so 2^-25
// of a turn of error) handed to sincospif in 32 bits.  A position of a million times a frequency of one would keep only
// four bits of its turn's fraction in 32 bits.
//
// Both operators move every byte once, so HBM bounds them, and next the instructions per access.  A thread owns one unit
// of one head for all the tokens of its block: what it turns with lies at a fixed place of a table of sines and cosines
// that the block makes once per token in shared memory (whatever the number of heads), its addresses move on by a
// constant, and the block's accesses run through a token's heads in the order they lie in memory.
#include <math.h>

#include "adsa_half.cuh"

namespace adsa {

constexpr int kTurnMaxThreads = 512;
constexpr int kTurnMaxPairs = ADSA_MAX_HEAD_DIM / 2;
constexpr int kTurnMaxTokens = 16;         // tokens of a block

struct TurnRows {            // rows of one tensor, element strides
    const void *src;
    void *dst;
    long long src_token, src_head, dst_token, dst_head;
    int heads;
};

struct TurnArgs {
    TurnRows q, k, v;        // k, v: dst is the pool, dst_token unused; any of them may have heads = 0
    const int32_t *pos;      // [tokens][n_axes]
    const int32_t *page_table, *n_rows, *cu_tokens;   // null page_table: no cache (rope alone)
    uint32_t *status;
    long long tokens;
    int per_row;             // tokens per batch row where cu_tokens is null
    int batch, max_pages, n_pages, page_rows, row_stride;
    int tokens_block;        // tokens a block takes
    int head_chunk;          // heads it walks (blockIdx.y: which)
    int d, n, n_axes;        // head elements, rotated pairs, axes
    int rot_units, units;    // units of a head that turn (halves only), all of them
};

// the last b of 0 .. batch with cu[b] <= t (the row of offsets `cu` that holds token t)
__device__ __forceinline__ int find_row(const int32_t *cu, int batch, long long t)
{
    int lo = 0, hi = batch;
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if ((long long)__ldg(cu + mid) <= t) lo = mid;
        else hi = mid - 1;
    }
    return lo;
}

// The same by a warp, for the token t + lane of each lane (within[0], [1]: that row's offsets), in a third of the dependent reads: 32
// rows are looked at at once, and the tokens of a block lie within a few of them (64 rows of 2 to 17 tokens: 9.54 -> 9.37 us)
__device__ __forceinline__ int find_rows(const int32_t *cu, int batch, long long t, int lane, int2 &within)
{
    int lo = 0, hi = batch;
    while (lo < hi) {
        const int step = (hi - lo + 31) / 32, at = lo + (lane + 1) * step;
        const bool before = at <= hi && (long long)__ldg(cu + min(at, hi)) <= t;
        lo += __popc(__ballot_sync(0xffffffffu, before)) * step;
        hi = min(hi, lo + step - 1);
    }
    const int next = lo + lane <= batch ? __ldg(cu + lo + lane) : 0x7fffffff;
    int b = 0;
#pragma unroll
    for (int s = 16; s > 0; s >>= 1)
        if ((long long)__shfl_sync(0xffffffffu, next, b + s) <= t + lane) b += s;
    within = make_int2(__shfl_sync(0xffffffffu, next, b), __shfl_sync(0xffffffffu, next, min(b + 1, 31)));
    if (b == 31) {                                                 // maybe further on
        b = find_row(cu, batch, t + lane) - lo;
        within = make_int2(__ldg(cu + lo + b), lo + b < batch ? __ldg(cu + lo + b + 1) : 0x7fffffff);
    }
    return lo + b;
}

// A unit of a head is ACC neighbouring elements (pairs side by side; with ACC = 1 a pair is two accesses), or ACC
// elements and their partners half a rotation further on.  The table holds, for the pairs of a unit two by two, their
// cosines and sines {c, c', s, s'}: entry [two][unit], so that neighbouring threads read neighbouring 16 bytes.
template <typename T, int ACC, bool HALVES>
struct Piece {
    typedef Pack<T, ACC> P;
    static constexpr bool kTwo = HALVES || ACC == 1;               // two accesses
    static constexpr int kPairs = kTwo ? ACC : ACC / 2;            // pairs of a unit
    static constexpr int kTwos = (kPairs + 1) / 2;
    P a, b;

    __device__ __forceinline__ void load(const T *src, int partner)
    {
        a = *reinterpret_cast<const P *>(src);
        if constexpr (kTwo)
            if (partner) b = *reinterpret_cast<const P *>(src + partner);
    }
    __device__ __forceinline__ void store(T *dst, int partner) const
    {
        *reinterpret_cast<P *>(dst) = a;
        if constexpr (kTwo)
            if (partner) *reinterpret_cast<P *>(dst + partner) = b;
    }
    // table: the unit's entries of the token, `units` apart; turned: pairs of the unit that turn
    __device__ __forceinline__ void turn(const float4 *table, int units, int turned)
    {
        if (ACC > 1 && turned == kPairs) {
            uint32_t *wa = reinterpret_cast<uint32_t *>(&a), *wb = reinterpret_cast<uint32_t *>(&b);
#pragma unroll
            for (int i = 0; i < kTwos; ++i) {
                const float4 t = table[i * units];
                if constexpr (HALVES) {
                    const float2 c = make_float2(t.x, t.y), s = make_float2(t.z, t.w), x = unpack2<T>(wa[i]), y = unpack2<T>(wb[i]);
                    const float2 u = fma2(x, c, mul2(y, make_float2(-s.x, -s.y))), v = fma2(x, s, mul2(y, c));
                    wa[i] = pack2<T>(u.x, u.y);
                    wb[i] = pack2<T>(v.x, v.y);
                } else {
                    const float2 x = unpack2<T>(wa[2 * i]);
                    wa[2 * i] = pack2<T>(x.x * t.x - x.y * t.z, x.x * t.z + x.y * t.x);
                    if (2 * i + 1 < kPairs) {
                        const float2 y = unpack2<T>(wa[2 * i + 1]);
                        wa[2 * i + 1] = pack2<T>(y.x * t.y - y.y * t.w, y.x * t.w + y.y * t.y);
                    }
                }
            }
        } else {                                                   // single elements, or a unit where the rotation ends
#pragma unroll
            for (int i = 0; i < kPairs; ++i) {
                if (i < turned) {
                    const float4 t = table[(i >> 1) * units];
                    const float c = i & 1 ? t.y : t.x, s = i & 1 ? t.w : t.z;
                    T *pa = kTwo ? &a.e[i] : &a.e[2 * i], *pb = kTwo ? &b.e[i] : &a.e[2 * i + 1];
                    const float x = to_f32(*pa), y = to_f32(*pb);
                    *pa = from_f32<T>(x * c - y * s);
                    *pb = from_f32<T>(x * s + y * c);
                }
            }
        }
    }
};

// blockIdx.x: tokens; blockIdx.y: a chunk of the q, k and v heads taken as one list.  Accesses of fewer than 16 bytes need
// all the warps an SM has to keep memory busy: 32 registers (2424 tokens x 32 heads of 100 elements: 13.0 -> 11.1 us, 60 to 120
// bytes a thread of spills included).
template <typename T, int ACC, bool HALVES>
__global__ void __launch_bounds__(kTurnMaxThreads, ACC < 8 ? 4 : 0)
turn_kernel(const __grid_constant__ TurnArgs a, const __grid_constant__ adsa_rotary rot)
{
    typedef Piece<T, ACC, HALVES> PieceT;
    extern __shared__ float4 table[];                              // [tokens][twos of a unit][units]
    __shared__ int s_row[kTurnMaxTokens], s_page[kTurnMaxTokens];  // row in its page (-1: not placed, -2: padding), page
    __shared__ int s_pos[kTurnMaxTokens * 4];
    __shared__ double s_turns[kTurnMaxPairs];
    __shared__ uint8_t s_axis[kTurnMaxPairs];
    const long long t0 = (long long)blockIdx.x * a.tokens_block;
    const int tokens = (int)min((long long)a.tokens_block, a.tokens - t0);
    const int h0 = blockIdx.y * a.head_chunk, heads = min(a.head_chunk, a.q.heads + a.k.heads + a.v.heads - h0);
    const int k_first = a.q.heads, v_first = a.q.heads + a.k.heads;
    // this thread's head and unit
    const int u = (int)threadIdx.x % a.units, h = h0 + (int)threadIdx.x / a.units;
    const bool live = h < h0 + heads;
    const int kind = h < k_first ? 0 : h < v_first ? 1 : 2, head = h - (kind == 0 ? 0 : kind == 1 ? k_first : v_first);
    const TurnRows &r = kind == 0 ? a.q : kind == 1 ? a.k : a.v;
    int e0, partner = 0, turned = 0;
    if constexpr (HALVES) {
        if (u < a.rot_units) { e0 = u * ACC; partner = a.n; turned = ACC; }
        else e0 = 2 * a.n + (u - a.rot_units) * ACC;
    } else if constexpr (ACC == 1) {
        e0 = 2 * u; partner = 1; turned = u < a.n ? 1 : 0;
    } else {
        e0 = u * ACC;
        turned = max(0, min(a.n - e0 / 2, PieceT::kPairs));
    }
    if (kind == 2) turned = 0;
    const long long head_rows = (long long)a.page_rows * a.row_stride, src_token = r.src_token, dst_token = r.dst_token;
    const T *src = (const T *)r.src + t0 * src_token + head * r.src_head + e0;
    T *dst = (T *)r.dst + (kind == 0 ? t0 * dst_token + head * r.dst_head : head * head_rows) + e0;
    const long long page_elements = (kind == 0 ? 0 : r.heads) * head_rows;
    const bool turns_here = h0 < v_first && a.n > 0;              // (v does not turn)
    if (turns_here)
        for (int i = threadIdx.x; i < a.n; i += blockDim.x) { s_turns[i] = rot.turns[i]; s_axis[i] = rot.axis[i]; }
    pdl_wait();
    pdl_launch();
    // everything that comes from memory is asked for at once: the first two tokens' elements, positions, rows
    PieceT p, q;
    if (live) {
        p.load(src, partner);
        if (tokens > 1) q.load(src + src_token, partner);
    }
    if (turns_here)
        for (int i = threadIdx.x; i < tokens * a.n_axes; i += blockDim.x) s_pos[i] = a.pos[t0 * a.n_axes + i];
    if (a.page_table) {                                            // where the tokens' rows go
        int2 within;
        int b = 0;
        if (threadIdx.x < 32 && a.cu_tokens) b = find_rows(a.cu_tokens, a.batch, t0, (int)threadIdx.x, within);
        if (threadIdx.x < tokens) {
            const long long t = t0 + threadIdx.x;
            int j, row = -2, page = 0;
            if (a.cu_tokens) {
                j = b < a.batch && t >= within.x && t < within.y ? (int)(t - within.x) : -1;
            } else {
                b = (int)(t / a.per_row);
                j = (int)(t - (long long)b * a.per_row);
            }
            if (j >= 0) {
                row = -1;
                const int first = a.n_rows[b];
                const long long at = (long long)first + j, pg = at / a.page_rows;
                if (first < 0 || pg >= a.max_pages) {
                    if (a.status && blockIdx.y == 0) atomicOr(a.status, ADSA_DEV_ROW_OVERFLOW);
                } else {
                    page = a.page_table[(size_t)b * a.max_pages + pg];
                    if (page < 0 || page >= a.n_pages) {
                        if (a.status && blockIdx.y == 0) atomicOr(a.status, ADSA_DEV_BAD_PAGE);
                    } else {
                        row = (int)(at - pg * a.page_rows);
                    }
                }
            }
            s_row[threadIdx.x] = row;
            s_page[threadIdx.x] = page;
        }
    }
    __syncthreads();
    // the tokens' sines and cosines
    const int turn_units = HALVES ? a.rot_units : a.units;         // units of the table
    if (turns_here) {
        float *out = reinterpret_cast<float *>(table);
        for (int i = threadIdx.x; i < tokens * a.n; i += blockDim.x) {
            const int t = i / a.n, pair = i - t * a.n, unit = pair / PieceT::kPairs, in = pair - unit * PieceT::kPairs;
            const double turns = (double)s_pos[t * a.n_axes + s_axis[pair]] * s_turns[pair];
            float sn, cs;
            sincospif((float)(2.0 * (turns - rint(turns))), &sn, &cs);
            float *entry = out + 4 * ((t * PieceT::kTwos + (in >> 1)) * turn_units + unit) + (in & 1);
            entry[0] = cs;
            entry[2] = sn;
        }
        __syncthreads();
    }
    if (!live) return;
    const float4 *entries = table + u;
    const int token_entries = PieceT::kTwos * turn_units;
    const auto placed = [&](int t) { return !a.page_table || (kind == 0 ? s_row[t] != -2 : s_row[t] >= 0); };
    const auto finish = [&](PieceT &p, int t) {
        if (turned) p.turn(entries + t * token_entries, turn_units, turned);
        T *o = dst + (kind == 0 ? t * dst_token : s_page[t] * page_elements + (long long)s_row[t] * a.row_stride);
        p.store(o, partner);
        if (kind != 0 && u == 0)                                   // the row's padding
            for (int e = a.d; e < a.row_stride; ++e) o[e] = from_f32<T>(0.f);
    };
    // two tokens in hand, (padding is read and not written)
    for (int t = 0; t < tokens; t += 2) {
        if (t > 0) {
            p.load(src + t * src_token, partner);
            if (t + 1 < tokens) q.load(src + (t + 1) * src_token, partner);
        }
        if (placed(t)) finish(p, t);
        if (t + 1 < tokens && placed(t + 1)) finish(q, t + 1);
    }
}

namespace {

// the widest access every row of `r` allows, at most `acc` elements (q, k and v of a call share one: a tensor that is not aligned
// to 16 bytes, or whose strides are not, slows the others too)
int fit(int acc, const TurnRows &r)
{
    if (r.heads == 0) return acc;
    for (; acc > 1; acc /= 2) {
        const uintptr_t bytes = (uintptr_t)acc * 2;
        if (((uintptr_t)r.src | (uintptr_t)r.dst) % bytes) continue;
        if ((r.src_token | r.src_head | r.dst_token | r.dst_head) % acc) continue;
        break;
    }
    return acc;
}

template <typename T>
cudaError_t launch_turn(const TurnArgs &a, const adsa_rotary &rot, int acc, bool halves, dim3 grid, unsigned threads, size_t smem, cudaStream_t st)
{
#define ADSA_TURN(A) \
    if (acc == A) return halves ? launch_pdl(turn_kernel<T, A, true>, grid, threads, smem, st, a, rot) \
                                : launch_pdl(turn_kernel<T, A, false>, grid, threads, smem, st, a, rot)
    ADSA_TURN(8);
    ADSA_TURN(4);
    ADSA_TURN(2);
    ADSA_TURN(1);
#undef ADSA_TURN
    return cudaErrorInvalidValue;
}

int run_turn(TurnArgs &a, const adsa_rotary &rot, int dtype, cudaStream_t st)
{
    a.d = rot.head_dim;
    a.n = rot.n_pairs;
    a.n_axes = rot.n_axes;
    const bool halves = rot.halves != 0;
    int acc = 8;
    while (acc > 1 && (halves ? a.n % acc || a.d % acc : a.d % acc)) acc /= 2;
    acc = fit(fit(fit(acc, a.q), a.k), a.v);
    a.rot_units = halves ? a.n / acc : 0;
    a.units = halves ? a.rot_units + (a.d - 2 * a.n) / acc : acc == 1 ? a.d / 2 : a.d / acc;
    const long long all_heads = (long long)a.q.heads + a.k.heads + a.v.heads;
    if (all_heads * a.units > 65535LL * kTurnMaxThreads) return ADSA_EINVAL;      // (a chunk of heads takes up to that many units)
    const int heads = (int)all_heads;
    // Heads a block: all of them if they make up to 512 units, fewer until every SM has a block.  Tokens a block: as many as
    // would let all blocks run at once at 2048 threads on each of 148 SMs, at most 16: a second, thinner wave costs as much as
    // a full one.  (The forms of under 16 bytes hold that many; the 16-byte forms, with 54 and 64 registers, hold half, and
    // take a second wave where 16 tokens a block are not enough: a long prompt's 1152 blocks of 256 threads run as nearly two.)
    int chunks = (heads * a.units + kTurnMaxThreads - 1) / kTurnMaxThreads;
    while (chunks < heads && (heads + chunks - 1) / chunks * a.units > kTurnMaxThreads) ++chunks;
    while (chunks < heads && a.tokens * chunks < 148 && (heads + chunks - 1) / chunks * a.units > 128) ++chunks;
    const int chunk = (heads + chunks - 1) / chunks;
    chunks = (heads + chunk - 1) / chunk;
    const unsigned threads = (unsigned)((chunk * a.units + 31) / 32 * 32);
    const long long resident = 148 * (2048 / threads);
    long long tokens = (a.tokens * chunks + resident - 1) / resident;
    tokens = tokens < 1 ? 1 : tokens > kTurnMaxTokens ? kTurnMaxTokens : tokens;
    const long long blocks = (a.tokens + tokens - 1) / tokens;
    if (blocks > 0x7fffffffLL || chunks > 65535) return ADSA_EINVAL;
    a.tokens_block = (int)tokens;
    a.head_chunk = chunk;
    // table bytes: at most kTurnMaxTokens x 128 pairs x 8 (with one pair a unit half of an entry is not used)
    const int pairs = halves || acc == 1 ? acc : acc / 2;
    const size_t smem = (size_t)tokens * ((pairs + 1) / 2) * (halves ? a.rot_units : a.units) * 16;
    const dim3 grid((unsigned)blocks, (unsigned)chunks);
    const cudaError_t e = dtype == ADSA_BF16 ? launch_turn<__nv_bfloat16>(a, rot, acc, halves, grid, threads, smem, st) : launch_turn<__half>(a, rot, acc, halves, grid, threads, smem, st);
    return e == cudaSuccess ? ADSA_OK : ADSA_ECUDA;
}

bool rotary_ok(const adsa_rotary *r)
{
    if (!r || r->head_dim < 2 || r->head_dim > ADSA_MAX_HEAD_DIM || r->head_dim % 2 || r->n_axes < 1 || r->n_axes > 4 || r->n_pairs < 0 ||
        2 * r->n_pairs > r->head_dim)
        return false;
    for (int i = 0; i < r->n_pairs; ++i)
        if (r->axis[i] >= r->n_axes) return false;
    return true;
}

bool rows_ok(const TurnRows &r) { return r.src && r.dst && !(((uintptr_t)r.src | (uintptr_t)r.dst) & 1); }

// rows of d elements that a stride puts on top of each other (a tensor expanded along tokens or heads), to be written by several threads
bool rows_overlap(const TurnRows &r, long long tokens, int d)
{
    return (tokens > 1 && r.dst_token > -d && r.dst_token < d) || (r.heads > 1 && r.dst_head > -d && r.dst_head < d);
}

}  // namespace
}  // namespace adsa

using namespace adsa;

extern "C" {

int adsa_rotary_init(adsa_rotary *rot, int head_dim, int n_axes, const int32_t *pairs, int halves, int restart, double base)
{
    if (!rot || !pairs || head_dim < 2 || head_dim > ADSA_MAX_HEAD_DIM || head_dim % 2 || n_axes < 1 || n_axes > 4) return ADSA_EINVAL;
    if (base == 0.0) base = 10000.0;
    if (!(base > 0.0) || !isfinite(base)) return ADSA_EINVAL;
    int n = 0;
    for (int a = 0; a < n_axes; ++a) {
        if (pairs[a] < 0 || pairs[a] > kTurnMaxPairs) return ADSA_EINVAL;
        n += pairs[a];
    }
    if (n < 1 || 2 * n > head_dim) return ADSA_EINVAL;
    adsa_rotary r = {};
    r.head_dim = head_dim;
    r.n_axes = n_axes;
    r.n_pairs = n;
    r.halves = halves != 0;
    for (int a = 0, i = 0; a < n_axes; ++a) {
        for (int j = 0; j < pairs[a]; ++j, ++i) {
            const double exponent = restart ? (double)j / pairs[a] : (double)i / n;
            r.turns[i] = pow(base, -exponent) / 6.283185307179586476925286766559;
            r.axis[i] = (uint8_t)a;
        }
    }
    *rot = r;
    return ADSA_OK;
}

int adsa_rope_axes(const adsa_rotary *rot, int dtype, const void *x, long long x_token, long long x_head, const int32_t *pos,
                   long long n_tokens, int n_heads, void *out, long long out_token, long long out_head, adsa_stream_t stream)
{
    if (!rotary_ok(rot) || (dtype != ADSA_BF16 && dtype != ADSA_F16) || n_tokens < 0 || n_heads < 0) return ADSA_EINVAL;
    if (n_tokens == 0 || n_heads == 0) return ADSA_OK;
    TurnArgs a = {};
    a.q = {x, out, x_token, x_head, out_token, out_head, n_heads};
    if (!rows_ok(a.q) || rows_overlap(a.q, n_tokens, rot->head_dim) || !pos || ((uintptr_t)pos & 3)) return ADSA_EINVAL;
    if (x == out && (x_token != out_token || x_head != out_head)) return ADSA_EINVAL;
    a.pos = pos;
    a.tokens = n_tokens;
    return run_turn(a, *rot, dtype, (cudaStream_t)stream);
}

int adsa_paged_append(const adsa_paged_kv *kv, const int32_t *page_table, int batch, int max_pages, const int32_t *n_rows,
                      const int32_t *cu_tokens, long long n_tokens, const void *k, long long k_token, long long k_head, const void *v,
                      long long v_token, long long v_head, const adsa_rotary *rot, const int32_t *pos, const void *q, int n_heads,
                      long long q_token, long long q_head, void *q_out, long long q_out_token, long long q_out_head, uint32_t *status,
                      adsa_stream_t stream)
{
    if (!paged_kv_ok(kv) || batch < 1 || max_pages < 1 || n_tokens < 0 || n_heads < 0) return ADSA_EINVAL;
    if (rot && (!rotary_ok(rot) || rot->head_dim != kv->head_dim)) return ADSA_EINVAL;
    if (!cu_tokens && n_tokens % batch) return ADSA_EINVAL;
    if (n_tokens > 0x7fffffffLL) return ADSA_EINVAL;          // cu_tokens are 32-bit offsets
    if (n_tokens == 0) return ADSA_OK;
    if (!page_table || !n_rows || !k || !v || (rot && !pos) || (n_heads && (!q || !q_out))) return ADSA_EINVAL;
    if (((uintptr_t)page_table | (uintptr_t)n_rows | (uintptr_t)cu_tokens | (uintptr_t)pos | (uintptr_t)status) & 3) return ADSA_EINVAL;
    if (n_heads && q == q_out && (q_token != q_out_token || q_head != q_out_head)) return ADSA_EINVAL;
    adsa_rotary none = {};
    none.head_dim = kv->head_dim;
    none.n_axes = 1;
    TurnArgs a = {};
    a.q = {q, q_out, q_token, q_head, q_out_token, q_out_head, n_heads};
    a.k = {k, kv->k_pool, k_token, k_head, 0, 0, kv->n_kv_heads};
    a.v = {v, kv->v_pool, v_token, v_head, 0, 0, kv->n_kv_heads};
    if ((n_heads && (!rows_ok(a.q) || rows_overlap(a.q, n_tokens, kv->head_dim))) || !rows_ok(a.k) || !rows_ok(a.v)) return ADSA_EINVAL;
    a.pos = pos;
    a.page_table = page_table; a.n_rows = n_rows; a.cu_tokens = cu_tokens; a.status = status;
    a.tokens = n_tokens; a.per_row = (int)(n_tokens / batch);
    a.batch = batch; a.max_pages = max_pages; a.n_pages = kv->n_pages;
    a.page_rows = kv->page_rows; a.row_stride = kv->row_stride;
    return run_turn(a, rot ? *rot : none, kv->dtype, (cudaStream_t)stream);
}

}  // extern "C"
