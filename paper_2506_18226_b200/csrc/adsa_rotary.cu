// Rotary positions with several axes, on their own (adsa_rope_axes) and on the way into a paged cache
// (adsa_paged_append).
//
// Pair i of a head turns by phi = pos[axis(i)] * theta_i: (a, b) -> (a cos - b sin, a sin + b cos).  The angle is
// taken as turns: pos * (theta_i / 2 pi) in 64 bits, the whole turns dropped, the rest (at most half a turn, so 2^-25
// of a turn of error) handed to sincospif in 32 bits.  A position of a million times a frequency of one would keep only
// four bits of its turn's fraction in 32 bits.
//
// Both operators move every byte once, so HBM bounds them; the sines are what could cost more.  A thread owns a few
// pairs of ONE token and walks the heads with them: one sine and cosine per pair and token, whatever the number of
// heads, and the accesses of a warp stay whole 128-byte lines (the units of a head lie side by side).
#include <math.h>

#include "adsa_half.cuh"

namespace adsa {

constexpr int kTurnThreads = 256;
constexpr int kTurnMaxPairs = ADSA_MAX_HEAD_DIM / 2;

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
    int head_chunk;          // heads a block walks
    int d, n, n_axes;        // head elements, rotated pairs, axes
    int rot_units, units;    // units of a head that turn (halves only), all of them
};

// the row of `cu` (offsets, [batch + 1]) that holds token t: the last b with cu[b] <= t
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

template <typename T, int ACC, bool HALVES, bool ROTATE>
__device__ __forceinline__ void turn_heads(const T *src, T *dst, long long src_head, long long dst_head, int count, int e0, int e1,
                                           const float (&cs)[ACC], const float (&sn)[ACC], int turned)
{
    typedef Pack<T, ACC> P;
#pragma unroll 4
    for (int h = 0; h < count; ++h) {
        const T *s = src + h * src_head;
        T *o = dst + h * dst_head;
        P a = *reinterpret_cast<const P *>(s + e0);
        if constexpr (HALVES || ACC == 1) {        // a second access: the partner elements (e1 < 0: a lone copied piece)
            if (e1 >= 0) {
                P b = *reinterpret_cast<const P *>(s + e1);
                if (ROTATE) {
#pragma unroll
                    for (int i = 0; i < ACC; ++i) {
                        if (i >= turned) break;
                        const float x = to_f32(a.e[i]), y = to_f32(b.e[i]);
                        a.e[i] = from_f32<T>(x * cs[i] - y * sn[i]);
                        b.e[i] = from_f32<T>(x * sn[i] + y * cs[i]);
                    }
                }
                *reinterpret_cast<P *>(o + e1) = b;
            }
        } else if (ROTATE) {
#pragma unroll
            for (int i = 0; i < ACC / 2; ++i) {
                if (i < turned) {
                    const float x = to_f32(a.e[2 * i]), y = to_f32(a.e[2 * i + 1]);
                    a.e[2 * i] = from_f32<T>(x * cs[i] - y * sn[i]);
                    a.e[2 * i + 1] = from_f32<T>(x * sn[i] + y * cs[i]);
                }
            }
        }
        *reinterpret_cast<P *>(o + e0) = a;
    }
}

// A unit of a head is ACC neighbouring elements (pairs side by side; with ACC = 1 a pair is two accesses), or ACC
// elements and their partners half a rotation further on.  blockIdx.y: a chunk of the q, k and v heads taken as one list.
template <typename T, int ACC, bool HALVES>
__global__ void __launch_bounds__(kTurnThreads)
turn_kernel(const __grid_constant__ TurnArgs a, const __grid_constant__ adsa_rotary rot)
{
    pdl_wait();
    pdl_launch();
    const long long idx = (long long)blockIdx.x * kTurnThreads + threadIdx.x;
    long long t;
    int u;
    if (a.tokens * a.units <= 0x7fffffffLL) { t = (uint32_t)idx / (uint32_t)a.units; u = (int)((uint32_t)idx - (uint32_t)t * (uint32_t)a.units); }
    else { t = idx / a.units; u = (int)(idx - t * a.units); }
    if (t >= a.tokens) return;

    // where the token's rows go
    long long cache_row = -1;            // ((page * heads) * page_rows + row) without the head, in rows
    int page = 0;
    if (a.page_table) {
        int b, j;
        if (a.cu_tokens) {
            b = find_row(a.cu_tokens, a.batch, t);
            if (b >= a.batch || t < a.cu_tokens[b] || t >= a.cu_tokens[b + 1]) return;   // padding behind or before the rows
            j = (int)(t - a.cu_tokens[b]);
        } else {
            b = (int)(t / a.per_row);
            j = (int)(t - (long long)b * a.per_row);
        }
        const long long row = (long long)a.n_rows[b] + j;
        const long long pg = row / a.page_rows;
        if (a.n_rows[b] < 0 || pg >= a.max_pages) {
            if (a.status && u == 0 && blockIdx.y == 0) atomicOr(a.status, ADSA_DEV_ROW_OVERFLOW);
        } else {
            page = a.page_table[(size_t)b * a.max_pages + pg];
            if (page < 0 || page >= a.n_pages) {
                if (a.status && u == 0 && blockIdx.y == 0) atomicOr(a.status, ADSA_DEV_BAD_PAGE);
            } else {
                cache_row = row - pg * a.page_rows;
            }
        }
    }

    // which elements, which pairs
    int e0, e1 = -1, pair0 = 0, turned = 0;
    if constexpr (HALVES) {
        if (u < a.rot_units) { e0 = u * ACC; e1 = e0 + a.n; pair0 = e0; turned = ACC; }
        else e0 = 2 * a.n + (u - a.rot_units) * ACC;
    } else if constexpr (ACC == 1) {
        e0 = 2 * u; e1 = e0 + 1; pair0 = u; turned = u < a.n ? 1 : 0;
    } else {
        e0 = u * ACC; pair0 = e0 / 2;
        turned = a.n - pair0;
        turned = turned < 0 ? 0 : turned > ACC / 2 ? ACC / 2 : turned;
    }
    const int h0 = blockIdx.y * a.head_chunk, h1 = min(h0 + a.head_chunk, a.q.heads + a.k.heads + a.v.heads);
    const int k_first = a.q.heads, v_first = a.q.heads + a.k.heads;
    float cs[ACC], sn[ACC];
    if (h0 < v_first) {                  // (v does not turn)
#pragma unroll
        for (int i = 0; i < ACC; ++i) {
            cs[i] = 1.f; sn[i] = 0.f;
            if (i < turned) {
                const double turns = (double)a.pos[t * a.n_axes + rot.axis[pair0 + i]] * rot.turns[pair0 + i];
                sincospif((float)(2.0 * (turns - rint(turns))), &sn[i], &cs[i]);
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < ACC; ++i) { cs[i] = 1.f; sn[i] = 0.f; }
    }

    if (h0 < k_first) {
        const int n = min(h1, k_first) - h0;
        const T *s = (const T *)a.q.src + t * a.q.src_token + h0 * a.q.src_head;
        T *o = (T *)a.q.dst + t * a.q.dst_token + h0 * a.q.dst_head;
        turn_heads<T, ACC, HALVES, true>(s, o, a.q.src_head, a.q.dst_head, n, e0, e1, cs, sn, turned);
    }
    if (cache_row < 0) return;
    const long long head_rows = (long long)a.page_rows * a.row_stride;
    if (h0 < v_first && h1 > k_first) {
        const int f = max(h0, k_first) - k_first, n = min(h1, v_first) - k_first - f;
        const T *s = (const T *)a.k.src + t * a.k.src_token + f * a.k.src_head;
        T *o = (T *)a.k.dst + ((long long)page * a.k.heads + f) * head_rows + cache_row * a.row_stride;
        turn_heads<T, ACC, HALVES, true>(s, o, a.k.src_head, head_rows, n, e0, e1, cs, sn, turned);
        if (u == 0)
            for (int h = 0; h < n; ++h)
                for (int e = a.d; e < a.row_stride; ++e) o[h * head_rows + e] = from_f32<T>(0.f);
    }
    if (h1 > v_first) {
        const int f = max(h0, v_first) - v_first, n = h1 - v_first - f;
        const T *s = (const T *)a.v.src + t * a.v.src_token + f * a.v.src_head;
        T *o = (T *)a.v.dst + ((long long)page * a.v.heads + f) * head_rows + cache_row * a.row_stride;
        turn_heads<T, ACC, HALVES, false>(s, o, a.v.src_head, head_rows, n, e0, e1, cs, sn, 0);
        if (u == 0)
            for (int h = 0; h < n; ++h)
                for (int e = a.d; e < a.row_stride; ++e) o[h * head_rows + e] = from_f32<T>(0.f);
    }
}

namespace {

// the widest access every row of `r` allows, at most `acc` elements
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
cudaError_t launch_turn(const TurnArgs &a, const adsa_rotary &rot, int acc, bool halves, dim3 grid, cudaStream_t st)
{
#define ADSA_TURN(A) \
    if (acc == A) return halves ? launch_pdl(turn_kernel<T, A, true>, grid, kTurnThreads, 0, st, a, rot) \
                                : launch_pdl(turn_kernel<T, A, false>, grid, kTurnThreads, 0, st, a, rot)
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
    const int heads = a.q.heads + a.k.heads + a.v.heads;
    const long long blocks = (a.tokens * a.units + kTurnThreads - 1) / kTurnThreads;
    if (blocks > 0x7fffffffLL) return ADSA_EINVAL;
    // Few tokens: a block per head, so that the call is one load deep; many: a thread keeps its sines for many heads.
    // 148 SMs hold eight blocks each.
    int chunk = heads;
    while (chunk > 1 && blocks * ((heads + chunk - 1) / chunk) < 148 * 8) chunk = (chunk + 1) / 2;
    if ((heads + chunk - 1) / chunk > 65535) chunk = (heads + 65534) / 65535;
    a.head_chunk = chunk;
    const dim3 grid((unsigned)blocks, (unsigned)((heads + chunk - 1) / chunk));
    const cudaError_t e = dtype == ADSA_BF16 ? launch_turn<__nv_bfloat16>(a, rot, acc, halves, grid, st) : launch_turn<__half>(a, rot, acc, halves, grid, st);
    return e == cudaSuccess ? ADSA_OK : ADSA_ECUDA;
}

bool rotary_ok(const adsa_rotary *r)
{
    return r && r->head_dim >= 2 && r->head_dim <= ADSA_MAX_HEAD_DIM && r->head_dim % 2 == 0 && r->n_axes >= 1 && r->n_axes <= 4 &&
           r->n_pairs >= 0 && 2 * r->n_pairs <= r->head_dim;
}

bool rows_ok(const TurnRows &r) { return r.src && r.dst && !(((uintptr_t)r.src | (uintptr_t)r.dst) & 1); }

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
    if (!rows_ok(a.q) || !pos || ((uintptr_t)pos & 3)) return ADSA_EINVAL;
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
    if ((n_heads && !rows_ok(a.q)) || !rows_ok(a.k) || !rows_ok(a.v)) return ADSA_EINVAL;
    a.pos = pos;
    a.page_table = page_table; a.n_rows = n_rows; a.cu_tokens = cu_tokens; a.status = status;
    a.tokens = n_tokens; a.per_row = (int)(n_tokens / batch);
    a.batch = batch; a.max_pages = max_pages; a.n_pages = kv->n_pages;
    a.page_rows = kv->page_rows; a.row_stride = kv->row_stride;
    return run_turn(a, rot ? *rot : none, kv->dtype, (cudaStream_t)stream);
}

}  // extern "C"
