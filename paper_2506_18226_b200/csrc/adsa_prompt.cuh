// What the kernels of adsa_packed_attn and adsa_chunk_attn share: their arguments, sequences as the device finds them, how the
// work is cut, and the attention of one query row by a warp.
#pragma once

#include "adsa_prefix.cuh"

namespace adsa {

// Division of numbers below 2^31 by a divisor that the host knows, by a product and a shift (Granlund and Montgomery 1994).
struct FastDiv {
    uint32_t mul, shift;
    FastDiv() = default;
    explicit FastDiv(uint32_t d)
    {
        shift = 0;
        while ((1ULL << shift) < d) ++shift;
        mul = (uint32_t)(((1ULL << 32) * ((1ULL << shift) - d)) / d + 1);
    }
    __device__ __forceinline__ int operator()(int n) const { return (int)((__umulhi(mul, (uint32_t)n) + (uint32_t)n) >> shift); }
};

struct PromptArgs {
    const void *q, *k, *v;                  // k, v: packed rows, or the pools
    long long q_token, q_head, k_token, k_head, v_token, v_head;   // element strides (k, v: of packed rows)
    const int32_t *cu_q, *cu_k;             // [batch + 1]; null: sequences of equal length
    // a paged cache: table != null
    const int32_t *table, *n_rows;          // [batch][max_pages], [batch]
    const int32_t *p_table, *p_rows, *start;   // [groups][max_p_pages], [groups], [groups + 1]
    uint32_t *status;
    long long n_q, n_k;                     // tokens of q; of packed k and v
    int batch, groups, kv_heads, per_kv;    // per_kv: query heads of a key head
    int max_pages, max_p_pages, page_rows, n_pages;
    int d, row_stride, causal;
    float scale_log2e;
    void *out;                              // 16-bit, or null
    float *out_f32, *lse;                   // or null
    int half_tokens;                        // of an item's half: 128 / per_kv
    FastDiv by_per_kv, by_page;
    // workspace: what each run leaves for the merge ({sequence of the item that it begins and leaves unfinished, or -1, key head, item, bit 0: an
    // item cut before ends here, bit 1: its block gave up a wait}, {that sequence's first token, tokens, own rows, rows of the prefix}), partial states [2 runs][16 or 32][256 rows][4 elements] and their (m, l)
    int4 *run_desc;
    float *state, *state_ml;
    int box_rows, box_shift;                // rows of a copy's box (a power of two, its logarithm); 0: K and V are copied row by row
    int q_boxes, tokens_first;              // q by boxes; the order in the maps of packed k (bit 1) and v (bit 2): tokens before heads
    int shifted, q_shifted;                 // packed k and v (q) by boxes that begin up to 7 elements before a head's row
    int split;                              // items may be cut (into partial states)
    int polls;                              // of a wait inside a kernel, before it gives up
};

// A sequence: its new tokens q0 .. q0 + m - 1, its own rows (k0 .. of packed ones), the prefix of its group.
struct PromptSeq {
    long long q0, k0;
    int m, n, p, group;
    // own rows that new token i attends
    __device__ __forceinline__ int seen(int i, int causal) const { return causal ? max(min(n - m + i + 1, n), 0) : n; }
};

// boundaries as given, kept inside 0 .. most and ascending for this sequence
__device__ __forceinline__ void prompt_range(const int32_t *cu, int b, int batch, long long most, long long &begin, int &count)
{
    long long lo, hi;
    if (cu) {
        lo = cu[b];
        hi = cu[b + 1];
    } else {
        const long long each = most / batch;
        lo = b * each;
        hi = lo + each;
    }
    begin = min(max(lo, 0LL), most);
    count = (int)(min(max(hi, begin), most) - begin);
}
__device__ __forceinline__ int prompt_group(const PromptArgs &a, int b)
{
    int lo = 0, hi = a.groups;              // start[lo] <= b < start[hi], where boundaries ascend
    if (hi == 0 || b < a.start[0] || b >= a.start[hi]) return -1;
    while (hi - lo > 1) {
        const int mid = (lo + hi) >> 1;
        if (a.start[mid] <= b) lo = mid;
        else hi = mid;
    }
    return lo;
}
__device__ __forceinline__ PromptSeq prompt_seq(const PromptArgs &a, int b)
{
    PromptSeq s;
    prompt_range(a.cu_q, b, a.batch, a.n_q, s.q0, s.m);
    s.k0 = 0;
    s.p = 0;
    s.group = -1;
    if (a.table) {
        s.n = clamp_rows(a.n_rows[b], a.max_pages, a.page_rows);
        s.group = prompt_group(a, b);
        if (s.group >= 0) s.p = clamp_rows(a.p_rows[s.group], a.max_p_pages, a.page_rows);
    } else {
        prompt_range(a.cu_k, b, a.batch, a.n_k, s.k0, s.n);
    }
    return s;
}
constexpr int kTileRows = 128;               // query rows of a half item, cached rows of a tile
constexpr unsigned kTileOver = 8;           // what an item costs beside its tiles, in units (half a tile's time for both halves)

// An item: the query rows of a run of tokens (all query heads of one key head), in one half of up to 128 rows or in two.
template <bool WIDE> __device__ __forceinline__ int item_tokens(const PromptArgs &a) { return WIDE ? a.half_tokens : 2 * a.half_tokens; }
// tiles of 128 rows (prefix, then own rows) that the tokens up to i attend
__device__ __forceinline__ int tiles_until(const PromptArgs &a, const PromptSeq &s, int i)
{
    return (s.p + kTileRows - 1) / kTileRows + (s.seen(i, a.causal) + kTileRows - 1) / kTileRows;
}
template <bool WIDE>
struct TileItem {
    int first, count, tiles;                // tokens; tiles
    bool pair;                              // two halves
    __device__ __forceinline__ TileItem(const PromptArgs &a, const PromptSeq &s, int q) : first(q * item_tokens<WIDE>(a))
    {
        count = min(s.m - first, item_tokens<WIDE>(a));
        tiles = tiles_until(a, s, first + count - 1);
        pair = !WIDE && count > a.half_tokens;
    }
    __device__ __forceinline__ unsigned tile_cost() const { return WIDE || pair ? 2u : 1u; }
    __device__ __forceinline__ unsigned cost(int shift) const { return max((kTileOver + tile_cost() * (unsigned)tiles) >> shift, 1u); }   // in units of 2^shift
};

// a page as a table names it; one outside the pool is reported, and read as page 0 (the result is then unspecified)
__device__ __forceinline__ int prompt_page(const PromptArgs &a, int page)
{
    if (page >= 0 && page < a.n_pages) return page;
    if (a.status) atomicOr(a.status, ADSA_DEV_BAD_PAGE);
    return 0;
}
// element offset of cached row j (prefix rows first) of a sequence, key head h, in k (v: their own strides when packed)
__device__ __forceinline__ size_t prompt_row(const PromptArgs &a, const PromptSeq &s, int b, int h, int j, bool value)
{
    if (!a.table) return (size_t)((s.k0 + j) * (value ? a.v_token : a.k_token) + h * (value ? a.v_head : a.k_head));
    const bool pre = j < s.p;
    const int row = pre ? j : j - s.p;
    const int32_t *pages = pre ? a.p_table + (size_t)s.group * a.max_p_pages : a.table + (size_t)b * a.max_pages;
    const int page = prompt_page(a, pages[a.by_page(row)]);
    return (((size_t)page * a.kv_heads + h) * a.page_rows + row - a.by_page(row) * a.page_rows) * a.row_stride;
}

// Magnitudes from here on are infinite in the 16-bit type (halfway from its largest value to the next power of two).  An output is a mean of
// values of that type and never as large, but weights that are rounded and a sum that is not can make it so.
template <typename T> struct TooLarge { static constexpr float value = 255.5f * 1.329227995784916e36f; };   // (2 - 2^-8) 2^127
template <> struct TooLarge<__half> { static constexpr float value = 65520.f; };
template <typename T> __device__ __forceinline__ bool prompt_fits(float x) { return fabsf(x) < TooLarge<T>::value; }   // (not NaN)

// bits that are all set in what is no finite number
template <typename T> struct Infinite { static constexpr uint32_t bits = 0x7f80u; };
template <> struct Infinite<__half> { static constexpr uint32_t bits = 0x7c00u; };
// the output element at `at`, as it was written, is no finite number
template <typename T>
__device__ __forceinline__ bool prompt_odd(const PromptArgs &a, size_t at)
{
    if (a.out) return (reinterpret_cast<const uint16_t *>(a.out)[at] & Infinite<T>::bits) == Infinite<T>::bits;
    return (reinterpret_cast<const uint32_t *>(a.out_f32)[at] & 0x7f800000u) == 0x7f800000u;
}
// A row whose scores or whose sum of weights are no numbers is NaN throughout, and rightly so: its first element is a NaN that no conversion makes, so
// that it is not looked at again.  (Not where scores have zeros times what lies beside a head's elements.)
__device__ __forceinline__ bool prompt_lost(const PromptArgs &a, float l) { return !a.shifted && !(l > 0.f && l < INFINITY); }
__device__ __forceinline__ void prompt_mark_lost(const PromptArgs &a, size_t at)
{
    if (a.out) reinterpret_cast<uint16_t *>(a.out)[at] = 0x7ffe;
    else reinterpret_cast<uint32_t *>(a.out_f32)[at] = 0x7ffffffeu;
}
__device__ __forceinline__ bool prompt_marked_lost(const PromptArgs &a, size_t at)
{
    return a.out ? reinterpret_cast<const uint16_t *>(a.out)[at] == 0x7ffe : reinterpret_cast<const uint32_t *>(a.out_f32)[at] == 0x7ffffffeu;
}

// One query row by one warp, as the formula has it: a cached row per lane for the scores, elements spread over the lanes for
// the sums.  All in 32 bits.  The running output is the mean so far, moved on by shares of the sum so far: it stays within the values' range,
// where a sum that is divided at the end passes 32 bits.  Elements c0 .. c1 - 1 of the output, at most 128 of them.
template <typename T>
__device__ __noinline__ void prompt_row_by_warp(const PromptArgs &a, const PromptSeq &s, int b, int i, int head, int lane, int c0, int c1)
{
    constexpr int PER = 2;                                   // pairs of elements a lane
    const int h = a.by_per_kv(head), n = s.p + s.seen(i, a.causal);
    const T *q = (const T *)a.q + (s.q0 + i) * a.q_token + head * a.q_head;
    float m = -INFINITY, l = 0.f;
    float2 o[PER];
#pragma unroll
    for (int e = 0; e < PER; ++e) o[e] = make_float2(0.f, 0.f);
    for (int j0 = 0; j0 < n; j0 += 32) {
        const int j = j0 + lane;
        float x = -INFINITY;
        size_t v_at = 0;
        if (j < n) {
            const T *k = (const T *)a.k + prompt_row(a, s, b, h, j, false);
            v_at = prompt_row(a, s, b, h, j, true);
            x = 0.f;
            for (int e = 0; e < a.d; ++e) x = fmaf(to_f32(q[e]), to_f32(k[e]), x);
            x *= a.scale_log2e;
        }
        // (a NaN score has to reach the result: max would drop it)
        const bool nan = __any_sync(0xffffffffu, isnan(x));
        float mx = x;
#pragma unroll
        for (int k = 16; k; k >>= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, k));
        const float m_new = nan ? NAN : fmaxf(m, mx);
        const float base = m_new == -INFINITY ? 0.f : m_new, before = l * pa_exp2(m - base), w = j < n ? pa_exp2(x - base) : 0.f;
        m = m_new;
        float sum = w;
#pragma unroll
        for (int k = 16; k; k >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, k);
        l = before + sum;
        const float inv = l == 0.f ? 0.f : 1.f / l, old = before * inv, share = w * inv;   // (no weight yet: as if nothing had come)
#pragma unroll
        for (int e = 0; e < PER; ++e) { o[e].x *= old; o[e].y *= old; }
        const int rows = min(n - j0, 32);
        for (int r = 0; r < rows; ++r) {
            const float p = __shfl_sync(0xffffffffu, share, r);
            const T *v = (const T *)a.v + __shfl_sync(0xffffffffu, v_at, r);
#pragma unroll
            for (int e = 0; e < PER; ++e) {
                const int at = c0 + 2 * (lane + 32 * e);
                if (at < c1) {
                    o[e].x = fmaf(p, to_f32(v[at]), o[e].x);
                    o[e].y = fmaf(p, to_f32(v[at + 1]), o[e].y);
                }
            }
        }
    }
    const size_t row = (size_t)(s.q0 + i) * a.kv_heads * a.per_kv + head;
#pragma unroll
    for (int e = 0; e < PER; ++e) {
        const int at = c0 + 2 * (lane + 32 * e);
        if (at >= c1) continue;
        if (n > 0 && l == 0.f) o[e] = make_float2(NAN, NAN);   // (scores of -infinity alone)
        if (a.out) *reinterpret_cast<uint32_t *>((T *)a.out + row * a.d + at) = pack2<T>(o[e].x, o[e].y);
        if (a.out_f32) *reinterpret_cast<float2 *>(a.out_f32 + row * a.d + at) = o[e];
    }
    if (a.lse && lane == 0 && c0 == 0) a.lse[row] = n > 0 ? (m + log2f(l)) * 0.693147180559945309f : -INFINITY;
}

// What V holds of infinities and NaN in the rows that were looked at, of one sequence and key head from row 0 on; a lane has the columns that it has in
// prompt_row_by_warp.
constexpr int kOddNone = 0x7fffffff;
struct PromptOdd {
    int b, head, rows, k_rows;              // looked at: rows of V, of K
    bool whole;                             // rows are made again as a whole: a block that gave up may not have written them
    int first[4][3], k_first;               // of a column of V: the row of the first NaN, infinity, -infinity; of K: the first that has one of them (a
                                            // NaN, for heads that begin between 16-byte pieces)
    __device__ __forceinline__ void reset(int b_, int head_)
    {
        b = b_;
        head = head_;
        rows = k_rows = 0;
        k_first = kOddNone;
#pragma unroll
        for (int e = 0; e < 12; ++e) first[e / 3][e % 3] = kOddNone;
    }
};
// Rows from .. to - 1 of V, until every column has a NaN; where it stopped.  (`first` in registers: through memory no load would pass a store.)
template <typename T>
__device__ __forceinline__ int prompt_look_v(const PromptArgs &a, const PromptSeq &s, int b, int h, int from, int to, int lane, int c0, int c1, int (&first)[4][3])
{
    constexpr uint32_t kInf = Infinite<T>::bits, kTop = 0x80008000u;
    uint32_t known[2][3];                                          // of a pair of columns: the highest bit of a half whose column has had one
#pragma unroll
    for (int e = 0; e < 6; ++e) known[e / 3][e % 3] = (first[e / 3 * 2][e % 3] != kOddNone ? 0x8000u : 0u) | (first[e / 3 * 2 + 1][e % 3] != kOddNone ? 0x80000000u : 0u);
    while (from < to) {
        bool open = false;
#pragma unroll
        for (int e = 0; e < 4; ++e) open = open || (c0 + 2 * (lane + 32 * (e / 2)) < c1 && first[e][0] == kOddNone);
        if (!__any_sync(0xffffffffu, open)) break;
        const size_t mine = from + lane < to ? prompt_row(a, s, b, h, from + lane, true) : 0;
        const int rows = min(to - from, 32);
        for (int r0 = 0; r0 < rows; r0 += 8) {
            uint32_t w[8][2], odd = 0;
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                const T *v = (const T *)a.v + __shfl_sync(0xffffffffu, mine, r0 + r);
#pragma unroll
                for (int e = 0; e < 2; ++e) {
                    const int col = c0 + 2 * (lane + 32 * e);
                    w[r][e] = r0 + r < rows && col < c1 ? __ldg(reinterpret_cast<const uint32_t *>(v + col)) : 0u;
                    odd |= (w[r][e] & 0x7fff7fffu) + (0x8000u - kInf) * 0x10001u;   // (the highest bit of a half whose exponent is full)
                }
            }
            if (!(odd & kTop)) continue;
            uint32_t any[2][3] = {};
#pragma unroll
            for (int e = 0; e < 16; ++e) {
                const uint32_t x = w[e / 2][e & 1], t = x & 0x7fff7fffu, full = t + (0x8000u - kInf) * 0x10001u, nan = t + (0x7fffu - kInf) * 0x10001u;
                any[e & 1][0] |= nan;
                any[e & 1][1] |= full & ~nan & ~x;
                any[e & 1][2] |= full & ~nan & x;
            }
            uint32_t more = 0;
#pragma unroll
            for (int e = 0; e < 6; ++e) more |= any[e / 3][e % 3] & ~known[e / 3][e % 3];
            if (!(more & kTop)) continue;                          // (all of kinds that their columns have had)
#pragma unroll
            for (int e = 0; e < 6; ++e) known[e / 3][e % 3] |= any[e / 3][e % 3] & kTop;
#pragma unroll
            for (int r = 0; r < 8; ++r) {
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const uint32_t x = w[r][e / 2] >> (e & 1) * 16 & 0x7fffu;
                    const bool minus = w[r][e / 2] >> (e & 1) * 16 & 0x8000u;
                    const int at = from + r0 + r;
                    if (x > kInf) first[e][0] = min(first[e][0], at);
                    if (x == kInf && !minus) first[e][1] = min(first[e][1], at);
                    if (x == kInf && minus) first[e][2] = min(first[e][2], at);
                }
            }
        }
        from += rows;
    }
    return from;
}
// Rows from .. to - 1 of K, until one has an infinity or a NaN (NAN_ALONE: a NaN): that one, or kOddNone.
template <typename T, bool NAN_ALONE>
__device__ __forceinline__ int prompt_look_k(const PromptArgs &a, const PromptSeq &s, int b, int h, int from, int to, int lane)
{
    constexpr uint32_t kInf = Infinite<T>::bits;
    for (; from < to; from += 32) {
        const size_t mine = from + lane < to ? prompt_row(a, s, b, h, from + lane, false) : 0;
        const int rows = min(to - from, 32);
        int first = kOddNone;
        for (int r0 = 0; r0 < rows; r0 += 8) {
            for (int e0 = 0; e0 < a.d; e0 += 64) {
                const int e = e0 + 2 * lane;
#pragma unroll
                for (int r = 0; r < 8; ++r) {
                    const T *k = (const T *)a.k + __shfl_sync(0xffffffffu, mine, r0 + r);
                    const uint32_t w = r0 + r < rows && e < a.d ? __ldg(reinterpret_cast<const uint32_t *>(k + e)) : 0u;
                    if (((w & 0x7fff7fffu) + ((NAN_ALONE ? 0x7fffu : 0x8000u) - kInf) * 0x10001u) & 0x80008000u) first = min(first, from + r0 + r);
                }
            }
        }
        first = __reduce_min_sync(0xffffffffu, first);
        if (first != kOddNone) return first;
    }
    return kOddNone;
}

// An output row with elements that are no finite numbers, by a warp: each is what the values that the row attends make it, whatever stands beside them in a
// tile.  A NaN among them makes NaN, an infinity that infinity, one of either sign NaN (weights are above zero, where no score is infinite); in half precision an
// infinity without one is an output past the largest value by its roundings.  What is left (a row beside infinities or NaN that it does not attend, values of
// bfloat16 near 2^127) is made again from the rows it attends.
// Rows of V are looked at once for all rows of a key head: made again row by row, one NaN in a prompt of 16384 tokens took 537 ms of a call of 0.26.
template <typename T>
__device__ __noinline__ void prompt_mend_row(const PromptArgs &a, const PromptSeq &s, int b, int i, int head, int lane, int c0, int c1, PromptOdd &odd)
{
    const int h = a.by_per_kv(head), n = s.p + s.seen(i, a.causal);
    if (odd.b != b || odd.head != h) odd.reset(b, h);
    const T *q = (const T *)a.q + (s.q0 + i) * a.q_token + head * a.q_head;
    if (odd.whole) {
        prompt_row_by_warp<T>(a, s, b, i, head, lane, c0, c1);
        return;
    }
    if (a.shifted) {                                               // NaN by its own scores, or by what lies beside them
        bool nan = false;
        for (int e = lane; e < a.d; e += 32) nan = nan || isnan(to_f32(q[e]));
        if (odd.k_rows < n && odd.k_first == kOddNone) {
            odd.k_first = prompt_look_k<T, true>(a, s, b, h, odd.k_rows, n, lane);
            odd.k_rows = n;
        }
        if (!__any_sync(0xffffffffu, nan) && odd.k_first >= n) prompt_row_by_warp<T>(a, s, b, i, head, lane, c0, c1);
        return;
    }
    int first[4][3];
#pragma unroll
    for (int e = 0; e < 12; ++e) first[e / 3][e % 3] = odd.first[e / 3][e % 3];
    if (odd.rows < n) {
        odd.rows = prompt_look_v<T>(a, s, b, h, odd.rows, n, lane, c0, c1, first);
#pragma unroll
        for (int e = 0; e < 12; ++e) odd.first[e / 3][e % 3] = first[e / 3][e % 3];
    }
    const size_t row = ((size_t)(s.q0 + i) * a.kv_heads * a.per_kv + head) * a.d;
    float y[4];
    bool fix[4], made = false, infinite = false, only16[4];
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int col = c0 + 2 * (lane + 32 * (e / 2)) + (e & 1);
        fix[e] = only16[e] = false;
        y[e] = 0.f;
        if (col >= c1 || !prompt_odd<T>(a, row + col)) continue;
        fix[e] = true;
        const bool nan = first[e][0] < n, plus = first[e][1] < n, minus = first[e][2] < n;
        const float x = a.out ? to_f32(((const T *)a.out)[row + col]) : a.out_f32[row + col];
        if (nan || (plus && minus)) y[e] = NAN;
        else if (plus || minus) {
            y[e] = plus ? INFINITY : -INFINITY;
            infinite = true;
        } else if (std::is_same<T, __half>::value && a.out && !isnan(x)) {
            y[e] = copysignf(65504.f, x);
            only16[e] = true;
        } else {
            made = true;
        }
    }
    made = __any_sync(0xffffffffu, made);
    if (!made && __any_sync(0xffffffffu, infinite)) {              // a weight of zero, or none: an infinite score
        bool bad = false;
        for (int e = lane; e < a.d; e += 32) bad = bad || !(fabsf(to_f32(q[e])) < INFINITY);
        if (odd.k_rows < n && odd.k_first == kOddNone) {
            odd.k_first = prompt_look_k<T, false>(a, s, b, h, odd.k_rows, n, lane);
            odd.k_rows = n;
        }
        made = odd.k_first < n || __any_sync(0xffffffffu, bad);
    }
    if (made) {
        prompt_row_by_warp<T>(a, s, b, i, head, lane, c0, c1);
        return;
    }
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        const int col = c0 + 2 * (lane + 32 * (e / 2)) + (e & 1);
        if (!fix[e]) continue;
        if (a.out) reinterpret_cast<uint16_t *>(a.out)[row + col] = (uint16_t)pack2<T>(y[e], 0.f);
        if (a.out_f32 && !only16[e]) a.out_f32[row + col] = y[e];
    }
}

size_t prompt_workspace(int head_dim, int sms, PromptArgs *a, void *workspace);   // lays the workspace out; its size
cudaError_t launch_prompt_tiles(int dtype, const PromptArgs &a, int sms, cudaStream_t st);

}  // namespace adsa
