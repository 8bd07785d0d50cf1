"""Rotary positions with several axes, the rotated append into a paged cache, decode attention over a shared prefix and
the norms with the gated residual, each against a plain implementation in 64 bits, and all four as one decode step.

Tolerances count roundings: a value rounded to type t is off by at most u = finfo(t).eps / 2 of itself; 32-bit steps are
counted at 2^-23 of the magnitudes they add up."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
HALF = [torch.bfloat16, torch.float16]


def _u(dtype):
    return torch.finfo(dtype).eps / 2


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _randn(gen, *shape, dtype=torch.bfloat16, scale=1.0):
    return (torch.randn(shape, generator=gen, device=DEV) * scale).to(dtype)


# ---- rotary positions ------------------------------------------------------------------------------------------------

def turn64(x, pos, pairs, style, restart, base=10000.0):
    """(turned x, sum of magnitudes of each pair) in 64 bits, pair by pair."""
    x = x.double()
    out, mag = x.clone(), x.abs()
    n = sum(pairs)
    i = 0
    for a, count in enumerate(pairs):
        for j in range(count):
            theta = base ** -(j / count if restart else i / n)
            ang = pos[:, a].double() * theta
            c, s = ang.cos()[:, None], ang.sin()[:, None]
            e0, e1 = (2 * i, 2 * i + 1) if style == "pairs" else (i, i + n)
            out[..., e0] = x[..., e0] * c - x[..., e1] * s
            out[..., e1] = x[..., e0] * s + x[..., e1] * c
            mag[..., e0] = mag[..., e1] = x[..., e0].abs() + x[..., e1].abs()
            i += 1
    return out, mag


def check_turned(got, want, mag, dtype, subnormal=0.0):
    # sine and cosine: the turn's fraction rounded to 32 bits (2^-25 turns = 1.9e-7 rad) and 2 ulp of the functions;
    # two products and a sum: together below 8 * 2^-23 of the pair's magnitude.  Then one rounding to the type (which
    # below its smallest normal number is half its smallest step).
    tol = _u(dtype) * want.abs() + 8 * 2.0 ** -23 * mag + torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
    assert ((got.double() - want).abs() <= tol).all(), float(((got.double() - want).abs() - tol).max())


ROPE = [  # tokens, heads, dim, pairs, base
    (1, 1, 2, (1,), 0.0),
    (1, 20, 64, (16, 16), 0.0),
    (37, 3, 64, (8, 12, 12), 10000.0),
    (130, 5, 100, (25, 25), 0.0),
    (65, 2, 100, (10, 0, 20, 7), 500.0),       # 37 of 50 pairs turn; an axis without pairs
    (33, 4, 128, (64,), 1e6),
    (29, 8, 128, (16, 24, 24), 0.0),
    (9, 2, 256, (43, 42, 43), 0.0),
    (700, 32, 96, (16, 32), 0.0),
    (3, 70, 30, (4, 5), 0.0),
]


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("style", ["pairs", "halves"])
@pytest.mark.parametrize("tokens,heads,dim,pairs,base", ROPE)
def test_rope_axes_matches_64_bits(tokens, heads, dim, pairs, base, style, dtype):
    import paper_2506_18226_b200 as A
    for restart in (True, False):
        g = _gen(tokens * 7 + dim)
        x = _randn(g, tokens, heads, dim, dtype=dtype)
        pos = torch.randint(0, 5000, (tokens, len(pairs)), generator=g, device=DEV, dtype=torch.int32)
        rot = A.Rotary(dim, pairs, base=base, style=style, restart=restart)
        want, mag = turn64(x, pos, pairs, style, restart, base or 10000.0)
        got = A.rope_axes(rot, x, pos)
        check_turned(got, want, mag, dtype)
        assert torch.equal(got[..., 2 * sum(pairs):], x[..., 2 * sum(pairs):])
        assert A.rope_axes(rot, x, pos, out=x) is x and torch.equal(x, got)      # in place


@pytest.mark.parametrize("style", ["pairs", "halves"])
def test_rope_axes_far_and_negative_positions(style):
    import paper_2506_18226_b200 as A
    g = _gen(3)
    x = _randn(g, 6, 4, 64)
    pos = torch.tensor([[2**31 - 1, -2**31], [10**9, 7], [-123456789, 2**30 + 1], [0, 0], [1, -1], [99999999, 5]], dtype=torch.int32,
                       device=DEV)
    want, mag = turn64(x, pos, (16, 16), style, True)
    # the reference's own angle: pos * theta in 64 bits is off by 2^-53 of up to 2^31 rad, 2.4e-7 rad
    got = A.rope_axes(A.Rotary(64, (16, 16), style=style), x, pos).double()
    tol = _u(torch.bfloat16) * want.abs() + (8 * 2.0 ** -23 + 1e-6) * mag
    assert ((got - want).abs() <= tol).all()
    assert torch.equal(got[3], x[3].double())                                    # position zero turns nothing


@pytest.mark.parametrize("offset,dim", [(0, 64), (1, 64), (2, 64), (4, 100), (0, 100), (3, 30)])
@pytest.mark.parametrize("style", ["pairs", "halves"])
def test_rope_axes_strides_and_alignment(style, offset, dim):
    """q of a packed projection whose rows start at any element; the output in another order; bytes around it untouched."""
    import paper_2506_18226_b200 as A
    g = _gen(offset + dim)
    T, H = 19, 6
    flat = _randn(g, T * (3 * H * dim + 5) + 8)
    x = flat[offset:offset + T * (3 * H * dim + 5)].view(T, -1)[:, :H * dim].unflatten(1, (H, dim))
    pos = torch.randint(-50, 900, (T, 2), generator=g, device=DEV, dtype=torch.int32)
    pairs = (dim // 4, dim // 4)
    room = torch.full((H, T, dim + 2), 7.0, dtype=torch.bfloat16, device=DEV)
    out = room[..., 1:dim + 1].transpose(0, 1) if offset % 2 else room[..., :dim].transpose(0, 1)
    want, mag = turn64(x, pos, pairs, style, False)
    before = flat.clone()
    got = A.rope_axes(A.Rotary(dim, pairs, style=style, restart=False), x, pos, out=out)
    check_turned(got, want, mag, torch.bfloat16)
    assert torch.equal(flat, before)
    edge = room[..., dim + 1] if offset % 2 else room[..., dim:]
    assert (edge == 7.0).all() and (offset % 2 == 0 or (room[..., 0] == 7.0).all())


def test_rope_axes_infinities_stay_in_their_pair():
    import paper_2506_18226_b200 as A
    x = torch.ones((2, 2, 64), dtype=torch.bfloat16, device=DEV)
    x[1, 0, 5], x[0, 1, 40] = float("inf"), float("nan")
    pos = torch.tensor([[3, 4], [5, 6]], dtype=torch.int32, device=DEV)
    got = A.rope_axes(A.Rotary(64, (8, 8)), x, pos)                               # elements 32 .. 63 do not turn
    bad = ~torch.isfinite(got)
    assert bad[1, 0, 4:6].all() and bad[0, 1, 40] and int(bad.sum()) == 3


def test_rope_axes_agrees_with_rope_2d():
    """Two axes of head_dim / 4 pairs that restart are adsa_rope_2d's angles (taken there in 32 bits: up to 47 rad here,
    2^-23 of it, twice)."""
    import paper_2506_18226_b200 as A
    eng = A.AdsaEngine(n_layers=1, batch=1, n_heads=4, head_dim=64, n_text=0, grid_h=48, grid_w=48, max_rows_per_stream=64, n_prefix=0)
    g = _gen(8)
    x = _randn(g, 2304, 4, 64)
    cell = torch.arange(2304, device=DEV, dtype=torch.int32)
    pos = torch.stack([cell // 48, cell % 48], 1).contiguous()
    got = A.rope_axes(A.Rotary(64, (16, 16)), x, pos).double()
    other = x.clone()
    eng.rope_2d(other, cell.repeat_interleave(4))
    want, mag = turn64(x, pos, (16, 16), "pairs", True)
    assert ((got - other.double()).abs() <= 2 * _u(torch.bfloat16) * want.abs() + 2e-5 * mag).all()


# ---- append ----------------------------------------------------------------------------------------------------------

def make_cache(gen, lengths, kv_heads, page_rows, dim, dtype, spare=3, stride=None, extra_pages=0):
    """Pools full of NaN, a table of distinct random pages for `lengths` rows each."""
    stride = (dim + 7) // 8 * 8 if stride is None else stride
    counts = [(n + page_rows - 1) // page_rows for n in lengths]
    pages = sum(counts) + spare
    most = max(1, max(counts)) + extra_pages
    order = torch.randperm(pages, generator=gen, device=DEV).to(torch.int32)
    table = torch.full((len(lengths), most), -12345, dtype=torch.int32, device=DEV)   # never read
    at = 0
    for b, c in enumerate(counts):
        table[b, :c] = order[at:at + c]
        at += c
    pools = [torch.full((pages, kv_heads, page_rows, stride), float("nan"), dtype=dtype, device=DEV) for _ in range(2)]
    return pools[0], pools[1], table


def rows_of(pool, table_row, n):
    """The logical rows 0 .. n-1: [n, heads, stride]."""
    r = torch.arange(n, device=DEV)
    pr = pool.shape[2]
    return pool[table_row[r // pr].long(), :, r % pr]


APPEND = [  # new tokens per batch row, rows before, kv heads, query heads, dim, stride, page rows
    ([1] * 32, [0] * 32, 20, 20, 64, 64, 64),
    ([1, 1, 1], [63, 64, 0], 2, 4, 64, 72, 64),
    ([5, 0, 130, 1], [3, 9, 0, 200], 4, 8, 100, 104, 48),
    ([17, 40], [15, 1], 3, 0, 128, 128, 16),
    ([64, 64], [0, 64], 1, 2, 256, 256, 1),
    ([9], [570], 2, 2, 30, 40, 572),
    ([300, 20, 411], [7, 100, 0], 8, 32, 128, 136, 24),
    ([0, 0], [5, 6], 2, 2, 64, 64, 16),
    ([0] * 40 + [3] + [0] * 70 + [1, 1] + [0] * 33 + [2, 0], list(range(148)), 1, 1, 64, 64, 16),
    ([n % 3 for n in range(1100)], [n % 50 for n in range(1100)], 1, 2, 64, 64, 32),
]


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("style", ["pairs", "halves"])
@pytest.mark.parametrize("case", range(len(APPEND)))
def test_paged_append_matches_64_bits(case, style, dtype):
    import paper_2506_18226_b200 as A
    new, have, kv, qh, dim, stride, page = APPEND[case]
    g = _gen(case)
    B, T, pad = len(new), sum(new), 4
    uniform = len(set(new)) == 1
    pairs = (dim // 8, dim // 4)
    for ragged in ([True, False] if uniform else [True]):
        first = 2 if ragged else 0                                                # padding tokens before and behind
        n_tokens = T + (first + pad if ragged else 0)
        k_pool, v_pool, table = make_cache(g, [n + h for n, h in zip(new, have)], kv, page, dim, dtype, stride=stride, extra_pages=2)
        k_before, v_before = k_pool.clone(), v_pool.clone()
        k, v = _randn(g, n_tokens, kv, dim, dtype=dtype), _randn(g, n_tokens, kv, dim, dtype=dtype)
        q = _randn(g, n_tokens, qh, dim, dtype=dtype) if qh else None
        q_out = torch.full_like(q, 7.0) if qh else None
        pos = torch.randint(0, 3000, (n_tokens, 2), generator=g, device=DEV, dtype=torch.int32)
        n_rows = torch.tensor(have, dtype=torch.int32, device=DEV)
        cu = [first]
        for n in new:
            cu.append(cu[-1] + n)
        rot = A.Rotary(dim, pairs, style=style)
        status = torch.zeros(1, dtype=torch.int32, device=DEV)
        got = A.paged_append(k, v, k_pool, v_pool, table, n_rows, cu_tokens=torch.tensor(cu, dtype=torch.int32, device=DEV) if ragged else None,
                             rotary=rot, pos=pos, q=q, q_out=q_out, status=status)
        assert int(status) == 0 and n_rows.tolist() == have
        want, mag = turn64(k, pos, pairs, style, True)
        for b in range(B):
            sl = slice(cu[b], cu[b + 1])
            r = torch.arange(have[b], have[b] + new[b], device=DEV)
            pg, row = table[b][r // page].long(), r % page
            check_turned(k_pool[pg, :, row][..., :dim], want[sl], mag[sl], dtype)
            assert torch.equal(v_pool[pg, :, row][..., :dim], v[sl])
            assert (k_pool[pg, :, row][..., dim:] == 0).all() and (v_pool[pg, :, row][..., dim:] == 0).all()
            k_pool[pg, :, row], v_pool[pg, :, row] = float("nan"), float("nan")
        # everything else is as it was (NaN compares by its bits)
        assert torch.equal(k_pool.view(torch.int16), k_before.view(torch.int16)) and torch.equal(v_pool.view(torch.int16), v_before.view(torch.int16))
        if qh:
            assert got is q_out
            want, mag = turn64(q, pos, pairs, style, True)
            check_turned(q_out[cu[0]:cu[-1]], want[cu[0]:cu[-1]], mag[cu[0]:cu[-1]], dtype)
            assert (q_out[:cu[0]] == 7.0).all() and (q_out[cu[-1]:] == 7.0).all()


def test_paged_append_from_a_packed_projection_in_place_and_without_rotation():
    import paper_2506_18226_b200 as A
    g = _gen(4)
    B, kv, qh, dim, page = 6, 2, 4, 64, 32
    qkv = _randn(g, B, (qh + 2 * kv), dim)
    plain = qkv.clone()
    q, k, v = qkv[:, :qh], qkv[:, qh:qh + kv], qkv[:, qh + kv:]
    have = torch.tensor([0, 31, 32, 5, 63, 64], dtype=torch.int32, device=DEV)
    k_pool, v_pool, table = make_cache(g, [n + 1 for n in have.tolist()], kv, page, dim, torch.bfloat16)
    pos = torch.stack([have, have + 9, have * 2], 1).contiguous()
    A.paged_append(k, v, k_pool, v_pool, table, have, rotary=A.Rotary(dim, (8, 12, 12)), pos=pos, q=q, q_out=q)
    want, mag = turn64(plain[:, :qh], pos, (8, 12, 12), "pairs", True)
    check_turned(qkv[:, :qh], want, mag, torch.bfloat16)
    assert torch.equal(qkv[:, qh:], plain[:, qh:])                                # k and v themselves are not changed
    A.paged_append(k, v, k_pool, v_pool, table, have)                             # the same rows, not turned
    r = have.long()
    pg = table[torch.arange(B, device=DEV), r // page].long()
    assert torch.equal(k_pool[pg, :, r % page], plain[:, qh:qh + kv]) and torch.equal(v_pool[pg, :, r % page], plain[:, qh + kv:])


def test_paged_append_skips_rows_it_cannot_place_and_says_so():
    import paper_2506_18226_b200 as A
    B = A.binding
    g = _gen(5)
    k_pool, v_pool, table = make_cache(g, [32, 32, 32, 32], 2, 16, 64, torch.bfloat16, spare=0)
    table[2, 1] = k_pool.shape[0]                                                 # outside the pool
    before = k_pool.clone()
    have = torch.tensor([31, 30, 16, -1], dtype=torch.int32, device=DEV)
    k, v = _randn(g, 8, 2, 64), _randn(g, 8, 2, 64)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    A.paged_append(k, v, k_pool, v_pool, table, have, status=status)              # row 0 runs over by one; row 3 starts at -1
    assert int(status) == B.DEV_ROW_OVERFLOW | B.DEV_BAD_PAGE
    assert torch.equal(k_pool[table[0, 1].long(), :, 15], k[0]) and torch.equal(k_pool[table[1, 1].long(), :, 14:16], k[2:4].transpose(0, 1))
    written = int((~torch.isnan(k_pool)).sum())
    assert written == 3 * 2 * 64 and torch.isnan(before).all()
    A.paged_append(k, v, k_pool, v_pool, table, have)                             # status not wanted: skipped all the same


# ---- attention -------------------------------------------------------------------------------------------------------

def attn64(q, k_pool, v_pool, table, n_rows, p_table, p_rows, start, scale):
    """out, lse, the tolerances' magnitudes: sum of w |v|, and the bound of a score's 32-bit error."""
    B, H, d = q.shape
    KV = k_pool.shape[1]
    G = H // KV
    out = torch.zeros((B, H, d), dtype=torch.float64, device=DEV)
    mag = torch.zeros_like(out)
    lse = torch.full((B, H), -math.inf, dtype=torch.float64, device=DEV)
    s_err = torch.zeros((B, H), dtype=torch.float64, device=DEV)
    for b in range(B):
        parts = [(table[b], int(n_rows[b]))]
        for gi in range(0 if start is None else len(start) - 1):
            if int(start[gi]) <= b < int(start[gi + 1]):
                parts.insert(0, (p_table[gi], int(p_rows[gi])))
        ks, vs = (torch.cat([rows_of(pool, t, n)[..., :d].double() for t, n in parts]) for pool in (k_pool, v_pool))   # [N, KV, d]
        if ks.shape[0] == 0:
            continue
        qq = q[b].double().view(KV, G, d)
        s = torch.einsum("hgd,nhd->hgn", qq, ks) * scale
        e = torch.einsum("hgd,nhd->hgn", qq.abs(), ks.abs()).amax(-1) * scale
        w = torch.softmax(s, -1)
        out[b] = torch.einsum("hgn,nhd->hgd", w, vs).reshape(H, d)
        mag[b] = torch.einsum("hgn,nhd->hgd", w, vs.abs()).reshape(H, d)
        lse[b] = torch.logsumexp(s, -1).reshape(H)
        s_err[b] = e.reshape(H)
    return out, lse, mag, s_err * (d / 16 + 2) * 2.0 ** -22


def check_attn(got, got32, lse, ref, dtype):
    out, want_lse, mag, s_err = ref
    # a weight is rounded to the type once (u of itself); a score is off by s_err, which moves a weight and the sum it is
    # divided by by that share each; exponentials, sums over up to 2^16 rows in 64-row pieces: below 2^-18 together
    inner = (_u(dtype) + 2 * s_err[..., None] + 2.0 ** -18) * mag
    assert ((got32.double() - out).abs() <= inner + 1e-30).all(), float(((got32.double() - out).abs() - inner).max())
    assert ((got.double() - out).abs() <= inner + _u(dtype) * (out.abs() + inner) + torch.finfo(dtype).smallest_normal).all()
    empty = torch.isinf(want_lse)
    assert torch.equal(torch.isinf(lse), empty) and (lse[empty] < 0).all() and (got[empty] == 0).all() and (got32[empty] == 0).all()
    # the logarithm of a sum that is off by 2^-18, in 32 bits
    tol = s_err + 2.0 ** -18 + 2.0 ** -22 * want_lse.abs()
    assert ((lse.double() - want_lse).abs()[~empty] <= tol[~empty]).all()


def attn_case(gen, own, prefix, start, kv, per, dim, page, dtype, stride=None, q_scale=1.5, room=0):
    """room: rows the tables have room for beyond the longest (the choice of kernel goes by what they can hold)."""
    lengths = list(own) + list(prefix)
    k_pool, v_pool, table = make_cache(gen, lengths, kv, page, dim, dtype, stride=stride, extra_pages=1 + room // page)
    for i, n in enumerate(lengths):
        if n:
            r = torch.arange(n, device=DEV)
            pg = table[i][r // page].long()
            k_pool[pg, :, r % page, :dim] = _randn(gen, n, kv, dim, dtype=dtype)
            v_pool[pg, :, r % page, :dim] = _randn(gen, n, kv, dim, dtype=dtype)
    B = len(own)
    q = _randn(gen, B, kv * per, dim, dtype=dtype, scale=q_scale)
    i32 = dict(dtype=torch.int32, device=DEV)
    return dict(q=q, k_pool=k_pool, v_pool=v_pool, page_table=table[:B].contiguous(), n_rows=torch.tensor(own, **i32),
                prefix_table=table[B:].contiguous() if prefix else None, prefix_rows=torch.tensor(prefix, **i32) if prefix else None,
                group_start=torch.tensor(start, **i32) if prefix else None)


def run_attn(c, scale=0.0, **kw):
    import paper_2506_18226_b200 as A
    q = c["q"]
    out = torch.full(q.shape, 7.0, dtype=q.dtype, device=q.device)
    out32 = torch.full(q.shape, 7.0, dtype=torch.float32, device=q.device)
    lse = torch.full(q.shape[:2], 7.0, dtype=torch.float32, device=q.device)
    status = torch.zeros(1, dtype=torch.int32, device=q.device)
    A.shared_prefix_attn(**c, scale=scale, out=out, out_f32=out32, lse=lse, status=status, **kw)
    assert int(status) == 0
    return out, out32, lse


ATTN = {  # own rows, prefix rows, group starts, key heads, query heads per key head, dim, page rows
    "one row": ([1], [], [], 1, 1, 64, 16),
    "nothing at all": ([0, 0], [0], [0, 2], 2, 1, 64, 16),
    "own rows only": ([5, 0, 64, 65, 300], [], [], 3, 1, 64, 32),
    "prefix only": ([0, 0, 0], [130], [0, 3], 2, 2, 64, 64),
    "prefix and own": ([7, 100, 1, 63], [120, 121], [0, 2, 4], 4, 1, 64, 64),
    "some rows of no group": ([9, 9, 9, 9, 0], [77, 33], [1, 2, 4], 2, 2, 64, 16),
    "empty groups and empty prefixes": ([3, 4, 5], [64, 10, 0, 1], [0, 0, 2, 3, 3], 2, 1, 128, 64),
    "sixteen query heads": ([200, 31], [257], [0, 2], 1, 16, 128, 48),
    "seventeen query heads": ([40, 64], [100], [0, 2], 1, 17, 64, 64),
    "sixty-four query heads": ([129, 1], [65], [0, 2], 2, 64, 64, 64),
    "33 queries share": ([10] * 33, [500], [0, 33], 2, 1, 64, 64),
    "many queries share": ([12] * 50, [333], [0, 50], 2, 5, 128, 64),
    "two big groups": ([20] * 70, [700, 65], [0, 41, 70], 1, 8, 64, 128),
    "wide heads": ([70, 2304, 5], [200], [0, 3], 3, 1, 100, 48),
    "pages of one row": ([5, 70], [66], [0, 2], 2, 2, 64, 1),
    "pages of seven": ([100, 6], [150], [0, 2], 2, 1, 128, 7),
    "pages of 572": ([600, 571, 572], [1000], [0, 3], 2, 1, 64, 572),
    "192 elements": ([90, 1], [70], [0, 2], 2, 2, 192, 32),
    "256 elements": ([90, 64], [129], [0, 2], 1, 4, 256, 16),
    "two elements": ([30, 1], [7], [0, 2], 2, 1, 2, 16),
    "30 elements": ([30, 257], [70], [0, 2], 2, 2, 30, 40),
    "long": ([3, 9000], [20000], [0, 2], 2, 4, 128, 64),
    "40 elements": ([130, 7], [260], [0, 2], 2, 3, 40, 24),
    "72 elements": ([130, 64, 1], [260], [0, 3], 2, 1, 72, 64),
    "130 elements": ([90, 63], [129], [0, 2], 2, 2, 130, 48),
    "200 elements": ([65, 1], [70], [0, 2], 1, 4, 200, 10),
    "forty query heads": ([70, 1, 200], [100, 30], [0, 1, 3], 2, 40, 64, 64),
    "large group, 100 elements": ([5] * 50, [900], [0, 50], 2, 2, 100, 48),
    "large group, 72 elements": ([1] * 70, [1500], [0, 70], 2, 4, 72, 64),
    "large group, 30 elements": ([2] * 40, [513, 3], [0, 39, 40], 1, 1, 30, 16),
    "large groups, one without rows": ([2] * 90, [0, 400], [0, 45, 90], 2, 1, 64, 16),
    "large group, pages of seven": ([2] * 300, [385], [0, 300], 1, 1, 128, 7),
    "large groups of all sizes": ([2] * 513, [100, 700, 130, 1, 128], [0, 40, 180, 480, 480, 513], 3, 1, 64, 16),
    "many large groups": ([1] * 480, list(range(1, 360, 30)), list(range(0, 481, 40)), 3, 1, 128, 32),
    "big batch": ([n % 90 for n in range(300)], [50, 60, 70], [0, 100, 200, 300], 2, 1, 64, 32),
}


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("room", [0, 1800, 30000])
@pytest.mark.parametrize("name", list(ATTN))
def test_shared_prefix_attn_matches_64_bits(name, room, dtype):
    own, prefix, start, kv, per, dim, page = ATTN[name]
    c = attn_case(_gen(len(name)), own, prefix, start, kv, per, dim, page, dtype, room=room)
    got = run_attn(c)
    ref = attn64(c["q"], c["k_pool"], c["v_pool"], c["page_table"], c["n_rows"], c["prefix_table"], c["prefix_rows"], c["group_start"],
                 1 / math.sqrt(dim))
    check_attn(*got, ref, dtype)
    again = run_attn(c)
    assert all(torch.equal(a, b) for a, b in zip(got, again))                     # the order of the sums is fixed


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("rows,room", [(3, 0), (3, 1800), (3, 30000), (50, 30000)])
def test_shared_prefix_attn_peaked_scores_scale_stride_and_strided_queries(rows, room, dtype):
    """Scores in the tens (one row takes nearly all the weight, and the maximum keeps moving), a scale of the caller's,
    padded pool rows that hold NaN, query rows out of a packed tensor that start on 4-byte boundaries only."""
    g = _gen(21)
    c = attn_case(g, [(70, 200, 33)[b % 3] for b in range(rows)], [300], [0, rows], 2, 4, 100, 24, dtype, stride=136, q_scale=2.0, room=room)
    packed = _randn(g, rows, 2, 30, 102, dtype=dtype, scale=2.0)
    c["q"] = packed[:, 1, 3:19:2, 2:]
    got = run_attn(c, scale=0.7)
    ref = attn64(c["q"], c["k_pool"], c["v_pool"], c["page_table"], c["n_rows"], c["prefix_table"], c["prefix_rows"], c["group_start"], 0.7)
    check_attn(*got, ref, dtype)


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("batch,groups", [(4096, 0), (2, 2047), (2000, 1048)])
def test_shared_prefix_attn_largest_batches(batch, groups, dim):
    own = [(7 * b) % 40 for b in range(batch)]
    start = sorted(((37 * g) % (batch + 1)) for g in range(groups + 1))
    c = attn_case(_gen(batch + dim), own, [(5 * g) % 30 for g in range(groups)], start, 1, 1, dim, 16, torch.bfloat16, room=4096)
    got = run_attn(c)
    some = sorted({0, 1, batch // 3, batch - 2, batch - 1} - {-1})
    ref = attn64(c["q"][some], c["k_pool"], c["v_pool"], c["page_table"][some], c["n_rows"][some], None, None, None, dim ** -0.5)
    for i, b in enumerate(some):                                                  # (a group of one row each, in the reference)
        g = [k for k in range(groups) if start[k] <= b < start[k + 1]]
        if g:
            one = attn64(c["q"][b:b + 1], c["k_pool"], c["v_pool"], c["page_table"][b:b + 1], c["n_rows"][b:b + 1], c["prefix_table"][g[0]:g[0] + 1],
                         c["prefix_rows"][g[0]:g[0] + 1], torch.tensor([0, 1]), dim ** -0.5)
            for whole, part in zip(ref, one):
                whole[i] = part[0]
    check_attn(*[x[some] for x in got], ref, torch.bfloat16)


def test_shared_prefix_attn_equals_private_copies_of_the_prefix():
    """The same rows as one cache per batch row and no prefix: equal up to the merge's roundings."""
    import paper_2506_18226_b200 as A
    g = _gen(31)
    own, P, dim, page = [40, 7, 90, 0], 150, 64, 16
    c = attn_case(g, own, [P], [0, 4], 2, 2, dim, page, torch.bfloat16)
    k2, v2, t2 = make_cache(g, [P + n for n in own], 2, page, dim, torch.bfloat16)
    for b, n in enumerate(own):
        r = torch.arange(P + n, device=DEV)
        for src, dst in ((c["k_pool"], k2), (c["v_pool"], v2)):
            dst[t2[b][r // page].long(), :, r % page] = torch.cat([rows_of(src, c["prefix_table"][0], P), rows_of(src, c["page_table"][b], n)])
    a = A.shared_prefix_attn(**c, out_f32=torch.empty(4, 4, dim, device=DEV))
    b = A.shared_prefix_attn(c["q"], k2, v2, t2, c["n_rows"] + P, out_f32=torch.empty(4, 4, dim, device=DEV))
    ref = attn64(c["q"], k2, v2, t2, c["n_rows"] + P, None, None, None, 1 / 8)
    tol = 2 * (_u(torch.bfloat16) + 2 * ref[3][..., None] + 2.0 ** -18) * ref[2]
    assert ((a.double() - b.double()).abs() <= tol).all()


@pytest.mark.parametrize("times", [1, 50, 500])
def test_shared_prefix_attn_lengths_and_boundaries_the_device_finds_wrong(times):
    """Lengths past the tables are cut to them, negative ones to zero; boundaries outside the batch are cut to it; a page
    outside the pool is reported, and touches no other batch row."""
    import paper_2506_18226_b200 as A
    g = _gen(41)
    c = attn_case(g, [32, 32, 32], [48], [0, 3], 2, 1, 64, 16, torch.bfloat16)
    c["page_table"] = c["page_table"][:, :2].repeat(1, times)                     # (longer tables, by the other kernels)
    c["prefix_table"] = c["prefix_table"][:, :3].repeat(1, times)
    c["n_rows"] *= times
    c["prefix_rows"] *= times
    want = A.shared_prefix_attn(**c)
    far = dict(c, n_rows=torch.tensor([10**9, 32 * times + 1, 32 * times], dtype=torch.int32, device=DEV), group_start=torch.tensor([-5, 99], dtype=torch.int32, device=DEV),
               prefix_rows=torch.tensor([2**31 - 1], dtype=torch.int32, device=DEV))
    assert torch.equal(A.shared_prefix_attn(**far), want)
    none = dict(c, n_rows=torch.full((3,), -4, dtype=torch.int32, device=DEV), prefix_rows=torch.tensor([-1], dtype=torch.int32, device=DEV))
    assert (A.shared_prefix_attn(**none) == 0).all()
    bad = dict(c, page_table=c["page_table"].clone())
    bad["page_table"][1, 1] = c["k_pool"].shape[0]
    bad["page_table"][1, 0] = -1
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = A.shared_prefix_attn(**bad, status=status)
    assert int(status) == A.binding.DEV_BAD_PAGE
    assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])


@pytest.mark.parametrize("rows,room", [(3, 0), (3, 1800), (3, 30000), (40, 30000)])
def test_shared_prefix_attn_scores_that_are_not_finite(rows, room):
    """A score of -inf has no weight; a softmax over -inf alone, +inf or NaN is NaN, for the rows that attend it and no other."""
    c = attn_case(_gen(47), [70, 9, 20] + [9] * (rows - 3), [150], [0, rows - 1], 1, 2, 64, 16, torch.bfloat16, room=room)
    c["q"] = c["q"].abs() + 0.1
    r = torch.arange(150, device=DEV)
    prefix = c["prefix_table"][0][r // 16].long()
    own = c["page_table"][0][33 // 16].long()
    was = c["k_pool"].clone()
    plain = run_attn(dict(c, prefix_rows=torch.zeros_like(c["prefix_rows"])))
    c["k_pool"][prefix, :, r % 16] = -float("inf")
    got = run_attn(c)
    # the same weights of the own rows, summed in 32 bits in either case
    for a, b in zip(got[1:], plain[1:]):
        assert ((a - b).abs() <= 2.0 ** -18 * (b.abs().amax() + 8)).all()
    alone = run_attn(dict(c, n_rows=torch.zeros_like(c["n_rows"])))
    assert alone[1][:-1].isnan().all() and (alone[2] == -float("inf")).all() and (alone[1][-1] == 0).all()
    c["k_pool"].copy_(was)
    for bad in (float("inf"), float("nan")):
        c["k_pool"][own, :, 33 % 16] = bad
        got = run_attn(c)
        assert got[1][0].isnan().all() and got[2][0].isnan().all() and got[1][1:].isfinite().all() and got[2][1:].isfinite().all()


@pytest.mark.parametrize("rows,room", [(8, 0), (8, 1800), (8, 30000), (100, 30000), (700, 0)])
def test_shared_prefix_attn_reports_boundaries_that_do_not_ascend(rows, room):
    import paper_2506_18226_b200 as A
    c = attn_case(_gen(43), [5 + b % 7 for b in range(rows)], [150, 20, 90], [0, rows // 2, rows // 4, rows], 2, 2, 64, 16, torch.bfloat16, room=room)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    got = A.shared_prefix_attn(**c, status=status)
    assert int(status) == A.binding.DEV_BAD_GROUPS and got.isfinite().all()
    status.zero_()
    c["group_start"].copy_(torch.tensor([0, rows // 4, rows // 2, rows], dtype=torch.int32))
    A.shared_prefix_attn(**c, status=status)
    assert int(status) == 0


@pytest.mark.parametrize("per,room", [(2, 0), (2, 1800), (2, 30000), (40, 30000)])
def test_shared_prefix_attn_replays_with_new_lengths_and_groups(per, room):
    """One captured call follows lengths, tables, boundaries and queries; another graph with a workspace of its own may
    run beside it."""
    import paper_2506_18226_b200 as A
    g = _gen(51)
    a = attn_case(g, [100, 37, 64, 1], [90, 200], [0, 2, 4], 2, per, 64, 32, torch.bfloat16, room=room)
    out = torch.empty_like(a["q"])
    graphs = []
    for _ in range(2):
        o = torch.empty_like(out)
        ws = A.shared_prefix_workspace(a["q"], a["k_pool"], a["page_table"], a["prefix_table"])
        A.shared_prefix_attn(**a, out=o, workspace=ws)
        torch.cuda.synchronize()
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            A.shared_prefix_attn(**a, out=o, workspace=ws)
        graphs.append((gr, o, torch.cuda.Stream(), ws))                           # a graph's workspace lives as long as the graph
    for own, prefix, start in (([100, 37, 64, 1], [90, 200], [0, 2, 4]), ([1, 0, 64, 1], [5, 64], [0, 1, 1]), ([99, 37, 0, 0], [0, 199], [0, 3, 4])):
        a["n_rows"].copy_(torch.tensor(own, dtype=torch.int32))
        a["prefix_rows"].copy_(torch.tensor(prefix, dtype=torch.int32))
        a["group_start"].copy_(torch.tensor(start, dtype=torch.int32))
        a["q"].normal_()
        want = A.shared_prefix_attn(**a)
        torch.cuda.synchronize()
        for gr, o, st, _ in graphs:
            with torch.cuda.stream(st):
                for _ in range(3):
                    gr.replay()
        torch.cuda.synchronize()
        for gr, o, st, _ in graphs:
            assert torch.equal(o, want)


# ---- norms and residual ----------------------------------------------------------------------------------------------

def norm64(y, x, w_pre, w_post, gate, scale, eps):
    z, x = y.double(), x.double()
    if w_post is not None:
        z = z / torch.sqrt(z.square().mean(1, keepdim=True) + eps) * w_post.double()
    if gate is not None:
        z = z * gate.double().repeat_interleave(y.shape[0] // gate.shape[0], 0)
    new = x + scale * z
    inv = 1 / torch.sqrt(new.square().mean(1, keepdim=True) + eps)
    mag = x.abs() + (scale * z).abs()
    return new, (new * inv * w_pre.double() if w_pre is not None else None), mag, inv


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("wide", [False, True])
@pytest.mark.parametrize("rows,dim,gates", [(1, 8, 0), (32, 1280, 32), (7, 96, 1), (129, 264, 3), (2, 16384, 2), (5, 8200, 0), (1000, 768, 10),
                                            (3, 4096, 3), (66, 2048, 0), (3000, 8, 0), (2400, 1280, 24), (2400, 2056, 1), (2368, 6000, 2),
                                            (2369, 16384, 1)])
def test_norm_residual_matches_64_bits(rows, dim, gates, wide, dtype):
    import paper_2506_18226_b200 as A
    g = _gen(rows + dim)
    xt = torch.float32 if wide else dtype
    y, x = _randn(g, rows, dim, dtype=dtype, scale=0.7), _randn(g, rows, dim, dtype=xt, scale=2.0)
    w_pre, w_post = _randn(g, dim, dtype=dtype), _randn(g, dim, dtype=dtype)
    gate = _randn(g, gates, dim, dtype=dtype) if gates else None
    for post in (w_post, None):
        for pre in (w_pre, None):
            want, want_h, mag, inv = norm64(y, x, pre, post, gate, -0.75, 1e-5)
            got, h = A.norm_residual(y, x, pre, w_post=post, gate=gate, scale=-0.75, eps=1e-5)
            # a mean of squares in 32 bits, half its relative error through the root, and five products: 2^-19 of what is added
            tol = 2.0 ** -19 * mag
            # below the smallest normal number a type's steps are all smallest_normal * eps apart: half of one is added
            step = 0.5 * torch.finfo(xt).smallest_normal * torch.finfo(xt).eps
            assert ((got.double() - want).abs() <= tol + _u(xt) * (want.abs() + tol) + step).all()
            if pre is None:
                assert h is None
                continue
            # h sees that error through its own norm, whose mean is off by no more than the largest element's share
            tol_h = (tol + 2.0 ** -18 * want.abs() + want.abs() * inv * tol.amax(1, keepdim=True)) * inv * pre.double().abs()
            small = torch.finfo(dtype).smallest_normal * torch.finfo(dtype).eps
            assert ((h.double() - want_h).abs() <= tol_h + _u(dtype) * (want_h.abs() + tol_h) + small).all()
    a, b = A.norm_residual(y, x, w_pre, w_post=w_post, gate=gate)
    y2, x2 = y.clone(), x.clone()
    c, d = A.norm_residual(y2, x2, w_pre, w_post=w_post, gate=gate, x_out=x2, h=y2)   # in place of both inputs
    assert c is x2 and d is y2 and torch.equal(a, c) and torch.equal(b, d)


def test_norm_residual_zero_rows_and_rows_that_are_not_finite():
    import paper_2506_18226_b200 as A
    y = torch.zeros((4, 64), dtype=torch.bfloat16, device=DEV)
    x = torch.zeros_like(y)
    w = torch.ones(64, dtype=torch.bfloat16, device=DEV)
    y[1, 3], x[2, 5] = float("nan"), float("inf")
    x[3] = 2.0
    new, h = A.norm_residual(y, x, w, w_post=w)
    assert (new[0] == 0).all() and (h[0] == 0).all()
    assert torch.isnan(new[1]).all() and torch.isnan(h[1]).all()
    assert torch.isinf(new[2, 5]) and int((~torch.isfinite(new[2])).sum()) == 1
    assert (new[3] == 2.0).all() and (h[3] == 1.0).all()
    assert A.norm_residual(y[:0], x[:0], w)[0].shape == (0, 64)


# ---- together, streams, devices ----------------------------------------------------------------------------------------

def test_a_decode_loop_of_all_four_operators():
    """Prompt rows enter the shared prefix, then eight decode steps of append, attention and norm on a stream of their
    own, captured once and replayed; every step against 64 bits on what the cache holds."""
    import paper_2506_18226_b200 as A
    g = _gen(61)
    G, M, H, KV, d, P, page = 2, 3, 4, 2, 64, 21, 16
    B, steps, D = G * M, 8, H * d
    k_pool, v_pool, table = make_cache(g, [steps] * B + [P] * G, KV, page, d, torch.bfloat16)
    own, pre = table[:B].contiguous(), table[B:].contiguous()
    rot = A.Rotary(d, (8, 12, 12))
    i32 = dict(dtype=torch.int32, device=DEV)
    pos = torch.arange(P, **i32).repeat(G)[:, None].expand(-1, 3).contiguous()
    A.paged_append(_randn(g, G * P, KV, d), _randn(g, G * P, KV, d), k_pool, v_pool, pre, torch.zeros(G, **i32), rotary=rot, pos=pos)
    p_rows, start = torch.full((G,), P, **i32), torch.tensor([0, M, B], **i32)
    n_before, n_after, tpos = torch.zeros(B, **i32), torch.ones(B, **i32), torch.full((B, 3), P, **i32)
    qkv = torch.empty(B, H + 2 * KV, d, dtype=torch.bfloat16, device=DEV)
    qt, attn = torch.empty(B, H, d, dtype=torch.bfloat16, device=DEV), torch.empty(B, H, d, dtype=torch.bfloat16, device=DEV)
    x, h = _randn(g, B, D), torch.empty(B, D, dtype=torch.bfloat16, device=DEV)
    x0 = x.clone()
    w = _randn(g, D)
    ws = A.shared_prefix_workspace(qt, k_pool, own, pre)

    def step():
        A.paged_append(qkv[:, H:H + KV], qkv[:, H + KV:], k_pool, v_pool, own, n_before, rotary=rot, pos=tpos, q=qkv[:, :H], q_out=qt)
        A.shared_prefix_attn(qt, k_pool, v_pool, own, n_after, pre, p_rows, start, out=attn, workspace=ws)
        A.norm_residual(attn.view(B, D), x, w, w_post=w, x_out=x, h=h)
        for t in (n_before, n_after, tpos):
            t.add_(1)

    side = torch.cuda.Stream()
    graph = None
    for i in range(steps):
        qkv.copy_(_randn(g, B, H + 2 * KV, d))
        x_old = x.clone()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            if i == 0:
                step()
            elif graph is None:
                side.synchronize()
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=side):
                    step()
                graph.replay()
            else:
                graph.replay()
        torch.cuda.current_stream().wait_stream(side)
        n = torch.full((B,), i + 1, **i32)
        assert n_before.tolist() == [i + 1] * B
        turned, mag = turn64(qkv[:, :H], torch.full((B, 3), P + i, **i32), (8, 12, 12), "pairs", True)
        check_turned(qt, turned, mag, torch.bfloat16)
        out, _, amag, s_err = attn64(qt, k_pool, v_pool, own, n, pre, p_rows, start, 1 / 8)
        inner = (_u(torch.bfloat16) + 2 * s_err[..., None] + 2.0 ** -18) * amag
        assert ((attn.double() - out).abs() <= inner + _u(torch.bfloat16) * (out.abs() + inner)).all()
        want, want_h, nmag, _ = norm64(attn.view(B, D), x_old, w, w, None, 1.0, 1e-5)
        assert ((x.double() - want).abs() <= 2.0 ** -18 * nmag + _u(torch.bfloat16) * want.abs()).all()
    assert not torch.equal(x, x0)


def test_the_binding_refuses_tensors_on_the_gpu_of_wrong_types_shapes_and_strides():
    import paper_2506_18226_b200 as A
    bf, i32 = torch.bfloat16, torch.int32
    x, pos = torch.zeros(4, 2, 64, dtype=bf, device=DEV), torch.zeros(4, 2, dtype=i32, device=DEV)
    rot = A.Rotary(64, (16, 16))
    A.rope_axes(rot, x, pos)
    wide = torch.zeros(4, 2, 128, dtype=bf, device=DEV)
    for args in ((x.float(), pos), (x[..., :62], pos), (wide[..., ::2], pos), (x[0], pos), (x, pos[:3]), (x, pos.long()), (x, pos[:, :1]), (x, pos.cpu()),
                 (x, pos.T.contiguous().T), (x, pos, x[:3]), (x, pos, x.half()), (x, pos, x.cpu()), (x.cpu(), pos)):
        with pytest.raises(ValueError, match="rope_axes: "):
            A.rope_axes(rot, *args)
    pool = torch.zeros(5, 2, 16, 64, dtype=bf, device=DEV)
    table, n = torch.zeros(4, 2, dtype=i32, device=DEV), torch.zeros(4, dtype=i32, device=DEV)
    table[:, 0] = torch.arange(4)
    one, cu = torch.zeros(1, dtype=i32, device=DEV), torch.arange(5, dtype=i32, device=DEV)
    good = dict(k=x, v=x, k_pool=pool, v_pool=pool.clone(), page_table=table, n_rows=n)
    A.paged_append(**good, rotary=rot, pos=pos, q=x, q_out=x.clone(), status=one, cu_tokens=cu)
    assert int(one) == 0
    for kw in (dict(v_pool=pool[:4]), dict(k_pool=pool.half()), dict(k_pool=pool[:, :1]), dict(n_rows=n[:3]), dict(n_rows=n[:, None]), dict(n_rows=None),
               dict(page_table=table.long()), dict(page_table=table[0]), dict(page_table=table.T), dict(k=x.half()), dict(v=x[:, :1]), dict(v=wide[..., ::2]),
               dict(rotary=rot), dict(rotary=rot, pos=pos[:2]), dict(rotary=A.Rotary(32, (8, 8)), pos=pos), dict(q=x.half()), dict(q=x[:3]),
               dict(q=x, q_out=x[:, :1]), dict(cu_tokens=n), dict(cu_tokens=cu.cpu()), dict(status=n), dict(status=cu[:1].long()), dict(v=x.cpu())):
        with pytest.raises(ValueError, match="paged_append: "):
            A.paged_append(**dict(good, **kw))
    good = dict(q=x, k_pool=pool, v_pool=pool, page_table=table, n_rows=n, prefix_table=table[:1], prefix_rows=one, group_start=cu[::4].contiguous())
    A.shared_prefix_attn(**good)
    for kw in (dict(q=x.half()), dict(q=x[0]), dict(q=wide[..., ::2]), dict(n_rows=n[:2]), dict(n_rows=None), dict(page_table=table[:3]), dict(v_pool=pool[:4]),
               dict(prefix_rows=n), dict(prefix_rows=None), dict(group_start=one), dict(group_start=None), dict(prefix_table=table[0]), dict(out=x.half()),
               dict(out=wide[..., ::2]), dict(lse=n), dict(out_f32=x), dict(status=n), dict(k_pool=pool.cpu()), dict(workspace=torch.zeros(8, dtype=torch.uint8))):
        with pytest.raises(ValueError, match="shared_prefix_attn: "):
            A.shared_prefix_attn(**dict(good, **kw))
    with pytest.raises(A.AdsaError):
        A.shared_prefix_attn(**good, workspace=torch.zeros(256, dtype=torch.uint8, device=DEV))
    y, w = torch.zeros(4, 64, dtype=bf, device=DEV), torch.zeros(64, dtype=bf, device=DEV)
    A.norm_residual(y, y.clone(), w)
    for a, kw in (((y.float(), y, w), {}), ((y[0], y, w), {}), ((y, y[:3], w), {}), ((y, None, w), {}), ((y, y, w[:32]), {}), ((y, y, w.float()), {}),
                  ((y, y.long(), w), {}), ((y, y, w), dict(gate=w)), ((y, y, w), dict(w_post=y)), ((y, y, w), dict(h=y.float())), ((y, y, None), dict(h=y)),
                  ((y, y, w), dict(x_out=y[:2])), ((y, y, w.cpu()), {}), ((y[:, ::2], y[:, ::2], w[:32]), {})):
        with pytest.raises(ValueError, match="norm_residual: "):
            A.norm_residual(*a, **kw)


def test_calls_on_another_stream_and_empty_calls():
    import paper_2506_18226_b200 as A
    g = _gen(71)
    c = attn_case(g, [40, 3], [50], [0, 2], 2, 2, 64, 16, torch.float16)
    want = A.shared_prefix_attn(**c)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(20_000_000)
        q = c["q"] * 1                                                             # produced on this stream, behind the pause
        got = A.shared_prefix_attn(**dict(c, q=q))
    torch.cuda.synchronize()
    assert torch.equal(got, want)
    assert A.shared_prefix_attn(**dict(c, q=c["q"][:0], page_table=c["page_table"][:0], n_rows=c["n_rows"][:0])).shape == (0, 4, 64)
    rot = A.Rotary(64, (32,))
    x = _randn(g, 4, 2, 64)
    assert A.rope_axes(rot, x[:0], torch.zeros((0, 1), dtype=torch.int32, device=DEV)).shape == (0, 2, 64)
    assert A.rope_axes(rot, x[:, :0], torch.zeros((4, 1), dtype=torch.int32, device=DEV)).shape == (4, 0, 64)


# ---- the model shell for images of one prompt ---------------------------------------------------------------------------

def _shells(**kw):
    from paper_2506_18226_b200.shell import LlamaGenShell, SharedPromptShell, ShellConfig
    cfg = ShellConfig(n_layers=3, dim=128, n_heads=2, ffn_hidden=256, vocab=512, n_text=8, grid_h=6, grid_w=6, n_images=3, top_k=50,
                      budget_fraction=1.0, **kw)
    g = _gen(4)
    text = torch.randn(2, cfg.n_text, cfg.dim, generator=g, device=DEV).to(torch.bfloat16)
    return cfg, text, LlamaGenShell, SharedPromptShell


def test_shared_prompt_shell_follows_the_shell_with_private_caches():
    """The same weights, every image with its own copy of the same condition and nothing evicted: the logits after the
    condition and after five steps (fed the same ids) agree as two bf16 evaluations of one decoder do."""
    cfg, text, Private, Shared = _shells()
    a, b = Private(cfg, seed=2, use_graphs=False), Shared(cfg, seed=2, use_graphs=False)
    a.prefill(text.repeat_interleave(cfg.n_images, 0).contiguous())
    b.prefill(text)
    for cell in range(1, 7):
        x, y = a.logits.double(), b.logits.double()
        assert float((x - y).norm() / x.norm()) <= 3e-2 and float((x * y).sum() / (x.norm() * y.norm())) >= 0.999
        a.tokens.copy_(b.tokens)
        if cell < 6:
            a.decode_step(cell)
            b.decode_step(cell)
    assert int(b.status) == 0 and a.eng.get_status()[0] == 0


@pytest.mark.parametrize("sandwich", [False, True])
def test_shared_prompt_shell_graph_and_eager_steps_draw_the_same_ids(sandwich):
    cfg, text, _, Shared = _shells(sandwich_norm=sandwich)
    ids = []
    for graphs in (True, False, True):
        sh = Shared(cfg, seed=3, use_graphs=graphs)
        ids.append(sh.generate(text).clone())
        assert int(sh.status) == 0 and sh.n_before.tolist() == [35] * cfg.batch
    assert torch.equal(ids[0], ids[1]) and torch.equal(ids[0], ids[2])
    assert int(ids[0].min()) >= 0 and int(ids[0].max()) < cfg.vocab and len(set(ids[0].flatten().tolist())) > 8
    again = sh.generate(text).clone()                                             # the cache and the graph serve a second generation
    assert torch.equal(again, ids[0])
