"""Attention of a chunk of new tokens over a paged cache against 64 bits: pages, prefixes, lengths, single tokens, what lies in
places that are not attended; and the calls of a prompt that enters in chunks."""
import math

import pytest
import torch

from prompt_ref import DEV, HALF, attend64, check, gen, randn, starts

pytestmark = pytest.mark.gpu


class Cache:
    """Pools filled row by row; what no sequence owns, and the padding of a row, is NaN."""

    def __init__(self, g, KV, page, d, dtype, stride=None, spare=3):
        self.g, self.KV, self.page, self.d, self.dtype = g, KV, page, d, dtype
        self.stride, self.spare = stride or (d + 7) // 8 * 8, spare
        self.rows = []

    def add(self, n):
        k, v = randn(self.g, n, self.KV, self.d, dtype=self.dtype), randn(self.g, n, self.KV, self.d, dtype=self.dtype)
        self.rows.append((k, v))
        return len(self.rows) - 1

    def build(self):
        """Pools and one table per sequence [pages], padded with pages that do not exist."""
        counts = [(len(k) + self.page - 1) // self.page for k, _ in self.rows]
        total = sum(counts) + self.spare
        order = torch.randperm(total, generator=self.g, device=DEV).tolist()
        pools = [torch.full((total, self.KV, self.page, self.stride), math.nan, dtype=self.dtype, device=DEV) for _ in range(2)]
        tables, at = [], 0
        for (k, v), c in zip(self.rows, counts):
            pages = order[at:at + c]
            at += c
            for i, pg in enumerate(pages):
                part = slice(i * self.page, (i + 1) * self.page)
                for pool, x in zip(pools, (k, v)):
                    x = x[part]
                    pool[pg, :, :len(x), :self.d] = x.transpose(0, 1)
            tables.append(pages)
        return pools[0], pools[1], tables


def table_of(tables, width=None):
    width = width or max(1, max(len(t) for t in tables))
    return torch.tensor([t + [-7] * (width - len(t)) for t in tables], dtype=torch.int32, device=DEV)


def call(cache, own, new, H, prefix=None, groups=None, equal=False, extra=0, **kw):
    """own: row counts, new: tokens; prefix: row counts, groups: members of each.  Returns everything for verify()."""
    import paper_2506_18226_b200 as A
    ids = [cache.add(n) for n in own]
    p_ids = [cache.add(n) for n in prefix or []]
    kp, vp, tables = cache.build()
    q = randn(cache.g, sum(new), H, cache.d, dtype=cache.dtype, scale=1.5)
    i32 = dict(dtype=torch.int32, device=DEV)
    args = dict(page_table=table_of([tables[i] for i in ids], max(1, max(len(tables[i]) for i in ids)) + extra), n_rows=torch.tensor(own, **i32),
                cu_tokens=None if equal else starts(new))
    if prefix is not None:
        args.update(prefix_table=table_of([tables[i] for i in p_ids]), prefix_rows=torch.tensor(prefix, **i32), group_start=starts(groups))
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
    status = torch.zeros(1, **i32)
    A.chunk_attn(q, kp, vp, **args, out=out, lse=lse, status=status, **kw)
    assert int(status) == 0
    verify(cache, ids, p_ids, groups, q, own, new, out, lse, kw.get("scale"))
    return q, kp, vp, args, out, lse


def verify(cache, ids, p_ids, groups, q, own, new, out, lse, scale=None):
    a = 0
    group = [g for g, c in enumerate(groups or []) for _ in range(c)]
    for b, (n, m) in enumerate(zip(own, new)):
        k, v = cache.rows[ids[b]]
        p = 0
        if b < len(group):
            pk, pv = cache.rows[p_ids[group[b]]]
            p, k, v = len(pk), torch.cat([pk, k]), torch.cat([pv, v])
        seen = [p + min(max(n - m + i + 1, 0), n) for i in range(m)]
        check(out[a:a + m], None if lse is None else lse[a:a + m], attend64(q[a:a + m], k, v, seen, scale), p + n, q.dtype, q.shape[2], f"b={b} m={m} n={n} p={p}")
        a += m


CASES = [  # own rows, new tokens, heads, key heads, dim, page
    ([1], [1], 1, 1, 64, 16),
    ([5, 1, 300], [1, 1, 1], 4, 2, 64, 64),
    ([129, 64, 1000], [4, 1, 9], 8, 2, 128, 64),
    ([257, 128, 127, 3], [130, 128, 127, 3], 2, 2, 64, 128),
    ([700, 40], [300, 40], 5, 1, 100, 48),
    ([333, 512, 600], [1, 17, 100], 6, 6, 100, 16),
    ([90, 700], [64, 13], 4, 4, 128, 7),
    ([61, 200], [50, 1], 4, 1, 64, 1),
    ([600, 1200], [33, 572], 4, 2, 64, 572),
    ([300, 77], [20, 77], 64, 1, 64, 32),
    ([260, 400], [129, 3], 6, 2, 80, 100),
    ([200, 300], [64, 300], 4, 2, 192, 64),
    ([400, 129], [200, 1], 3, 1, 256, 24),
    ([3000], [2], 8, 1, 128, 64),
    ([40, 50, 60], [0, 50, 0], 2, 1, 64, 16),
    ([3500, 10], [1, 1], 16, 1, 36, 256),
    ([5, 40], [9, 40], 2, 2, 64, 16),              # fewer rows than tokens: the first tokens attend nothing
    ([0, 70], [3, 2], 2, 2, 64, 16),
]


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("own,new,H,KV,d,page", CASES)
def test_chunks_over_their_own_rows(own, new, H, KV, d, page, dtype):
    call(Cache(gen(sum(own) + d), KV, page, d, dtype), own, new, H)


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("own,new,prefix,groups,H,KV,d,page", [
    ([40, 200, 33, 90], [8, 16, 33, 1], [120, 77], [2, 2], 4, 4, 64, 64),
    ([300, 20, 1], [257, 20, 1], [500], [2], 8, 2, 128, 64),              # the last sequence is of no group
    ([64, 64, 64], [1, 1, 1], [1, 0, 300], [1, 1, 1], 2, 1, 100, 48),     # a prefix of no rows
    ([0, 3], [4, 7], [200], [2], 2, 2, 64, 16),                           # tokens that attend the prefix alone
    ([150, 20], [140, 20], [129, 128], [1, 1], 2, 2, 256, 10),
])
def test_chunks_under_shared_prefixes(own, new, prefix, groups, H, KV, d, page, dtype):
    call(Cache(gen(sum(own) + d), KV, page, d, dtype), own, new, H, prefix, groups)


@pytest.mark.parametrize("extra", [0, 5, 400])
def test_tables_wider_than_their_rows_and_equal_chunks(extra):
    call(Cache(gen(1), 2, 64, 64, torch.bfloat16), [200, 300, 64], [16, 16, 16], 4, equal=True, extra=extra, scale=0.2)


@pytest.mark.parametrize("batch,H,KV,d,n", [(3, 8, 2, 64, 500), (40, 20, 20, 64, 260), (2, 32, 4, 128, 2100), (1, 4, 4, 100, 5000)])
def test_single_tokens_agree_with_shared_prefix_attn(batch, H, KV, d, n):
    """One token a sequence: the decode step's call, whose weights meet V as two values; both within their own tolerance of 64 bits."""
    import paper_2506_18226_b200 as A
    cache = Cache(gen(n), KV, 64, d, torch.bfloat16)
    own = [max(1, n - 37 * b) for b in range(batch)]
    q, kp, vp, args, out, lse = call(cache, own, [1] * batch, H)
    other = torch.empty_like(lse)
    A.shared_prefix_attn(q, kp, vp, args["page_table"], args["n_rows"], lse=other)
    assert (lse - other).abs().max() < 1e-5


def test_lengths_out_of_range_are_clamped():
    import paper_2506_18226_b200 as A
    cache = Cache(gen(2), 2, 16, 64, torch.bfloat16)
    ids = [cache.add(n) for n in (48, 32, 16)]
    kp, vp, tables = cache.build()
    q = randn(cache.g, 9, 2, 64)
    table = table_of([tables[i] for i in ids])
    table[1, 2], table[2, 1:] = table[1, 1], table[2, 0]
    n = torch.tensor([1000, -5, 16], dtype=torch.int32, device=DEV)
    out, lse = torch.empty_like(q), torch.empty(9, 2, device=DEV)
    A.chunk_attn(q, kp, vp, table, n, out=out, lse=lse)
    verify(cache, ids, [], None, q[:3], [48], [3], out[:3], lse[:3])
    assert (out[3:6] == 0).all() and (lse[3:6] == -math.inf).all()
    verify(cache, ids[2:], [], None, q[6:], [16], [3], out[6:], lse[6:])


@pytest.mark.parametrize("bad", [-1, 10 ** 6])
def test_a_page_outside_the_pool_is_reported(bad):
    import paper_2506_18226_b200 as A
    cache = Cache(gen(3), 2, 16, 64, torch.bfloat16)
    ids = [cache.add(100), cache.add(60)]
    kp, vp, tables = cache.build()
    kp.nan_to_num_(), vp.nan_to_num_()
    table = table_of([tables[i] for i in ids])
    table[0, 2] = bad
    q, status = randn(cache.g, 20, 2, 64), torch.zeros(1, dtype=torch.int32, device=DEV)
    out = A.chunk_attn(q, kp, vp, table, torch.tensor([100, 60], dtype=torch.int32, device=DEV), status=status)
    assert int(status) == A.binding.DEV_BAD_PAGE
    verify(cache, ids[1:], [], None, q[10:], [60], [10], out[10:], None)            # the other sequence is as it should be
    A.chunk_attn(q, kp, vp, table, torch.tensor([100, 60], dtype=torch.int32, device=DEV))   # no status wanted


@pytest.mark.parametrize("KV,d,page", [(2, 64, 64), (2, 128, 20)])
def test_infinities_in_rows_that_a_token_does_not_attend(KV, d, page):
    cache = Cache(gen(9), KV, page, d, torch.bfloat16)
    ids = [cache.add(300)]
    k, v = cache.rows[0]
    q_seen = 260                                   # the chunk's last 40 rows hold infinities: tokens before them are as without
    import paper_2506_18226_b200 as A
    q = randn(cache.g, 140, 2 * KV, d)
    want = attend64(q, k.clone(), v.clone(), list(range(161, 301)))
    k[q_seen:, :, 1], v[q_seen:] = math.inf, -math.inf
    kp, vp, tables = cache.build()
    lse = torch.empty(140, 2 * KV, device=DEV)
    out = A.chunk_attn(q, kp, vp, table_of(tables), torch.tensor([300], dtype=torch.int32, device=DEV), lse=lse)
    check(out[:100], lse[:100], [w[:100] for w in want], 260, torch.bfloat16, d)
    assert not torch.isfinite(out[100:]).any()


@pytest.mark.parametrize("sizes", [[64, 64, 64, 64], [1, 2, 130, 67, 56], [200, 56]])
def test_a_prompt_that_enters_in_chunks(sizes):
    """Rotation and append, then attention, chunk by chunk under a shared prefix; the whole prompt at once by packed_attn."""
    import paper_2506_18226_b200 as A
    g, H, KV, d, page, B = gen(11), 4, 2, 64, 16, 3
    T = sum(sizes)
    pairs = (16, 16)
    rot = A.Rotary(d, pairs)
    q, k, v = randn(g, B * T, H, d), randn(g, B * T, KV, d), randn(g, B * T, KV, d)
    pos = torch.stack([torch.arange(T, device=DEV) // 16, torch.arange(T, device=DEV) % 16], 1).to(torch.int32).repeat(B, 1)
    qt, kt = A.rope_axes(rot, q, pos), A.rope_axes(rot, k, pos)
    cu = starts([T] * B)
    whole = A.packed_attn(qt, kt, v, cu)
    per = T // page + 1
    kp, vp = (torch.zeros(B * per, KV, page, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    table = torch.randperm(B * per, generator=g, device=DEV).to(torch.int32).view(B, per)
    n = torch.zeros(B, dtype=torch.int32, device=DEV)
    got = torch.empty(B, T, H, d, dtype=torch.bfloat16, device=DEV)
    at = 0
    ws = A.prompt_workspace(q, KV, B)
    for m in sizes:
        part = [x.view(B, T, -1, d)[:, at:at + m].reshape(B * m, -1, d) for x in (q, k, v)]
        p = pos.view(B, T, 2)[:, at:at + m].reshape(B * m, 2).clone()
        A.paged_append(part[1], part[2], kp, vp, table, n, rotary=rot, pos=p, q=part[0], q_out=part[0])
        n += m
        got[:, at:at + m] = A.chunk_attn(part[0], kp, vp, table, n, workspace=ws).view(B, m, H, d)
        at += m
    for b in range(B):
        want = attend64(qt[b * T:(b + 1) * T], kt[b * T:(b + 1) * T], v[b * T:(b + 1) * T], list(range(1, T + 1)))
        check(got[b], None, want, T, torch.bfloat16, d)
        check(whole[b * T:(b + 1) * T], None, want, T, torch.bfloat16, d)


def test_a_step_captured_into_a_graph_and_on_another_stream():
    import paper_2506_18226_b200 as A
    cache = Cache(gen(14), 2, 64, 128, torch.bfloat16)
    ids = [cache.add(n) for n in (700, 900)]
    kp, vp, tables = cache.build()
    q, out, lse = randn(cache.g, 8, 8, 128), None, torch.empty(8, 8, device=DEV)
    out = torch.empty_like(q)
    n, ws, table = torch.tensor([700, 900], dtype=torch.int32, device=DEV), A.prompt_workspace(q, 2, 2), table_of([tables[i] for i in ids])
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        A.chunk_attn(q, kp, vp, table, n, out=out, lse=lse, workspace=ws)
    side.synchronize()
    verify(cache, ids, [], None, q, [700, 900], [4, 4], out, lse)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        A.chunk_attn(q, kp, vp, table, n, out=out, lse=lse, workspace=ws)
    rows = cache.rows
    for now in ([700, 900], [5, 320], [64, 0]):
        n.copy_(torch.tensor(now, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        cache.rows = [(k[:c], v[:c]) for (k, v), c in zip(rows, now)]
        verify(cache, ids, [], None, q, now, [4, 4], out, lse)
