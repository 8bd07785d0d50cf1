"""Prompt attention where items are cut between blocks, where element offsets pass 32 bits, with many sequences, and two calls at once."""
import math

import pytest
import torch

from prompt_ref import DEV, HALF, attend64, check, gen, randn, starts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("lens,H,KV,d", [([2600, 1900], 2, 1, 256), ([3100], 2, 2, 128), ([2900, 5], 4, 1, 64), ([2700], 3, 1, 100), ([2048, 2049], 1, 1, 192),
                                         ([6000], 1, 1, 36)])
@pytest.mark.parametrize("causal", [True, False])
def test_items_cut_between_blocks(lens, H, KV, d, causal, dtype):
    """Few long items: every one lies in the runs of several blocks."""
    import paper_2506_18226_b200 as A
    g, T = gen(sum(lens)), sum(lens)
    q, k, v = randn(g, T, H, d, dtype=dtype, scale=1.5), randn(g, T, KV, d, dtype=dtype), randn(g, T, KV, d, dtype=dtype)
    out, f32, lse = torch.empty_like(q), torch.empty(T, H, d, device=DEV), torch.empty(T, H, device=DEV)
    A.packed_attn(q, k, v, starts(lens), causal=causal, out=out, out_f32=f32, lse=lse)
    only16 = A.packed_attn(q, k, v, starts(lens), causal=causal)
    a = 0
    for n in lens:
        want = attend64(q[a:a + n], k[a:a + n], v[a:a + n], list(range(1, n + 1)) if causal else [n] * n)
        check(out[a:a + n], lse[a:a + n], want, n, dtype, d)
        check(f32[a:a + n], None, want, n, dtype, d)
        check(only16[a:a + n], None, want, n, dtype, d)
        a += n


@pytest.mark.parametrize("H,KV,d", [(2, 1, 128), (2, 2, 64), (1, 1, 256), (3, 3, 100)])
@pytest.mark.parametrize("bad", [math.inf, math.nan])
def test_cut_items_and_what_their_rows_do_not_attend(H, KV, d, bad):
    import paper_2506_18226_b200 as A
    g, n, first = gen(d), 3000, 2300
    q, k, v = randn(g, n, H, d, scale=1.5), randn(g, n, KV, d), randn(g, n, KV, d)
    want = attend64(q, k, v, list(range(1, n + 1)))
    k[first:, :, 1], v[first:] = bad, bad
    lse = torch.empty(n, H, device=DEV)
    out = A.packed_attn(q, k, v, lse=lse)
    check(out[:first], lse[:first], [w[:first] for w in want], first, torch.bfloat16, d)
    assert not torch.isfinite(out[first:]).any()


@pytest.mark.parametrize("new,H,KV,d,prefix", [(1, 4, 1, 64, 0), (3, 8, 2, 128, 700), (20, 1, 1, 100, 0), (300, 2, 1, 256, 500), (200, 4, 4, 64, 1000)])
def test_chunks_cut_between_blocks(new, H, KV, d, prefix):
    import paper_2506_18226_b200 as A
    g, page, B, n = gen(new + d), 64, 2, 5000
    per, p_per = (n + page - 1) // page, (prefix + page - 1) // page
    pools = torch.full((2, B * per + p_per, KV, page, (d + 7) // 8 * 8), math.nan, dtype=torch.bfloat16, device=DEV)
    k, v = randn(g, B, n, KV, d), randn(g, B, n, KV, d)
    pk, pv = randn(g, prefix, KV, d), randn(g, prefix, KV, d)
    for pool, own, pre in zip(pools, (k, v), (pk, pv)):
        for b in range(B):
            for i in range(per):
                x = own[b, i * page:(i + 1) * page]
                pool[b * per + i, :, :len(x), :d] = x.transpose(0, 1)
        for i in range(p_per):
            x = pre[i * page:(i + 1) * page]
            pool[B * per + i, :, :len(x), :d] = x.transpose(0, 1)
    i32 = dict(dtype=torch.int32, device=DEV)
    kw = dict(prefix_table=torch.arange(B * per, B * per + p_per, **i32)[None], prefix_rows=torch.tensor([prefix], **i32), group_start=torch.tensor([0, B], **i32)) if prefix else {}
    q, rows = randn(g, B * new, H, d, scale=1.5), torch.tensor([n, n - 777], **i32)
    lse = torch.empty(B * new, H, device=DEV)
    out = A.chunk_attn(q, pools[0], pools[1], torch.arange(B * per, **i32).view(B, per), rows, lse=lse, **kw)
    for b in range(B):
        m = int(rows[b])
        part = slice(b * new, (b + 1) * new)
        want = attend64(q[part], torch.cat([pk, k[b, :m]]), torch.cat([pv, v[b, :m]]), [prefix + m - new + i + 1 for i in range(new)])
        check(out[part], lse[part], want, prefix + m, torch.bfloat16, d, f"b={b}")


@pytest.mark.parametrize("batch,tokens", [(300, 3), (4000, 1), (2000, 2), (700, 40)])
def test_many_sequences(batch, tokens):
    import paper_2506_18226_b200 as A
    g, H, KV, d = gen(batch), 2, 1, 64
    lens = [(tokens + b % 3) if b % 7 else 0 for b in range(batch)]
    T = sum(lens)
    q, k, v = randn(g, T, H, d), randn(g, T, KV, d), randn(g, T, KV, d)
    out = A.packed_attn(q, k, v, starts(lens))
    # in one go: sequences as blocks of a mask
    seq = torch.repeat_interleave(torch.arange(batch, device=DEV), torch.tensor(lens, device=DEV))
    at = torch.arange(T, device=DEV)
    for r in range(0, T, 4096):
        rows = slice(r, min(r + 4096, T))
        lo = max(0, r - 64)
        cols = slice(lo, rows.stop)
        seen = (seq[rows, None] == seq[None, cols]) & (at[None, cols] <= at[rows, None])
        x = torch.einsum("thd,jd->htj", q[rows].double(), k[cols, 0].double()) / math.sqrt(d)
        w = torch.softmax(x.masked_fill(~seen, -math.inf), -1)
        want = torch.einsum("htj,jd->thd", w, v[cols, 0].double())
        mag = torch.einsum("htj,jd->thd", w, v[cols, 0].double().abs())
        assert ((out[rows].double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 1e-4) * mag).all()


def test_offsets_past_32_bits():
    """Rows of q and of the outputs, and pages of the pools, beyond 2^31 elements."""
    import paper_2506_18226_b200 as A
    g, H, d = gen(1), 128, 128
    T, lens = 135000, [500, 331]
    first = T - sum(lens)
    q, out = torch.empty(T, H, d, dtype=torch.bfloat16, device=DEV), torch.empty(T, H, d, dtype=torch.bfloat16, device=DEV)
    q[first:].normal_(generator=g)
    k, v = (torch.empty(T, 2, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    k[first:].normal_(generator=g), v[first:].normal_(generator=g)
    A.packed_attn(q, k, v, starts(lens, first), out=out)
    a = first
    for n in lens:
        want = attend64(q[a:a + n, ::37], k[a:a + n], v[a:a + n], list(range(1, n + 1)))   # (heads 0, 37, 74, 111: two on each key head)
        check(out[a:a + n, ::37], None, want, n, torch.bfloat16, d)
        a += n
    del out, k, v
    page, pages = 64, 2 ** 31 // (2 * 64 * d) + 50
    kp, vp = (torch.empty(pages, 2, page, d, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    kp[-20:].normal_(generator=g), vp[-20:].normal_(generator=g)
    table = torch.arange(pages - 20, pages, dtype=torch.int32, device=DEV).view(2, 10)
    n = torch.tensor([600, 333], dtype=torch.int32, device=DEV)
    for new in (2, 70):
        qq = q[-2 * new:, :4].contiguous()
        got = A.chunk_attn(qq, kp, vp, table, n)
        for b in range(2):
            rows = [x[table[b].long()].transpose(1, 2).reshape(-1, 2, d)[:int(n[b])] for x in (kp, vp)]
            part = slice(b * new, (b + 1) * new)
            check(got[part], None, attend64(qq[part], *rows, [int(n[b]) - new + i + 1 for i in range(new)]), 600, torch.bfloat16, d)


def test_two_calls_at_once_and_two_graphs():
    """Calls on two streams with a workspace each, and two captured calls replayed side by side, give what they give alone."""
    import paper_2506_18226_b200 as A
    g = gen(2)
    sets = []
    for lens in ([2500, 100], [1, 3000]):
        T = sum(lens)
        q, k, v = randn(g, T, 4, 64), randn(g, T, 2, 64), randn(g, T, 2, 64)
        cu = starts(lens)
        sets.append((q, k, v, cu, A.prompt_workspace(q, 2, 2), torch.empty_like(q), A.packed_attn(q, k, v, cu)))
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(5):
        for s, (q, k, v, cu, ws, out, _) in zip(streams, sets):
            with torch.cuda.stream(s):
                A.packed_attn(q, k, v, cu, out=out, workspace=ws)
    torch.cuda.synchronize()
    for *_, out, want in sets:
        assert torch.equal(out, want)
        out.zero_()
    graphs = []
    for q, k, v, cu, ws, out, _ in sets:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            A.packed_attn(q, k, v, cu, out=out, workspace=ws)
        graphs.append(graph)
    torch.cuda.synchronize()
    for s, graph in zip(streams, graphs):
        with torch.cuda.stream(s):
            graph.replay()
    torch.cuda.synchronize()
    for *_, out, want in sets:
        assert torch.equal(out, want)


def test_pages_of_any_size_and_a_small_workspace():
    import paper_2506_18226_b200 as A
    g, d = gen(5), 64
    for page in (1, 2, 3, 5, 8, 40, 250):
        n, new = 421, 30
        per = (n + page - 1) // page
        kp, vp = randn(g, per, 2, page, d), randn(g, per, 2, page, d)
        table = torch.randperm(per, generator=g, device=DEV).to(torch.int32)[None]
        rows = [x[table[0].long()].transpose(1, 2).reshape(-1, 2, d)[:n] for x in (kp, vp)]
        for m in (1, new, 250):
            q = randn(g, m, 4, d)
            out = A.chunk_attn(q, kp, vp, table, torch.tensor([n], dtype=torch.int32, device=DEV))
            check(out, None, attend64(q, *rows, [n - m + i + 1 for i in range(m)]), n, torch.bfloat16, d, f"page={page} m={m}")
    with pytest.raises(A.AdsaError) as e:
        A.packed_attn(q, q, q, workspace=torch.empty(256, dtype=torch.uint8, device=DEV))
    assert e.value.status == A.binding.ENOMEM
