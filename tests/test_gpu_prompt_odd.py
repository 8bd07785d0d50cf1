"""Prompt attention of values that are no finite numbers: every output element is what the rows that it attends make it, and a call takes about as long as
any other (an output made again by itself takes as long as its row has rows)."""
import math

import pytest
import torch

from prompt_ref import DEV, HALF, gen, randn, starts, u

pytestmark = pytest.mark.gpu


def reference(q, k, v, seen):
    """In 64 bits, with every weight above zero where its score is finite: infinities and NaN of V by themselves, the finite rest by products."""
    m, H, d = q.shape
    out = torch.empty(m, H, d, dtype=torch.float64, device=DEV)
    bound = torch.empty_like(out)
    n = torch.as_tensor(seen, device=DEV)
    mask = torch.arange(k.shape[0], device=DEV)[None] < n[:, None]
    for h in range(H):
        kk, vv = (x[:, h * k.shape[1] // H].double() for x in (k, v))
        x = (q[:, h].double() @ kk.T / math.sqrt(d))
        w = torch.softmax(x.masked_fill(~mask, -math.inf), 1)
        w = torch.where(mask, w, 0.0)
        odd = ~torch.isfinite(vv)
        fine = torch.where(odd, 0.0, vv)
        o = torch.where(torch.isnan(w).any(1, keepdim=True), math.nan, w.nan_to_num() @ fine)
        bound[:, h] = w.nan_to_num() @ fine.abs()
        has = [(mask.double() @ y.double()) > 0 for y in (torch.isnan(vv), vv == math.inf, vv == -math.inf)]
        o = torch.where(has[1], math.inf, o)
        o = torch.where(has[2], -math.inf, o)
        o = torch.where(has[0] | (has[1] & has[2]) | torch.isnan(w).any(1, keepdim=True), math.nan, o)
        out[:, h] = o
    return out, bound


def verify(out, want, dtype):
    ref, mag = want
    assert torch.equal(torch.isnan(out), torch.isnan(ref))
    inf = torch.isinf(ref)
    assert torch.equal(out.double()[inf], ref[inf]) and not torch.isinf(out[~inf]).any()
    fine = torch.isfinite(ref)
    err = (out.double() - ref).abs() - (u(dtype) * ref.abs() + (u(dtype) + 2e-4) * mag + 1e-6)
    assert (err[fine] <= 0).all()


def spoil(k, v, q, kind, g):
    n = v.shape[0]
    some = torch.randperm(n, generator=g, device=DEV)[:max(n // 40, 2)]
    if kind == "a column of infinities":
        v[:, :, 3] = math.inf
    elif kind == "some infinities of a column":
        v[some, :, 3] = math.inf
    elif kind == "either sign":
        v[some[::2], :, 5], v[some[1::2], :, 5], v[some, 0, 1] = math.inf, -math.inf, -math.inf
    elif kind == "a NaN value":
        v[n // 3, :, 2], v[n // 2, 0] = math.nan, math.nan
    elif kind == "NaN and infinities":
        v[some[::3], :, 7], v[some[1::3], :, 7], v[some[2::3], :, 8] = math.nan, math.inf, -math.inf
    elif kind == "late ones":
        v[n - 5:, :, 4], v[n - 1] = math.inf, math.nan
    elif kind == "a NaN key":
        k[n // 2, 0, 3] = math.nan
        v[some, :, 3] = math.inf
    elif kind == "NaN queries":
        q[::7] = math.nan
        v[some, :, 2] = -math.inf


KINDS = ["a column of infinities", "some infinities of a column", "either sign", "a NaN value", "NaN and infinities", "late ones", "a NaN key", "NaN queries"]


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("n,m,H,KV,d", [(600, 600, 4, 2, 64), (700, 700, 2, 1, 128), (500, 500, 2, 2, 256), (450, 450, 3, 3, 100), (2500, 3, 4, 2, 128), (5000, 2, 1, 1, 64),
                                        (3300, 3300, 1, 1, 64), (3000, 3000, 2, 2, 36), (2700, 200, 6, 6, 100)])
@pytest.mark.parametrize("f32", [0, 1, 2])
def test_each_element_by_what_it_attends(n, m, H, KV, d, kind, f32, dtype):
    import paper_2506_18226_b200 as A
    g = gen(n + d)
    q, k, v = randn(g, m, H, d, dtype=dtype), randn(g, n, KV, d, dtype=dtype), randn(g, n, KV, d, dtype=dtype)
    spoil(k, v, q, kind, g)
    for causal in (True, False):
        want = reference(q, k, v, [n - m + i + 1 for i in range(m)] if causal else [n] * m)
        out = torch.empty_like(q) if f32 < 2 else None
        also = torch.empty(q.shape, device=DEV) if f32 else None
        A.packed_attn(q, k, v, starts([m]), starts([n]), causal=causal, out=out, out_f32=also)
        if out is not None:
            verify(out, want, dtype)
        if also is not None:
            verify(also, want, dtype)


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("new,H,KV,d,page", [(1, 4, 2, 64, 16), (300, 4, 2, 128, 64), (9, 2, 2, 100, 20)])
def test_in_pages(new, H, KV, d, page, kind, dtype):
    import paper_2506_18226_b200 as A
    g, n, batch = gen(new), 900, 3
    per = n // page
    pools = randn(g, 2, batch * per, KV, page, (d + 7) // 8 * 8, dtype=dtype)
    q = randn(g, batch * new, H, d, dtype=dtype)
    k, v = (pools[i].transpose(1, 2).reshape(batch, per * page, KV, -1)[..., :d].clone() for i in range(2))
    for b in range(batch):
        spoil(k[b], v[b], q[b * new:(b + 1) * new], kind, g)
    for pool, x in zip(pools, (k, v)):
        pool[..., :d] = x.reshape(batch * per, page, KV, d).transpose(1, 2)
    n = per * page
    out = A.chunk_attn(q, pools[0], pools[1], torch.arange(batch * per, dtype=torch.int32, device=DEV).view(batch, per), torch.full((batch,), n, dtype=torch.int32, device=DEV))
    for b in range(batch):
        part = slice(b * new, (b + 1) * new)
        verify(out[part], reference(q[part], k[b], v[b], [n - new + i + 1 for i in range(new)]), dtype)


@pytest.mark.parametrize("dtype", HALF)
def test_a_value_of_infinity_whose_weight_is_zero(dtype):
    """A key of infinity makes a score of -infinity and a weight of zero: zero times infinity is NaN, as the formula has it."""
    import paper_2506_18226_b200 as A
    g, n = gen(9), 400
    q, k, v = (randn(g, n, 1, 64, dtype=dtype) for _ in range(3))
    q[:, :, 0], k[100, 0, 0], v[100, 0, 7], v[150, 0, 9] = 1.0, -math.inf, math.inf, math.inf
    out = A.packed_attn(q, k, v)[:, 0]
    assert torch.isfinite(out[:100]).all() and torch.isnan(out[100:, 7]).all()
    assert torch.isfinite(out[100:150, 9]).all() and (out[150:, 9] == math.inf).all()
    rest = [c for c in range(64) if c not in (7, 9)]
    assert torch.isfinite(out[:, rest]).all()


@pytest.mark.parametrize("what,dtype", [(what, dtype) for dtype in HALF for what in ("a NaN key", "NaN queries", "a NaN value", "a column of infinities",
                                                                                        "a column of infinities from the middle on")] + [("the largest values", torch.float16)])
def test_a_call_takes_no_longer_by_orders(what, dtype):
    """One sequence of 16384 tokens.  With every row made again by itself: 2000 times as long; with V and K looked at for eight rows at a time a tenth of that
    at most (half's largest values are known by their roundings alone; bfloat16's are made again row by row; the bound is there to tell the two apart, not to say how quick a call is)."""
    import paper_2506_18226_b200 as A
    g, n, H, KV, d = gen(3), 16384, 4, 1, 128
    q, k, v = randn(g, n, H, d, dtype=dtype), randn(g, n, KV, d, dtype=dtype), randn(g, n, KV, d, dtype=dtype)
    out, ws = torch.empty_like(q), A.prompt_workspace(q, KV, 1)

    def time():
        best = math.inf
        for _ in range(3):
            a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
            a.record()
            A.packed_attn(q, k, v, out=out, workspace=ws)
            b.record()
            torch.cuda.synchronize()
            best = min(best, a.elapsed_time(b))
        return best

    usual = time()
    if what == "a NaN key":
        k[0] = math.nan
    elif what == "NaN queries":
        q.fill_(math.nan)
    elif what == "a NaN value":
        v[0] = math.nan
    elif what == "a column of infinities":
        v[:, :, 3] = math.inf
    elif what == "a column of infinities from the middle on":
        v[n // 2:, :, 3] = math.inf
    else:
        v.fill_(65504.0)
    took = time()
    print(f"{what}: {took:.2f} ms, usually {usual:.2f}")
    assert took < 200 * usual
