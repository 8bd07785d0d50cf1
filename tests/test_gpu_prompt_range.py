"""Prompt attention whose values are the largest of their type: an output is a mean of them, and so fits the type, whatever the
roundings on its way do."""
import math

import pytest
import torch

from prompt_ref import DEV, HALF, attend64, check, gen, starts

pytestmark = pytest.mark.gpu


def inputs(n_q, n_k, H, KV, d, dtype):
    """One row in 128 has a score of 0, the others ln 0.50026: half-type weights relative to them, times 2^6, are 32.0166, which
    rounds up by just under 2^-11 of itself, so that a mean taken with weights that are rounded and a sum that is not comes out
    2^-11.05 too large; 65504 (1 + 2^-12) would round to infinity.  (bfloat16: two products of the largest value are beyond 32 bits.)"""
    q, k = torch.zeros(n_q, H, d, dtype=dtype, device=DEV), torch.zeros(n_k, KV, d, dtype=dtype, device=DEV)
    x = math.log(0.50026)
    big = float(torch.tensor(x).to(dtype))
    q[..., :2] = 1.0
    k[..., 0], k[..., 1] = big, x - big
    k[::128] = 0.0
    v = torch.full((n_k, KV, d), torch.finfo(dtype).max, dtype=dtype, device=DEV)
    v[..., 1::2] *= -1
    return q, k, v


def expect(out, f32, v, H):
    """Every value of a column is the same, and so is their mean (in 32 bits up to what the sums round)."""
    want = v[:1].repeat_interleave(H // v.shape[1], 1).expand(out.shape)
    assert torch.equal(out, want), f"{int((out != want).sum())} of {out.numel()} differ, {int(torch.isinf(out).sum())} infinite"
    if f32 is not None:
        rel = (f32.double() / want.double() - 1).abs().max()
        # weights that are rounded once may stand where the output fits its type all the same
        assert torch.isfinite(f32).all() and float(rel) <= torch.finfo(v.dtype).eps / 2 + 1e-4


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("n,H,KV,d", [(1024, 4, 4, 64), (1030, 8, 2, 128), (700, 2, 1, 256), (900, 3, 3, 100), (6000, 1, 1, 64), (3100, 2, 1, 192)])
@pytest.mark.parametrize("f32", [False, True])
def test_prompts(n, H, KV, d, f32, dtype):
    import paper_2506_18226_b200 as A
    q, k, v = inputs(n, n, H, KV, d, dtype)
    out, also = torch.empty_like(q), torch.empty(q.shape, device=DEV) if f32 else None
    A.packed_attn(q, k, v, scale=1.0, out=out, out_f32=also)
    expect(out, also, v, H)


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("lens_k,m,H,KV,d", [([1000, 5], 1, 4, 4, 64), ([1024, 2048, 300], 3, 8, 2, 128), ([9000], 2, 4, 1, 64), ([9000], 7, 2, 2, 128)])
def test_few_rows(lens_k, m, H, KV, d, dtype):
    import paper_2506_18226_b200 as A
    q, k, v = inputs(m * len(lens_k), sum(lens_k), H, KV, d, dtype)
    out, f32 = torch.empty_like(q), torch.empty(q.shape, device=DEV)
    A.packed_attn(q, k, v, starts([m] * len(lens_k)), starts(lens_k), scale=1.0, out=out, out_f32=f32)
    expect(out, f32, v, H)


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("n,m,H,KV,d,page", [(2048, 1, 4, 2, 64, 64), (9000, 5, 4, 1, 128, 64), (2000, 300, 4, 2, 64, 128), (1500, 200, 2, 2, 100, 20), (6000, 130, 1, 1, 256, 16)])
def test_chunks(n, m, H, KV, d, page, dtype):
    import paper_2506_18226_b200 as A
    q, k, v = inputs(m, n, H, KV, d, dtype)
    pages, stride = (n + page - 1) // page, (d + 7) // 8 * 8
    pools = torch.zeros(2, pages * page, KV, stride, dtype=dtype, device=DEV)
    pools[0, :n, :, :d], pools[1, :n, :, :d] = k, v
    pools = pools.view(2, pages, page, KV, stride).transpose(2, 3).contiguous()
    out, f32 = torch.empty_like(q), torch.empty(q.shape, device=DEV)
    A.chunk_attn(q, pools[0], pools[1], torch.arange(pages, dtype=torch.int32, device=DEV)[None], torch.tensor([n], dtype=torch.int32, device=DEV), scale=1.0, out=out,
                 out_f32=f32)
    expect(out, f32, v, H)


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("n,m,H,KV,d", [(600, 600, 4, 2, 64), (5000, 3, 4, 2, 128)])
def test_large_values_of_either_sign(n, m, H, KV, d, dtype):
    """Random values up to the largest, random scores: within the tolerance of any other call."""
    import paper_2506_18226_b200 as A
    g = gen(n)
    q, k = (torch.randn(*shape, d, generator=g, device=DEV).to(dtype) for shape in ((m, H), (n, KV)))
    v = ((torch.rand(n, KV, d, generator=g, device=DEV) * 2 - 1) * torch.finfo(dtype).max).to(dtype)
    lse = torch.empty(m, H, device=DEV)
    out = A.packed_attn(q, k, v, starts([m]), starts([n]), lse=lse)
    check(out, lse, attend64(q, k, v, [n - m + i + 1 for i in range(m)]), n, dtype, d)
