"""Forms of the calls with many query rows per sequence that ordinary callers take: 16-bit outputs alone, single tokens beside long chunks, and where lse is no
number."""
import math

import pytest
import torch

from prompt_ref import DEV, HALF, attend64, gen, randn, starts, u
from test_gpu_chunk_attn import Cache, call
from test_gpu_packed_attn import CASES, inputs, verify

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens,H,KV,d", CASES)
def test_16_bit_outputs_alone(lens, H, KV, d, causal, dtype):
    import paper_2506_18226_b200 as A
    q, k, v = inputs(gen(sum(lens) + 5 * H + d), lens, lens, H, KV, d, dtype)
    lse = torch.empty(q.shape[:2], device=DEV)
    out = A.packed_attn(q, k, v, starts(lens), causal=causal, lse=lse)
    verify(q, k, v, lens, lens, causal, out, lse)
    assert torch.equal(A.packed_attn(q, k, v, starts(lens), causal=causal), out)


# 32 query rows a sequence and key head on the mean at most: calls that the kernel for few rows takes, with sequences of many of its items
MIXED = [([1] * 60 + [900] + [1] * 3, 1, 1, 64), ([1] * 40 + [200], 16, 4, 128), ([2, 700, 1, 0, 5] + [1] * 60, 2, 2, 128), ([1] * 130 + [500, 300], 12, 3, 64),
         ([1] * 60 + [33], 17, 1, 64), ([1] * 200 + [5], 31, 1, 128)]


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens,H,KV,d", MIXED)
def test_single_tokens_beside_a_prompt(lens, H, KV, d, causal, dtype):
    import paper_2506_18226_b200 as A
    assert sum(lens) * H // KV <= 32 * len(lens)
    lens_k = [n if n > 9 else 40 * n + 3 for n in lens]
    q, k, v = inputs(gen(sum(lens) + d), lens, lens_k, H, KV, d, dtype)
    lse = torch.empty(q.shape[:2], device=DEV)
    out = A.packed_attn(q, k, v, starts(lens), starts(lens_k), causal=causal, lse=lse)
    verify(q, k, v, lens, lens_k, causal, out, lse)


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("new,H,KV,d,page,prefix", [([1] * 50 + [700], 2, 2, 64, 64, None), ([1] * 30 + [150] + [1] * 20, 12, 3, 128, 16, 200), ([1, 1, 400] + [1] * 40, 4, 2, 100, 48, 77)])
def test_single_tokens_beside_a_long_chunk(new, H, KV, d, page, prefix, dtype):
    assert sum(new) * H // KV <= 32 * len(new)
    own = [n + 30 * (b % 7) for b, n in enumerate(new)]
    if prefix is None:
        call(Cache(gen(sum(new)), KV, page, d, dtype), own, new, H)
    else:
        call(Cache(gen(sum(new)), KV, page, d, dtype), own, new, H, [prefix, 33], [len(new) - 5, 5])


@pytest.mark.parametrize("batch,H,KV,d,n", [(3, 8, 2, 64, 500), (40, 20, 20, 64, 260), (2, 32, 4, 128, 2100)])
def test_single_tokens_give_what_the_decode_step_gives(batch, H, KV, d, n):
    """Outputs of both calls, each off by its own roundings: of the output (u of itself) in both, of the weights (u of what they add up) in one."""
    import paper_2506_18226_b200 as A
    cache = Cache(gen(n + 1), KV, 64, d, torch.bfloat16)
    own = [max(1, n - 37 * b) for b in range(batch)]
    q, kp, vp, args, out, _ = call(cache, own, [1] * batch, H)
    other = A.shared_prefix_attn(q, kp, vp, args["page_table"], args["n_rows"])
    for b in range(batch):
        want, _, mag, _ = attend64(q[b:b + 1], *cache.rows[b], [own[b]])
        tol = 2.01 * u(torch.bfloat16) * want.abs() + 1.01 * u(torch.bfloat16) * mag + 1e-4 * mag
        assert ((out[b:b + 1].double() - other[b:b + 1].double()).abs() <= tol).all()


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("n,m,H,KV,d", [(300, 300, 2, 2, 64), (1500, 2, 4, 1, 128), (700, 200, 2, 1, 256), (4000, 300, 1, 1, 64)])
def test_where_lse_is_no_number(n, m, H, KV, d, dtype):
    """NaN where a score that the row attends is NaN; -infinity (and an output of NaN) where all of them are -infinity; else as without."""
    import paper_2506_18226_b200 as A
    g = gen(n + d)
    q, k, v = randn(g, m, H, d, dtype=dtype), randn(g, n, KV, d, dtype=dtype), randn(g, n, KV, d, dtype=dtype)
    q[:, :, 0] = 1.0
    k[::3, 0, 0] = -math.inf                                               # (a weight of 0)
    q[m // 2, 0, 3] = math.nan
    k[n - 1, KV - 1, 1] = math.nan                                         # (the last token's last key head)
    for causal in (True, False):
        lse = torch.empty(m, H, device=DEV)
        out = A.packed_attn(q, k, v, starts([m]), starts([n]), causal=causal, lse=lse)
        want, ref, mag, _ = attend64(q, k, v, [n - m + i + 1 for i in range(m)] if causal else [n] * m)
        assert torch.equal(torch.isnan(lse), torch.isnan(ref)) and torch.equal(torch.isnan(out), torch.isnan(want))
        assert torch.equal(lse.double()[torch.isinf(ref)], ref[torch.isinf(ref)])
        fine = torch.isfinite(ref)
        assert fine.any() or not causal                                    # (both ways every token attends the last one, NaN in a call of one key head)
        assert ((lse.double() - ref)[fine].abs() < 1e-4).all()
        rows = torch.isfinite(want)
        assert ((out.double() - want).abs() <= u(dtype) * want.abs() + (u(dtype) + 1e-4) * mag + 1e-6)[rows].all()
    k[:, :, 0] = -math.inf
    k[:, :, 1:] = 0
    q.nan_to_num_(0.0)
    lse = torch.empty(m, H, device=DEV)
    out = A.packed_attn(q, k, v, starts([m]), starts([n]), causal=False, lse=lse)
    assert torch.isnan(out).all() and (lse == -math.inf).all()
