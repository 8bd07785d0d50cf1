"""Prompt attention with as much work in a call as memory holds: many tokens in many sequences, and more units of work than 32 bits count."""
import math

import pytest
import torch

from prompt_ref import DEV, attend64, check, gen, randn, starts

pytestmark = pytest.mark.gpu


def test_a_thousand_prompts_of_a_thousand_tokens():
    import paper_2506_18226_b200 as A
    g, H, KV, d, batch = gen(1), 32, 8, 16, 1024
    lens = [1024 + (b * 37) % 101 - 50 for b in range(batch)]
    T = sum(lens)
    q, k, v = randn(g, T, H, d, scale=1.5), randn(g, T, KV, d), randn(g, T, KV, d)
    out, lse = torch.full_like(q, math.nan), torch.full((T, H), math.nan, device=DEV)
    cu = starts(lens)
    A.packed_attn(q, k, v, cu, out=out, lse=lse)
    assert torch.isfinite(out).all() and torch.isfinite(lse).all()
    at = cu.tolist()
    for b in (0, 1, 511, 700, batch - 1):
        part = slice(at[b], at[b + 1])
        check(out[part], lse[part], attend64(q[part], k[part], v[part], list(range(1, lens[b] + 1))), lens[b], torch.bfloat16, d, f"b={b}")


def test_more_units_than_32_bits_count():
    """537.6 million items of nothing (a token and head each, no rows to attend, 8 units an item): every row of every one is written."""
    import paper_2506_18226_b200 as A
    batch, H, d = 4000, 134400, 2
    assert batch * H * 8 > 2 ** 32
    q = torch.ones(batch, H, d, dtype=torch.bfloat16, device=DEV)
    kv = torch.ones(0, H, d, dtype=torch.bfloat16, device=DEV)
    out, lse = torch.full_like(q, 7.0), torch.full((batch, H), 7.0, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    cu = torch.arange(batch + 1, dtype=torch.int32, device=DEV)
    A.packed_attn(q, kv, kv, cu, torch.zeros_like(cu), out=out, lse=lse, status=status)
    assert int(status) == 0 and not bool(out.any()) and bool((lse == -math.inf).all())
