"""Prompt attention whose rows are copied one by one (no box fits their strides): every call of many gives the same bits, and the right ones."""
import pytest
import torch

from prompt_ref import DEV, attend64, check, gen, randn, starts

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("H,KV,d,pad", [(4, 2, 64, 2), (6, 3, 100, 6), (2, 1, 128, 4), (2, 1, 256, 2)])
def test_row_copies_over_and_over(H, KV, d, pad):
    import paper_2506_18226_b200 as A
    lens, g = [700, 130, 3, 1500], gen(d)
    T = sum(lens)
    q, k, v = (randn(g, T, h, d + pad)[..., :d] for h in (H, KV, KV))
    cu, ws, lse = starts(lens), A.prompt_workspace(q, KV, len(lens)), torch.empty(T, H, device=DEV)
    first = A.packed_attn(q, k, v, cu, lse=lse, workspace=ws).clone()
    a = 0
    for n in lens:
        check(first[a:a + n], lse[a:a + n], attend64(q[a:a + n], k[a:a + n], v[a:a + n], list(range(1, n + 1))), n, torch.bfloat16, d)
        a += n
    out = torch.empty_like(first)
    for _ in range(50):
        out.zero_()
        A.packed_attn(q, k, v, cu, out=out, workspace=ws)
        assert torch.equal(out, first)
