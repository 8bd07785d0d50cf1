"""The packed call with a status: refusals found on the host.  Addresses here are made up and never dereferenced."""
import pytest
import torch

import paper_2506_18226_b200 as A
from paper_2506_18226_b200 import binding as B

P = 0x10000000


def _packed(status, wsb=0, **kw):
    a = dict(dtype=0, q=P, qt=256, qh=64, k=P, kt=128, kh=64, v=P, vt=128, vh=64, cu_q=P, cu_k=P, batch=2, n_q=10, n_k=10, heads=4, kv=2, d=64, causal=1,
             scale=0.0, out=P, out32=None, lse=None, ws=P)
    a.update(kw)
    return A.load().adsa_packed_attn_status(*a.values(), wsb, status, None)


def test_a_status_has_to_be_aligned():
    assert _packed(P + 2) == B.EINVAL and _packed(P) == B.ENOMEM and _packed(None) == B.ENOMEM
    assert _packed(P, n_q=0) == 0 and _packed(P, heads=3) == B.EINVAL


def test_the_binding_takes_one_int32():
    bf = torch.bfloat16
    x, kv = torch.zeros(6, 4, 64, dtype=bf), torch.zeros(6, 2, 64, dtype=bf)
    for status in (torch.zeros(2, dtype=torch.int32), torch.zeros(1), torch.zeros(1, dtype=torch.int64), 3):
        with pytest.raises(ValueError):
            A.packed_attn(x, kv, kv, status=status)


def test_patience():
    lib = A.load()
    assert lib.adsa_prompt_wait_polls(3) == -1
    assert lib.adsa_prompt_wait_polls(-5) == 3
    assert lib.adsa_prompt_wait_polls(-1) == -1
