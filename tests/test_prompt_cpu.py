"""What the calls with many query rows per sequence refuse, found on the host before anything is launched, and the size of their
workspace.  Addresses here are made up and never dereferenced."""
import ctypes as C
import math

import pytest
import torch

import paper_2506_18226_b200 as A
from paper_2506_18226_b200 import binding as B

P = 0x10000000      # a 256-byte aligned address


def _packed(**kw):
    a = dict(dtype=0, q=P, qt=256, qh=64, k=P, kt=128, kh=64, v=P, vt=128, vh=64, cu_q=P, cu_k=P, batch=2, n_q=10, n_k=10, heads=4, kv=2, d=64, causal=1,
             scale=0.0, out=P, out32=None, lse=None, ws=P, wsb=1 << 40)
    a.update(kw)
    return A.load().adsa_packed_attn(*a.values(), None)


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(dtype=-1), dict(q=None), dict(k=None), dict(v=None), dict(out=None), dict(ws=None), dict(ws=P + 128),
                                dict(q=P + 2), dict(k=P + 2), dict(v=P + 1), dict(qt=255), dict(qh=63), dict(kt=127), dict(kh=63), dict(vt=1), dict(vh=3),
                                dict(cu_q=P + 2), dict(cu_k=P + 1), dict(lse=P + 2), dict(out=P + 2), dict(out32=P + 4), dict(batch=0), dict(batch=-1),
                                dict(batch=4097), dict(n_q=-1), dict(n_k=-1), dict(n_q=2**31), dict(n_k=2**31), dict(n_q=2**29), dict(heads=3), dict(heads=1),
                                dict(heads=0), dict(kv=0), dict(kv=-2), dict(heads=130), dict(d=63), dict(d=0), dict(d=258), dict(scale=-1.0),
                                dict(scale=math.nan), dict(cu_q=None, n_q=9), dict(cu_k=None, n_k=9)])
def test_packed_refusals(kw):
    assert _packed(**kw) == B.EINVAL


def test_nothing_to_do_is_ok():
    assert _packed(n_q=0) == 0 and _chunk(n=0) == 0


def _kv(**kw):
    a = dict(k_pool=P, v_pool=P, dtype=0, n_pages=10, n_kv_heads=2, page_rows=16, head_dim=64, row_stride=64)
    a.update(kw)
    return B.AdsaPagedKv(*a.values())


def _chunk(kv=None, **kw):
    a = dict(kv=C.byref(_kv(**(kv or {}))), q=P, qt=256, qh=64, cu=P, batch=2, n=10, heads=4, table=P, max_pages=3, n_rows=P, pt=P, mpp=2, pr=P, start=P,
             groups=1, scale=0.0, out=P, out32=None, lse=None, ws=P, wsb=1 << 40, status=None)
    a.update(kw)
    return A.load().adsa_chunk_attn(*a.values(), None)


@pytest.mark.parametrize("kv", [dict(k_pool=None), dict(v_pool=P + 8), dict(dtype=2), dict(n_pages=0), dict(n_kv_heads=0), dict(page_rows=0),
                                dict(page_rows=4097), dict(head_dim=63), dict(head_dim=72), dict(row_stride=60), dict(row_stride=264, head_dim=260),
                                dict(n_pages=2**25, n_kv_heads=4, page_rows=16)])
def test_chunk_refuses_bad_pools(kv):
    assert _chunk(kv=kv) == B.EINVAL


@pytest.mark.parametrize("kw", [dict(q=None), dict(table=None), dict(n_rows=None), dict(out=None), dict(ws=None), dict(ws=P + 128), dict(q=P + 2), dict(qt=255),
                                dict(qh=65), dict(batch=0), dict(batch=4097), dict(n=-1), dict(n=2**31), dict(heads=3), dict(heads=1), dict(heads=130),
                                dict(max_pages=0), dict(mpp=0), dict(pt=None), dict(pr=None), dict(start=None), dict(groups=-1), dict(groups=4097),
                                dict(scale=-1.0), dict(scale=math.nan), dict(out=P + 2), dict(out32=P + 4), dict(lse=P + 1), dict(status=P + 1),
                                dict(max_pages=2**27), dict(mpp=2**27), dict(cu=None, n=9), dict(cu=P + 2), dict(table=P + 2), dict(start=P + 1)])
def test_chunk_refusals(kw):
    assert _chunk(**kw) == B.EINVAL


def test_workspace_size_and_its_check():
    def size(*a):
        out = C.c_size_t(0)
        return A.load().adsa_prompt_workspace_bytes(*a, C.byref(out)), out.value
    rc, small = size(2, 4, 2, 64)
    assert rc == 0 and small > 0 and size(2, 4, 2, 128)[1] >= small
    for bad in ((0, 4, 2, 64), (4097, 4, 2, 64), (2, 4, 3, 64), (2, 4, 0, 64), (2, 4, 2, 65), (2, 4, 2, 258), (2, 130, 2, 64)):
        assert size(*bad)[0] == B.EINVAL
    assert A.load().adsa_prompt_workspace_bytes(2, 4, 2, 64, None) == B.EINVAL
    assert _packed(wsb=small - 1) == B.ENOMEM and _chunk(wsb=small - 1) == B.ENOMEM


def test_the_binding_refuses_wrong_types_shapes_and_devices():
    bf, i32 = torch.bfloat16, torch.int32
    x, kv, cu = torch.zeros(6, 4, 64, dtype=bf), torch.zeros(6, 2, 64, dtype=bf), torch.zeros(3, dtype=i32)
    for kw in (dict(), dict(q=x.float()), dict(q=x[0]), dict(k=kv.half()), dict(k=kv[..., :32]), dict(v=kv[:5]), dict(v=kv[:, :1]), dict(cu_q=cu.long()),
               dict(cu_q=cu[:1]), dict(cu_k=cu[:2]), dict(cu_q=None, cu_k=cu), dict(out=x.half()), dict(out_f32=x), dict(lse=cu), dict(q=x.transpose(1, 2))):
        with pytest.raises(ValueError):                                            # the first: not on a GPU
            A.packed_attn(**dict(dict(q=x, k=kv, v=kv, cu_q=cu), **kw))
    pool, table, n = torch.zeros(5, 2, 16, 64, dtype=bf), torch.zeros(2, 2, dtype=i32), torch.zeros(2, dtype=i32)
    for kw in (dict(), dict(q=x.half()), dict(k_pool=pool[..., :32]), dict(v_pool=pool[:3]), dict(page_table=n), dict(n_rows=cu), dict(cu_tokens=n),
               dict(prefix_rows=n), dict(group_start=n), dict(prefix_table=table, prefix_rows=n, group_start=n), dict(out=kv), dict(lse=x), dict(status=n)):
        with pytest.raises(ValueError):
            A.chunk_attn(**dict(dict(q=x, k_pool=pool, v_pool=pool, page_table=table, n_rows=n, cu_tokens=cu), **kw))
