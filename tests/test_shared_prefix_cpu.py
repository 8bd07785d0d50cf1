"""What the calls on a paged whole-token cache refuse, found on the host before anything is launched; the rotary's table;
the workspace's size.  Addresses here are made up and never dereferenced."""
import ctypes as C
import math

import pytest
import torch

import paper_2506_18226_b200 as A
from paper_2506_18226_b200 import binding as B

P = 0x10000000      # a 256-byte aligned address


def _rot(head_dim=64, pairs=(16, 16), halves=0, restart=1, base=0.0):
    r = B.AdsaRotary()
    rc = A.load().adsa_rotary_init(C.byref(r), head_dim, len(pairs), (C.c_int32 * max(1, len(pairs)))(*pairs), halves, restart, base)
    return rc, r


def test_rotary_table():
    rc, r = _rot(100, (10, 0, 20), restart=1)
    assert rc == 0 and (r.head_dim, r.n_axes, r.n_pairs, r.halves) == (100, 3, 30, 0)
    assert list(r.axis)[:30] == [0] * 10 + [2] * 20
    for i in range(30):
        j, n = (i, 10) if i < 10 else (i - 10, 20)
        assert math.isclose(r.turns[i] * 2 * math.pi, 10000.0 ** (-j / n), rel_tol=1e-14)
    rc, r = _rot(128, (16, 24, 24), halves=1, restart=0, base=500.0)
    assert rc == 0 and r.halves == 1
    for i in range(64):
        assert math.isclose(r.turns[i] * 2 * math.pi, 500.0 ** (-i / 64), rel_tol=1e-14)


@pytest.mark.parametrize("kw", [dict(head_dim=63), dict(head_dim=0), dict(head_dim=258), dict(pairs=()), dict(pairs=(4,) * 5), dict(pairs=(0, 0)),
                                dict(pairs=(-1, 5)), dict(pairs=(20, 13)), dict(pairs=(2**31 - 1, 2)), dict(base=-1.0), dict(base=math.nan), dict(base=math.inf)])
def test_rotary_refusals(kw):
    assert _rot(**kw)[0] == B.EINVAL
    if "base" not in kw or kw["base"] == -1.0:
        with pytest.raises(A.AdsaError):
            A.Rotary(kw.get("head_dim", 64), kw.get("pairs", (16, 16)), base=kw.get("base", 0.0))


def test_rotary_style_is_checked():
    with pytest.raises(ValueError):
        A.Rotary(64, (32,), style="both")


def _rope(**kw):
    a = dict(rot=C.byref(_rot()[1]), dtype=0, x=P, xt=128, xh=64, pos=P, tokens=4, heads=2, out=P + 4096, ot=128, oh=64)
    a.update(kw)
    return A.load().adsa_rope_axes(*a.values(), None)


def test_a_rotary_with_an_axis_it_does_not_have_is_refused():
    r = _rot()[1]
    r.axis[5] = 2
    assert _rope(rot=C.byref(r)) == B.EINVAL and _append(rot=C.byref(r), pos=P) == B.EINVAL


def test_the_header_is_plain_c():
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-fsyntax-only", "-x", "c", os.path.join(root, "include", "adsa.h")], check=True)


@pytest.mark.parametrize("kw", [dict(rot=None), dict(dtype=2), dict(dtype=-1), dict(x=None), dict(out=None), dict(pos=None), dict(tokens=-1),
                                dict(heads=-1), dict(x=P + 1), dict(out=P + 1), dict(pos=P + 2), dict(out=P, ot=256)])
def test_rope_axes_refusals(kw):
    assert _rope(**kw) == B.EINVAL


def test_nothing_to_do_is_ok():
    assert _rope(tokens=0) == 0 and _rope(heads=0) == 0
    assert _append(n_tokens=0) == 0 and _attn(batch=0) == 0 and _norm(rows=0) == 0


def _kv(**kw):
    a = dict(k_pool=P, v_pool=P, dtype=0, n_pages=10, n_kv_heads=2, page_rows=16, head_dim=64, row_stride=64)
    a.update(kw)
    return B.AdsaPagedKv(*a.values())


BAD_KV = [dict(k_pool=None), dict(v_pool=P + 8), dict(dtype=2), dict(n_pages=0), dict(n_kv_heads=0), dict(page_rows=0), dict(page_rows=4097),
          dict(head_dim=63), dict(head_dim=0), dict(head_dim=72), dict(row_stride=60), dict(row_stride=264, head_dim=260),
          dict(n_pages=2**25, n_kv_heads=4, page_rows=16)]


def _append(kv=None, **kw):
    a = dict(kv=C.byref(_kv(**(kv or {}))), table=P, batch=2, max_pages=3, n_rows=P, cu=None, n_tokens=4, k=P, kt=128, kh=64, v=P, vt=128, vh=64,
             rot=None, pos=None, q=None, heads=0, qt=0, qh=0, qo=None, qot=0, qoh=0, status=None)
    a.update(kw)
    return A.load().adsa_paged_append(*a.values(), None)


@pytest.mark.parametrize("kv", BAD_KV)
def test_append_and_attention_refuse_bad_pools(kv):
    assert _append(kv=kv) == B.EINVAL
    assert _attn(kv=kv) == B.EINVAL


@pytest.mark.parametrize("kw", [dict(table=None), dict(n_rows=None), dict(k=None), dict(v=None), dict(batch=0), dict(max_pages=0), dict(n_tokens=-1),
                                dict(n_tokens=3), dict(n_tokens=2**31), dict(heads=2), dict(heads=2, q=P), dict(heads=-1), dict(k=P + 1), dict(cu=P + 2),
                                dict(status=P + 1), dict(heads=2, q=P, qo=P, qt=128, qot=256, qh=64, qoh=64)])
def test_append_refusals(kw):
    assert _append(**kw) == B.EINVAL


def test_append_refuses_a_rotary_that_does_not_fit():
    rot = _rot()[1]
    assert _append(rot=C.byref(rot)) == B.EINVAL                                  # no positions
    assert _append(rot=C.byref(_rot(128, (64,))[1]), pos=P) == B.EINVAL           # another head dimension
    assert _append(rot=C.byref(B.AdsaRotary()), pos=P) == B.EINVAL                # never initialised


def _attn(kv=None, **kw):
    a = dict(kv=C.byref(_kv(**(kv or {}))), q=P, qr=256, qh=64, batch=2, heads=4, table=P, max_pages=3, n_rows=P, pt=P, mpp=2, pr=P, start=P, groups=1,
             scale=0.0, out=P, out32=None, lse=None, ws=P, wsb=1 << 40, status=None)
    a.update(kw)
    return A.load().adsa_shared_prefix_attn(*a.values(), None)


@pytest.mark.parametrize("kw", [dict(q=None), dict(table=None), dict(n_rows=None), dict(out=None), dict(ws=None), dict(ws=P + 128), dict(q=P + 2),
                                dict(qr=255), dict(qh=65), dict(batch=-1), dict(batch=4095), dict(heads=3), dict(heads=1), dict(heads=130),
                                dict(max_pages=0), dict(mpp=0), dict(pt=None), dict(pr=None), dict(start=None), dict(groups=-1), dict(groups=2048),
                                dict(scale=-1.0), dict(scale=math.nan), dict(out=P + 2), dict(out32=P + 4), dict(lse=P + 1), dict(status=P + 1),
                                dict(max_pages=2**27), dict(mpp=2**27), dict(max_pages=2**27 - 8)])
def test_attention_refusals(kw):
    assert _attn(**kw) == B.EINVAL


def test_workspace_size_and_its_check():
    def size(*a):
        out = C.c_size_t(0)
        rc = A.load().adsa_shared_prefix_workspace_bytes(*a, C.byref(out))
        return rc, out.value
    rc, small = size(2, 1, 4, 2, 64)
    assert rc == 0 and small > 0
    assert size(64, 1, 32, 8, 128)[1] > small
    for bad in ((0, 1, 4, 2, 64), (2, -1, 4, 2, 64), (2, 1, 4, 3, 64), (2, 1, 4, 0, 64), (2, 1, 4, 2, 65), (2, 1, 4, 2, 258), (4095, 1, 4, 2, 64),
                (2, 1, 130, 2, 64)):
        assert size(*bad)[0] == B.EINVAL
    assert A.load().adsa_shared_prefix_workspace_bytes(2, 1, 4, 2, 64, None) == B.EINVAL
    assert _attn(wsb=small - 1) == B.ENOMEM


def _norm(**kw):
    a = dict(dtype=0, xdtype=0, y=P, x=P, w_post=P, gate=P, n_gates=2, w_pre=P, x_out=P, h=P, rows=4, dim=64, scale=1.0, eps=1e-5)
    a.update(kw)
    return A.load().adsa_norm_residual(*a.values(), None)


@pytest.mark.parametrize("kw", [dict(dtype=2), dict(xdtype=1), dict(xdtype=3), dict(y=None), dict(x=None), dict(x_out=None), dict(h=None), dict(w_pre=None),
                                dict(n_gates=3), dict(n_gates=0), dict(rows=-1), dict(rows=2**31), dict(dim=60), dict(dim=0), dict(dim=16392), dict(eps=-1.0),
                                dict(eps=math.nan), dict(y=P + 8), dict(gate=P + 2), dict(x_out=P + 4)])
def test_norm_residual_refusals(kw):
    assert _norm(**kw) == B.EINVAL


def test_a_copy_of_a_rotary_has_a_schedule_of_its_own():
    import copy
    import gc
    import pickle
    rot = A.Rotary(64, (8, 12), base=500.0, style="halves", restart=False)
    want = bytes(rot.c)
    copies = [copy.copy(rot), copy.deepcopy(rot), pickle.loads(pickle.dumps(rot))]
    assert len({r.ref for r in copies + [rot]}) == 4
    del rot
    gc.collect()
    for r in copies:
        assert r.ref == C.addressof(r.c) and bytes(r.c) == want and (r.head_dim, r.n_axes) == (64, 2)


def test_the_binding_refuses_wrong_types_shapes_and_devices():
    bf, i32 = torch.bfloat16, torch.int32
    x, pos = torch.zeros(4, 2, 64, dtype=bf), torch.zeros(4, 2, dtype=i32)
    rot = A.Rotary(64, (16, 16))
    for args in ((x.float(), pos), (x[..., :62], pos), (x, pos[:3]), (x, pos.long()), (x, pos[:, :1]), (x, pos), (x.transpose(1, 2), pos)):
        with pytest.raises(ValueError):                                            # the last but one: not on a GPU
            A.rope_axes(rot, *args)
    pool = torch.zeros(5, 2, 16, 64, dtype=bf)
    table, n = torch.zeros(4, 2, dtype=i32), torch.zeros(4, dtype=i32)
    for kw in (dict(), dict(v_pool=pool[:4]), dict(k_pool=pool.half()), dict(n_rows=n[:3]), dict(page_table=table.long()), dict(k=x.half()), dict(v=x[:, :1]),
               dict(rotary=rot), dict(rotary=rot, pos=pos[:2]), dict(q=x.half()), dict(q=x, q_out=x[:, :1]), dict(cu_tokens=n), dict(status=n)):
        a = dict(dict(k=x, v=x, k_pool=pool, v_pool=pool, page_table=table, n_rows=n), **kw)
        with pytest.raises(ValueError):
            A.paged_append(**a)
    for kw in (dict(), dict(q=x.half()), dict(n_rows=n[:2]), dict(prefix_table=table, prefix_rows=n, group_start=n), dict(out=x.half()), dict(lse=n),
               dict(out_f32=x), dict(status=n)):
        a = dict(dict(q=x, k_pool=pool, v_pool=pool, page_table=table, n_rows=n, workspace=torch.zeros(1, dtype=torch.uint8)), **kw)
        with pytest.raises(ValueError):
            A.shared_prefix_attn(**a)
    y, w = torch.zeros(4, 64, dtype=bf), torch.zeros(64, dtype=bf)
    for a, kw in (((y, y, w), {}), ((y.float(), y, w), {}), ((y, y[:3], w), {}), ((y, y, w[:32]), {}), ((y, y, w.float()), {}), ((y, y.long(), w), {}),
                  ((y, y, w), dict(gate=w)), ((y, y, w), dict(w_post=y)), ((y, y, w), dict(h=y.float())), ((y, y, w), dict(x_out=y[:2]))):
        with pytest.raises(ValueError):
            A.norm_residual(*a, **kw)
