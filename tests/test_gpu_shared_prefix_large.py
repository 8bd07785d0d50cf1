"""The calls on a paged whole-token cache where element offsets pass 32 bits: the far ends of tensors of more than 2^31 elements."""
import pytest
import torch

from test_gpu_shared_prefix import DEV, _gen, _randn, _u, attn64, check_attn, check_turned, norm64, turn64

pytestmark = pytest.mark.gpu

BF = torch.bfloat16


@pytest.fixture(autouse=True)
def memory_back():
    yield
    torch.cuda.empty_cache()


@pytest.mark.parametrize("style", ["pairs", "halves"])
@pytest.mark.parametrize("heads,dim", [(16, 128), (21, 100)])
def test_rope_axes_beyond_32_bits(heads, dim, style):
    import paper_2506_18226_b200 as A
    g = _gen(1)
    tokens = 2**31 // (heads * dim) + 5000
    x = torch.empty(tokens, heads, dim, dtype=BF, device=DEV)
    ends = [slice(0, 40), slice(tokens - 3000, tokens)]
    for e in ends:
        x[e] = _randn(g, x[e].shape[0], heads, dim)
    pos = torch.randint(0, 5000, (tokens, 2), generator=g, device=DEV, dtype=torch.int32)
    pairs = (dim // 8, dim // 4)
    out = A.rope_axes(A.Rotary(dim, pairs, style=style), x, pos)
    for e in ends:
        want, mag = turn64(x[e], pos[e], pairs, style, True)
        check_turned(out[e], want, mag, BF)


@pytest.mark.parametrize("kv,dim,page", [(8, 128, 64), (8, 100, 48), (4, 64, 64)])
def test_append_and_attention_at_the_end_of_a_large_pool(kv, dim, page):
    """Every page lies where its elements' offsets pass 32 bits; a group large enough for the wide kernel, a small one, own rows."""
    import paper_2506_18226_b200 as A
    g = _gen(2)
    stride = (dim + 7) // 8 * 8
    per_page = kv * page * stride
    pages = 2**32 // per_page + 600
    k_pool, v_pool = (torch.empty(pages, kv, page, stride, dtype=BF, device=DEV) for _ in range(2))
    own, prefix, members = [3 + (17 * b) % 200 for b in range(44)], [9000, 300], [40, 4]
    lengths = own + prefix
    first = 2**32 // per_page + 1                                                 # of the pages used
    order = torch.randperm(pages - first, generator=g, device=DEV).to(torch.int32) + first
    most = max(lengths) // page + 1
    table, at = torch.zeros(len(lengths), most, dtype=torch.int32, device=DEV), 0
    for i, n in enumerate(lengths):
        c = (n + page - 1) // page
        table[i, :c] = order[at:at + c]
        at += c
    i32 = dict(dtype=torch.int32, device=DEV)
    cu = torch.tensor([0] + lengths, **i32).cumsum(0).to(torch.int32)
    T = int(cu[-1])
    k, v, pos = _randn(g, T, kv, dim), _randn(g, T, kv, dim), torch.randint(0, 4000, (T, 2), generator=g, **i32)
    pairs = (dim // 8, dim // 4)
    status = torch.zeros(1, **i32)
    A.paged_append(k, v, k_pool, v_pool, table, torch.zeros(len(lengths), **i32), cu_tokens=cu, rotary=A.Rotary(dim, pairs), pos=pos, status=status)
    want, mag = turn64(k, pos, pairs, "pairs", True)
    for i in (0, 43, 44, 45):
        r = torch.arange(lengths[i], device=DEV)
        pg, row, sl = table[i][r // page].long(), r % page, slice(int(cu[i]), int(cu[i + 1]))
        check_turned(k_pool[pg, :, row][..., :dim], want[sl], mag[sl], BF)
        assert torch.equal(v_pool[pg, :, row][..., :dim], v[sl])
    q = _randn(g, 44, kv * 2, dim)
    n_rows, p_rows = torch.tensor(own, **i32), torch.tensor(prefix, **i32)
    out, out32, lse = torch.empty_like(q), torch.empty(q.shape, device=DEV), torch.empty(q.shape[:2], device=DEV)
    for groups in ([0, 40, 44], [0, 0, 44]):                                      # the long prefix for forty rows; for none, and no row left out
        A.shared_prefix_attn(q, k_pool, v_pool, table[:44].contiguous(), n_rows, table[44:].contiguous(), p_rows, torch.tensor(groups, **i32), out=out, out_f32=out32,
                             lse=lse, status=status)
        ref = attn64(q, k_pool, v_pool, table[:44], n_rows, table[44:], p_rows, groups, dim ** -0.5)
        check_attn(out, out32, lse, ref, BF)
    narrow = table[:44, :max(own) // page + 1].contiguous()                       # no prefix, narrow tables: a block per batch row and key head
    A.shared_prefix_attn(q, k_pool, v_pool, narrow, n_rows, out=out, out_f32=out32, lse=lse, status=status)
    check_attn(out, out32, lse, attn64(q, k_pool, v_pool, narrow, n_rows, None, None, None, dim ** -0.5), BF)
    assert int(status) == 0


@pytest.mark.parametrize("xt", [BF, torch.float32])
def test_norm_residual_beyond_32_bits(xt):
    import paper_2506_18226_b200 as A
    g = _gen(3)
    dim = 16384
    rows = 2**31 // dim + 1000
    y, x = torch.empty(rows, dim, dtype=BF, device=DEV), torch.empty(rows, dim, dtype=xt, device=DEV)
    e = slice(rows - 1500, rows)
    y[e], x[e] = _randn(g, 1500, dim), _randn(g, 1500, dim, dtype=xt)
    gate, w = _randn(g, rows // 8, dim) if rows % 8 == 0 else _randn(g, 1, dim), _randn(g, dim)
    got, h = A.norm_residual(y, x, w, w_post=w, gate=gate)
    per = rows // gate.shape[0]
    full = gate[(torch.arange(rows - 1500, rows, device=DEV) // per)]
    want, want_h, mag, inv = norm64(y[e], x[e], w, w, full, 1.0, 1e-5)
    tol = 2.0 ** -19 * mag
    assert ((got[e].double() - want).abs() <= tol + _u(xt) * (want.abs() + tol)).all()
    tol_h = (tol + 2.0 ** -18 * want.abs() + want.abs() * inv * tol.amax(1, keepdim=True)) * inv * w.double().abs()
    assert ((h[e].double() - want_h).abs() <= tol_h + _u(BF) * (want_h.abs() + tol_h) + 1e-40).all()
