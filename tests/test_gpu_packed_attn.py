"""Attention over whole prompts laid end to end against 64 bits: lengths, heads, masks, strides, what lies in places that are not
attended."""
import math

import pytest
import torch

from prompt_ref import DEV, HALF, attend64, check, gen, randn, starts

pytestmark = pytest.mark.gpu


def inputs(g, lens_q, lens_k, H, KV, d, dtype):
    return (randn(g, sum(lens_q), H, d, dtype=dtype, scale=1.5), randn(g, sum(lens_k), KV, d, dtype=dtype), randn(g, sum(lens_k), KV, d, dtype=dtype))


def verify(q, k, v, lens_q, lens_k, causal, out, lse, scale=None, out_f32=None):
    a = b = 0
    for m, n in zip(lens_q, lens_k):
        seen = [min(max(n - m + i + 1, 0), n) if causal else n for i in range(m)]
        want = attend64(q[a:a + m], k[b:b + n], v[b:b + n], seen, scale)
        what = f"m={m} n={n} at {a}"
        check(None if out is None else out[a:a + m], None if lse is None else lse[a:a + m], want, n, q.dtype, q.shape[2], what)
        if out_f32 is not None:
            check(out_f32[a:a + m], None, want, n, q.dtype, q.shape[2], what)
        a, b = a + m, b + n


CASES = [  # lengths, heads, key heads, dim
    ([1], 1, 1, 2),
    ([1], 4, 2, 64),
    ([1, 1, 1], 3, 1, 128),
    ([0, 5, 0, 0, 9, 0], 4, 4, 64),
    ([2, 17, 33], 6, 2, 30),
    ([127, 128, 129], 2, 2, 64),
    ([255, 256, 257, 1], 2, 1, 128),
    ([300, 41], 12, 12, 64),
    ([385, 7, 513], 5, 1, 100),
    ([700], 8, 1, 128),
    ([1144, 143, 600], 8, 2, 128),
    ([90, 200], 64, 1, 64),
    ([120, 60], 10, 2, 36),
    ([333, 20], 7, 1, 72),
    ([260, 129, 40], 4, 2, 130),
    ([200, 300], 3, 1, 192),
    ([129, 400], 4, 4, 256),
    ([2500], 1, 1, 64),
]


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens,H,KV,d", CASES)
def test_prompts_of_different_lengths(lens, H, KV, d, causal, dtype):
    import paper_2506_18226_b200 as A
    g = gen(sum(lens) + 7 * H + d)
    q, k, v = inputs(g, lens, lens, H, KV, d, dtype)
    out, lse = torch.empty_like(q), torch.empty(q.shape[:2], device=DEV)
    f32 = torch.empty(q.shape, device=DEV)
    got = A.packed_attn(q, k, v, starts(lens), causal=causal, out=out, out_f32=f32, lse=lse)
    assert got is out
    verify(q, k, v, lens, lens, causal, out, lse, out_f32=f32)


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("lens_q,lens_k", [([5, 300], [9, 200]), ([200, 1, 64], [64, 0, 500]), ([1, 1, 1], [1, 700, 3000]), ([130, 3], [0, 0]),
                                           ([300], [17]), ([2], [5000])])
def test_lengths_of_q_and_k_that_differ(lens_q, lens_k, causal, dtype):
    """Causal with fewer rows than tokens: the first tokens attend nothing and get zeros and -inf."""
    import paper_2506_18226_b200 as A
    g = gen(sum(lens_q) * 3 + sum(lens_k))
    q, k, v = inputs(g, lens_q, lens_k, 4, 2, 64, dtype)
    lse = torch.empty(q.shape[:2], device=DEV)
    out = A.packed_attn(q, k, v, starts(lens_q), starts(lens_k), causal=causal, lse=lse)
    verify(q, k, v, lens_q, lens_k, causal, out, lse)
    empty = [i for m, n in [(lens_q[0], lens_k[0])] for i in range(m) if (n - m + i < 0 if causal else n == 0)]
    assert (out[empty] == 0).all() and (lse[empty] == -math.inf).all()


def test_one_sequence_without_boundaries_and_a_scale():
    import paper_2506_18226_b200 as A
    g = gen(5)
    q, k, v = inputs(g, [200], [200], 4, 4, 64, torch.bfloat16)
    lse = torch.empty(200, 4, device=DEV)
    out = A.packed_attn(q, k, v, scale=0.3, lse=lse)
    verify(q, k, v, [200], [200], True, out, lse, scale=0.3)
    f32 = torch.empty(q.shape, device=DEV)
    assert A.packed_attn(q, k, v, out_f32=f32) is f32


@pytest.mark.parametrize("d,offset", [(64, 0), (64, 2), (100, 0), (100, 4), (128, 8), (128, 6)])
@pytest.mark.parametrize("layout", ["packed", "heads first"])
def test_strides_and_alignment(d, offset, layout):
    """q, k and v out of one projection whose rows start at any even element, or with their heads outermost; bytes around untouched."""
    import paper_2506_18226_b200 as A
    lens, H, KV = [150, 301], 4, 2
    T, g = sum(lens), gen(d + offset)
    if layout == "packed":
        flat = randn(g, T * ((H + 2 * KV) * d + 6) + 16)
        x = flat[offset:offset + T * ((H + 2 * KV) * d + 6)].view(T, -1)[:, :(H + 2 * KV) * d].unflatten(1, (-1, d))
        q, k, v = x[:, :H], x[:, H:H + KV], x[:, H + KV:]
    else:
        flat = randn(g, (H + 2 * KV) * T * (d + 2) + 16)
        x = flat[offset:offset + (H + 2 * KV) * T * (d + 2)].view(H + 2 * KV, T, d + 2)[..., :d].transpose(0, 1)
        q, k, v = x[:, :H], x[:, H:H + KV], x[:, H + KV:]
    before = flat.clone()
    lse = torch.empty(T, H, device=DEV)
    out = A.packed_attn(q, k, v, starts(lens), lse=lse)
    verify(q, k, v, lens, lens, True, out, lse)
    assert torch.equal(flat, before)


@pytest.mark.parametrize("d,H,KV", [(100, 6, 6), (100, 6, 3), (36, 4, 4), (50, 8, 8), (112, 5, 5), (66, 16, 16), (30, 8, 4)])
@pytest.mark.parametrize("bad", [False, True])
def test_heads_that_begin_between_16_byte_pieces(d, H, KV, bad):
    """Dense rows whose tokens are 16-byte aligned and whose heads are not (they are read with what lies before them): the neighbours'
    infinities and NaN have no effect."""
    import paper_2506_18226_b200 as A
    lens, g, pad = [300, 7, 129, 260], gen(d), -KV * d % 8
    T = sum(lens)
    q = randn(g, T, H * d + (-H * d % 8), scale=1.5)[:, :H * d].unflatten(1, (H, d))
    k, v = (randn(g, T, KV * d + pad)[:, :KV * d].unflatten(1, (KV, d)) for _ in range(2))
    if bad:
        k[:, 1], v[:, 1], q[:, H // KV] = math.nan, math.inf, math.inf
    out, lse = torch.empty(T, H, d, dtype=torch.bfloat16, device=DEV), torch.empty(T, H, device=DEV)
    A.packed_attn(q, k, v, starts(lens), out=out, lse=lse)
    g_ = H // KV
    heads = [h for h in range(H) if not bad or h // g_ != 1]
    verify(q[:, heads], k[:, [h // g_ for h in heads]], v[:, [h // g_ for h in heads]], lens, lens, True, out[:, heads].contiguous(), lse[:, heads].contiguous())


def test_a_head_dimension_shared_by_all_key_heads():
    """k and v expanded over heads (a stride of zero)."""
    import paper_2506_18226_b200 as A
    g = gen(8)
    q, k = randn(g, 170, 6, 64), randn(g, 170, 1, 64)
    v = randn(g, 170, 1, 64)
    lse = torch.empty(170, 6, device=DEV)
    out = A.packed_attn(q, k.expand(-1, 3, -1), v.expand(-1, 3, -1), lse=lse)
    verify(q, k, v, [170], [170], True, out, lse)


@pytest.mark.parametrize("causal", [True, False])
def test_padding_is_left_as_it_is_and_has_no_part(causal):
    import paper_2506_18226_b200 as A
    lens, g = [70, 0, 200, 131], gen(21)
    T = sum(lens)
    q, k, v = inputs(g, [5 + T + 40], [5 + T + 40], 4, 2, 64, torch.bfloat16)
    k[:5], v[:5], k[5 + T:], v[5 + T:] = math.nan, math.inf, math.inf, math.nan
    q[:5], q[5 + T:] = math.nan, math.inf
    out, lse = torch.full_like(q, 7.0), torch.full(q.shape[:2], 7.0, device=DEV)
    A.packed_attn(q, k, v, starts(lens, 5), causal=causal, out=out, lse=lse)
    verify(q[5:5 + T], k[5:5 + T], v[5:5 + T], lens, lens, causal, out[5:5 + T], lse[5:5 + T])
    for x in (out, lse):
        assert (x[:5] == 7.0).all() and (x[5 + T:] == 7.0).all()


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("d", [64, 100, 128, 256])
@pytest.mark.parametrize("bad", [math.inf, -math.inf, math.nan])
def test_what_a_row_does_not_attend_has_no_effect(bad, d, dtype):
    """The keys and values of later tokens, and of the next sequence, hold infinities and NaN: earlier tokens get what they get without."""
    import paper_2506_18226_b200 as A
    lens, g = [150, 300, 33], gen(d)
    q, k, v = inputs(g, lens, lens, 4, 2, d, dtype)
    lse = torch.empty(q.shape[:2], device=DEV)
    want = attend64(q[150:450], k[150:450], v[150:450], list(range(1, 301)))
    k[150 + 210:150 + 300, :, 3], v[150 + 205:150 + 300] = bad, bad
    k[450:], v[450:] = bad, bad
    out = A.packed_attn(q, k, v, starts(lens), lse=lse)
    check(out[150:355], lse[150:355], [w[:205] for w in want], 205, dtype, d)
    verify(q[:150], k[:150], v[:150], lens[:1], lens[:1], True, out[:150], lse[:150])
    assert not torch.isfinite(out[355:]).any()


@pytest.mark.parametrize("dtype", HALF)
def test_infinities_and_nan_that_are_attended(dtype):
    import paper_2506_18226_b200 as A
    g = gen(31)
    q, k, v = inputs(g, [260], [260], 2, 2, 64, dtype)
    v[40, 0, 5], v[130, 0, 9], v[50, 1, 3], v[70, 1, 3] = math.inf, -math.inf, math.inf, -math.inf
    q[200, 0], k[100, 1] = math.nan, math.nan
    lse = torch.empty(260, 2, device=DEV)
    out = A.packed_attn(q, k, v, lse=lse)
    verify(q, k, v, [260], [260], True, out, lse)
    assert torch.isnan(lse[200, 0]) and torch.isnan(lse[100:, 1]).all()


@pytest.mark.parametrize("dtype", HALF)
def test_scores_far_apart(dtype):
    """Scores that rise by hundreds from row to row (the running maximum moves all the time) and fall by as much; weights that all
    but one row lose; the lowest scores a type can make."""
    import paper_2506_18226_b200 as A
    g = gen(77)
    n = 700
    q, k, v = randn(g, n, 3, 64, dtype=dtype), randn(g, n, 3, 64, dtype=dtype), randn(g, n, 3, 64, dtype=dtype)
    ramp = torch.linspace(0, 60, n, device=DEV)
    q[:, :, 0] = 40.0
    k[:, 0, 0], k[:, 1, 0] = ramp.to(dtype), (-ramp).to(dtype)
    q[:, 2], k[:, 2] = 200.0, -200.0                                               # every score alike: -320000
    lse = torch.empty(n, 3, device=DEV)
    out = A.packed_attn(q, k, v, lse=lse)
    verify(q, k, v, [n], [n], True, out, lse)


def test_workspace_of_the_callers_and_equal_results():
    import paper_2506_18226_b200 as A
    lens, g = [500, 300, 1, 700], gen(3)
    q, k, v = inputs(g, lens, lens, 8, 2, 128, torch.bfloat16)
    cu = starts(lens)
    ws = A.prompt_workspace(q, 2, len(lens))
    ws.fill_(255)
    first = A.packed_attn(q, k, v, cu, workspace=ws)
    for _ in range(3):
        assert torch.equal(A.packed_attn(q, k, v, cu, workspace=ws), first)
    assert torch.equal(A.packed_attn(q, k, v, cu), first)
    assert A.packed_attn(q[:0], k[:0], v[:0], starts([0, 0])).shape == (0, 8, 128)


def test_other_streams_and_a_captured_call():
    import paper_2506_18226_b200 as A
    lens, g = [129, 400], gen(4)
    q, k, v = inputs(g, lens, lens, 4, 4, 64, torch.float16)
    cu, out, ws = starts(lens), torch.empty_like(q), A.prompt_workspace(q, 4, 2)
    want = A.packed_attn(q, k, v, cu)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        assert torch.equal(A.packed_attn(q, k, v, cu, out=out, workspace=ws), want)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        A.packed_attn(q, k, v, cu, out=out, workspace=ws)
    lens2 = [400, 77]                                                              # lengths are read when the graph runs
    for lens_now in (lens, lens2, lens):
        cu.copy_(starts(lens_now))
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        n = sum(lens_now)
        verify(q[:n], k[:n], v[:n], lens_now, lens_now, True, out[:n], None)
        assert (out[n:] == 0).all()


def test_boundaries_past_the_tokens_are_clamped():
    import paper_2506_18226_b200 as A
    g = gen(6)
    q, k, v = inputs(g, [100], [100], 2, 2, 64, torch.bfloat16)
    out = torch.full_like(q, 7.0)
    A.packed_attn(q, k, v, torch.tensor([-50, 60, 2000, 3000], dtype=torch.int32, device=DEV), out=out)
    verify(q, k, v, [60, 40], [60, 40], True, out, None)


def test_boundaries_that_do_not_ascend_write_no_row_outside():
    """The sequences overlap; rows around the outputs stay as they were."""
    import paper_2506_18226_b200 as A
    g = gen(77)
    q, k, v = inputs(g, [90], [90], 4, 2, 64, torch.bfloat16)
    around = torch.full((90 + 64, 4, 64), 7.0, dtype=torch.bfloat16, device=DEV)
    cu = torch.tensor([0, 90, 20, 200, -5, 90, 0, 90], dtype=torch.int32, device=DEV)
    A.packed_attn(q, k, v, cu, out=around[32:122])
    assert (around[:32] == 7).all() and (around[122:] == 7).all()
    assert torch.isfinite(around.float()).all()


@pytest.mark.parametrize("which", ["q", "k", "v", "half of q", "lse", "workspace"])
def test_outputs_on_top_of_inputs_are_refused(which):
    import paper_2506_18226_b200 as A
    g = gen(78)
    q, k, v = inputs(g, [40], [40], 2, 2, 64, torch.bfloat16)
    both = torch.zeros(60, 2, 64, dtype=torch.bfloat16, device=DEV)
    out = {"q": q, "k": k, "v": v}.get(which, torch.empty_like(q))
    kw = {}
    if which == "half of q":
        both[:40] = q
        q, out = both[:40], both[20:]
    if which == "lse":
        kw["lse"] = out.view(torch.float32).view(-1)[:80].view(40, 2)
    if which == "workspace":
        kw["workspace"] = A.prompt_workspace(q, 2, 1)
        out = kw["workspace"][:q.numel() * 2].view(torch.bfloat16).view(q.shape)
    with pytest.raises(ValueError, match="overlap"):
        A.packed_attn(q, k, v, out=out, **kw)
    # beside one another they are taken: three parts of one projection
    qkv = randn(g, 40, 6, 64)
    A.packed_attn(qkv[:, :2], qkv[:, 2:4], qkv[:, 4:], out=torch.empty_like(v))
