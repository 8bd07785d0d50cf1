"""The draw of the next token against 64 bits: borders inside ties, settings per row, guidance, logits that are no numbers, the ends of the
uniform numbers; rows by themselves, captured, on another stream."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = [torch.bfloat16, torch.float16, torch.float32]


def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def draw64(x, u, T, top_k, top_p, min_p):
    """(token, logprob) of one row of logits (float32 values), rule by rule, in 64 bits."""
    x = torch.where(torch.isnan(x), -math.inf, x).double().cpu()
    top = float(x.max())
    if top == -math.inf:
        return -1, -math.inf
    if not T > 0:
        T, top_k = 1.0, 1
    w = torch.exp((x - top) / T) if math.isfinite(top) else (x == top).double()
    w[x == top] = 1.0
    ids = sorted(torch.nonzero(x > -math.inf).flatten().tolist(), key=lambda i: (-float(x[i]), i)) if x.numel() < 5000 else \
        [i for i in torch.argsort(-x, stable=True).tolist() if x[i] > -math.inf]
    if not math.isfinite(top):
        ids = [i for i in ids if x[i] == top]
    if top_k > 0:
        ids = ids[:top_k]
    if top_p < 1:
        run = torch.cumsum(w[ids], 0)
        ids = ids[:int((run < max(top_p, 0.0) * run[-1]).sum()) + 1]
    if min_p > 0:
        ids = [i for i in ids if w[i] >= min(min_p, 1.0)]
    ids = sorted(ids)
    run = torch.cumsum(w[ids], 0)
    at = min(int((run < u * run[-1]).sum()), len(ids) - 1)
    return ids[at], float((x[ids[at]] - top) / T if math.isfinite(top) else 0.0) - math.log(float(run[-1]))


def verify(logits, u, tokens, logprobs, T=1.0, top_k=0, top_p=1.0, min_p=0.0):
    def of(s, r):
        return s[r].item() if torch.is_tensor(s) else torch.tensor(s, dtype=torch.float32).item() if isinstance(s, float) else s
    for r in range(logits.shape[0]):
        token, lp = draw64(logits[r].float(), of(u, r), of(T, r), of(top_k, r), of(top_p, r), of(min_p, r))
        assert int(tokens[r]) == token, (r, int(tokens[r]), token)
        if logprobs is not None:
            # one rounding to 32 bits of a value made in 64, whose sum is in steps of 2^-42 (2^20 of them at most)
            got = float(logprobs[r])
            assert got == lp or abs(got - lp) <= 2.0 ** -24 * abs(lp) + 2.0 ** -22 * 2.0 ** -20, (r, got, lp)


SETTINGS = [dict(), dict(T=0.7), dict(top_k=1), dict(top_k=5), dict(top_k=50, top_p=0.9), dict(top_p=0.5, T=1.3), dict(top_p=0.95, min_p=0.02),
            dict(min_p=0.3), dict(top_k=2000, top_p=0.99, min_p=0.001, T=0.9), dict(T=0.0), dict(top_p=0.0), dict(min_p=2.0), dict(top_k=10 ** 6),
            dict(T=0.01), dict(T=100.0, top_p=0.3)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("vocab", [1, 2, 31, 33, 1000, 1025, 4099, 16384])
@pytest.mark.parametrize("kw", SETTINGS)
def test_rows_against_64_bits(vocab, kw, dtype):
    import paper_2506_18226_b200 as A
    g = _gen(vocab)
    x = (torch.randn(6, vocab, generator=g, device=DEV) * 2.5).to(dtype)
    u = torch.rand(6, generator=g, device=DEV)
    lp = torch.empty(6, device=DEV)
    names = dict(T="temperature")
    t = A.sample(x, u, **{names.get(k, k): v for k, v in kw.items()}, logprobs=lp)
    verify(x, u, t, lp, **kw)


@pytest.mark.parametrize("vocab,rows", [(50001, 3), (131072, 2), (1 << 20, 1)])
@pytest.mark.parametrize("kw", [dict(), dict(top_k=40, top_p=0.9), dict(top_p=0.9), dict(top_k=60000, top_p=0.97, min_p=1e-4)])
def test_large_vocabularies(vocab, rows, kw):
    import paper_2506_18226_b200 as A
    g = _gen(vocab)
    for dtype in (torch.bfloat16, torch.float32):
        x = (torch.randn(rows, vocab, generator=g, device=DEV) * 2).to(dtype)
        u = torch.rand(rows, generator=g, device=DEV)
        lp = torch.empty(rows, device=DEV)
        verify(x, u, A.sample(x, u, **kw, logprobs=lp), lp, **kw)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("kw", [dict(top_k=7), dict(top_k=100), dict(top_p=0.4), dict(top_p=0.8, top_k=300), dict(top_p=0.05), dict(min_p=0.5)])
def test_borders_inside_ties(kw, dtype):
    """Few distinct logits: every border falls among equal ones, and the lower ids are kept.  -0 and 0 are equal."""
    import paper_2506_18226_b200 as A
    g = _gen(4)
    x = torch.randint(-2, 3, (16, 700), generator=g, device=DEV).to(dtype)
    x[x == 0] *= torch.where(torch.rand(x[x == 0].shape, generator=g, device=DEV) < 0.5, -1.0, 1.0).to(dtype)
    x[1], x[2] = 1.5, 0.0
    u = torch.rand(16, generator=g, device=DEV)
    verify(x, u, A.sample(x, u, **kw), None, **kw)


def test_the_running_sum_is_followed_to_its_ends():
    """The same row under a sweep of uniform numbers, 0 and the one below 1 among them: every id gets its share."""
    import paper_2506_18226_b200 as A
    g = _gen(5)
    n = 4000
    row = torch.randn(64, generator=g, device=DEV)
    x = row.expand(n, 64)                                                          # (a row stride of zero)
    u = (torch.arange(n, device=DEV) + 0.5) / n
    u[0], u[-1] = 0.0, 1 - 2.0 ** -24
    t = A.sample(x, u)
    assert (t[1:] >= t[:-1]).all() and int(t[0]) == 0 and int(t[-1]) == 63
    share = torch.bincount(t, minlength=64) / n
    assert (share - torch.softmax(row.double(), 0)).abs().max() <= 1.5 / n
    u[:3] = torch.tensor([-1.0, 1.0, 7.0])
    t = A.sample(x[:3], u[:3], top_k=9)
    kept = row.topk(9).indices.sort().values
    assert t.tolist() == [int(kept[0]), int(kept[-1]), int(kept[-1])]


@pytest.mark.parametrize("dtype", TYPES)
def test_settings_per_row(dtype):
    import paper_2506_18226_b200 as A
    g = _gen(6)
    R, V = 24, 3000
    x = (torch.randn(R, V, generator=g, device=DEV) * 3).to(dtype)
    u = torch.rand(R, generator=g, device=DEV)
    T = torch.rand(R, generator=g, device=DEV) + 0.3
    k = torch.randint(-1, 200, (R,), generator=g, device=DEV, dtype=torch.int32)
    p = torch.rand(R, generator=g, device=DEV) * 1.2
    m = torch.rand(R, generator=g, device=DEV) * 0.2 - 0.05
    T[3], k[4], p[5], m[6] = 0.0, 0, 1.0, 0.0
    lp = torch.empty(R, device=DEV)
    t = A.sample(x, u, temperature=T, top_k=k, top_p=p, min_p=m, logprobs=lp)
    verify(x, u, t, lp, T=T, top_k=k, top_p=p, min_p=m)
    # NaN per row: the largest logit; no top_p; no min_p
    T[0], p[1], m[2] = math.nan, math.nan, math.nan
    k[:3] = 0
    p[[0, 2]], m[[0, 1]] = 1.0, 0.0
    t = A.sample(x, u, temperature=T, top_k=k, top_p=p, min_p=m)
    T[0], p[1], m[2] = 0.0, 1.0, 0.0
    verify(x[:3], u[:3], t[:3], None, T=T, top_k=k, top_p=p, min_p=m)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("guidance", [7.5, 1.0, 0.0, -2.3])
def test_guidance(guidance, dtype):
    import paper_2506_18226_b200 as A
    g = _gen(7)
    c, n = (torch.randn(2, 5, 2000, generator=g, device=DEV) * 2).to(dtype)
    u = torch.rand(5, generator=g, device=DEV)
    lp = torch.empty(5, device=DEV)
    t = A.sample(c, u, uncond=n, guidance=guidance, top_k=300, top_p=0.9, logprobs=lp)
    x = n.float() + torch.tensor(guidance, device=DEV) * (c.float() - n.float())
    verify(x, u, t, lp, top_k=300, top_p=0.9)


def test_it_draws_as_cfg_sample_does():
    """The same rule with top_k alone, for bf16 rows of both halves: the older call's weights are in 32 bits, so a few draws may differ."""
    import paper_2506_18226_b200 as A
    g = _gen(8)
    n, V = 64, 16384
    x = (torch.randn(2 * n, V, generator=g, device=DEV) * 1.5).to(torch.bfloat16)
    u = torch.rand(n, generator=g, device=DEV)
    a = A.cfg_sample(x, 4.0, 500, 0.8, u)
    b = A.sample(x[:n], u, uncond=x[n:], guidance=4.0, top_k=500, temperature=0.8)
    assert (a == b).sum() >= n - 1


@pytest.mark.parametrize("dtype", TYPES)
def test_logits_that_are_no_numbers(dtype):
    import paper_2506_18226_b200 as A
    g = _gen(9)
    x = torch.randn(10, 500, generator=g, device=DEV).to(dtype)
    inf = math.inf
    x[0, :400], x[1, ::2], x[2], x[3], x[4, 7] = -inf, math.nan, -inf, math.nan, inf
    x[5, [3, 90, 91]], x[6] = inf, inf
    x[7, 1:] = -inf
    x[8, :] = torch.finfo(dtype).min
    u = torch.rand(10, generator=g, device=DEV)
    u[4] = 0.0
    for kw in (dict(), dict(top_k=450), dict(top_p=0.9), dict(top_k=20, top_p=0.7, min_p=0.1), dict(T=0.0), dict(top_k=2)):
        lp = torch.empty(10, device=DEV)
        t = A.sample(x, u, **{"temperature" if k == "T" else k: v for k, v in kw.items()}, logprobs=lp)
        verify(x, u, t, lp, **kw)
        assert t[2] == -1 and t[3] == -1 and t[4] == 7 and t[7] == 0


def test_strides_streams_and_a_captured_call():
    import paper_2506_18226_b200 as A
    g = _gen(10)
    room = (torch.randn(12, 3011, generator=g, device=DEV) * 2).to(torch.bfloat16)
    x = room[:, 1:3002]
    u = torch.rand(12, generator=g, device=DEV)
    kw = dict(temperature=0.8, top_k=100, top_p=0.9)
    want = A.sample(x.contiguous(), u, **kw)
    assert torch.equal(A.sample(x, u, **kw), want)
    verify(x, u, want, None, T=0.8, top_k=100, top_p=0.9)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = A.sample(x, u, **kw)
    side.synchronize()
    assert torch.equal(got, want)
    out = torch.empty(12, dtype=torch.int32, device=DEV)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        A.sample(x, u, **kw, tokens=out)
    for seed in range(3):
        u.copy_(torch.rand(12, generator=_gen(seed), device=DEV))
        graph.replay()
        torch.cuda.synchronize()
        verify(x, u, out, None, T=0.8, top_k=100, top_p=0.9)
    assert A.sample(x[:0], u[:0]).shape == (0,)
