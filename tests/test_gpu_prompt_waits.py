"""Prompt attention whose waits run out: with no patience at all, kernels give up on copies that are under way.  The call ends, its status says so, what was
written is right and nothing else was, and the next call is as any other.  No part of the GPU fails here: every copy lands."""
import contextlib
import math

import pytest
import torch

from prompt_ref import DEV, gen, randn, starts

pytestmark = pytest.mark.gpu


@contextlib.contextmanager
def patience(polls):
    import paper_2506_18226_b200 as A
    lib = A.load()
    was = lib.adsa_prompt_wait_polls(polls)
    try:
        yield
    finally:
        lib.adsa_prompt_wait_polls(was)


def verify(call, shape, dtype, long=True):
    """call(out, lse, status) with patience, without, and with again.  A poll itself waits for 4 us, so
    only waits that are longer run out: a call of many or long items has them, a short one may not, and is then right throughout."""
    import paper_2506_18226_b200 as A
    want, lse = torch.empty(shape, dtype=dtype, device=DEV), torch.empty(shape[:2], device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    call(want, lse, status)
    torch.cuda.synchronize()
    assert int(status) == 0
    out, out_lse = torch.full_like(want, 7.0), torch.full_like(lse, 7.0)
    with patience(0):
        call(out, out_lse, status)
    torch.cuda.synchronize()
    left = (out == 7.0).all(-1)
    gave_up = int(status)
    assert gave_up == A.binding.DEV_COPY_TIMEOUT or (gave_up == 0 and not long)
    assert gave_up or not bool(left.any())
    assert torch.equal(out[~left], want[~left])
    assert torch.equal(out_lse[out_lse != 7.0], lse[out_lse != 7.0])
    status.zero_()
    call(out, out_lse, status)
    torch.cuda.synchronize()
    assert int(status) == 0 and torch.equal(out, want) and torch.equal(out_lse, lse)


@pytest.mark.parametrize("n,H,KV,d,pad,f32", [(8192, 4, 1, 128, 0, False), (6000, 4, 4, 64, 0, True), (5000, 2, 1, 256, 0, False), (4000, 4, 2, 64, 2, False),
                                              (5000, 6, 6, 100, 0, False), (700, 2, 1, 128, 0, False)])
def test_prompts(n, H, KV, d, pad, f32):
    """By boxes, with 32-bit outputs, of wide heads, by row copies, by boxes that begin between heads; whole items and cut ones."""
    import paper_2506_18226_b200 as A
    g = gen(n)
    q, k, v = (randn(g, n, h, d + pad)[..., :d] for h in (H, KV, KV))
    ws = A.prompt_workspace(q, KV, 1)
    also = torch.empty(q.shape, device=DEV) if f32 else None
    verify(lambda out, lse, status: A.packed_attn(q, k, v, out=out, out_f32=also, lse=lse, workspace=ws, status=status), q.shape, q.dtype, n > 2000)


@pytest.mark.parametrize("batch,m,n,H,KV,d,page,long", [(4, 1, 20000, 8, 2, 64, 64, False), (40, 3, 3000, 8, 8, 128, 16, True), (2, 300, 8000, 8, 2, 128, 64, False)])
def test_chunks(batch, m, n, H, KV, d, page, long):
    """One part of an item a block (no wait of 4 us need be); items of 24 tiles one after another, for which the next one's rows of q wait; one part of many rows."""
    import paper_2506_18226_b200 as A
    g, per = gen(n), (n + page - 1) // page
    kp, vp = (randn(g, batch * per, KV, page, d) for _ in range(2))
    table = torch.randperm(batch * per, generator=g, device=DEV).to(torch.int32).view(batch, per)
    rows = torch.full((batch,), n, dtype=torch.int32, device=DEV)
    q = randn(g, batch * m, H, d)
    ws = A.prompt_workspace(q, KV, batch)
    verify(lambda out, lse, status: A.chunk_attn(q, kp, vp, table, rows, out=out, lse=lse, workspace=ws, status=status), q.shape, q.dtype, long)


@pytest.mark.parametrize("n,m,d", [(8192, 8192, 128), (6000, 400, 64), (30000, 2, 128)])
def test_rows_that_held_infinities_before_are_left_or_right(n, m, d):
    """Values of infinity make rows that are mended after the others; what was not written is not taken for one of them."""
    import paper_2506_18226_b200 as A
    g, H, KV, batch = gen(n), 4, 1, 40 if m < 10 else 1
    q, k, v = randn(g, batch * m, H, d), randn(g, batch * n, KV, d), randn(g, batch * n, KV, d)
    v[n // 2, :, 3] = math.inf
    ws, cu = A.prompt_workspace(q, KV, batch), starts([m] * batch)
    want = A.packed_attn(q, k, v, cu, starts([n] * batch), workspace=ws)
    out, status = torch.full_like(want, math.inf), torch.zeros(1, dtype=torch.int32, device=DEV)
    with patience(0):
        A.packed_attn(q, k, v, cu, starts([n] * batch), out=out, workspace=ws, status=status)
    torch.cuda.synchronize()
    left = (out == math.inf).all(-1)
    assert m == 400 or (int(status) == A.binding.DEV_COPY_TIMEOUT and bool(left.any()))   # (400 tokens: a part of an item a block, no wait of 4 us need be)
    # (a row made again as a whole has its weights in 32 bits)
    got, ref = out[~left].float(), want[~left].float()
    odd = ~torch.isfinite(ref)
    assert torch.equal(torch.isfinite(got), ~odd) and torch.equal(got[odd], ref[odd])
    assert ((got - ref)[~odd].abs() <= 0.05).all()


def test_a_call_without_a_status():
    import paper_2506_18226_b200 as A
    g = gen(1)
    q, k, v = (randn(g, 4000, 2, 128) for _ in range(3))
    want = A.packed_attn(q, k, v)
    with patience(0):
        A.packed_attn(q, k, v)
    torch.cuda.synchronize()
    assert torch.equal(A.packed_attn(q, k, v), want)


def test_the_patience_that_was_is_returned():
    import paper_2506_18226_b200 as A
    lib = A.load()
    was = lib.adsa_prompt_wait_polls(5)
    assert lib.adsa_prompt_wait_polls(-7) == 5 and lib.adsa_prompt_wait_polls(was) == -1
