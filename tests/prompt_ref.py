"""Attention of many query rows per sequence in 64 bits, with the error that the documented arithmetic may have.

Tolerances count roundings, u = finfo(t).eps / 2 of a value each.  With weights w_j (their sum 1) and A = sum_j w_j |v_j|:
the output is rounded to its type (u of itself); every weight is rounded once to the 16-bit type (u of itself, half: 2^-31 of the
largest where that is more); a score is a sum of d products and a scaling in 32 bits, (d + 4) 2^-23 of the magnitudes it adds up
(S), and so is its weight relative to itself, once in the numerator and once in the sum; exponentials, sums over rows and rescaling
in 32 bits: 16 roundings for a tile of 128 rows, 2^-23 each."""
import math

import torch

DEV = "cuda:0"
HALF = [torch.bfloat16, torch.float16]


def u(dtype):
    return torch.finfo(dtype).eps / 2


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def randn(g, *shape, dtype=torch.bfloat16, scale=1.0):
    return (torch.randn(shape, generator=g, device=DEV) * scale).to(dtype)


def starts(lengths, first=0):
    at = [first]
    for n in lengths:
        at.append(at[-1] + n)
    return torch.tensor(at, dtype=torch.int32, device=DEV)


def attend64(q, k, v, seen, scale=None):
    """q [m][H][d], k, v [n][KV][d], seen: rows each token attends, from the front [m] (a list) -> out, lse, A, S in 64 bits."""
    m, H, d = q.shape
    n, KV, _ = k.shape
    scale = 1 / math.sqrt(d) if not scale else scale
    out = torch.zeros(m, H, d, dtype=torch.float64, device=q.device)
    mag, lse, s_mag = torch.zeros_like(out), torch.full((m, H), -math.inf, dtype=torch.float64, device=q.device), torch.zeros(m, H, dtype=torch.float64, device=q.device)
    count = torch.as_tensor(seen, device=q.device)
    mask = torch.arange(n, device=q.device)[None] < count[:, None]
    some = (count > 0)
    if n == 0 or m == 0 or not bool(some.any()):
        return out, lse, mag, s_mag
    for h in range(H):
        kk, vv, qq = k[:, h * KV // H].double(), v[:, h * KV // H].double(), q[:, h].double()
        x = (qq @ kk.T * scale).masked_fill(~mask, -math.inf)[some]
        w = torch.softmax(x, 1)
        # rows that are not attended have no part, whatever they hold
        w_, v_ = w.masked_fill(~mask[some], 0.0), vv
        if not bool(torch.isfinite(vv).all()):
            o = torch.stack([w_[i, :c] @ vv[:c] for i, c in enumerate(count[some].tolist())])
        else:
            o = w_ @ v_
        out[some, h] = o
        mag[some, h] = w_ @ torch.nan_to_num(vv).abs()
        lse[some, h] = torch.logsumexp(x, 1)
        s_mag[some, h] = ((qq.abs() @ kk.abs().T * scale).masked_fill(~mask, 0.0).amax(1))[some]
    return out, lse, mag, s_mag


def check(got, lse, want, rows, dtype, d, what=""):
    """got [m][H][d] (or None), lse [m][H] (or None) against attend64's values; rows: cached rows at most."""
    out, ref_lse, mag, s_mag = want
    score = (d + 4) * 2.0 ** -23 * s_mag
    sums = 16 * (rows / 128 + 1) * 2.0 ** -23
    if got is not None:
        weights = u(dtype) + 2 * score[..., None] + sums
        finite = mag[mag < 1e30]
        floor = 2.0 ** -31 * max(rows, 1) * float(finite.max()) if dtype == torch.float16 and finite.numel() else 0.0
        tol = u(got.dtype) * out.abs() + weights * mag + floor + torch.finfo(got.dtype).smallest_normal * torch.finfo(got.dtype).eps
        fine = torch.isfinite(out)
        assert torch.equal(torch.isnan(got.double()), torch.isnan(out)), what
        assert torch.equal(got.double()[~fine & ~torch.isnan(out)], out[~fine & ~torch.isnan(out)]), what
        err = ((got.double() - out).abs() - tol)[fine]
        assert err.numel() == 0 or float(err.max()) <= 0, f"{what}: {float(err.max())} over"
    if lse is not None:
        fine = torch.isfinite(ref_lse)
        assert torch.equal(lse.double()[~fine], ref_lse[~fine]) or bool(torch.isnan(ref_lse[~fine]).any()), what
        # the score's error, the sum's, the logarithm and the output's rounding (of up to |lse| + the largest score)
        tol = score + sums + 8 * 2.0 ** -23 * (1 + ref_lse.abs() + s_mag)
        err = ((lse.double() - ref_lse).abs() - tol)[fine]
        assert err.numel() == 0 or float(err.max()) <= 0, f"{what}: lse {float(err.max())} over"
