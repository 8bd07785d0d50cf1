"""adsa_shared_prefix_attn against 64 bits, as near as its 32-bit sums of 16-bit products can come.

Tolerances.  A weight enters the second product as the sum of two 16-bit values (cut, then rounded): bfloat16 keeps 16 bits of it
(off by at most 2^-16), float16 22 (2^-22), but no less than 2^-30 of the largest weight.  A score's 32-bit error is counted as in
test_gpu_shared_prefix.py, which moves a weight and the sum it is divided by.  A state of n cached rows takes 2 n / 16 matrix products
and as many rescalings at most into its 32-bit sums, each off by 2^-23 of what has been summed (tensor cores cut);
the merge, exponentials and the rest: 2^-18."""
import pytest
import torch

from test_gpu_shared_prefix import HALF, _gen, _u, attn64, attn_case, run_attn

pytestmark = pytest.mark.gpu


def attn64_of(c, rows, scale):
    """attn64 for some batch rows, each as a group of its own; and the largest |v| there is."""
    start = c["group_start"].tolist() if c["group_start"] is not None else []
    parts = []
    for b in rows:
        g = [k for k in range(len(start) - 1) if start[k] <= b < start[k + 1]]
        pre = (c["prefix_table"][g[0]:g[0] + 1], c["prefix_rows"][g[0]:g[0] + 1], torch.tensor([0, 1])) if g else (None, None, None)
        parts.append(attn64(c["q"][b:b + 1], c["k_pool"], c["v_pool"], c["page_table"][b:b + 1], c["n_rows"][b:b + 1], *pre, scale))
    return [torch.cat(x) for x in zip(*parts)]


def check_close(c, got, rows, ref, dtype, state_rows, most_rows):
    """state_rows: cached rows of a state at most; most_rows: cached rows of a batch row at most."""
    (out16, out32, lse), (want, want_lse, mag, s_err) = [x[rows].double() for x in got], ref
    sums = state_rows / 4 * 2.0 ** -23 + 2.0 ** -18
    inner = (2.0 ** -16 if dtype == torch.bfloat16 else 2.0 ** -22) * mag + (2 * s_err[..., None] + sums) * mag
    if dtype == torch.float16:
        v = c["v_pool"]
        inner = inner + most_rows * 2.0 ** -30 * float(v.abs().nan_to_num(0.0).max())
    assert ((out32 - want).abs() <= inner).all(), float(((out32 - want).abs() / inner).max())
    assert ((out16 - want).abs() <= inner + _u(dtype) * (want.abs() + inner) + torch.finfo(dtype).smallest_normal).all()
    tol = s_err + sums + 2.0 ** -22 * want_lse.abs()
    assert ((lse - want_lse).abs() <= tol).all(), float(((lse - want_lse).abs() / tol).max())


# ---- precision -------------------------------------------------------------------------------------------------------

WEIGHTS = {  # own rows, prefix rows, group starts, key heads, query heads per key head, dim, page rows
    "a query per key head": ([7, 100, 1, 300], [120, 200], [0, 2, 4], 4, 1, 64, 64),
    "three": ([7, 100, 1], [120], [0, 3], 2, 3, 128, 32),
    "four": ([200, 31], [57], [0, 2], 2, 4, 40, 16),
    "five": ([200, 31], [57], [0, 2], 2, 5, 64, 16),
    "eight, wide heads": ([60, 250], [100], [0, 2], 1, 8, 200, 16),
    "four, wide heads": ([60, 250], [100], [0, 2], 2, 4, 256, 16),
    "sixteen": ([200, 31], [257], [0, 2], 1, 16, 128, 48),
    "forty": ([70, 1, 200], [100, 30], [0, 1, 3], 2, 40, 64, 64),
    "100 elements": ([70, 300, 5], [200], [0, 3], 3, 1, 100, 48),
    "two elements": ([30, 1], [7], [0, 2], 2, 1, 2, 16),
    "a large group": ([20] * 70, [300, 65], [0, 41, 70], 1, 8, 64, 128),
    "a large group, 128 elements": ([12] * 50, [333], [0, 50], 2, 5, 128, 64),
    "a large group, 100 elements": ([5] * 50, [400], [0, 50], 2, 2, 100, 48),
}


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("room", [0, 1800, 30000])
@pytest.mark.parametrize("name", list(WEIGHTS))
def test_weights_are_not_rounded_to_16_bits(name, room, dtype):
    """The 32-bit output is as near as 32-bit sums of 16-bit products can be; with weights of 8 (11) bits it would not be."""
    own, prefix, start, kv, per, dim, page = WEIGHTS[name]
    c = attn_case(_gen(len(name) + dim), own, prefix, start, kv, per, dim, page, dtype, room=room, q_scale=0.5)
    got = run_attn(c)
    rows = list(range(len(own)))
    most = max(own) + max(prefix)
    check_close(c, got, rows, attn64_of(c, rows, dim ** -0.5), dtype, most, most)


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("per", [1, 4, 8, 40])
@pytest.mark.parametrize("room", [0, 1800, 30000])
def test_infinities_in_attended_values(per, room, dtype):
    """An infinity of V under a weight above zero is that infinity, in its own column alone."""
    c = attn_case(_gen(per + 3), [70, 9, 20] + [9] * 37, [150], [0, 39], 2, per, 64, 16, dtype, room=room, q_scale=0.5)
    plain = run_attn(c)
    r = 77                                                                        # of the prefix; 33 of batch row 0's own
    c["v_pool"][c["prefix_table"][0][r // 16].long(), :, r % 16, 5] = float("inf")
    c["v_pool"][c["page_table"][0][33 // 16].long(), 1, 33 % 16, 8] = -float("inf")
    got = run_attn(c)
    for a, b in zip(got[:2], plain[:2]):
        want = b.clone()
        want[:39, :, 5] = float("inf")
        want[0, per:, 8] = -float("inf")
        assert torch.equal(a, want)
    assert torch.equal(got[2], plain[2])
