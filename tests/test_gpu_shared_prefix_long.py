"""adsa_shared_prefix_attn against 64 bits where a block has long runs: many tiles of a prefix on tcgen05, and lists that are cut
into runs of several sizes, with items that go on from one run to the next.

Tolerances.  A weight enters the second product as the sum of two 16-bit values (cut, then rounded): bfloat16 keeps 16 bits of it
(off by at most 2^-16), float16 22 (2^-22), but no less than 2^-30 of the largest weight.  A score's 32-bit error is counted as in
test_gpu_shared_prefix.py, which moves a weight and the sum it is divided by.  A state of n cached rows takes 2 n / 16 matrix products
and as many rescalings at most into its 32-bit sums, each off by 2^-23 of what has been summed (tensor cores cut);
the merge, exponentials and the rest: 2^-18."""
import math

import pytest
import torch

from prefix_cut import Cut, WideCut, sweep_units, wide_units
from test_gpu_shared_prefix import DEV, HALF, _gen, _randn, _u, attn64, attn_case, run_attn

pytestmark = pytest.mark.gpu


def attn64_of(c, rows, scale):
    """attn64 for some batch rows, each as a group of its own."""
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


# ---- many tiles a block on tcgen05 --------------------------------------------------------------------------------------

def steps_of_scores(c, dim, prefix):
    """Moves each prefix's keys along a direction that every query shares, further from tile to tile and back again: maxima rise by about three
    (log2) a tile of 128 rows, so that sums are rescaled, and a run may begin anywhere on the slope."""
    page = c["k_pool"].shape[2]
    c["q"].add_(0.5)
    for g, n in enumerate(prefix):
        r = torch.arange(n, device=DEV)
        pg = c["prefix_table"][g][r // page].long()
        rise = ((r // 128) % 11).double() * (3 * math.log(2) / (0.5 * math.sqrt(dim)))
        at = c["k_pool"][pg, :, r % page, :dim].double() * 0.3 + rise[:, None, None]
        c["k_pool"][pg, :, r % page, :dim] = at.to(c["k_pool"].dtype)


WIDE = {  # batch rows of each group, prefix rows, key heads, query heads per key head, dim, page rows
    "256 query rows, 128 elements": ([64], [33000], 8, 4, 128, 64),
    "256 and 64, 64 elements": ([80], [33000], 4, 4, 64, 64),
    "256 and 144, 100 elements": ([100], [33001], 4, 4, 100, 64),
    "100 in turns, 64 elements": ([50], [50000], 8, 2, 64, 128),
    "70 in turns, 128 elements": ([35], [40077], 8, 2, 128, 48),
    "three groups, 128 elements": ([64, 30, 45], [30000, 9000, 18001], 4, 4, 128, 64),
    "three groups, 64 elements": ([65, 45, 3, 30], [30000, 19000, 500, 9127], 4, 4, 64, 572),
    "three groups, 30 elements": ([128, 33, 66], [30000, 31000, 18001], 4, 2, 30, 40),
}


@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("rising", [False, True])
@pytest.mark.parametrize("name", list(WIDE))
def test_many_tiles_of_a_prefix_in_a_block(name, rising, dtype):
    members, prefix, kv, per, dim, page = WIDE[name]
    start = [0]
    for m in members:
        start.append(start[-1] + m)
    batch = start[-1]
    own = [(7 * b) % 41 for b in range(batch)]
    c = attn_case(_gen(len(name) + dim), own, prefix, start, kv, per, dim, page, dtype, q_scale=1.0)
    if rising:
        steps_of_scores(c, dim, prefix)
    units = wide_units(prefix, start, kv, per)
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    assert units / WideCut(units, sms).runs > 12 and batch * per > 32 * len(prefix)   # the ring goes round more than twice
    got = run_attn(c)
    rows = sorted({0, 1, 31, batch // 2, batch - 2, batch - 1} | {min(batch - 1, s + d) for s in start for d in (0, 17)} - {-1})
    state = (units // sms + 2) * 128
    check_close(c, got, rows, attn64_of(c, rows, dim ** -0.5), dtype, state, max(prefix) + 41)
    assert all(torch.equal(a, b) for a, b in zip(got, run_attn(c)))


# ---- runs of several sizes ---------------------------------------------------------------------------------------------

@pytest.mark.parametrize("dtype", HALF)
@pytest.mark.parametrize("dim", [64, 100, 128, 200])
@pytest.mark.parametrize("K,rows", [(2, 11), (3, 24), (4, 52), (5, 88)])
def test_runs_of_several_sizes(K, rows, dim, dtype):
    """Ragged own rows and the prefixes of four groups in one list that is cut into 2 .. 5 sizes of runs: items of up to 40 tiles lie
    across runs of different sizes."""
    heads = {64: 32, 100: 16, 128: 16, 200: 8}[dim]
    own = [[100 + (877 * b) % 2200, 0, 2300, 64 * (b % 30)][b % 4 if b % 5 == 0 else 0] for b in range(rows)]
    prefix, start = [2424, 1, 700, 2500], [0, rows // 4, rows // 4 + 1, rows // 2, rows - 1]
    units = sweep_units(own, prefix, start, heads, 1, dim)
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    cut = Cut(units, sms * (2 if dim <= 128 else 1))
    assert cut.K == K or sms != 148
    c = attn_case(_gen(K + dim), own, prefix, start, heads, 1, dim, 64 if dim != 100 else 48, dtype, room=6000)
    got = run_attn(c)
    some = sorted({0, 1, 5, rows // 4, rows // 2, rows - 2, rows - 1} | set(range(0, rows, 7)))
    ref = attn64_of(c, some, dim ** -0.5)
    check_close(c, got, some, ref, dtype, 4800, 4800)
    assert all(torch.equal(a, b) for a, b in zip(got, run_attn(c)))
