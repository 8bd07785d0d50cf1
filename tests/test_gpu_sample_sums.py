"""The draw's sums: weights are whole multiples of 2^-42 of the largest, so a sum of n of them is off by n 2^-43 of it at most.  A peak over a flat tail, whose
roundings all go one way, shows it whole."""
import math

import pytest
import torch

pytestmark = pytest.mark.gpu

DEV = "cuda:0"


@pytest.mark.parametrize("vocab", [1000, 16384, 131072, 2 ** 20])
@pytest.mark.parametrize("depth", [5.0, 20.0, 28.5, 29.0, 29.5, 30.0, 33.0])
def test_a_peak_over_a_flat_tail(vocab, depth):
    """Every drawn id has the uniform number within its edges, up to the bound; so do the borders of top_p."""
    import paper_2506_18226_b200 as A
    us = [0.0, 0.25, 0.5, 1 - 2.0 ** -10, 1 - 2.0 ** -20, 1 - 2.0 ** -23, 1 - 2.0 ** -24]
    peak = vocab // 3
    x = torch.full((len(us), vocab), -depth, device=DEV)
    x[:, peak] = 0.0
    u, lp = torch.tensor(us, device=DEV), torch.empty(len(us), device=DEV)
    w = math.exp(-depth)
    total, bound = 1 + (vocab - 1) * w, vocab * 2.0 ** -43
    for i, token in enumerate(A.sample(x, u, logprobs=lp).tolist()):
        before = token * w + (1 - w if token > peak else 0.0)             # real sums before and after the id
        after = before + (1.0 if token == peak else w)
        assert before - 2 * bound <= us[i] * total <= after + 2 * bound, (us[i], token)
        want = (0.0 if token == peak else -depth) - math.log(total)
        assert abs(float(lp[i]) - want) <= bound + 2.0 ** -24 * abs(want)
    # the mass that top_p keeps, by the share of the peak (drawn: all ids before it have less than u = 0.3 of the mass, or top_p leaves them out)
    for p in (1 - 2.0 ** -24, 1 - 2.0 ** -20, 0.999):
        head = torch.full((1, vocab), -depth, device=DEV)
        head[0, 0] = 0.0                                                   # (the first id: drawn with u = 0)
        one = torch.empty(1, device=DEV)
        assert A.sample(head, torch.zeros(1, device=DEV), top_p=p, logprobs=one).item() == 0
        kept = math.exp(-float(one))
        goal = torch.tensor(p, dtype=torch.float32).item() * total
        # (lp is rounded to 32 bits, half a step 2^-24 of |lp| at most, and exp makes that a relative error of the mass: 4.8 2^-24 for a mass of 111)
        off = 2.0 ** -24 * abs(float(one)) + 1e-12
        assert max(goal, 1.0) - 3 * bound <= kept * (1 + off) and kept * (1 - off) <= max(goal, 1.0) + w + 3 * bound
