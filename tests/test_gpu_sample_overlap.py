"""adsa_sample's outputs on top of its inputs: rows are drawn side by side, so a token written there could change another row's."""
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def test_outputs_over_inputs_are_refused():
    import paper_2506_18226_b200 as A
    n, vocab = 4, 64
    x, u = torch.randn(n, vocab, device=DEV), torch.rand(n, device=DEV)
    y = torch.randn(n, vocab, device=DEV)
    each = dict(temperature=torch.ones(n, device=DEV), top_k=torch.full((n,), 5, dtype=torch.int32, device=DEV), top_p=torch.full((n,), 0.9, device=DEV),
                min_p=torch.zeros(n, device=DEV))
    want = A.sample(x, u, uncond=y, guidance=2.0, **each)
    spare = torch.empty(n, dtype=torch.int32, device=DEV)
    before = [t.clone() for t in (x, y, u, *each.values())]
    for target in (x[1, 3:7], y[3, 60:], u, each["temperature"], each["top_k"], each["top_p"], each["min_p"]):
        with pytest.raises(ValueError, match="overlap"):
            A.sample(x, u, uncond=y, guidance=2.0, tokens=target.view(torch.int32), **each)
        with pytest.raises(ValueError, match="overlap"):
            A.sample(x, u, uncond=y, guidance=2.0, tokens=spare, logprobs=target.view(torch.float32), **each)
    with pytest.raises(ValueError, match="overlap"):
        A.sample(x, u, tokens=spare, logprobs=spare.view(torch.float32))
    assert all(torch.equal(a, b) for a, b in zip(before, (x, y, u, *each.values())))
    # beside one another they are taken
    both = torch.empty(2 * n, dtype=torch.int32, device=DEV)
    got = A.sample(x, u, uncond=y, guidance=2.0, tokens=both[:n], logprobs=both[n:].view(torch.float32), **each)
    assert torch.equal(got, want)
