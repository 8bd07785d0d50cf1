"""What the draw of a token refuses, found on the host before anything is launched.  Addresses here are made up and never dereferenced."""
import ctypes as C
import math

import pytest
import torch

import paper_2506_18226_b200 as A
from paper_2506_18226_b200 import binding as B

P = 0x10000000


def _sample(how=None, **kw):
    s = dict(temperature=1.0, top_k=5, top_p=0.9, min_p=0.0, temperatures=None, top_ks=None, top_ps=None, min_ps=None, guidance=1.0)
    s.update(how or {})
    a = dict(how=C.byref(B.AdsaSampling(*s.values())), dtype=0, logits=P, row=100, uncond=P, uncond_row=100, rows=2, vocab=100, u=P, tokens=P, logprobs=P)
    a.update(kw)
    return A.load().adsa_sample(*a.values(), None)


@pytest.mark.parametrize("kw", [dict(how=None), dict(dtype=3), dict(dtype=-1), dict(logits=None), dict(u=None), dict(tokens=None), dict(rows=-1), dict(vocab=0),
                                dict(vocab=2**20 + 1), dict(logits=P + 1), dict(dtype=2, logits=P + 2), dict(uncond=P + 1), dict(u=P + 2), dict(tokens=P + 1),
                                dict(logprobs=P + 2)])
def test_refusals(kw):
    if "how" in kw:
        assert A.load().adsa_sample(None, 0, P, 100, None, 0, 2, 100, P, P, None, None) == B.EINVAL
    else:
        assert _sample(**kw) == B.EINVAL


@pytest.mark.parametrize("how", [dict(temperature=math.nan), dict(top_p=math.nan), dict(min_p=math.nan), dict(guidance=math.inf), dict(guidance=math.nan),
                                 dict(temperatures=P + 1), dict(top_ks=P + 2), dict(top_ps=P + 3), dict(min_ps=P + 1)])
def test_settings_refused(how):
    assert _sample(how) == B.EINVAL


def test_nothing_to_do_is_ok():
    assert _sample(rows=0) == 0


def test_the_binding_refuses_wrong_types_shapes_and_devices():
    x, u, i = torch.zeros(3, 10), torch.zeros(3), torch.zeros(3, dtype=torch.int32)
    for kw in (dict(), dict(logits=x.double()), dict(logits=x[0]), dict(logits=x.t()), dict(uniforms=u[:2]), dict(uniforms=u.double()), dict(uncond=x.half()),
               dict(uncond=x[:, :5]), dict(tokens=u), dict(logprobs=i), dict(temperature=u[:2]), dict(top_k=u), dict(top_p=i), dict(min_p=u.double()), dict(top_k=2**40)):
        with pytest.raises(ValueError):                                            # the first: not on a GPU
            A.sample(**dict(dict(logits=x, uniforms=u), **kw))
