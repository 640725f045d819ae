"""Gradients of logits some of which are masked, at temperatures and weights of the entropy whose product with the mask's value is past fp32's largest number."""
import math

import pytest
import torch

from rows_util import DEV, Logprobs, order, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("temperature,weight", [(1e-3, 1e3), (0.01, 1e5), (1.0, 1e9), (1.0, 0.3), (50.0, 1e20)])
@pytest.mark.parametrize("low", [-math.inf, "lowest", -1e30, -1e4])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("pad,lead", [(7, 0), (0, 1)])
def test_masked_entries(temperature, weight, low, f32, pad, lead):
    """A masked entry has probability 0 and takes part in nothing.  The others lie within 30 of each other in units of the temperature: none of their probabilities is below fp32's normal numbers."""
    t, vocab, top = 7, 9001, 5
    lowest = torch.finfo(torch.float32 if f32 else torch.bfloat16).min if low == "lowest" else low
    v = 2.0 + (randn((t, vocab), 4) * 3.0).clamp(-12, 12) * temperature
    hide = randn((t, vocab), 5) > -0.3
    hide[:, 4] = False
    hide[1] = True
    hide[1, 8123] = False                                               # one is left
    hide[2] = False
    hide[3] = True
    hide[3, 10:17] = False
    l = Logprobs(torch.where(hide, lowest, v), top, temperature, targets=torch.tensor([4, 5, 8123, 11, 0, 9000, 8999], dtype=torch.int32, device=DEV), pad=pad, lead=lead, f32=f32)
    ids = order(l.logits.v)[:, :top].to(torch.int32).contiguous()
    sign = torch.where(randn((t,), 6) > 0, 1.0, -1.0)
    for out32 in (False, True):
        for kw in (dict(dentropy=(sign * weight).float()), dict(dentropy=(sign * weight).float(), dlogprob=randn((t,), 7).float(), dtop=randn((t, top), 8).float(), ids=ids)):
            l.backward(out32=out32, **kw)
            torch.cuda.synchronize()
            assert bool(torch.isfinite(l.dl.v).all())
            l.check_back()
