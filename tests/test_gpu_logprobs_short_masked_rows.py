"""Alternatives of rows so short that many threads have no logit, where fewer than are asked for are not -inf."""
import math

import pytest
import torch

from rows_util import DEV, Logprobs, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("vocab", [1, 2, 5, 9, 44, 179, 500, 1000])
@pytest.mark.parametrize("top", [1, 2, 20, 64])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("lead", [0, 1])
def test_fewer_than_alternatives(vocab, top, f32, lead):
    """Row r keeps r logits (the first ones, then random ones), row 0 none."""
    t = 70
    v = randn((t, vocab), vocab, 3.0)
    v = torch.where(torch.argsort(torch.argsort(randn((t, vocab), vocab + 1), dim=1), dim=1) < torch.arange(t, device=DEV)[:, None], v, -math.inf)
    v[1] = -math.inf
    v[1, 0] = -2.0
    l = Logprobs(v, min(top, vocab), f32=f32, lead=lead)
    for entropy in (True, False):
        l.forward(entropy=entropy)
        torch.cuda.synchronize()
        l.check()
