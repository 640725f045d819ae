"""Alternatives of rows that a cluster shares out, where the candidates of one thread block are too many and those of the others are not."""
import pytest
import torch

from rows_util import DEV, Logprobs, order, randn

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("t", [1, 9, 60])
@pytest.mark.parametrize("top", [1, 20, 64])
def test_ties_in_one_share(top, t, f32):
    """Every block of the cluster takes the same way, however long one of them needs for its share: the answer is the same in each of many calls.  Ties of 700 logits lie in one share at a time (a
    share is vocab / 8 at least), a few larger logits in the others."""
    vocab = 72000
    calls = []
    for at in range(0, vocab - 4500, 9000):
        v = randn((t, vocab), at + 1, 0.5)
        v[:, at + 1800:at + 2500] = 9.0
        v[:, 11::17777] = 9.5
        calls.append(Logprobs(v, top, f32=f32))
    want = [order(l.logits.v)[:, :top] for l in calls]
    for _ in range(20):
        for l in calls:
            l.forward(entropy=False, stats=False)
        torch.cuda.synchronize()
        assert all(bool((l.ids[:-1].reshape(t, top).long() == w).all()) for l, w in zip(calls, want))
    for l in calls:
        l.check()
