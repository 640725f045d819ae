"""Gradients of ids that are given more than once: the weights are added in the order in which they are given, the target's behind them, in every call alike."""
import numpy as np
import pytest
import torch

from rows_util import DEV, Logprobs, randn

pytestmark = pytest.mark.gpu
BIG = float(2 ** 30)                          # (next to it 1 is lost)


@pytest.mark.parametrize("weights", [(BIG, -BIG, 1.0), (BIG, 1.0, -BIG), (1.0, BIG, -BIG), (0.1, 0.7, -0.3)], ids=str)
@pytest.mark.parametrize("top", [3, 40, 64])
@pytest.mark.parametrize("with_target", [False, True])
@pytest.mark.parametrize("f32", [False, True])
def test_order_of_the_weights(weights, top, with_target, f32):
    """Three and more weights at one id whose probability is 0, so that its gradient is their sum in fp32 and nothing else."""
    t, vocab, id = 4, 3001, (7, 3000, 2, 1500)
    v = randn((t, vocab), 8, 3.0)
    for r in range(t):
        v[r, id[r]] = -400.0
    at = np.linspace(0, top - (2 if with_target else 1), 2 if with_target else 3).astype(int)
    ids = torch.arange(100, 100 + top, dtype=torch.int32, device=DEV).repeat(t, 1)
    d, dt = torch.zeros(t, device=DEV), torch.zeros((t, top), device=DEV)
    places = list(at) + ([None] if with_target else [])
    for r in range(t):
        for j, w in zip(places, weights):
            if j is None:
                d[r] = w
            else:
                ids[r, j], dt[r, j] = id[r], w
    l = Logprobs(v, top, targets=torch.tensor(id, dtype=torch.int32, device=DEV), f32=f32)
    a, b, c = (np.float32(w) for w in weights)
    want = float(np.float32(a + b) + c)
    runs = []
    for _ in range(10):
        l.backward(dlogprob=d if with_target else None, dtop=dt, ids=ids, out32=True)
        torch.cuda.synchronize()
        assert [float(l.dl.v[r, id[r]]) for r in range(t)] == [want] * t
        runs.append(l.dl.v.clone())
    assert all(torch.equal(runs[0], r) for r in runs)
