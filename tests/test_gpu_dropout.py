"""dbspmspv_dropout: the numbers of the published generator, entry by entry, whatever the strides, the type and the call."""
import numpy as np
import pytest
import torch

from paper_2608_16308_b200 import binding as B
from rows_util import DEV, Join, Rows, TYPE, at, keep, numbers, randn, seeded

pytestmark = pytest.mark.gpu


def dropped(x, drop, random, f32, y=None):
    t, n = x.v.shape
    y = y or Rows(t, n, x.ld - n, 0, None, x.buf.dtype)
    B.dbspmspv_dropout(*at(x), int(f32), t, n, drop, random, *at(y))
    torch.cuda.synchronize()
    return y


def want(x, drop, random, f32):
    t, n = x.shape
    below = int(np.floor(65536 * float(np.float32(drop)) + 0.5))
    scale = np.float32(65536) / np.float32(65536 - below) if below < 65536 else np.float32(0)
    kept = torch.from_numpy(numbers(random, t, n) >= below).to(DEV)
    return torch.where(kept, x.float() * float(scale), 0.0).to(TYPE[f32])


@pytest.mark.parametrize("t,n", [(1, 1), (1, 8), (3, 9), (5, 64), (17, 100), (1, 4096), (33, 1025), (2, 30001), (1030, 40), (4100, 3)])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("pad,lead", [(0, 0), (1, 0), (8, 3)])
def test_entries(t, n, f32, pad, lead):
    x = Rows(t, n, pad, lead, randn((t, n), t + n).to(TYPE[f32]), TYPE[f32])
    for drop, seed, offset in ((0.1, 5, 0), (0.5, -1, -1), (0.9, 1 << 62, 1 << 40)):
        y = dropped(x, drop, seeded(seed, offset), f32)
        assert torch.equal(y.v, want(x.v, drop, (seed, offset), f32)) and y.untouched()


def test_probabilities_at_the_ends():
    x = Rows(20, 1000, 0, 0, randn((20, 1000), 3).to(torch.bfloat16), torch.bfloat16)
    x.v[3, 5] = float("inf")
    x.v[4, 6] = float("nan")
    for drop in (1.0, 0.999999):
        assert bool((dropped(x, drop, seeded(1), False).v == 0).all())
    assert torch.equal(dropped(x, 0.0, None, False).v.view(torch.int16), x.v.view(torch.int16))
    assert torch.equal(dropped(x, 1e-7, seeded(1), False).v.view(torch.int16), x.v.view(torch.int16))
    y = dropped(x, 0.5, seeded(7), False)
    gone = ~keep((7, 0), 20, 1000, 0.5).bool()
    assert bool((y.v[gone] == 0).all()) and bool(torch.isfinite(y.v[~gone][:1].float()).all())


def test_the_gradient_is_the_same_call_and_joins_draw_the_same():
    t, n, drop, random = 50, 777, 0.3, seeded(99, 7)
    x = Rows(t, n, 0, 0, randn((t, n), 1).float(), torch.float32)
    y = dropped(x, drop, random, True)
    ones = Rows(t, n, 0, 0, torch.ones((t, n), device=DEV), torch.float32)
    mask = dropped(ones, drop, random, True).v
    assert torch.equal(y.v, x.v * mask)
    j = Join(t, n, "none", "none", scale=1.0, drop=drop, stream=True, blk=True, has_r=False)
    j.b, j.random = x, random
    j.forward(h=False, stats=False)
    torch.cuda.synchronize()
    assert torch.equal(j.out.v, y.v)


def test_in_place_and_share_of_dropped():
    x = Rows(700, 3001, 0, 0, torch.ones((700, 3001), device=DEV), torch.float32)
    y = dropped(x, 0.25, seeded(3, 4), True, y=x)
    share = float((y.v == 0).double().mean())
    # (2.1 million entries: five standard deviations are 0.0015)
    assert abs(share - 0.25) < 0.0015
    a, b = (dropped(Rows(64, 512, 0, 0, torch.ones((64, 512), device=DEV), torch.float32), 0.5, r, True).v for r in (seeded(3, 4), seeded(3, 5)))
    assert 0.4 < float((a == b).double().mean()) < 0.6


def test_a_long_batch():
    """rows past 2^31 entries: t * ld in 64 bits"""
    t, n = 70000, 40
    buf = torch.ones(t * 32768, dtype=torch.bfloat16, device=DEV)
    x = buf.reshape(t, 32768)[:, :n]
    random = seeded(8, 1)
    B.dbspmspv_dropout(x, 32768, 0, t, n, 0.5, random, x, 32768)
    torch.cuda.synchronize()
    assert torch.equal(x.double(), keep((8, 1), t, n, 0.5))
    assert bool((buf.reshape(t, 32768)[-5:, n:] == 1).all())
