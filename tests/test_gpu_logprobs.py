"""dbspmspv_logprobs and its gradient against 64 bits: vocabularies from one entry on, alternatives with ties, masks, rows with nothing left, infinities and NaN."""
import math

import numpy as np
import pytest
import torch

from paper_2608_16308_b200 import binding as B
from rows_util import DEV, Logprobs, Rows, at, order, randn

pytestmark = pytest.mark.gpu


def forward(l, **kw):
    l.forward(**kw)
    torch.cuda.synchronize()
    l.check()


def vec(t, seed, k=None):
    return randn((t,) if k is None else (t, k), seed).float()


def back(l, **kw):
    """every gradient at once, then each by itself"""
    t = l.t
    d, e = vec(t, 1), vec(t, 2) * 0.3
    ids = order(l.logits.v)[:, :l.top].to(torch.int32).contiguous() if l.top else None
    dt = vec(t, 3, l.top) if l.top else None
    for some in (dict(dlogprob=d, dentropy=e, dtop=dt, ids=ids), dict(dlogprob=d), dict(dentropy=e), dict(dtop=dt, ids=ids)):
        if any(v is not None for v in some.values()):
            l.backward(**some, **kw)
            torch.cuda.synchronize()
            l.check_back()


@pytest.mark.parametrize("vocab", [1, 2, 7, 8, 9, 31, 100, 1000, 4096, 4097, 8191, 32000, 50001, 131072])
@pytest.mark.parametrize("t", [1, 3])
@pytest.mark.parametrize("f32", [False, True])
def test_vocabularies(vocab, t, f32):
    l = Logprobs(randn((t, vocab), vocab, 3.0), min(vocab, 20), f32=f32)
    forward(l)
    back(l)


@pytest.mark.parametrize("pad,lead", [(0, 1), (1, 0), (3, 2), (5, 5), (8, 7)])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("vocab", [5, 519, 4103, 20001])
def test_strides(vocab, f32, pad, lead):
    l = Logprobs(randn((7, vocab), vocab, 3.0), min(vocab, 5), 0.7, pad=pad, lead=lead, f32=f32)
    forward(l)
    back(l)
    l.backward(dlogprob=vec(7, 1), out32=not f32)
    torch.cuda.synchronize()
    l.check_back()


@pytest.mark.parametrize("t", [18, 19, 37, 74, 75, 148, 149, 600])
def test_tokens(t):
    """every share of a row: clusters of eight to one"""
    l = Logprobs(randn((t, 17000), t, 3.0), 10, 1.3)
    forward(l)
    back(l)


@pytest.mark.parametrize("top", [0, 1, 2, 16, 17, 32, 33, 63, 64])
@pytest.mark.parametrize("f32", [False, True])
def test_alternatives(top, f32):
    """rounded to bf16 (and here to halves) logits tie all over the row"""
    for t, vocab in ((2, 40000), (200, 3000)):
        forward(Logprobs((randn((t, vocab), top, 3.0) * 2).round() / 2, top, f32=f32))
        forward(Logprobs(randn((t, vocab), top, 3.0), top, f32=f32))


@pytest.mark.parametrize("t", [1, 150])
@pytest.mark.parametrize("top", [1, 20, 64])
def test_orders_that_make_selection_hard(t, top):
    vocab = 36000
    up = torch.arange(vocab, device=DEV).double().repeat(t, 1)
    forward(Logprobs(up / 1000, top))                                   # ever larger
    forward(Logprobs(-up / 1000, top))
    forward(Logprobs(up * 0, top))                                      # all alike
    forward(Logprobs(torch.where(up % 2048 < 8, 5.0 + up / vocab, 0.0), top))      # the largest all belong to the same few threads
    forward(Logprobs(torch.where(up % 4096 < 4, 5.0, -up), top))
    forward(Logprobs(torch.where(up >= vocab - 700, 9.0, 0.0), top))    # at the end
    forward(Logprobs(torch.where(up % 2 == 0, 0.0, -0.0), top))         # both zeros


@pytest.mark.parametrize("top", [5, 30])
@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("low", [-math.inf, "lowest"])
def test_masks(top, f32, low):
    lowest = torch.finfo(torch.float32 if f32 else torch.bfloat16).min if low == "lowest" else low
    v = randn((8, 9000), 4, 3.0)
    hide = randn((8, 9000), 5) > -0.5
    hide[1] = True
    hide[2] = True
    hide[2, 8123] = False                                               # one is left
    hide[3, :] = True
    hide[3, 10:13] = False                                              # fewer than alternatives
    hide[4] = False
    l = Logprobs(torch.where(hide, lowest, v), top, f32=f32, targets=torch.tensor([1, 5, 8123, 11, 0, 7, 8999, 4], dtype=torch.int32, device=DEV))
    forward(l)
    back(l)
    forward(Logprobs(torch.where(hide, lowest, v), top, 0.5, f32=f32))


def test_nothing_left_has_no_gradient():
    l = Logprobs(torch.full((3, 700), -math.inf, device=DEV), 4)
    forward(l)
    assert bool((l.logprob[:3] == -math.inf).all()) and bool((l.entropy[:3] == 0).all())
    back(l)
    assert bool((l.dl.v == 0).all())


@pytest.mark.parametrize("bad", [math.nan, math.inf])
@pytest.mark.parametrize("t", [2, 300])
def test_spoiled_rows(bad, t):
    v = randn((t, 20000), 6, 3.0)
    clean = Logprobs(v, 9)
    forward(clean)
    w = v.clone()
    w[1, 777] = bad
    w[1, 15000] = bad
    l = Logprobs(w, 9)
    l.forward()
    torch.cuda.synchronize()
    rows = [r for r in range(t) if r != 1]
    for a, b in ((l.logprob, clean.logprob), (l.entropy, clean.entropy), (l.stats, clean.stats)):
        assert torch.equal(a[rows], b[rows])
    assert torch.equal(l.ids[:-1].reshape(t, 9)[rows], clean.ids[:-1].reshape(t, 9)[rows])
    assert math.isnan(float(l.logprob[1])) and math.isnan(float(l.entropy[1])) and bool(torch.isnan(l.lps[9:18]).all())
    assert torch.equal(l.ids[9:18].long(), order(l.logits.v)[1, :9])
    # the gradient from what the forward call kept
    d = vec(t, 1)
    out = Rows(t, 20000, 0, 0, None, torch.float32)
    B.dbspmspv_logprobs_backward(*at(l.logits), 1, t, 20000, 1.0, l.targets, l.stats, None, 0, None, d, None, None, *at(out), 1)
    torch.cuda.synchronize()
    assert bool(torch.isnan(out.v[1]).all()) and bool(torch.isfinite(out.v[rows]).all())


def test_only_nan():
    l = Logprobs(torch.full((2, 3000), math.nan, device=DEV), 3)
    l.forward()
    torch.cuda.synchronize()
    assert bool(torch.isnan(l.logprob[:2]).all()) and l.ids[:6].tolist() == [0, 1, 2, 0, 1, 2]


def test_targets():
    v = randn((6, 500), 7, 3.0)
    l = Logprobs(v, 3, targets=torch.tensor([-1, -100, 499, 500, 2 ** 31 - 1, 0], dtype=torch.int32, device=DEV))
    forward(l)
    d = vec(6, 1)
    l.backward(dlogprob=d)
    torch.cuda.synchronize()
    assert bool((l.dl.v[:2] == 0).all()) and bool(torch.isnan(l.dl.v[3:5]).all()) and bool(torch.isfinite(l.dl.v[[2, 5]]).all())


def test_alternatives_given_by_the_caller():
    """the same one twice, the target among them, ids that are none"""
    v = randn((4, 3000), 8, 3.0)
    l = Logprobs(v, 6, 0.8, targets=torch.tensor([5, 2999, 0, 17], dtype=torch.int32, device=DEV))
    ids = torch.tensor([[5, 5, 5, 9, 9, 1], [2999, 0, 1, 2, 3, 2998], [-1, 3000, 2 ** 31 - 1, -(2 ** 31), 0, 0], [1, 2, 3, 4, 5, 6]], dtype=torch.int32, device=DEV)
    l.backward(dlogprob=vec(4, 1), dentropy=vec(4, 2), dtop=vec(4, 3, 6), ids=ids)
    torch.cuda.synchronize()
    l.check_back()


@pytest.mark.parametrize("f32", [False, True])
@pytest.mark.parametrize("vocab,pad,lead", [(4103, 2, 1), (12345, 0, 0), (9, 0, 3)])
def test_in_place(f32, vocab, pad, lead):
    l = Logprobs(randn((5, vocab), 9, 3.0), 4, pad=pad, lead=lead, f32=f32)
    ids = order(l.logits.v)[:, :4].to(torch.int32).contiguous()
    l.backward(dlogprob=vec(5, 1), dentropy=vec(5, 2), dtop=vec(5, 3, 4), ids=ids, in_place=True)
    torch.cuda.synchronize()
    l.check_back()


def test_outputs_one_by_one():
    v = randn((5, 2000), 10, 3.0)
    for which in ("logprob", "entropy", "stats"):
        l = Logprobs(v, 0)
        forward(l, **{k: k == which for k in ("logprob", "entropy", "stats")})
    l = Logprobs(v, 7)
    forward(l, logprob=False, entropy=False, stats=False)
    ids = l.ids.clone()
    for a, b in ((l.ids, None), (None, l.lps)):
        B.dbspmspv_logprobs(*at(l.logits), 1, 5, 2000, 1.0, None, None, None, None, 7, a, b)
    torch.cuda.synchronize()
    l.check()
    assert torch.equal(ids, l.ids)


@pytest.mark.parametrize("temperature", [1e-3, 0.3, 50.0])
def test_temperatures(temperature):
    l = Logprobs(randn((6, 5000), 11, 3.0), 5, temperature)
    forward(l)
    back(l)


def test_logits_of_any_size():
    v = randn((6, 5000), 12, 3.0)
    v[0] += 1e30
    v[1] *= 1e35
    v[2] -= 3e38
    v[3] *= 1e-38
    l = Logprobs(v.clamp(-3e38, 3e38), 5)
    forward(l)
    back(l)


def test_gradients_against_differences():
    """central differences of the definition in 64 bits"""
    t, vocab, T = 3, 50, 0.9
    v = randn((t, vocab), 13, 2.0).float().double()
    l = Logprobs(v, 4, T)
    ids = order(v)[:, :4]
    d, e, dt = vec(t, 1), vec(t, 2), vec(t, 3, 4)
    l.backward(dlogprob=d, dentropy=e, dtop=dt, ids=ids.to(torch.int32).contiguous())
    torch.cuda.synchronize()

    def loss(z):
        logp = torch.log_softmax(z / float(np.float32(T)), dim=1)
        H = -(logp.exp() * logp).sum(dim=1)
        return (logp.gather(1, l.targets.long()[:, None])[:, 0] * d).sum() + (H * e).sum() + (logp.gather(1, ids) * dt).sum()

    for s in range(4):
        w = torch.randn(v.shape, generator=torch.Generator(device=DEV).manual_seed(s), device=DEV, dtype=torch.float64)
        want = (loss(v + 1e-5 * w) - loss(v - 1e-5 * w)) / 2e-5
        got = l.dl.f64() * w
        assert abs(float(got.sum() - want)) <= 1e-5 * float(got.abs().sum())


def test_rows_far_apart():
    """row offsets past 2^31 entries"""
    t, vocab, ld = 9, 1000, 1 << 28
    buf = torch.empty(t * ld, dtype=torch.bfloat16, device=DEV)
    v = buf.reshape(t, ld)[:, :vocab]
    v.copy_(randn((t, vocab), 14, 3.0))
    small = Logprobs(v.double(), 5, f32=False)
    forward(small)
    lp, ids = torch.empty(t, device=DEV), torch.empty((t, 5), dtype=torch.int32, device=DEV)
    B.dbspmspv_logprobs(v, ld, 0, t, vocab, 1.0, small.targets, lp, None, None, 5, ids, None)
    small.backward(dlogprob=vec(t, 1))
    B.dbspmspv_logprobs_backward(v, ld, 0, t, vocab, 1.0, small.targets, small.kept, None, 0, None, vec(t, 1), None, None, v, ld, 0)
    torch.cuda.synchronize()
    assert torch.equal(lp, small.logprob[:t]) and torch.equal(ids.reshape(-1), small.ids[:-1]) and torch.equal(v, small.dl.v)
