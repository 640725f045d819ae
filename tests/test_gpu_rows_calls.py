"""Joins, dropout and log probabilities as a program uses them: a step of a pruned network forwards and backwards, captured and replayed calls, other streams, memory that is not the device's, rows far apart."""
import math
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2608_16308_b200 import binding as B
from linear_util import DEV, Layer, act, normal, room
from rows_util import HALF, Join, Logprobs, Rows, keep, near, randn, seeded

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


class Step:
    """h = norm(x); b = down(gated(h)); out, h2 = join(x, b) with norms on both sides, a gate and dropout; logits = head(h2); log probabilities of targets, and the gradients of all of it."""

    def __init__(self, t=37, n=264, hidden=520, vocab=1111, drop=0.1):
        self.t, self.n, self.hidden, self.vocab, self.drop = t, n, hidden, vocab, drop
        self.gate, self.up, self.down, self.head = Layer(hidden, n, seed=1), Layer(hidden, n, seed=2), Layer(n, hidden, seed=3), Layer(vocab, n, seed=4)
        self.x = normal((t, n), 5)
        self.w = {k: (randn((n,), i, 0.2, 1.0)).to(torch.bfloat16) for i, k in enumerate(("first", "block", "gate", "next"))}
        self.targets = torch.from_numpy(np.random.default_rng(6).integers(-1, vocab, t)).to(DEV).to(torch.int32)
        self.random = seeded(42, 7)
        self.dlogprob = torch.full((t,), -1.0 / t, device=DEV)
        self.first, self.join = B.default_join_opts(), B.default_join_opts()
        self.join.norm_block, self.join.scale, self.join.drop = B.NORM_RMS, 0.5, drop
        e = lambda *shape, dtype=torch.bfloat16: torch.empty(shape, dtype=dtype, device=DEV)
        for k, w in dict(h=n, g=hidden, u=hidden, y=hidden, b=n, out=n, h2=n, dh2=n, dout=n, db=n, dy=hidden, dh=n, dx=n, dlogits=vocab).items():
            setattr(self, k, e(t, w))
        self.logits, self.logprob, self.stats, self.kept, self.kept0 = e(t, vocab, dtype=torch.float32), e(t, dtype=torch.float32), e(t, 2, dtype=torch.float32), e(t, 4, dtype=torch.float32), e(t, 4, dtype=torch.float32)
        self.dw = {k: e(n, dtype=torch.float32) for k in self.w}
        self.ws = [room(l, u, t, True) for l, u in ((self.gate, self.up), (self.down, None), (self.head, None))]
        nb = B.dbspmspv_join_workspace(self.join, t, n)
        self.jw = torch.empty(nb, dtype=torch.uint8, device=DEV), nb

    def run(self, stream=None):
        t, n, hid, v, w = self.t, self.n, self.hidden, self.vocab, self.w
        B.dbspmspv_join(self.first, t, n, self.x, n, None, 0, None, None, None, 0, w["first"], None, None, None, 0, self.h, n, self.kept0, stream)
        B.dbspmspv_gated(self.gate.h, self.up.h, self.h, n, t, B.ACT_SILU, self.y, hid, self.g, self.u, hid, *self.ws[0], stream)
        B.dbspmspv_linear(self.down.h, self.y, hid, t, None, B.ACT_NONE, None, 0, self.b, n, 0, None, 0, *self.ws[1], stream)
        B.dbspmspv_join(self.join, t, n, self.x, n, self.b, n, w["block"], None, w["gate"], 0, w["next"], None, self.random, self.out, n, self.h2, n, self.kept, stream)
        B.dbspmspv_linear(self.head.h, self.h2, n, t, None, B.ACT_NONE, None, 0, self.logits, v, 1, None, 0, *self.ws[2], stream)
        B.dbspmspv_logprobs(self.logits, v, 1, t, v, 1.0, self.targets, self.logprob, None, self.stats, 0, None, None, stream)
        B.dbspmspv_logprobs_backward(self.logits, v, 1, t, v, 1.0, self.targets, self.stats, None, 0, None, self.dlogprob, None, None, self.dlogits, v, 0, stream)
        B.dbspmspv_linear_backward(self.head.h, self.h2, n, t, B.ACT_NONE, None, 0, self.dlogits, v, self.dh2, n, None, None, *self.ws[2], stream)
        B.dbspmspv_join_backward(self.join, t, n, self.out, n, self.b, n, self.kept, w["block"], None, w["gate"], 0, w["next"], self.random, self.dh2, n, None, 0, self.dout, n, self.db, n,
                                 self.dw["block"], None, self.dw["gate"], 0, self.dw["next"], None, *self.jw, stream)
        B.dbspmspv_linear_backward(self.down.h, self.y, hid, t, B.ACT_NONE, None, 0, self.db, n, self.dy, hid, None, None, *self.ws[1], stream)
        B.dbspmspv_gated_backward(self.gate.h, self.up.h, self.h, n, t, B.ACT_SILU, self.g, self.u, hid, self.dy, hid, self.dh, n, None, None, *self.ws[0], stream)
        B.dbspmspv_join_backward(self.first, t, n, self.x, n, None, 0, self.kept0, None, None, None, 0, w["first"], None, self.dh, n, self.dout, n, self.dx, n, None, 0, None, None, None, 0,
                                 self.dw["first"], None, *self.jw, stream)

    def want(self):
        x = self.x.double().requires_grad_()
        w = {k: v.double().requires_grad_() for k, v in self.w.items()}
        rms = lambda v, g: v / (v.square().mean(dim=1, keepdim=True) + 1e-5).sqrt() * g
        h = rms(x, w["first"])
        b = (act(h @ self.gate.dense.T, "silu") * (h @ self.up.dense.T)) @ self.down.dense.T
        out = x + 0.5 * keep(self.random.tolist(), self.t, self.n, self.drop) * w["gate"] * rms(b, w["block"])
        logp = torch.log_softmax(rms(out, w["next"]) @ self.head.dense.T, dim=1)
        has = self.targets >= 0
        lp = torch.where(has, logp.gather(1, self.targets.long().clamp(min=0)[:, None])[:, 0], 0.0)
        (lp * self.dlogprob.double()).sum().backward()
        return lp.detach(), x.grad, {k: v.grad for k, v in w.items()}

    def close(self):
        for l in (self.gate, self.up, self.down, self.head):
            l.close()


def test_a_step_of_a_network():
    """Nine arrays are rounded to bf16 on the way to a gradient (h, g and u, y, b, out, h2, dlogits, dh2, db, dy ...), each off by 2^-8 of its entries at most and by half of that in the 2-norm; norms and products
    hand the error on unmagnified, SiLU by 1.1: 9 * 2^-9 * 1.1 = 0.02, where no two of them cancel, and twice that where they add up with the layers' own 2.3e-3."""
    s = Step()
    s.run()
    torch.cuda.synchronize()
    lp, dx, dw = s.want()
    off = lambda a, b: float((a.double() - b).norm() / b.norm())
    assert off(s.logprob, lp) < 0.04 and off(s.dx, dx) < 0.04
    for k in dw:
        assert off(s.dw[k], dw[k]) < 0.04, k
    s.close()


def test_captured_steps_draw_what_the_device_says():
    s = Step(drop=0.3)
    outs = lambda: [v.clone() for v in (s.out, s.logprob, s.dx, s.db, *s.dw.values())]
    s.run()
    torch.cuda.synchronize()
    eager = outs()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        s.run()
    for v in (s.out, s.dx, s.db):
        v.zero_()
    g.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(eager, outs()))
    s.random[1] += 1                                             # another step's numbers, the same graph
    g.replay()
    torch.cuda.synchronize()
    replayed = outs()
    assert not torch.equal(eager[0], replayed[0])
    s.run()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(outs(), replayed))
    lp, dx, _ = s.want()
    assert float((s.dx.double() - dx).norm() / dx.norm()) < 0.04
    del g
    s.close()


def test_captured_before_any_other_call():
    """kernels that no call has loaded yet, in a process of its own"""
    code = r"""
import sys, os
sys.path.insert(0, os.getcwd()); sys.path.insert(0, os.path.join(os.getcwd(), "tests"))
import torch
from rows_util import Join, Logprobs, randn
j, l = Join(40, 5000, gate="shared", drop=0.1), Logprobs(randn((3, 40000), 1, 3.0), 5)
j.set_kept()
torch.cuda.synchronize()
st = torch.cuda.Stream()
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g, stream=st):
    j.forward(); kept = j.out, j.h, j.stats
    l.forward()
g.replay(); torch.cuda.synchronize()
j.check(); l.check()
print("right")
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert "right" in r.stdout, r.stdout[-2000:] + r.stderr[-2000:]


def test_two_streams_at_once():
    a, b = Join(900, 3000, gate="shared", drop=0.1, seed=1), Join(900, 3000, gate="shared", drop=0.1, seed=50)
    la, lb = Logprobs(randn((300, 20000), 1, 3.0), 5), Logprobs(randn((300, 20000), 2, 3.0), 5)
    for j in (a, b):
        j.set_kept()
    torch.cuda.synchronize()
    s, u = torch.cuda.Stream(), torch.cuda.Stream()
    for _ in range(5):
        with torch.cuda.stream(s):
            a.backward()
            la.forward()
        with torch.cuda.stream(u):
            b.backward()
            lb.forward()
    torch.cuda.synchronize()
    a.check_back(), b.check_back(), la.check(), lb.check()
    x = Join(20, 300, seed=3)
    torch.cuda.synchronize()
    x.forward(stream=s.cuda_stream)                              # a raw stream
    torch.cuda.synchronize()
    x.check()


def status(f, *args, **kw):
    with pytest.raises(B.DbSpmspvError) as e:
        f(*args, **kw)
    return e.value.status


def test_memory_of_the_host_is_refused():
    """an address that kernels could not read (a numpy array's) is found out before anything runs"""
    h = np.zeros(4096, np.float32)
    d = torch.zeros(4096, device=DEV)
    random = seeded(1)
    o = B.default_join_opts()
    o.stream_f32 = 1
    for a, b in ((h, d), (d, h)):
        assert status(B.dbspmspv_join, o, 2, 8, a, 8, None, 0, None, None, None, 0, None, None, None, b, 8, None, 0, None) == B.ERR_INVALID_ARG
        assert status(B.dbspmspv_dropout, a, 8, 1, 2, 8, 0.5, random, b, 8) == B.ERR_INVALID_ARG
        assert status(B.dbspmspv_logprobs_backward, a, 8, 1, 2, 8, 1.0, None, d, None, 0, None, None, None, None, b, 8, 1) == B.ERR_INVALID_ARG
    assert status(B.dbspmspv_logprobs, h, 8, 1, 2, 8, 1.0, None, None, d, None, 0, None, None) == B.ERR_INVALID_ARG
    assert status(B.dbspmspv_join_backward, o, 2, 8, None, 0, None, 0, d, None, None, None, 0, None, None, None, 0, h, 8, d, 8, None, 0, None, None, None, 0, None, None, None, 0) == B.ERR_INVALID_ARG
    torch.cuda.synchronize()


def test_workspace():
    j = Join(50, 520, gate="shared")
    j.set_kept()
    nb = B.dbspmspv_join_workspace(j.opts, 50, 520)
    assert nb > 0 and B.dbspmspv_join_workspace(j.opts, 0, 520) == 0
    d = torch.empty(520, device=DEV)
    args = lambda ws, n, dw: (j.opts, 50, 520, j.out.start, 520, j.b.start, 520, j.kept, j.wb, None, j.gate, 0, j.wn, None, j.dh.start, 520, j.dout.start, 520, j.res_dr, 520, None, 0, None, None, None, 0, dw, None, ws, n)
    j.res_dr = torch.empty((50, 520), dtype=torch.bfloat16, device=DEV)
    ws = torch.empty(nb, dtype=torch.uint8, device=DEV)
    B.dbspmspv_join_backward(*args(ws, nb, d))
    B.dbspmspv_join_backward(*args(None, 0, None))               # (no sums: none is needed)
    assert status(B.dbspmspv_join_backward, *args(ws, nb - 1, d)) == B.ERR_INVALID_ARG
    assert status(B.dbspmspv_join_backward, *args(None, nb, d)) == B.ERR_INVALID_ARG
    torch.cuda.synchronize()


def test_no_tokens_zero_the_sums():
    j = Join(3, 100, "layer", "layer", c=True, gate="shared", seed=2)
    j.set_kept()
    v = [torch.full((101,), 77.0, device=DEV) for _ in range(5)]
    B.dbspmspv_join_backward(j.opts, 0, 100, None, 0, None, 0, None, j.wb, j.cb, j.gate, 0, j.wn, None, None, 0, None, 0, None, 0, None, 0, v[0], v[1], v[2], 0, v[3], v[4], None, 0)
    torch.cuda.synchronize()
    assert all(bool((x[:100] == 0).all()) and float(x[100]) == 77.0 for x in v)


def test_no_memory_is_allocated():
    j, l = Join(300, 2000, gate="shared", drop=0.1), Logprobs(randn((100, 30000), 1, 3.0), 5)
    j.forward(), l.forward()
    j.backward()
    torch.cuda.synchronize()
    ws = torch.empty(B.dbspmspv_join_workspace(j.opts, j.t, j.n), dtype=torch.uint8, device=DEV)
    j.backward(workspace=ws)
    d = torch.zeros(100, device=DEV)
    l.backward(dlogprob=d)
    torch.cuda.synchronize()
    torch.cuda.empty_cache()
    before = torch.cuda.mem_get_info()[0]
    o = j.opts
    for _ in range(20):
        B.dbspmspv_join(o, j.t, j.n, j.r.start, j.r.ld, j.b.start, j.b.ld, j.wb, None, j.gate, 0, j.wn, None, j.random, j.out.start, j.out.ld, j.h.start, j.h.ld, j.stats)
        B.dbspmspv_logprobs(l.logits.start, l.logits.ld, 1, l.t, l.vocab, 1.0, l.targets, l.logprob, l.entropy, l.stats, 5, l.ids, l.lps)
    torch.cuda.synchronize()
    assert torch.cuda.mem_get_info()[0] == before


def test_joins_of_rows_far_apart():
    """offsets past 2^31 entries, and rows whose stride in bytes needs more than 32 bits"""
    for t, n, ld in ((70, 520, 1 << 25), (3, 264, (1 << 31) + 8)):
        j = Join(t, n, gate="shared", drop=0.2, seed=4)
        j.forward()
        want = j.out.v.clone(), j.h.v.clone()
        buf = torch.empty((t - 1) * ld + n, dtype=torch.bfloat16, device=DEV)
        far = torch.as_strided(buf, (t, n), (ld, 1))
        far.copy_(j.r.v)
        B.dbspmspv_join(j.opts, t, n, far, ld, j.b.start, j.b.ld, j.wb, None, j.gate, 0, j.wn, None, j.random, far, ld, j.h.start, j.h.ld, j.stats)
        torch.cuda.synchronize()
        assert torch.equal(far, want[0]) and torch.equal(j.h.v, want[1])
        del buf, far


def test_a_batch_in_parts_is_the_batch():
    """rows do not depend on one another, nor on how many there are"""
    j = Join(700, 1300, "layer", "rms", c=True, gate="shared", seed=6)
    j.forward()
    whole = j.out.v.clone(), j.h.v.clone(), j.stats.clone()
    out, h, st = torch.empty_like(whole[0]), torch.empty_like(whole[1]), torch.empty((700, 4), device=DEV)
    for a, b in ((0, 1), (1, 150), (150, 700)):
        B.dbspmspv_join(j.opts, b - a, 1300, j.r.v[a:], j.r.ld, j.b.v[a:], j.b.ld, j.wb, j.cb, j.gate, 0, j.wn, j.cn, None, out[a:], 1300, h[a:], 1300, st[a:])
    torch.cuda.synchronize()
    # (a row may be shared out to fewer or more lanes: its sums are added in another order, 23 roundings)
    near(out, whole[0].double(), 2 * HALF * whole[0].double().abs() + 1e-4)
    near(h, whole[1].double(), 2 * HALF * whole[1].double().abs() + 1e-4)
    near(st, whole[2][:700].double(), 1e-5 * (1 + whole[2][:700].double().abs()))
