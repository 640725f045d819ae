"""Plain forms in 64 bits and error bounds for the tests of dbspmspv_join, dbspmspv_dropout, dbspmspv_logprobs and their gradients.

E is a rounding to fp32.  A sum over a row passes at most 8 + 5 + 8 roundings where a thread's own terms, a warp's and a team's follow one another, and what is made of it a few more: MANY of
them cover a norm or a slope, relative to the magnitudes that enter it."""
import math

import numpy as np
import torch

from paper_2608_16308_b200 import binding as B
from linear_util import DEV, HALF, Rows, near  # noqa: F401

E = 2.0 ** -24
MANY = 64 * E
NORM = {"none": B.NORM_NONE, "rms": B.NORM_RMS, "layer": B.NORM_LAYER}
TYPE = {False: torch.bfloat16, True: torch.float32}


def philox(c, k):
    """Philox 4x32-10 on Python integers: counter of four words, key of two."""
    c, k = list(c), list(k)
    for _ in range(10):
        p, q = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(q >> 32) ^ c[1] ^ k[0], q & 0xFFFFFFFF, (p >> 32) ^ c[3] ^ k[1], p & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def numbers(random, tokens, n):
    """The 16 bits of every entry (numpy, unsigned 64-bit words)."""
    seed, offset = (int(v) & 0xFFFFFFFFFFFFFFFF for v in random)
    eights = (n + 7) // 8
    c = [np.broadcast_to(np.arange(eights, dtype=np.uint64), (tokens, eights)), np.broadcast_to(np.arange(tokens, dtype=np.uint64)[:, None], (tokens, eights)),
         np.full((tokens, eights), offset & 0xFFFFFFFF, np.uint64), np.full((tokens, eights), offset >> 32, np.uint64)]
    k = [seed & 0xFFFFFFFF, seed >> 32]
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        p, q = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(q >> half) ^ c[1] ^ np.uint64(k[0]), q & low, (p >> half) ^ c[3] ^ np.uint64(k[1]), p & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    w = np.stack(c, axis=-1)
    return np.stack([w & np.uint64(0xFFFF), w >> np.uint64(16)], axis=-1).reshape(tokens, eights * 8)[:, :n].astype(np.int64)


def keep(random, tokens, n, drop, dev=None):
    """What each entry is multiplied with, in 64 bits."""
    if not drop:
        return torch.ones((tokens, n), dtype=torch.float64, device=dev or DEV)
    below = math.floor(65536 * float(np.float32(drop)) + 0.5)
    scale = 65536 / (65536 - below) if below < 65536 else 0.0
    return torch.from_numpy((numbers(random, tokens, n) >= below) * scale).to(dev or DEV)


def seeded(seed, offset=0):
    return torch.tensor([seed, offset], dtype=torch.int64, device=DEV)


def randn(shape, seed, scale=1.0, mean=0.0):
    return torch.from_numpy(np.random.default_rng(seed).standard_normal(shape) * scale + mean).to(DEV)


def stats_of(x, norm, eps):
    mean = x.mean(dim=1, keepdim=True) if norm == "layer" else torch.zeros_like(x[:, :1])
    if norm == "none":
        return mean, mean + 1
    return mean, ((x - mean).square().mean(dim=1, keepdim=True) + eps) ** -0.5


def mean(x):
    return x.mean(dim=1, keepdim=True)


class Join:
    """The operands of a join, what it and its gradient are in 64 bits, with bounds, and the calls."""

    def __init__(self, t, n, block="rms", next="rms", w=True, c=False, gate="none", scale=0.75, drop=0.0, stream=False, blk=False, params=False, dblk=False, pad=0, lead=0, seed=0, eps=1e-5,
                 has_b=True, has_r=True):
        self.t, self.n, self.block, self.next, self.gate_kind, self.scale, self.drop, self.eps = t, n, block, next, gate, scale, drop, eps
        self.st, self.bt, self.pt, self.dt = TYPE[stream], TYPE[blk], TYPE[params], TYPE[dblk]
        self.pad, self.lead = pad, lead
        row = lambda dtype, seed_, **kw: Rows(t, n, pad, lead, randn((t, n), seed_, **kw).to(dtype), dtype)
        vec = lambda seed_, m: randn((n,), seed_, 0.3, m).to(self.pt)
        self.r, self.b = row(self.st, seed + 1, scale=1.5) if has_r else None, row(self.bt, seed + 2, scale=0.7, mean=0.2) if has_b else None
        self.wb, self.cb = (vec(seed + 3, 1.0) if w and block != "none" else None), (vec(seed + 4, 0.0) if c and block != "none" else None)
        self.wn, self.cn = (vec(seed + 5, 1.0) if w and next != "none" else None), (vec(seed + 6, 0.0) if c and next != "none" else None)
        self.gate = None if gate == "none" else vec(seed + 7, 0.5) if gate == "shared" else row(self.pt, seed + 7, scale=0.3, mean=0.5)
        self.random = seeded(1234567890123 + seed, 99 << 32 | seed) if drop else None
        self.dh, self.dout = row(torch.bfloat16, seed + 8), row(self.st, seed + 9)
        o = B.default_join_opts()
        o.norm_block, o.norm_next, o.eps_block, o.eps_next, o.scale, o.drop = NORM[block], NORM[next], eps, eps, scale, drop
        o.stream_f32, o.block_f32, o.params_f32, o.dblock_f32 = int(stream), int(blk), int(params), int(dblk)
        self.opts = o
        f = lambda v, d: torch.full((n,), d, dtype=torch.float64, device=DEV) if v is None else v.double()
        self.wbd, self.cbd, self.wnd, self.cnd = f(self.wb, 1.0), f(self.cb, 0.0), f(self.wn, 1.0), f(self.cn, 0.0)
        self.gd = f(None, 1.0) if self.gate is None else self.gate.double() if gate == "shared" else self.gate.f64()
        self.mask = keep(self.random.tolist() if drop else None, t, n, drop)

    def rows(self, dtype):
        return Rows(self.t, self.n, self.pad, self.lead, None, dtype)

    # ---- forward
    def forward(self, out=None, h=True, stats=True, stream=None, want_out=True):
        self.out = out if out is not None else self.rows(self.st) if want_out else None
        self.h = self.rows(torch.bfloat16) if h else None
        self.stats = torch.full((self.t + 1, 4), 77.0, device=DEV) if stats else None
        g = self.gate
        B.dbspmspv_join(self.opts, self.t, self.n, *at(self.r), *at(self.b), self.wb, self.cb, g.start if isinstance(g, Rows) else g, g.ld if isinstance(g, Rows) else 0, self.wn, self.cn,
                        self.random, *at(self.out), *at(self.h), self.stats, stream)

    def want(self):
        r = self.r.f64() if self.r else torch.zeros((self.t, self.n), dtype=torch.float64, device=DEV)
        if self.b is None:
            m0 = torch.zeros((self.t, 1), dtype=torch.float64, device=DEV)
            i0, out, e = m0 + 1, r, E * r.abs()
        else:
            b = self.b.f64()
            m0, i0 = stats_of(b, self.block, self.eps)
            y = ((b - m0) * i0 * self.wbd + self.cbd) * self.gd * self.scale * self.mask
            size = ((b.abs() + mean(b.abs())) * i0 * self.wbd.abs() + self.cbd.abs()) * self.gd.abs() * abs(self.scale) * self.mask
            out, e = r + y, MANY * size + E * (r.abs() + y.abs())
        m1, i1 = stats_of(out, self.next, self.eps)
        xh = (out - m1) * i1
        h = xh * self.wnd + self.cnd
        rms = lambda v: mean(v.square()).sqrt()
        eh = self.wnd.abs() * ((e + mean(e)) * i1 + MANY * (out.abs() + mean(out.abs())) * i1 + xh.abs() * rms(e) * i1) + 4 * E * (h.abs() + self.cnd.abs())
        return out, e, h, eh, torch.cat([m0, i0, m1, i1], dim=1)

    def check(self):
        out, e, h, eh, st = self.want()
        step = HALF if self.st == torch.bfloat16 else E
        if self.out is not None:
            near(self.out.v, out, e + step * (out.abs() + e))
            assert self.out.untouched()
        if self.h is not None:
            near(self.h.v, h, eh + HALF * (h.abs() + eh))
            assert self.h.untouched()
        if self.stats is not None:
            err = torch.cat([MANY * mean(self.b.f64().abs()) if self.b else mean(out) * 0, MANY * st[:, 1:2], MANY * mean(out.abs()) + mean(e), (MANY + 2 * mean(e.square()).sqrt() * st[:, 3:4]) * st[:, 3:4]], dim=1)
            near(self.stats[:self.t], st, err)
            assert bool((self.stats[self.t] == 77.0).all())

    # ---- backward, from `out` and `stats` as a forward call leaves them (here: rounded 64-bit values)
    def set_kept(self):
        out, _, _, _, st = self.want()
        self.out = Rows(self.t, self.n, self.pad, self.lead, out.to(self.st), self.st)
        self.kept = st.float()

    def backward(self, wanted=("dr", "db", "dgate", "dw_block", "dc_block", "dw_next", "dc_next"), dh=True, dout=True, in_place=False, stream=None, workspace=None):
        n = self.n
        g = self.gate
        self.set_kept() if not hasattr(self, "kept") else None
        self.res = {}
        if "dr" in wanted:
            self.res["dr"] = self.dout if in_place else self.rows(self.st)
        if "db" in wanted:
            self.res["db"] = self.rows(self.dt)
        if "dgate" in wanted and g is not None:
            self.res["dgate"] = self.rows(self.pt) if isinstance(g, Rows) else torch.full((n + 1,), 77.0, device=DEV)
        for k, has in (("dw_block", self.block != "none"), ("dc_block", self.block != "none"), ("dw_next", self.next != "none"), ("dc_next", self.next != "none")):
            if k in wanted and has:
                self.res[k] = torch.full((n + 1,), 77.0, device=DEV)
        self.dout_was = self.dout.f64().clone()
        room = B.dbspmspv_join_workspace(self.opts, self.t, n)
        ws = torch.full((room + 64,), 0xAB, dtype=torch.uint8, device=DEV) if workspace is None else workspace
        q = self.res.get
        dg = q("dgate")
        B.dbspmspv_join_backward(self.opts, self.t, n, *at(self.out), *at(self.b), self.kept, self.wb, self.cb, g.start if isinstance(g, Rows) else g, g.ld if isinstance(g, Rows) else 0, self.wn,
                                 self.random, *at(self.dh if dh else None), *at(self.dout if dout else None), *at(q("dr")), *at(q("db")), q("dw_block"), q("dc_block"),
                                 dg.start if isinstance(dg, Rows) else dg, dg.ld if isinstance(dg, Rows) else 0, q("dw_next"), q("dc_next"), ws, room, stream)
        if workspace is None:
            assert bool((ws[room:] == 0xAB).all())
        self.used = dh, dout

    def want_back(self):
        use_dh, use_dout = self.used
        zero = torch.zeros((self.t, self.n), dtype=torch.float64, device=DEV)
        dh, dout = self.dh.f64() if use_dh else zero, self.dout_was if use_dout else zero
        k = self.kept.double()
        out = self.out.f64()
        xh, X = (out - k[:, 2:3]) * k[:, 3:4], (out.abs() + k[:, 2:3].abs()) * k[:, 3:4]

        def back(u, eu, xh, X, inv, norm):
            if norm == "none":
                return u, eu
            m = mean(u) if norm == "layer" else 0.0
            d = inv * (u - m - xh * mean(u * xh))
            e = inv * (eu + mean(eu) + X * mean(eu * X) + MANY * (u.abs() + mean(u.abs()) + X * mean(u.abs() * X)))
            return d, e

        u = dh * self.wnd
        d, e = back(u, E * u.abs(), xh, X, k[:, 3:4], self.next)
        G, eG = dout + d, e + E * (dout.abs() + d.abs())
        w = {"dr": (G, eG)}
        total = lambda v, ev, size: (v.sum(dim=0), ev.sum(dim=0) + (self.t + 64) * E * size.sum(dim=0))
        w["dw_next"], w["dc_next"] = total(dh * xh, 4 * E * dh.abs() * X, dh.abs() * X), total(dh, 0 * dh, dh.abs())
        q, eq = self.scale * self.mask * G, abs(self.scale) * self.mask * (eG + 4 * E * G.abs())
        b = self.b.f64() if self.b is not None else zero
        bh, BX = (b - k[:, 0:1]) * k[:, 1:2], (b.abs() + k[:, 0:1].abs()) * k[:, 1:2]
        g = self.gd
        dp, edp = q * g, (eq + 2 * E * q.abs()) * g.abs()
        w["dw_block"] = total(dp * bh, edp * BX + 4 * E * dp.abs() * BX, dp.abs() * BX)
        w["dc_block"] = total(dp, edp, dp.abs())
        P, PS = bh * self.wbd + self.cbd, BX * self.wbd.abs() + self.cbd.abs()
        dg, edg = q * P, eq * PS + 8 * E * q.abs() * PS
        w["dgate"] = (dg, edg) if isinstance(self.gate, Rows) else total(dg, edg, q.abs() * PS)
        w["db"] = back(dp * self.wbd, (edp + 2 * E * dp.abs()) * self.wbd.abs(), bh, BX, k[:, 1:2], self.block)
        return w

    def check_back(self):
        w = self.want_back()
        for name, got in self.res.items():
            want, err = w[name]
            if isinstance(got, Rows):
                step = HALF if got.buf.dtype == torch.bfloat16 else E
                near(got.v, want, err + step * (want.abs() + err) + 1e-30)
                assert got.untouched()
            else:
                near(got[:-1], want, err + 2 * E * want.abs() + 1e-30)
                assert float(got[-1]) == 77.0


def at(rows):
    return (None, 0) if rows is None else (rows.start, rows.ld)


# ---- log probabilities ---------------------------------------------------------------------------
def order(logits):
    """Places of the logits, largest first, NaN before everything, equal ones by their index."""
    l = torch.where(torch.isnan(logits), torch.inf, logits.double())
    first = torch.isnan(logits).to(torch.int8)
    by_value = torch.sort(l, dim=1, descending=True, stable=True).indices
    return by_value.gather(1, torch.sort(first.gather(1, by_value), dim=1, descending=True, stable=True).indices)


class Logprobs:
    def __init__(self, values, top=0, temperature=1.0, targets=None, pad=0, lead=0, f32=True):
        t, v = values.shape
        self.t, self.vocab, self.top, self.temperature, self.f32 = t, v, top, temperature, f32
        self.logits = Rows(t, v, pad, lead, values.to(TYPE[f32]), TYPE[f32])
        self.pad, self.lead = pad, lead
        self.targets = targets if targets is not None else torch.from_numpy(np.random.default_rng(t + v).integers(0, v, t)).to(DEV).to(torch.int32)

    def forward(self, logprob=True, entropy=True, stats=True, stream=None):
        full = lambda on, *shape: torch.full(shape, 77.0, device=DEV) if on else None
        self.logprob, self.entropy, self.stats = full(logprob, self.t + 1), full(entropy, self.t + 1), full(stats, self.t + 1, 2)
        self.ids = torch.full((self.t * self.top + 1,), 77, dtype=torch.int32, device=DEV) if self.top else None
        self.lps = full(self.top > 0, self.t * self.top + 1)
        B.dbspmspv_logprobs(*at(self.logits), int(self.f32), self.t, self.vocab, self.temperature, self.targets, self.logprob, self.entropy, self.stats, self.top, self.ids, self.lps, stream)

    def want(self):
        l = self.logits.f64()
        M = l.amax(dim=1, keepdim=True)
        nothing = M == -math.inf
        x = torch.where(nothing, -math.inf, (l - torch.where(nothing, 0.0, M)) / float(np.float32(self.temperature)))
        total = torch.logsumexp(x, dim=1, keepdim=True)
        logp = torch.where(nothing, -math.inf, x - total)
        p = torch.where(nothing, 0.0, logp.exp())
        spread = (p * torch.where(p > 0, x, 0.0).abs()).sum(dim=1)
        err = (self.vocab / 2048 + 40) * 2.0 ** -22 + 6 * E * spread
        H = torch.special.entr(p).sum(dim=1)
        return {"M": M[:, 0], "total": total[:, 0], "logp": logp, "p": p, "H": H, "err": err, "eH": err * (2 + 2 * spread) + 8 * E * (total[:, 0].abs().clamp(max=1e30) + spread), "x": x}

    def check(self):
        w = self.want()
        eq = lambda a, b: bool(((a == b) | (torch.isnan(a) & torch.isnan(b))).all())
        fine = torch.isfinite(w["total"])

        def close(got, want, bound):
            got = got.double()
            # (the outputs are fp32: what is past its largest number, a masked logit over a small temperature, is an infinity there)
            want = torch.where(want.abs() > torch.finfo(torch.float32).max, torch.sign(want) * math.inf, want)
            ok = torch.isfinite(want)
            assert eq(torch.where(ok, 0.0, got), torch.where(ok, 0.0, want))
            near(torch.where(ok, got, 0.0), torch.where(ok, want, 0.0), torch.where(ok, bound, 0.0) + 1e-30)

        t = self.t
        if self.logprob is not None:
            at_ = self.targets.long().clamp(0, self.vocab - 1)[:, None]
            lp = w["logp"].gather(1, at_)[:, 0]
            bound = w["err"] + 8 * E * (w["x"].gather(1, at_)[:, 0].abs() + w["total"].abs())
            lp = torch.where(self.targets < 0, 0.0, torch.where(self.targets >= self.vocab, math.nan, lp))
            close(self.logprob[:t], lp, torch.where(torch.isfinite(bound), bound, 0.0))
            assert float(self.logprob[t]) == 77.0
        if self.entropy is not None:
            close(self.entropy[:t], w["H"], torch.where(fine, w["eH"], 0.0))
            assert float(self.entropy[t]) == 77.0
        if self.stats is not None:
            assert eq(self.stats[:t, 0].double(), w["M"])
            close(self.stats[:t, 1], w["total"], torch.where(fine, w["err"] + 4 * E * w["total"].abs(), 0.0))
            assert bool((self.stats[t] == 77.0).all())
        if self.top:
            ids = order(self.logits.v)[:, :self.top]
            assert bool((self.ids[:-1].reshape(t, self.top).long() == ids).all())
            lp = w["logp"].gather(1, ids)
            bound = w["err"][:, None] + 8 * E * (w["x"].gather(1, ids).abs() + w["total"].abs()[:, None])
            close(self.lps[:-1].reshape(t, self.top), lp, torch.where(torch.isfinite(bound), bound, 0.0))
            assert int(self.ids[-1]) == 77 and float(self.lps[-1]) == 77.0

    def backward(self, dlogprob=None, dentropy=None, dtop=None, ids=None, out32=None, in_place=False, stream=None):
        w = self.want()
        self.kept = torch.stack([w["M"], w["total"]], dim=1).float().contiguous()
        self.H = w["H"].float()
        self.d = dlogprob, dentropy, dtop, ids
        self.was = self.logits.f64().clone()
        out32 = self.f32 if out32 is None else out32
        self.dl = self.logits if in_place else Rows(self.t, self.vocab, self.pad, self.lead, None, TYPE[out32])
        B.dbspmspv_logprobs_backward(*at(self.logits), int(self.f32), self.t, self.vocab, self.temperature, self.targets, self.kept, self.H if dentropy is not None else None,
                                     self.top if dtop is not None else 0, ids, dlogprob, dentropy, dtop, *at(self.dl), int(out32), stream)

    def check_back(self):
        dlogprob, dentropy, dtop, ids = self.d
        T = float(np.float32(self.temperature))
        k, H = self.kept.double(), self.H.double()[:, None]
        nothing = k[:, :1] == -math.inf
        x = (self.was - torch.where(nothing, 0.0, k[:, :1])) / T
        logp = torch.where(nothing, -math.inf, x - k[:, 1:])
        p = torch.exp(logp)
        own, size = torch.zeros_like(p), torch.zeros_like(p)
        rows = torch.arange(self.t, device=DEV)
        if dlogprob is not None:
            has = (self.targets >= 0) & (self.targets < self.vocab)
            own.index_put_((rows[has], self.targets[has].long()), dlogprob[has].double(), accumulate=True)
        if dtop is not None:
            for j in range(self.top):
                has = (ids[:, j] >= 0) & (ids[:, j] < self.vocab)
                own.index_put_((rows[has], ids[has, j].long()), dtop[has, j].double(), accumulate=True)
                size.index_put_((rows[has], ids[has, j].long()), dtop[has, j].double().abs(), accumulate=True)
        size = size + own.abs()
        S, SA = own.sum(dim=1, keepdim=True), size.sum(dim=1, keepdim=True)
        dH = torch.zeros((self.t, 1), dtype=torch.float64, device=DEV) if dentropy is None else dentropy.double()[:, None]
        lp0 = torch.where(p > 0, logp, 0.0)
        want = (own - p * (S + dH * (lp0 + H))) / T
        ax = torch.where(p > 0, x.abs() + k[:, 1:].abs(), 0.0)
        bound = (size * 80 * E + p * (2.0 ** -21 + 8 * E * ax) * (SA + dH.abs() * (lp0.abs() + H)) + p * (80 * E * SA + 8 * E * dH.abs() * (ax + H))) / T
        # (the exponent is taken from a reference that is M log2(e) / T rounded, off by E |M| log2(e) / T at most; what makes up for that is itself rounded: E times as much again.  It shows where
        # all else is 0: the only logit left)
        ref = torch.where(nothing, 0.0, k[:, :1]).abs() * 1.45 / T + k[:, 1:].abs() * 1.45
        bound = bound + torch.where(ref <= 4200, 8 * E * E * ref * p * (SA + dH.abs()) / T, 0.0)
        want, bound = torch.where(nothing, 0.0, want), torch.where(nothing, 0.0, bound)
        step = HALF if self.dl.buf.dtype == torch.bfloat16 else E
        near(self.dl.v, want, bound + step * (want.abs() + bound) + 1e-37)
        assert self.dl.untouched()
