"""Layers, plain forms in 64 bits and error bounds for the tests of dbspmspv_linear, dbspmspv_gated and their gradients."""
import math

import numpy as np
import torch

from paper_2608_16308_b200 import binding as B
from paper_2608_16308_b200 import workloads as wl

DEV = "cuda:0"
ACT = {"none": B.ACT_NONE, "relu": B.ACT_RELU, "silu": B.ACT_SILU, "gelu": B.ACT_GELU}
HALF = 2.0 ** -8        # a rounding to bf16, relative to the value
SUM = 2e-5              # fp32 sums, relative to the sum of the magnitudes (the library's bound for its products)
FUN = 1e-5              # exp, erf, the divide and the few roundings around them in fp32, relative to |z| + 1


def act(z, name):
    return {"none": lambda: z, "relu": lambda: torch.relu(z), "silu": lambda: z * torch.sigmoid(z),
            "gelu": lambda: z * 0.5 * (1 + torch.erf(z / math.sqrt(2)))}[name]()


def slope(z, name):
    s = torch.sigmoid(z)
    return {"none": lambda: torch.ones_like(z), "relu": lambda: (z > 0).double(), "silu": lambda: s + z * s * (1 - s),
            "gelu": lambda: 0.5 * (1 + torch.erf(z / math.sqrt(2))) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)}[name]()


class Layer:
    """A pruned layer: its handle, the dense matrix in 64 bits, the stored places row by row.  Row 0 and column 0 are empty where the layer is
    large enough; the first stored values are -0 and 0."""

    def __init__(self, m, n, keep=0.5, seed=0, linear=1, scale=None):
        rng = np.random.default_rng(seed)
        w = rng.standard_normal((m, n)) * (scale or 1.0 / math.sqrt(max(1.0, n * keep)))
        mask = rng.random((m, n)) < keep
        if m > 4 and n > 4:
            mask[0, :] = False
            mask[:, 0] = False
        w = np.where(mask, wl.bf16_bits_to_f32(wl.f32_to_bf16_bits(w.astype(np.float32))), np.float32(0.0)).astype(np.float32)
        rows, cols = np.nonzero(mask)
        vals = w[rows, cols].copy()
        if vals.size > 4:
            vals[:2] = (-0.0, 0.0)
            w[rows[:2], cols[:2]] = 0.0
        ptr = np.zeros(m + 1, np.int64)
        np.cumsum(mask.sum(axis=1), out=ptr[1:])
        self.m, self.n, self.nnz = m, n, vals.size
        self.dense = torch.from_numpy(w.astype(np.float64)).to(DEV)
        self.at = torch.from_numpy(np.flatnonzero(mask)).to(DEV)
        opts = B.default_create_opts()
        opts.linear = linear
        up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
        self.h = B.dbspmspv_create_csr(m, n, self.nnz, up(ptr), up(cols.astype(np.int32)), up(wl.f32_to_bf16_bits(vals).view(np.int16)), B.BF16, 16, opts)

    def close(self):
        if self.h:
            h, self.h = self.h, None
            B.dbspmspv_get_stats(h)              # (raises if a wait ran out)
            B.dbspmspv_destroy(h)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Rows:
    """tokens x width in a buffer whose rows are `pad` entries longer and which begins `lead` entries late; the rest holds a marker."""

    def __init__(self, t, width, pad=0, lead=0, values=None, dtype=torch.bfloat16, mark=77.0):
        self.ld = width + pad
        self.buf = torch.full((lead + t * self.ld + 8,), mark, dtype=dtype, device=DEV)
        self.v = self.buf[lead:lead + t * self.ld].reshape(t, self.ld)[:, :width] if t else self.buf[:0].reshape(0, width)
        self.start = self.buf[lead:]
        if values is not None:
            self.v.copy_(values)
        self.inside = torch.zeros_like(self.buf, dtype=torch.bool)
        if t:
            self.inside[lead:lead + t * self.ld].reshape(t, self.ld)[:, :width] = True
        self.mark = mark

    def f64(self):
        return self.v.double()

    def untouched(self):
        return bool((self.buf[~self.inside] == self.mark).all())


def normal(shape, seed, zeros=0.0, scale=1.0):
    rng = np.random.default_rng(seed)
    v = rng.standard_normal(shape) * scale * (rng.random(shape) >= zeros)
    return torch.from_numpy(v.astype(np.float32)).to(DEV).to(torch.bfloat16)


def room(layer, up, tokens, backward):
    b = B.dbspmspv_linear_workspace(layer.h, up.h if up is not None else None, tokens, backward)
    return torch.full((b,), 0xAB, dtype=torch.uint8, device=DEV), b


def near(got, want, bound):
    got, want, bound = got.double(), want.double(), bound.double()
    bad = ~((got - want).abs() <= bound)
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} out of bounds, worst {float(((got - want).abs() / bound.clamp(min=1e-300))[bad].max()):.3g} times"


def linear_want(layer, x, bias, name, residual):
    """y, z and the bounds of their errors"""
    z = x @ layer.dense.T
    dz = SUM * (x.abs() @ layer.dense.abs().T)
    if bias is not None:
        z = z + bias.double()
        dz = dz + SUM * bias.double().abs()
    y = act(z, name)
    dy = 1.2 * dz + FUN * (z.abs() + 1) * (name not in ("none", "relu"))        # (the activations' slopes stay under 1.13)
    if residual is not None:
        y = y + residual
        dy = dy + 2.0 ** -23 * (y.abs() + residual.abs())
    return y, dy, z, dz


def gated_want(gate, up, x, name):
    a, da, g, dg = linear_want(gate, x, None, name, None)
    u = x @ up.dense.T
    du = SUM * (x.abs() @ up.dense.abs().T)
    return a * u, da * u.abs() + a.abs() * du + da * du + 2.0 ** -23 * (a * u).abs(), g, dg, u, du


def slopes(dy, z, u, name):
    """what the products of a gradient take, with the bound of its error: rounded to bf16 once"""
    if u is None:
        d = [dy * slope(z, name)]
        scale = [dy.abs()]
    else:
        d = [dy * u * slope(z, name), dy * act(z, name)]
        scale = [(dy * u).abs(), dy.abs()]
    exact = u is None and name in ("none", "relu")
    return d, [torch.zeros_like(v) if exact else HALF * v.abs() + FUN * s * (z.abs() + 1) for v, s in zip(d, scale)]


def grads_want(layers, x, d, e):
    dx = sum(v @ w.dense for v, w in zip(d, layers))
    bx = sum((q + SUM * v.abs()) @ w.dense.abs() for v, q, w in zip(d, e, layers))
    dw = [(v.T @ x).reshape(-1)[w.at] for v, w in zip(d, layers)]
    bw = [((q + SUM * v.abs()).T @ x.abs()).reshape(-1)[w.at] for v, q, w in zip(d, e, layers)]
    return dx, bx, dw, bw
