"""The activations of linear and gated layers and their slopes, for every finite bf16 value in front of them: relative to the result, down to the
smallest normal number.

A layer of one column whose weights are those values hands each of them to the activation exactly (x = 1); its gradients with dy = x = 1 are the slopes,
in bf16 as dw and unrounded as dbias.

Bounds, in units of 2^-23 relative to the result, from the error bounds that CUDA states for its functions:
  GELU    z Phi(z) by erfc (3): its argument is off by 1 (a constant and a product, half each), which erfc magnifies by at most z^2 + 1; two products: z^2 + 5
  SiLU    z / (1 + exp(-z)) by exp of -|z| (2 + 1.173 |z|), a sum, a divide (2) and products: 1.2 |z| + 8
  slopes  sums of two terms, relative to the sum of their magnitudes: GELU Phi(z), as above, and z phi(z), 2 + 1.173 z^2 / 2 and three roundings: z^2 + 7;
          SiLU p (1 + z (1 - p)): 1.2 |z| + 12
Below the smallest normal number nothing is promised."""
import math

import numpy as np
import pytest
import torch

from paper_2608_16308_b200 import binding as B
from paper_2608_16308_b200 import workloads as wl
from linear_util import ACT, DEV, HALF, near

pytestmark = pytest.mark.gpu
ULP, TINY = 2.0 ** -23, 2.0 ** -126


@pytest.fixture(scope="module")
def column():
    """handle of the layer, its weights as bf16 and in 64 bits"""
    vals = wl.bf16_bits_to_f32(np.arange(65536, dtype=np.uint16))
    vals = vals[np.isfinite(vals)]
    m = len(vals)
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    o = B.default_create_opts()
    o.linear = 1
    h = B.dbspmspv_create_csr(m, 1, m, up(np.arange(m + 1, dtype=np.int64)), up(np.zeros(m, np.int32)), up(wl.f32_to_bf16_bits(vals).view(np.int16)), B.BF16, 16, o)
    z = up(vals)
    yield h, m, z.to(torch.bfloat16), z.double()
    B.dbspmspv_destroy(h)


def phi(z):
    return 0.5 * torch.special.erfc(-z / math.sqrt(2))             # (torch's ndtr is 1 + erf, which cancels on the left in 64 bits too)


def act(z, name):
    """value and error of its fp32 form"""
    if name == "gelu":
        v = z * phi(z)
        return v, v.abs() * ULP * (z * z).clamp(max=400) + 5 * ULP * v.abs() + TINY            # (under -20 the result is below the smallest number)
    if name == "silu":
        v = z * torch.sigmoid(z)
        return v, v.abs() * ULP * (1.2 * z.abs().clamp(max=200) + 8) + TINY
    return {"none": z, "relu": z.clamp(min=0)}[name], torch.zeros_like(z)


def slope(z, name):
    if name == "gelu":
        a, b = phi(z), z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        return a + b, (a + b.abs()) * ULP * ((z * z).clamp(max=400) + 7) + TINY
    if name == "silu":
        p, q = torch.sigmoid(z), torch.sigmoid(-z)
        return p * (1 + z * q), p * (1 + z.abs() * q) * ULP * (1.2 * z.abs().clamp(max=200) + 12) + TINY
    return {"none": torch.ones_like(z), "relu": (z > 0).double()}[name], torch.zeros_like(z)


def rounded(want, err):
    return err + HALF * (want.abs() + err)


@pytest.mark.parametrize("t", [1, 17])
@pytest.mark.parametrize("name", ["none", "relu", "silu", "gelu"])
def test_values(column, name, t):
    """over the column and on the tensor cores, in bf16 and in fp32, as a layer and as a gate"""
    h, m, zb, z = column
    x = torch.zeros((t, 8), dtype=torch.bfloat16, device=DEV)
    x[:, 0] = 1
    y, g, u = (torch.empty((t, m), dtype=torch.bfloat16, device=DEV) for _ in range(3))
    y32 = torch.empty((t, m), device=DEV)
    B.dbspmspv_linear(h, x, 8, t, None, ACT[name], None, 0, y, m, 0, None, 0, None, 0)
    B.dbspmspv_linear(h, x, 8, t, None, ACT[name], None, 0, y32, m, 1, None, 0, None, 0)
    torch.cuda.synchronize()
    want, err = act(z, name)
    for k in (0, t - 1):
        near(y[k], want, rounded(want, err))
        near(y32[k], want, err)
    B.dbspmspv_gated(h, h, x, 8, t, ACT[name], y, m, g, u, m, None, 0)
    torch.cuda.synchronize()
    assert torch.equal(g[t - 1], zb) and torch.equal(u[0], zb)
    want, err = want * z, err * z.abs() + ULP * (want * z).abs()
    ok = (want.abs() + err < 1.7 * 2.0 ** 127)                     # (the square of a large value overflows)
    for k in (0, t - 1):
        near(y[k][ok], want[ok], rounded(want, err)[ok] + TINY)
        assert torch.isinf(y[k][want > 2.0 ** 128]).all()


@pytest.mark.parametrize("name", ["none", "relu", "silu", "gelu"])
def test_slopes(column, name):
    h, m, zb, z = column
    one = torch.ones(8, dtype=torch.bfloat16, device=DEV)
    ones, zeros = torch.ones(m, dtype=torch.bfloat16, device=DEV), torch.zeros(m, dtype=torch.bfloat16, device=DEV)
    dw, du = (torch.empty(m, dtype=torch.bfloat16, device=DEV) for _ in range(2))
    db = torch.empty(m, device=DEV)
    nb = B.dbspmspv_linear_workspace(h, h, 1, True)
    ws = torch.empty(nb, dtype=torch.uint8, device=DEV)
    want, err = slope(z, name)
    B.dbspmspv_linear_backward(h, one, 8, 1, ACT[name], zb, m, ones, m, None, 0, dw, None, ws, nb)
    torch.cuda.synchronize()
    near(dw, want, rounded(want, err))
    dw.fill_(9.0)
    B.dbspmspv_linear_backward(h, one, 8, 1, ACT[name], zb, m, ones, m, None, 0, dw, db, ws, nb)
    torch.cuda.synchronize()
    near(dw, want, rounded(want, err))
    near(db, want, err)
    B.dbspmspv_gated_backward(h, h, one, 8, 1, ACT[name], zb, ones, m, ones, m, None, 0, dw, du, ws, nb)
    torch.cuda.synchronize()
    near(dw, want, rounded(want, err))
    want, err = act(z, name)
    near(du, want, rounded(want, err))
    B.dbspmspv_gated_backward(h, h, one, 8, 1, ACT[name], zb, zeros, m, ones, m, None, 0, dw, du, ws, nb)
    torch.cuda.synchronize()
    assert not dw.any()
    near(du, want, rounded(want, err))


@pytest.mark.parametrize("t", [1, 17])
def test_infinities(t):
    """An infinite entry in front of an activation: what the formula gives in arithmetic with infinities."""
    w = np.array([1.0, -1.0, 0.5, -2.0], np.float32)
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    o = B.default_create_opts()
    o.linear = 1
    h = B.dbspmspv_create_csr(4, 1, 4, up(np.arange(5, dtype=np.int64)), up(np.zeros(4, np.int32)), up(wl.f32_to_bf16_bits(w).view(np.int16)), B.BF16, 16, o)
    nan, inf = float("nan"), float("inf")
    want = {"none": (inf, -inf), "relu": (inf, 0.0), "silu": (inf, nan), "gelu": (inf, nan)}
    for name, (pos, neg) in want.items():
        x = torch.full((t, 8), inf, dtype=torch.bfloat16, device=DEV)
        y = torch.empty((t, 4), device=DEV)
        B.dbspmspv_linear(h, x, 8, t, None, ACT[name], None, 0, y, 4, 1, None, 0, None, 0)
        torch.cuda.synchronize()
        assert torch.equal(torch.nan_to_num(y, 5.0, 7.0, -7.0), torch.nan_to_num(torch.tensor([[pos, neg, pos, neg]] * t, device=DEV), 5.0, 7.0, -7.0))
        x.fill_(nan)
        B.dbspmspv_linear(h, x, 8, t, None, ACT[name], None, 0, y, 4, 1, None, 0, None, 0)
        torch.cuda.synchronize()
        assert torch.isnan(y).all()
    B.dbspmspv_destroy(h)
