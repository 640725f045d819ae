"""dbspmspv_linear and dbspmspv_gated with their gradients, against plain forms in 64 bits: sizes off every tile, one token to
several tiles of them, strides and starts that TMA cannot address, every activation, empty rows and columns."""
import pytest
import torch

from paper_2608_16308_b200 import binding as B
from linear_util import ACT, DEV, HALF, SUM, Layer, Rows, gated_want, grads_want, linear_want, near, normal, room, slopes

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (64, 64), (65, 17), (200, 333), (1030, 130), (129, 2050), (520, 1032)]
TOKENS = [1, 2, 3, 17, 65, 250, 301]
# few tiles and many tokens, which clusters of two, four and eight share
LONG = [((1000, 1100), 1040), ((520, 640), 2100), ((300, 250), 2600)]
# enough tiles that two thread blocks work on each
PAIRS = [((2050, 1930), 1900)]
CASES = [(s, t) for s in SHAPES for t in TOKENS] + LONG + PAIRS


def run_linear(layer, t, name, pad, lead, bias, residual, keep, f32, zeros, seed):
    m, n = layer.m, layer.n
    x = Rows(t, n, pad, lead, normal((t, n), seed, zeros))
    b = normal((m,), seed + 1) if bias else None
    r = Rows(t, m, pad, lead, normal((t, m), seed + 2)) if residual else None
    y = Rows(t, m, pad, lead, dtype=torch.float32 if f32 else torch.bfloat16)
    z = Rows(t, m, pad, lead) if keep else None
    ws, nb = room(layer, None, t, False)
    B.dbspmspv_linear(layer.h, x.start, x.ld, t, b, ACT[name], r.start if r else None, r.ld if r else 0, y.start, y.ld, int(f32),
                      z.start if z else None, z.ld if z else 0, ws, nb)
    torch.cuda.synchronize()
    wy, ey, wz, ez = linear_want(layer, x.f64(), b, name, r.f64() if r else None)
    near(y.v, wy, ey + (2.0 ** -24 if f32 else HALF) * (wy.abs() + ey))
    assert y.untouched()
    if z:
        near(z.v, wz, ez + HALF * (wz.abs() + ez))
        assert z.untouched()


@pytest.mark.parametrize("shape,t", CASES, ids=str)
def test_linear(shape, t):
    layer = Layer(*shape, seed=t)
    for k, (name, pad, lead, bias, residual, keep, f32, zeros) in enumerate([
            ("none", 0, 0, False, False, False, False, 0.0), ("relu", 3, 1, True, True, True, True, 0.5), ("silu", 8, 0, True, False, False, True, 0.9),
            ("gelu", 1, 8, False, True, True, False, 0.0)]):
        run_linear(layer, t, name, pad, lead, bias, residual, keep, f32, zeros, 10 * k + t)
    layer.close()


@pytest.mark.parametrize("shape,t", CASES, ids=str)
def test_gated(shape, t):
    m, n = shape
    gate, up = Layer(m, n, 0.5, seed=1), Layer(m, n, 0.3, seed=2)
    for name, pad, lead, keep in (("silu", 0, 0, True), ("gelu", 3, 1, False), ("relu", 8, 8, True), ("none", 0, 3, False)):
        x = Rows(t, n, pad, lead, normal((t, n), t + pad, 0.3))
        y, g, u = Rows(t, m, pad, lead), Rows(t, m, pad, lead), Rows(t, m, pad, lead)
        ws, nb = room(gate, up, t, False)
        B.dbspmspv_gated(gate.h, up.h, x.start, x.ld, t, ACT[name], y.start, y.ld, g.start if keep else None, u.start if keep else None, g.ld, ws, nb)
        torch.cuda.synchronize()
        wy, ey, wg, eg, wu, eu = gated_want(gate, up, x.f64(), name)
        near(y.v, wy, ey + HALF * (wy.abs() + ey))
        assert y.untouched() and g.untouched() and u.untouched()
        if keep:
            near(g.v, wg, eg + HALF * (wg.abs() + eg))
            near(u.v, wu, eu + HALF * (wu.abs() + eu))
    gate.close(), up.close()


@pytest.mark.parametrize("shape,t", CASES, ids=str)
def test_linear_backward(shape, t):
    layer = Layer(*shape, seed=3)
    m, n = shape
    for name, pad, lead in (("none", 0, 0), ("none", 3, 1), ("relu", 8, 0), ("silu", 1, 3), ("gelu", 0, 8)):
        x = Rows(t, n, pad, lead, normal((t, n), t, 0.2))
        z = Rows(t, m, pad, lead, normal((t, m), t + 1, scale=2.0))
        dy = Rows(t, m, pad, lead, normal((t, m), t + 2))
        dx = Rows(t, n, pad, lead)
        dw = torch.full((layer.nnz + 1,), 77.0, dtype=torch.bfloat16, device=DEV)
        db = torch.full((m + 1,), 77.0, dtype=torch.float32, device=DEV)
        ws, nb = room(layer, None, t, True)
        B.dbspmspv_linear_backward(layer.h, x.start, x.ld, t, ACT[name], z.start if name != "none" else None, z.ld, dy.start, dy.ld, dx.start, dx.ld, dw, db, ws, nb)
        torch.cuda.synchronize()
        d, e = slopes(dy.f64(), z.f64(), None, name)
        wx, bx, (ww,), (bw,) = grads_want([layer], x.f64(), d, e)
        near(dx.v, wx, bx + HALF * (wx.abs() + bx))
        near(dw[:-1], ww, bw + HALF * (ww.abs() + bw))
        near(db[:-1], d[0].sum(dim=0), SUM * d[0].abs().sum(dim=0) + 1e-5 * (dy.f64().abs() * (z.f64().abs() + 1)).sum(dim=0))
        assert dx.untouched() and float(dw[-1]) == 77.0 and float(db[-1]) == 77.0
    layer.close()


@pytest.mark.parametrize("shape,t", CASES, ids=str)
def test_gated_backward(shape, t):
    m, n = shape
    gate, up = Layer(m, n, 0.5, seed=4), Layer(m, n, 0.3, seed=5)
    for name, pad, lead in (("silu", 0, 0), ("gelu", 3, 1), ("relu", 8, 8), ("none", 1, 0)):
        x = Rows(t, n, pad, lead, normal((t, n), t))
        g, u = Rows(t, m, pad, lead, normal((t, m), t + 1, scale=2.0)), Rows(t, m, pad, lead, normal((t, m), t + 2))
        dy = Rows(t, m, pad, lead, normal((t, m), t + 3))
        dx = Rows(t, n, pad, lead)
        dw = [torch.full((w.nnz + 1,), 77.0, dtype=torch.bfloat16, device=DEV) for w in (gate, up)]
        ws, nb = room(gate, up, t, True)
        B.dbspmspv_gated_backward(gate.h, up.h, x.start, x.ld, t, ACT[name], g.start, u.start, g.ld, dy.start, dy.ld, dx.start, dx.ld, dw[0], dw[1], ws, nb)
        torch.cuda.synchronize()
        d, e = slopes(dy.f64(), g.f64(), u.f64(), name)
        wx, bx, ww, bw = grads_want([gate, up], x.f64(), d, e)
        near(dx.v, wx, bx + HALF * (wx.abs() + bx))
        for k in range(2):
            near(dw[k][:-1], ww[k], bw[k] + HALF * (ww[k].abs() + bw[k]))
            assert float(dw[k][-1]) == 77.0
        assert dx.untouched()
    gate.close(), up.close()
