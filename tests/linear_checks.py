"""One call of a linear or gated layer, or of their gradients, against the plain form in 64 bits."""
import torch

from paper_2608_16308_b200 import binding as B
from linear_util import ACT, DEV, HALF, Rows, gated_want, grads_want, linear_want, near, normal, room, slopes


def check_linear(layer, t, name="none", pad=0, lead=0, bias=False, residual=False, keep=False, f32=False, zeros=0.0, seed=1):
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


def check_gated(gate, up, t, name="silu", pad=0, lead=0, keep=False, zeros=0.0, seed=1):
    m, n = gate.m, gate.n
    x = Rows(t, n, pad, lead, normal((t, n), seed, zeros))
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


def check_backward(layers, t, name="none", pad=0, lead=0, want_dx=True, want_dw=True, seed=1):
    m, n = layers[0].m, layers[0].n
    x = Rows(t, n, pad, lead, normal((t, n), seed))
    z, u, dy = (Rows(t, m, pad, lead, normal((t, m), seed + 1 + k, scale=2.0 if k == 0 else 1.0)) for k in range(3))
    dx = Rows(t, n, pad, lead)
    dw = [torch.full((w.nnz + 1,), 77.0, dtype=torch.bfloat16, device=DEV) for w in layers]
    ask = [d if want_dw else None for d in dw]
    out = (dx.start if want_dx else None, dx.ld)
    if len(layers) == 1:
        ws, nb = room(layers[0], None, t, True)
        B.dbspmspv_linear_backward(layers[0].h, x.start, x.ld, t, ACT[name], z.start if name != "none" else None, z.ld, dy.start, dy.ld, *out, ask[0], None, ws, nb)
        d, e = slopes(dy.f64(), z.f64(), None, name)
    else:
        ws, nb = room(layers[0], layers[1], t, True)
        B.dbspmspv_gated_backward(layers[0].h, layers[1].h, x.start, x.ld, t, ACT[name], z.start, u.start, z.ld, dy.start, dy.ld, *out, ask[0], ask[1], ws, nb)
        d, e = slopes(dy.f64(), z.f64(), u.f64(), name)
    torch.cuda.synchronize()
    wx, bx, ww, bw = grads_want(layers, x.f64(), d, e)
    if want_dx:
        near(dx.v, wx, bx + HALF * (wx.abs() + bx))
    if want_dw:
        for k in range(len(layers)):
            near(dw[k][:-1], ww[k], bw[k] + HALF * (ww[k].abs() + bw[k]))
    assert dx.untouched() and all(float(v[-1]) == 77.0 for v in dw)
