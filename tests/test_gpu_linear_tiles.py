"""Linear and gated layers with more tiles than the GPU has thread blocks for: a block takes three and more of them, so both of its accumulators
are written again behind their first tile.  Against plain forms in 64 bits, over pairs of thread blocks and single ones."""
import pytest
import torch

from paper_2608_16308_b200 import binding as B
from linear_util import ACT, DEV, HALF, SUM, Layer, Rows, gated_want, grads_want, linear_want, near, normal, room, slopes

pytestmark = pytest.mark.gpu


def check_linear(layer, t, name="none", pad=0, lead=0, bias=False, residual=False, keep=False, f32=False, seed=1):
    m, n = layer.m, layer.n
    x = Rows(t, n, pad, lead, normal((t, n), seed))
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


# 16 x 11 tiles of 256 x 256 for 74 pairs; with rows off 16 bytes 32 x 42 of 128 x 64 for 296 blocks
@pytest.mark.parametrize("n", [130, 700])
@pytest.mark.parametrize("pad,lead", [(0, 0), (3, 1)])
def test_linear(n, pad, lead):
    layer = Layer(4090, n, seed=1)
    check_linear(layer, 2650, "relu", pad, lead, bias=True, residual=True, keep=True)
    check_linear(layer, 2650, "none", pad, lead, f32=True)
    layer.close()


@pytest.mark.parametrize("n", [130, 700])
@pytest.mark.parametrize("pad,lead", [(0, 0), (3, 1)])
def test_gated(n, pad, lead):
    gate, up = Layer(2500, n, 0.5, seed=1), Layer(2500, n, 0.3, seed=2)
    check_gated(gate, up, 2300, "silu", pad, lead, keep=True)
    check_gated(gate, up, 2300, "gelu", pad, lead)
    gate.close(), up.close()


@pytest.mark.parametrize("m", [130, 700])
def test_gradient_of_x(m):
    gate, up = Layer(m, 4090, 0.5, seed=1), Layer(m, 4090, 0.3, seed=2)
    check_backward([gate], 2650, "relu", want_dw=False)
    check_backward([gate, up], 2650, "silu", 3, 1, want_dw=False)
    gate.close(), up.close()


# 13 x 13 tiles of one layer, 338 of two
@pytest.mark.parametrize("t", [20, 65, 300])
def test_gradient_of_weights(t):
    gate, up = Layer(3250, 3130, 0.5, seed=1), Layer(3250, 3130, 0.3, seed=2)
    check_backward([gate], t, want_dx=False)
    check_backward([gate, up], t, "silu", want_dx=False)
    gate.close(), up.close()


def test_a_million_tokens_of_one_sign():
    """The gradient of weights over a million tokens whose terms are all positive: an accumulator cuts off up to 2^-23 of itself per step of 16 terms,
    which 131,072 terms make 8192 * 2^-23 at most, and one rounding to bf16."""
    m, n, t = 1800, 1160, 1 << 20
    layer = Layer(m, n, 0.05, seed=1)
    gen = torch.Generator(device=DEV).manual_seed(1)
    x, dy = (torch.empty((t, w), dtype=torch.bfloat16, device=DEV).uniform_(0.5, 1.5, generator=gen) for w in (n, m))
    dw = torch.full((layer.nnz + 1,), 77.0, dtype=torch.bfloat16, device=DEV)
    B.dbspmspv_linear_backward(layer.h, x, n, t, B.ACT_NONE, None, 0, dy, m, None, 0, dw, None, None, 0)
    rows = 8
    want = sum(dy[k:k + 16384, -rows:].double().T @ x[k:k + 16384].double() for k in range(0, t, 16384))
    torch.cuda.synchronize()
    last = layer.at >= (m - rows) * n
    want = want.reshape(-1)[layer.at[last] - (m - rows) * n]
    near(dw[:-1][last], want, (HALF + 8192 * 2.0 ** -23) * want)
    assert int(last.sum()) > 100 and float(dw[-1]) == 77.0
    layer.close()
