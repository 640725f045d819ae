"""dbspmspv_linear and dbspmspv_gated as a program uses them: refusals, handles of every kind, a block chained forwards and backwards,
gradients against differences, captured and replayed calls, other streams, rows far apart, entries that are not finite."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2608_16308_b200 import binding as B
from paper_2608_16308_b200 import workloads as wl
from linear_util import ACT, DEV, HALF, SUM, Layer, Rows, act, gated_want, grads_want, linear_want, near, normal, room, slope, slopes

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def linear(layer, x, y, t=None, bias=None, name="none", residual=None, f32=0, z=None, ws=None, nb=0, stream=None):
    B.dbspmspv_linear(layer.h, x.start, x.ld, x.v.shape[0] if t is None else t, bias, ACT[name], residual.start if residual else None, residual.ld if residual else 0,
                      y.start, y.ld, f32, z.start if z else None, z.ld if z else 0, ws, nb, stream)


def check_linear(layer, t, seed):
    x, y = Rows(t, layer.n, 0, 0, normal((t, layer.n), seed)), Rows(t, layer.m)
    ws, nb = room(layer, None, t, False)
    linear(layer, x, y, ws=ws, nb=nb)
    torch.cuda.synchronize()
    wy, ey, _, _ = linear_want(layer, x.f64(), None, "none", None)
    near(y.v, wy, ey + HALF * (wy.abs() + ey))


def check_backward(layer, t, seed):
    x, dy, dx = Rows(t, layer.n, 0, 0, normal((t, layer.n), seed)), Rows(t, layer.m, 0, 0, normal((t, layer.m), seed + 1)), Rows(t, layer.n)
    dw = torch.full((layer.nnz + 1,), 77.0, dtype=torch.bfloat16, device=DEV)
    ws, nb = room(layer, None, t, True)
    B.dbspmspv_linear_backward(layer.h, x.start, x.ld, t, B.ACT_NONE, None, 0, dy.start, dy.ld, dx.start, dx.ld, dw, None, ws, nb)
    torch.cuda.synchronize()
    d, e = slopes(dy.f64(), dy.f64(), None, "none")
    wx, bx, (ww,), (bw,) = grads_want([layer], x.f64(), d, e)
    near(dx.v, wx, bx + HALF * (wx.abs() + bx))
    near(dw[:-1], ww, bw + HALF * (ww.abs() + bw))
    assert float(dw[-1]) == 77.0


@pytest.mark.parametrize("keep", [0.002, 0.05, 0.15, 0.3, 0.95, 1.0])
@pytest.mark.parametrize("t", [1, 5, 130])
def test_every_sparsity(keep, t):
    """From blocks without a payload to dense ones: the copy by columns does not depend on how the elements are stored."""
    layer = Layer(333, 270, keep, seed=7)
    check_linear(layer, t, 3)
    check_backward(layer, t, 5)
    layer.close()


@pytest.mark.parametrize("m,n", [(3, 30000), (70, 70001), (1, 513), (513, 1), (64, 25601)])
@pytest.mark.parametrize("t", [1, 2, 20])
def test_narrow_and_wide(m, n, t):
    layer = Layer(m, n, 0.5, seed=8)
    check_linear(layer, t, 3)
    check_backward(layer, t, 5)
    layer.close()


def test_triples_in_any_order_with_duplicates():
    """dw follows the stored weights row by row, whatever order they were given in; duplicates are one weight."""
    rng = np.random.default_rng(3)
    m, n, k, t = 150, 90, 4000, 33
    row, col = rng.integers(0, m, k).astype(np.int32), rng.integers(0, n, k).astype(np.int32)
    val = (rng.integers(-3, 4, k) / 4).astype(np.float32)                # (sums of a few are exact in bf16)
    dense = np.zeros((m, n))
    np.add.at(dense, (row, col), val)
    mask = np.zeros((m, n), bool)
    mask[row, col] = True
    o = B.default_create_opts()
    o.linear = 1
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    layer = Layer.__new__(Layer)
    layer.m, layer.n, layer.nnz = m, n, int(mask.sum())
    layer.dense, layer.at = up(dense), up(np.flatnonzero(mask))
    layer.h = B.dbspmspv_create_coo(m, n, k, up(row), up(col), up(wl.f32_to_bf16_bits(val).view(np.int16)), B.BF16, 16, o)
    assert B.dbspmspv_get_stats(layer.h).nnz == layer.nnz
    check_linear(layer, t, 3)
    check_backward(layer, t, 5)
    layer.close()


def status(f, *args, **kw):
    with pytest.raises(B.DbSpmspvError) as e:
        f(*args, **kw)
    return e.value.status


def test_handles_that_do_not_serve():
    small, large = Layer(100, 64, linear=0), Layer(1040, 64, linear=0)      # (the large one is decoded by columns, so it has the copy)
    x, y, dx = Rows(4, 64, values=normal((4, 64), 1)), Rows(4, 1040), Rows(4, 64)
    assert status(linear, small, x, y) == B.ERR_UNSUPPORTED
    assert status(B.dbspmspv_linear_workspace, small.h, None, 4, False) == B.ERR_UNSUPPORTED
    check_linear(large, 3, 9)
    dw = torch.zeros(large.nnz, dtype=torch.bfloat16, device=DEV)
    ws, nb = room(large, None, 4, True)
    args = (large.h, x.start, x.ld, 4, B.ACT_NONE, None, 0, y.start, y.ld)
    B.dbspmspv_linear_backward(*args, dx.start, dx.ld, None, None, ws, nb)
    assert status(B.dbspmspv_linear_backward, *args, dx.start, dx.ld, dw, None, ws, nb) == B.ERR_UNSUPPORTED
    a = wl.random_sparse(64, 64, 500, 1)
    up = lambda v: torch.from_numpy(np.ascontiguousarray(v)).to(DEV)
    o = B.default_create_opts()
    f32 = B.dbspmspv_create_csr(64, 64, a.nnz, up(a.row_ptr), up(a.col_idx), up(a.val), B.F32)
    assert status(B.dbspmspv_linear, f32, x.start, x.ld, 4, None, 0, None, 0, y.start, y.ld, 0, None, 0, None, 0) == B.ERR_UNSUPPORTED
    B.dbspmspv_destroy(f32)
    o.linear = 1
    assert status(B.dbspmspv_create_csr, 64, 64, a.nnz, up(a.row_ptr), up(a.col_idx), up(a.val), B.F32, 16, o) == B.ERR_UNSUPPORTED
    bad = a.val.copy()
    bad[7] = np.inf
    bits = up(wl.f32_to_bf16_bits(bad).view(np.int16))
    assert status(B.dbspmspv_create_csr, 64, 64, a.nnz, up(a.row_ptr), up(a.col_idx), bits, B.BF16, 16, o) == B.ERR_UNSUPPORTED
    small.close(), large.close()


def test_refused_arguments():
    a, b, c = Layer(96, 72), Layer(96, 72), Layer(96, 80)
    t = 20
    x, y, z = Rows(t, 72, 8, values=normal((t, 72), 1)), Rows(t, 96), Rows(t, 96)
    ok = dict(h=a.h, x=x.start, ldx=x.ld, tokens=t, bias=None, act=0, residual=None, ldr=0, y=y.start, ldy=y.ld, y_f32=0, z=None, ldz=0, workspace=None, workspace_bytes=0)
    B.dbspmspv_linear(**ok)
    odd = torch.zeros(4096, dtype=torch.uint8, device=DEV)[1:]
    for change in (dict(x=None), dict(y=None), dict(tokens=-1), dict(act=4), dict(act=-1), dict(ldx=71), dict(ldy=95), dict(residual=z.start, ldr=95), dict(z=z.start, ldz=95),
                   dict(workspace_bytes=-1), dict(workspace=odd, workspace_bytes=1000), dict(y=odd), dict(y_f32=1, y=y.buf[1:]), dict(x=odd), dict(ldx=73),
                   dict(ldx=73, workspace=odd[15:], workspace_bytes=20 * 72 * 2 - 1), dict(h=None)):
        assert status(B.dbspmspv_linear, **{**ok, **change}) == B.ERR_INVALID_ARG, change
    g = dict(gate=a.h, up=b.h, x=x.start, ldx=x.ld, tokens=t, act=2, y=y.start, ldy=y.ld, g=None, u=None, ldgu=0, workspace=None, workspace_bytes=0)
    B.dbspmspv_gated(**g)
    for change in (dict(up=c.h), dict(up=None), dict(gate=None), dict(g=z.start, ldgu=90), dict(u=z.start, ldgu=90), dict(x=None), dict(act=9)):
        assert status(B.dbspmspv_gated, **{**g, **change}) == B.ERR_INVALID_ARG, change
    ws, nb = room(a, b, t, True)
    bw = dict(h=a.h, x=x.start, ldx=x.ld, tokens=t, act=1, z=z.start, ldz=z.ld, dy=y.start, lddy=y.ld, dx=Rows(t, 72).start, lddx=72, dw=None, dbias=None, workspace=ws, workspace_bytes=nb)
    B.dbspmspv_linear_backward(**bw)
    dw = torch.zeros(a.nnz, dtype=torch.bfloat16, device=DEV)
    for change in (dict(z=None), dict(dy=None), dict(dw=dw, x=None), dict(dw=dw, ldx=71), dict(ldz=95), dict(lddy=95), dict(lddx=71), dict(workspace=None), dict(workspace_bytes=100)):
        assert status(B.dbspmspv_linear_backward, **{**bw, **change}) == B.ERR_INVALID_ARG, change
    gb = dict(gate=a.h, up=b.h, x=x.start, ldx=x.ld, tokens=t, act=2, g=z.start, u=z.start, ldgu=z.ld, dy=y.start, lddy=y.ld, dx=Rows(t, 72).start, lddx=72, dw_gate=None, dw_up=None,
              workspace=ws, workspace_bytes=nb)
    B.dbspmspv_gated_backward(**gb)
    for change in (dict(u=None), dict(g=None), dict(up=c.h), dict(workspace_bytes=nb // 4), dict(ldgu=95)):
        assert status(B.dbspmspv_gated_backward, **{**gb, **change}) == B.ERR_INVALID_ARG, change
    torch.cuda.synchronize()
    a.close(), b.close(), c.close()


def test_no_tokens():
    a, b = Layer(96, 72), Layer(96, 72, 0.3, seed=2)
    B.dbspmspv_linear(a.h, None, 72, 0, None, 1, None, 0, None, 96, 0, None, 0, None, 0)
    B.dbspmspv_gated(a.h, b.h, None, 72, 0, 1, None, 96, None, None, 0, None, 0)
    dw = [torch.full((w.nnz + 1,), 5.0, dtype=torch.bfloat16, device=DEV) for w in (a, b)]
    db = torch.full((97,), 5.0, device=DEV)
    B.dbspmspv_linear_backward(a.h, None, 72, 0, 0, None, 0, None, 96, None, 0, dw[0], db, None, 0)
    torch.cuda.synchronize()
    assert not dw[0][:-1].any() and not db[:-1].any() and float(dw[0][-1]) == 5.0 and float(db[-1]) == 5.0
    dw[0].fill_(5.0)
    B.dbspmspv_gated_backward(a.h, b.h, None, 72, 0, 2, None, None, 96, None, 96, None, 0, dw[0], dw[1], None, 0)
    torch.cuda.synchronize()
    assert not dw[0][:-1].any() and not dw[1][:-1].any() and float(dw[0][-1]) == 5.0 and float(dw[1][-1]) == 5.0
    a.close(), b.close()


@pytest.mark.parametrize("wanted", [(0, 0, 0), (1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 0)])
def test_some_of_the_gradients(wanted):
    """What is not asked for is not computed, and what is does not change."""
    gate, up = Layer(200, 140, 0.5, seed=1), Layer(200, 140, 0.4, seed=2)
    t = 70
    x, g, u, dy = (Rows(t, w, values=normal((t, w), k)) for k, w in enumerate((140, 200, 200, 200)))
    ws, nb = room(gate, up, t, True)

    def call(ask):
        dx = Rows(t, 140)
        dw = [torch.full((w.nnz,), 9.0, dtype=torch.bfloat16, device=DEV) for w in (gate, up)]
        B.dbspmspv_gated_backward(gate.h, up.h, x.start, x.ld, t, B.ACT_SILU, g.start, u.start, g.ld, dy.start, dy.ld, dx.start if ask[0] else None, dx.ld,
                                  dw[0] if ask[1] else None, dw[1] if ask[2] else None, ws, nb)
        torch.cuda.synchronize()
        return dx.v.clone(), dw[0], dw[1]

    every, some = call((1, 1, 1)), call(wanted)
    for ask, p, q, mark in zip(wanted, every, some, (77.0, 9.0, 9.0)):
        assert torch.equal(q, p) if ask else bool((q == mark).all())
    gate.close(), up.close()


@pytest.mark.parametrize("t", [1, 3, 130])
def test_nothing_left_of_a_layer(t):
    """Every weight is pruned: sums are zeros, bias and residual remain, no gradient of weights is written."""
    layer, up = Layer(200, 140, 0.0, seed=1), Layer(200, 140, 0.5, seed=2)
    assert layer.nnz == 0
    x, r, y, z, dx = Rows(t, 140, values=normal((t, 140), 1)), Rows(t, 200, values=normal((t, 200), 2)), Rows(t, 200), Rows(t, 200), Rows(t, 140)
    bias = normal((200,), 3)
    ws, nb = room(layer, up, t, True)
    linear(layer, x, y, bias=bias, name="relu", residual=r, z=z, ws=ws, nb=nb)
    torch.cuda.synchronize()
    assert torch.equal(z.v, bias.expand(t, -1))
    near(y.v, torch.relu(bias.double()) + r.f64(), (HALF + 2.0 ** -23) * (torch.relu(bias.double()) + r.f64()).abs())      # (both terms exact, their sum rounded to fp32 and to bf16)
    dw = torch.full((8,), 9.0, dtype=torch.bfloat16, device=DEV)
    db = torch.full((200,), 9.0, device=DEV)
    B.dbspmspv_linear_backward(layer.h, x.start, x.ld, t, B.ACT_NONE, None, 0, r.start, r.ld, dx.start, dx.ld, dw, db, ws, nb)
    torch.cuda.synchronize()
    assert not dx.v.any() and bool((dw == 9.0).all())
    near(db, r.f64().sum(0), SUM * r.f64().abs().sum(0))
    B.dbspmspv_gated(layer.h, up.h, x.start, x.ld, t, B.ACT_SILU, y.start, y.ld, None, None, 0, ws, nb)
    torch.cuda.synchronize()
    assert not y.v.any()
    layer.close(), up.close()


@pytest.mark.parametrize("t", [1, 40, 300])
def test_one_handle_as_both_layers(t):
    """y = act(W x) * (W x), and its gradients: those of the two uses, which a program adds up."""
    w = Layer(264, 200, 0.5, seed=5)
    x, y, g, u = Rows(t, 200, values=normal((t, 200), 1)), Rows(t, 264), Rows(t, 264), Rows(t, 264)
    dy, dx = Rows(t, 264, values=normal((t, 264), 2)), Rows(t, 200)
    dw = [torch.zeros(w.nnz, dtype=torch.bfloat16, device=DEV) for _ in range(2)]
    ws, nb = room(w, w, t, True)
    B.dbspmspv_gated(w.h, w.h, x.start, x.ld, t, B.ACT_GELU, y.start, y.ld, g.start, u.start, g.ld, ws, nb)
    B.dbspmspv_gated_backward(w.h, w.h, x.start, x.ld, t, B.ACT_GELU, g.start, u.start, g.ld, dy.start, dy.ld, dx.start, dx.ld, dw[0], dw[1], ws, nb)
    torch.cuda.synchronize()
    wy, ey, wg, eg, wu, eu = gated_want(w, w, x.f64(), "gelu")
    near(y.v, wy, ey + HALF * (wy.abs() + ey))
    near(g.v, wg, eg + HALF * (wg.abs() + eg))
    assert torch.equal(g.v, u.v)
    d, e = slopes(dy.f64(), g.f64(), u.f64(), "gelu")
    wx, bx, ww, bw = grads_want([w, w], x.f64(), d, e)
    near(dx.v, wx, bx + HALF * (wx.abs() + bx))
    for a, b, c in zip(dw, ww, bw):
        near(a, b, c + HALF * (b.abs() + c))
    w.close()


def test_two_streams_at_once():
    """One handle, two streams, two workspaces: calls that overlap give what they give alone."""
    gate, up = Layer(1030, 777, 0.5, seed=1), Layer(1030, 777, 0.4, seed=2)
    t = 150
    x = [Rows(t, 777, values=normal((t, 777), k)) for k in range(2)]
    dy = [Rows(t, 1030, values=normal((t, 1030), 5 + k)) for k in range(2)]
    rooms = [room(gate, up, t, True) for _ in range(2)]

    def call(k, stream):
        y, g, u, dx = Rows(t, 1030), Rows(t, 1030), Rows(t, 1030), Rows(t, 777)
        dw = [torch.zeros(w.nnz, dtype=torch.bfloat16, device=DEV) for w in (gate, up)]
        torch.cuda.synchronize()
        ws, nb = rooms[k]

        def go():
            B.dbspmspv_gated(gate.h, up.h, x[k].start, x[k].ld, t, B.ACT_SILU, y.start, y.ld, g.start, u.start, g.ld, ws, nb, stream)
            B.dbspmspv_gated_backward(gate.h, up.h, x[k].start, x[k].ld, t, B.ACT_SILU, g.start, u.start, g.ld, dy[k].start, dy[k].ld, dx.start, dx.ld, dw[0], dw[1], ws, nb, stream)
        return go, (y.v, g.v, u.v, dx.v, dw[0], dw[1])

    alone = []
    for k in range(2):
        go, out = call(k, None)
        go()
        torch.cuda.synchronize()
        alone.append([v.clone() for v in out])
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(10):
        pair = [call(k, streams[k].cuda_stream) for k in range(2)]
        for _ in range(3):
            for go, _ in pair:
                go()
        torch.cuda.synchronize()
        for k in range(2):
            assert all(torch.equal(a, b) for a, b in zip(alone[k], pair[k][1]))
    gate.close(), up.close()


@pytest.mark.parametrize("t", [1, 7, 300])
def test_block_forwards_and_backwards(t):
    """norm's output -> gated block -> projection back onto the residual stream, then the gradients of all of it; the layers in
    between hand their bf16 results on.  In 64 bits from the same bf16 results in between, and once against differences."""
    m, n = 330, 136
    gate, up, down = Layer(m, n, 0.5, seed=1), Layer(m, n, 0.4, seed=2), Layer(n, m, 0.5, seed=3)
    x, res, dy = Rows(t, n, values=normal((t, n), 1)), Rows(t, n, values=normal((t, n), 2)), Rows(t, n, values=normal((t, n), 3))
    h, g, u, y = Rows(t, m), Rows(t, m), Rows(t, m), Rows(t, n)
    dh, dx = Rows(t, m), Rows(t, n)
    dwd = torch.empty(down.nnz, dtype=torch.bfloat16, device=DEV)
    dw = [torch.empty(w.nnz, dtype=torch.bfloat16, device=DEV) for w in (gate, up)]
    ws, nb = room(gate, up, t, True)
    ws2, nb2 = room(down, None, t, True)
    B.dbspmspv_gated(gate.h, up.h, x.start, x.ld, t, B.ACT_SILU, h.start, h.ld, g.start, u.start, g.ld, ws, nb)
    linear(down, h, y, residual=res, ws=ws2, nb=nb2)
    B.dbspmspv_linear_backward(down.h, h.start, h.ld, t, B.ACT_NONE, None, 0, dy.start, dy.ld, dh.start, dh.ld, dwd, None, ws2, nb2)
    B.dbspmspv_gated_backward(gate.h, up.h, x.start, x.ld, t, B.ACT_SILU, g.start, u.start, g.ld, dh.start, dh.ld, dx.start, dx.ld, dw[0], dw[1], ws, nb)
    torch.cuda.synchronize()
    wh, eh, _, _, _, _ = gated_want(gate, up, x.f64(), "silu")
    near(h.v, wh, eh + HALF * (wh.abs() + eh))
    wy, ey, _, _ = linear_want(down, h.f64(), None, "none", res.f64())
    near(y.v, wy, ey + HALF * (wy.abs() + ey))
    wx, bx, (ww,), (bw,) = grads_want([down], h.f64(), *slopes(dy.f64(), dy.f64(), None, "none"))
    near(dh.v, wx, bx + HALF * (wx.abs() + bx))
    near(dwd, ww, bw + HALF * (ww.abs() + bw))
    wx, bx, ww, bw = grads_want([gate, up], x.f64(), *slopes(dh.f64(), g.f64(), u.f64(), "silu"))
    near(dx.v, wx, bx + HALF * (wx.abs() + bx))
    for k in range(2):
        near(dw[k], ww[k], bw[k] + HALF * (ww[k].abs() + bw[k]))

    # differences of the whole block in 64 bits: loss = sum(dy * y); every intermediate result is off by its own roundings,
    # at most HALF of it: dg = dh u s(g) by those of dh, u and its own, and by s' (under 0.5) times g's; du = dh act(g) by those of dh and its own, and by act' (under
    # 1.1) times g's; dx and dw by one more.  6 HALF of the terms' magnitudes covers them and their products.
    def loss(xv, wg, wu, wd):
        return (dy.f64() * ((act(xv @ wg.T, "silu") * (xv @ wu.T)) @ wd.T + res.f64())).sum()

    xv, ws64 = x.f64(), [gate.dense, up.dense, down.dense]
    step = 1e-5

    def difference(k, i, j):
        parts = [xv] + ws64
        ends = []
        for sign in (1, -1):
            moved = parts[k].clone()
            moved[i, j] += sign * step
            ends.append(loss(*(moved if q == k else p for q, p in enumerate(parts))))
        return float((ends[0] - ends[1]) / (2 * step))

    gg, uu = xv @ gate.dense.T, xv @ up.dense.T
    dha = dy.f64().abs() @ down.dense.abs()
    dga, dua = dha * uu.abs() * (slope(gg, "silu").abs() + 0.5 * gg.abs()), dha * (act(gg, "silu").abs() + 1.1 * gg.abs())
    rng = np.random.default_rng(t)
    for _ in range(6):
        i, j = int(rng.integers(0, t)), int(rng.integers(0, n))
        b = float((dga[i] * gate.dense[:, j].abs() + dua[i] * up.dense[:, j].abs()).sum())
        assert abs(float(dx.v[i, j]) - difference(0, i, j)) <= 6 * HALF * b + 1e-6
        for k, (w, terms) in enumerate(((gate, dga), (up, dua))):
            p = int(rng.integers(0, w.nnz))
            r, c = divmod(int(w.at[p]), n)
            b = float((terms[:, r] * xv[:, c].abs()).sum())
            assert abs(float(dw[k][p]) - difference(1 + k, r, c)) <= 6 * HALF * b + 1e-6
    gate.close(), up.close(), down.close()


@pytest.mark.parametrize("t", [1, 4, 40, 300])
def test_same_bits_again_and_in_place(t):
    layer = Layer(520, 264, seed=4)
    x, r = Rows(t, 264, values=normal((t, 264), 1)), Rows(t, 520, values=normal((t, 520), 2))
    y, y2 = Rows(t, 520), Rows(t, 520, values=r.v)
    ws, nb = room(layer, None, t, False)
    linear(layer, x, y, name="gelu", residual=r, ws=ws, nb=nb)
    for _ in range(3):
        y3 = Rows(t, 520)
        linear(layer, x, y3, name="gelu", residual=r, ws=ws, nb=nb)
        assert torch.equal(y.v, y3.v)
    linear(layer, x, y2, name="gelu", residual=y2, ws=ws, nb=nb)           # the residual stream is updated where it lies
    assert torch.equal(y.v, y2.v)
    for pad in (1, 3):
        q = Rows(t, 520, pad, pad, values=r.v)
        linear(layer, x, q, name="gelu", residual=q, ws=ws, nb=nb)
        assert torch.equal(y.v, q.v) and q.untouched()
    layer.close()


@pytest.mark.parametrize("t", [1, 3, 130])
def test_entries_that_are_not_finite(t):
    """A token's infinite or NaN entry reaches every row of that token and no other token."""
    layer = Layer(300, 200, seed=5)
    for bad in (float("inf"), float("-inf"), float("nan")):
        x, y = Rows(t, 200, values=normal((t, 200), 1)), Rows(t, 300)
        x.v[t // 2, 77] = bad
        ws, nb = room(layer, None, t, False)
        linear(layer, x, y, ws=ws, nb=nb)
        torch.cuda.synchronize()
        want = x.f64() @ layer.dense.T
        assert not torch.isfinite(y.v[t // 2]).any()
        assert torch.equal(torch.isnan(want), torch.isnan(y.v)) and torch.equal(want[torch.isinf(want)], y.v.double()[torch.isinf(want)])
        good = torch.arange(t, device=DEV) != t // 2
        near(y.v[good], want[good], (SUM + 2 * HALF) * (x.f64()[good].abs() @ layer.dense.abs().T))
    layer.close()


def test_activations_far_out():
    """Every bf16 value in front of an activation: no overflow on the way to a finite result."""
    n = 64
    layer = Layer.__new__(Layer)
    o = B.default_create_opts()
    o.linear = 1
    up = lambda a: torch.from_numpy(np.ascontiguousarray(a)).to(DEV)
    ptr = np.arange(n + 1, dtype=np.int64)
    layer.h = B.dbspmspv_create_csr(n, n, n, up(ptr), up(np.arange(n, dtype=np.int32)), up(wl.f32_to_bf16_bits(np.ones(n, np.float32)).view(np.int16)), B.BF16, 16, o)
    layer.m = layer.n = n
    layer.dense = torch.eye(n, dtype=torch.float64, device=DEV)
    bits = np.arange(65536, dtype=np.uint16)
    vals = wl.bf16_bits_to_f32(bits)
    vals = vals[np.isfinite(vals)]
    vals = np.concatenate([vals, np.zeros(-len(vals) % n, np.float32)]).reshape(-1, n)
    t = vals.shape[0]
    x = Rows(t, n, values=torch.from_numpy(vals).to(DEV))
    for name in ("relu", "silu", "gelu"):
        y = Rows(t, n)
        linear(layer, x, y, name=name)
        one = Rows(1, n)
        torch.cuda.synchronize()
        want = act(x.f64(), name)
        # (exp underflows from -87 on, where the result is under 1e-35; 1 + erf is rounded next to 1, half of that times z)
        lost = 1e-35 + (2e-7 * x.f64().abs().clamp(max=8) if name == "gelu" else 0)
        near(y.v, want, 1.01 * HALF * want.abs() + lost)
        for k in (0, t // 2, t - 1):
            linear(layer, Rows(1, n, values=x.v[k:k + 1]), one, name=name)
            torch.cuda.synchronize()
            near(one.v, want[k:k + 1], 1.01 * HALF * want[k:k + 1].abs() + (lost if isinstance(lost, float) else lost[k:k + 1]))
    layer.close()


def test_captured_and_replayed():
    """A forward and backward pass in a CUDA graph, replayed on other inputs; two graphs with a workspace each."""
    gate, up = Layer(400, 210, 0.5, seed=1), Layer(400, 210, 0.5, seed=2)
    t, graphs = 90, []
    side = torch.cuda.Stream()
    for k in range(2):
        x, dy = Rows(t, 210, 1, values=normal((t, 210), k)), Rows(t, 400, values=normal((t, 400), 10 + k))
        y, g, u, dx = Rows(t, 400), Rows(t, 400), Rows(t, 400), Rows(t, 210)
        dw = [torch.empty(w.nnz, dtype=torch.bfloat16, device=DEV) for w in (gate, up)]
        ws, nb = room(gate, up, t, True)

        def both(x=x, dy=dy, y=y, g=g, u=u, dx=dx, dw=dw, ws=ws, nb=nb):
            B.dbspmspv_gated(gate.h, up.h, x.start, x.ld, t, B.ACT_SILU, y.start, y.ld, g.start, u.start, g.ld, ws, nb)
            B.dbspmspv_gated_backward(gate.h, up.h, x.start, x.ld, t, B.ACT_SILU, g.start, u.start, g.ld, dy.start, dy.ld, dx.start, dx.ld, dw[0], dw[1], ws, nb)

        with torch.cuda.stream(side):
            both()
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            both()
        graphs.append((graph, x, dy, y, g, u, dx, dw, both))
    for rnd in range(3):
        for k, (graph, x, dy, *_rest) in enumerate(graphs):
            x.v.copy_(normal((t, 210), 100 + 2 * rnd + k))
            dy.v.copy_(normal((t, 400), 200 + 2 * rnd + k))
        torch.cuda.synchronize()
        streams = [torch.cuda.Stream(), torch.cuda.Stream()]
        for s, (graph, *_rest) in zip(streams, graphs):                  # (side by side)
            with torch.cuda.stream(s):
                graph.replay()
        torch.cuda.synchronize()
        for graph, x, dy, y, g, u, dx, dw, both in graphs:
            got = [v.clone() for v in (y.v, g.v, u.v, dx.v, dw[0], dw[1])]
            both()
            torch.cuda.synchronize()
            for p, q in zip(got, (y.v, g.v, u.v, dx.v, dw[0], dw[1])):
                assert torch.equal(p, q)
            wy, ey, *_ = gated_want(gate, up, x.f64(), "silu")
            near(y.v, wy, ey + HALF * (wy.abs() + ey))
    del graphs
    gate.close(), up.close()


def test_calls_behind_each_other_on_a_busy_stream():
    """Products, single tokens, decode calls and gradients one behind the other without a wait in between: each reads what the one before wrote."""
    m = 1040
    a, b = Layer(m, m, 0.5, seed=1, scale=0.04), Layer(m, m, 0.5, seed=2, scale=0.04)
    x = Rows(6, m, values=normal((6, m), 1))
    y = [Rows(6, m) for _ in range(3)]
    dec = torch.empty((6, m), device=DEV)
    ws, nb = room(a, b, 6, True)
    results = []
    for wait in (True, False):
        torch.cuda.synchronize()
        pause = torch.cuda.synchronize if wait else (lambda: None)
        if not wait:
            torch.cuda._sleep(20_000_000)                                # (the calls below are queued while the stream is busy)
        out = []
        for rnd in range(4):
            src = x if rnd == 0 else y[2]
            linear(a, src, y[0], name="gelu", ws=ws, nb=nb); pause()
            B.dbspmspv_gated(a.h, b.h, y[0].start, m, 6, B.ACT_SILU, y[1].start, m, None, None, 0, ws, nb); pause()
            B.dbspmspv_decode_batch(b.h, y[1].start, m, dec, m, 6); pause()
            held = y[1].v.clone(); pause()
            linear(b, y[1], y[2], t=1, residual=y[0], ws=ws, nb=nb); pause()
            linear(b, y[1], y[2], residual=y[0], ws=ws, nb=nb); pause()
            B.dbspmspv_linear_backward(a.h, None, m, 6, B.ACT_RELU, y[0].start, m, y[2].start, m, y[1].start, m, None, None, ws, nb); pause()
            out += [y[0].v.clone(), y[1].v.clone(), y[2].v.clone()]
        torch.cuda.synchronize()
        near(dec, held.double() @ b.dense.T, SUM * (held.double().abs() @ b.dense.abs().T) + 1e-30)
        results.append(out)
    for p, q in zip(*results):
        assert torch.equal(p, q)
    a.close(), b.close()


def test_rows_far_apart():
    """Offsets past 32 bits: three tokens whose rows begin more than 2^31 entries apart."""
    layer = Layer(300, 100, seed=6)
    ld = (1 << 31) + 8
    far = torch.empty(2 * ld + 512, dtype=torch.bfloat16, device=DEV)
    x = Rows(3, 100, values=normal((3, 100), 1))
    want, e, _, _ = linear_want(layer, x.f64(), None, "none", None)
    rows = lambda w: torch.stack([far[k * ld:k * ld + w] for k in range(3)])
    ws, nb = room(layer, None, 3, True)
    for t in (2, 3):
        far[:300] = 0
        B.dbspmspv_linear(layer.h, x.start, x.ld, t, None, 0, None, 0, far, ld, 0, None, 0, ws, nb)
        torch.cuda.synchronize()
        near(rows(300)[:t], want[:t], (e + HALF * (want.abs() + e))[:t])
    for k in range(3):
        far[k * ld:k * ld + 100] = x.v[k]
    y = Rows(3, 300)
    for t in (2, 3):
        B.dbspmspv_linear(layer.h, far, ld, t, None, 0, None, 0, y.start, y.ld, 0, None, 0, ws, nb)
        torch.cuda.synchronize()
        near(y.v[:t], want[:t], (e + HALF * (want.abs() + e))[:t])
    layer.close()


def test_small_cases_pass_under_the_range_checked_library():
    from paper_2608_16308_b200 import build
    env = dict(os.environ, DBSPMSPV_LIBRARY=build.build_library(checked=True))
    r = subprocess.run([sys.executable, "-m", "pytest", "-x", "-q", "-m", "gpu", "-p", "no:cacheprovider", "tests/test_gpu_linear.py", "-k", "linear_backward or gated_backward"],
                       cwd=ROOT, env=env, capture_output=True, text=True, timeout=900)
    assert r.returncode == 0 and "passed" in r.stdout, r.stdout[-4000:] + r.stderr[-2000:]
