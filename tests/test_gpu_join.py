"""dbspmspv_join and its gradient against the formulas in 64 bits: norms, gates, biases, types, strides off every vector, rows from one column to a cluster's."""
import pytest
import torch

from rows_util import Join

pytestmark = pytest.mark.gpu


def both(j, **kw):
    j.forward()
    torch.cuda.synchronize()
    j.check()
    j.backward(**kw)
    torch.cuda.synchronize()
    j.check_back()


@pytest.mark.parametrize("n", [1, 7, 8, 9, 255, 256, 257, 264, 1000, 2056, 4096, 4099, 8192, 11008, 32768])
@pytest.mark.parametrize("t", [1, 5])
def test_widths(n, t):
    both(Join(t, n, "rms", "layer", c=n % 2 == 0, gate="shared", drop=0.25, seed=n))


@pytest.mark.parametrize("block", ["none", "rms", "layer"])
@pytest.mark.parametrize("next", ["none", "rms", "layer"])
@pytest.mark.parametrize("gate", ["none", "shared", "token"])
@pytest.mark.parametrize("c", [False, True])
def test_norms_gates_biases(block, next, gate, c):
    both(Join(9, 200, block, next, c=c, gate=gate, drop=0.1, seed=5))
    both(Join(3, 513, block, next, w=False, c=c, gate=gate, params=True, seed=6))


@pytest.mark.parametrize("stream", [False, True])
@pytest.mark.parametrize("blk", [False, True])
@pytest.mark.parametrize("params", [False, True])
@pytest.mark.parametrize("dblk", [False, True])
@pytest.mark.parametrize("pad,lead", [(0, 0), (8, 8), (3, 1), (5, 0)])
def test_types_and_strides(stream, blk, params, dblk, pad, lead):
    both(Join(6, 1037, "layer", "rms", c=True, gate="token", drop=0.3, stream=stream, blk=blk, params=params, dblk=dblk, pad=pad, lead=lead, seed=7))
    both(Join(6, 600, "rms", "rms", gate="shared", stream=stream, blk=blk, params=params, dblk=dblk, pad=pad, lead=lead, seed=8))


@pytest.mark.parametrize("t,n", [(148, 1024), (149, 96), (1000, 64), (2500, 8), (700, 520), (301, 4096), (333, 5000), (160, 9000), (40, 20000), (7001, 33)])
def test_many_tokens(t, n):
    both(Join(t, n, "rms", "rms", gate="shared", drop=0.1, seed=t))
    both(Join(t, n, "layer", "layer", c=True, gate="token", stream=True, seed=t))


def test_every_piece_of_the_widest_types():
    """all operands in 32 bits, gate rows too: the most shared memory a row can take"""
    for n in (4096, 8192, 32768):
        both(Join(5, n, "rms", "rms", gate="token", drop=0.5, stream=True, blk=True, params=True, dblk=True, seed=3))


@pytest.mark.parametrize("kw", [dict(has_b=False), dict(has_r=False), dict(has_b=False, next="none"), dict(has_r=False, block="none", drop=0.9)], ids=str)
def test_parts_of_a_join(kw):
    j = Join(11, 777, seed=4, **kw)
    j.forward()
    torch.cuda.synchronize()
    j.check()
    for out, h, stats in ((True, False, False), (False, True, True), (True, False, True)):
        j.forward(h=h, stats=stats, want_out=out)
        torch.cuda.synchronize()
        j.check()


@pytest.mark.parametrize("norms", ["none", "rms"])
@pytest.mark.parametrize("t,n,pad,lead", [(20, 1000, 0, 0), (700, 1037, 0, 0), (700, 1037, 4, 1), (90, 5001, 0, 3)])
@pytest.mark.parametrize("stream", [False, True])
def test_in_place(norms, t, n, pad, lead, stream):
    """r becomes out, dout becomes dr: rows in words too, whose neighbours' halves a warp writes while another one reads"""
    kw = dict(block=norms, next=norms, gate="shared", drop=0.1, seed=2, pad=pad, lead=lead, stream=stream)
    j = Join(t, n, **kw)
    want = j.want()
    j.forward(out=j.r)
    torch.cuda.synchronize()
    j.want = lambda: want
    j.check()
    j = Join(t, n, **kw)
    j.backward(in_place=True)
    torch.cuda.synchronize()
    j.check_back()


@pytest.mark.parametrize("has_b,has_r,out,h", [(False, True, False, True), (False, True, True, True), (True, False, True, True), (True, True, False, True), (True, True, True, False)])
@pytest.mark.parametrize("n,pad", [(4096, 0), (520, 0), (521, 0), (11008, 8)])
def test_what_is_missing(has_b, has_r, out, h, n, pad):
    for t in (3, 400):
        j = Join(t, n, gate="shared", drop=0.1, seed=3, pad=pad, has_b=has_b, has_r=has_r)
        j.forward(want_out=out, h=h)
        torch.cuda.synchronize()
        j.check()


ALL = ("dr", "db", "dgate", "dw_block", "dc_block", "dw_next", "dc_next")


@pytest.mark.parametrize("wanted", [(k,) for k in ALL] + [("dr", "db"), ("dw_block", "dw_next"), ("dc_block", "dgate")], ids=str)
@pytest.mark.parametrize("gate", ["shared", "token"])
def test_gradients_one_by_one(wanted, gate):
    j = Join(37, 520, "layer", "layer", c=True, gate=gate, drop=0.2, seed=9)
    j.backward(wanted=wanted)
    torch.cuda.synchronize()
    j.check_back()


@pytest.mark.parametrize("dh,dout", [(True, False), (False, True)])
@pytest.mark.parametrize("next", ["none", "rms"])
def test_one_way_back(dh, dout, next):
    j = Join(13, 300, "rms", next, gate="shared", drop=0.2, seed=10)
    j.backward(dh=dh, dout=dout)
    torch.cuda.synchronize()
    j.check_back()


def test_gradient_of_a_norm_alone():
    """b is there for the forward call only: its gradient passes the gate and the dropout, nothing else needs it"""
    j = Join(13, 300, "none", "rms", gate="shared", drop=0.2, seed=10)
    j.set_kept()
    j.b = None
    j.backward(wanted=("dr", "db", "dw_next"))
    torch.cuda.synchronize()
    j.check_back()


def test_large_means():
    """rows far from zero: the layer norm's variance is that of the differences"""
    j = Join(5, 2000, "layer", "layer", stream=True, blk=True, seed=11)
    j.b.v.add_(300.0)
    j.r.v.add_(-500.0)
    both(j)


def test_constant_and_zero_rows():
    j = Join(6, 264, "layer", "rms", stream=True, blk=True, seed=12, has_r=True)
    j.b.v[1] = 0.0
    j.b.v[2] = 3.0
    j.r.v[1] = 0.0
    both(j)


@pytest.mark.parametrize("drop", [0.0, 1e-6, 0.5, 0.99999, 1.0])
def test_probabilities(drop):
    both(Join(9, 1000, "rms", "rms", gate="shared", drop=drop, seed=13))


def test_a_spoiled_token_spoils_no_other():
    bad = float("nan"), float("inf"), -float("inf")
    j, clean = Join(12, 520, "rms", "layer", c=True, seed=14), Join(12, 520, "rms", "layer", c=True, seed=14)
    for i, v in enumerate(bad):
        j.b.v[2 + i, 7 * i] = v
        j.r.v[6 + i, 7 * i] = v
    rows = [t for t in range(12) if not 2 <= t < 5 and not 6 <= t < 9]
    for x in (j, clean):
        x.forward()
    torch.cuda.synchronize()
    for a, b in ((j.out, clean.out), (j.h, clean.h)):
        assert torch.equal(a.v[rows], b.v[rows])
        assert not bool(torch.isfinite(a.v[2:5].float()).all(dim=1).any()) and not bool(torch.isfinite(a.v[6:9].float()).all(dim=1).any())
    assert torch.equal(j.stats[rows], clean.stats[rows])


@pytest.mark.parametrize("norm", ["rms", "layer"])
def test_gradients_against_differences(norm):
    """Central differences of the formula in 64 bits, along random directions of every input."""
    j = Join(4, 40, norm, norm, c=True, gate="shared", drop=0.25, stream=True, blk=True, params=True, dblk=True, seed=15)
    j.backward()
    torch.cuda.synchronize()
    dh, dout = j.dh.f64(), j.dout.f64()
    base = dict(r=j.r.f64(), b=j.b.f64(), wb=j.wbd, cb=j.cbd, g=j.gd, wn=j.wnd, cn=j.cnd)

    def loss(r, b, wb, cb, g, wn, cn):
        def normed(x, w, c):
            m = x.mean(dim=1, keepdim=True) if norm == "layer" else 0.0
            return (x - m) / ((x - m).square().mean(dim=1, keepdim=True) + j.eps).sqrt() * w + c
        out = r + j.scale * j.mask * g * normed(b, wb, cb)
        return (out * dout).sum() + (normed(out, wn, cn) * dh).sum()

    names = dict(r="dr", b="db", wb="dw_block", cb="dc_block", g="dgate", wn="dw_next", cn="dc_next")
    for k, v in base.items():
        got = j.res[names[k]]
        got = got.f64() if hasattr(got, "f64") else got[:-1].double()
        for s in range(3):
            d = torch.randn(v.shape, generator=torch.Generator(device=v.device).manual_seed(s), device=v.device, dtype=torch.float64)
            step = 1e-5
            want = (loss(**{**base, k: v + step * d}) - loss(**{**base, k: v - step * d})) / (2 * step)
            # (`out` was handed back in 32 bits: 2^-24 of its entries, a few roundings of the sums; differences are off by 1e-9)
            assert abs(float((got * d).sum() - want)) <= 1e-5 * float((got.abs() * d.abs()).sum()), k


def test_same_results_again():
    j = Join(999, 1500, gate="shared", drop=0.1, seed=16)
    bits = lambda rows: [v.buf.clone() if hasattr(v, "buf") else v.clone() for v in rows]
    runs = []
    for _ in range(2):
        j.forward()
        runs.append(bits([j.out, j.h, j.stats]))
    j.set_kept()
    for _ in range(2):
        j.backward()
        runs.append(bits(j.res.values()))
    torch.cuda.synchronize()
    for a, b in (runs[:2], runs[2:]):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
