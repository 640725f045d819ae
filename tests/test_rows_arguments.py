"""Joins, dropout and log probabilities refuse what they cannot do before they look for a device; the generator's known answers."""
import ctypes

import numpy as np
import pytest

from paper_2608_16308_b200 import binding as B
from rows_util import numbers, philox

A = np.zeros(4096, np.float32)                    # (an aligned address; no call below gets as far as using it)
A = A[(-A.ctypes.data // 4) % 16:][:64]
ODD = A.view(np.uint8)[1:]


def status(f, *args, **kw):
    with pytest.raises(B.DbSpmspvError) as e:
        f(*args, **kw)
    return e.value.status


def opts(**kw):
    o = B.default_join_opts()
    for k, v in kw.items():
        setattr(o, k, v)
    return o


JOIN = dict(opts=opts(), tokens=2, n=8, r=A, ldr=8, b=A, ldb=8, w_block=None, c_block=None, gate=None, ldg=0, w_next=None, c_next=None, random=None, out=A, ldo=8, h=A, ldh=8, stats=None, stream=0)
BACK = dict(opts=opts(), tokens=2, n=8, out=A, ldo=8, b=A, ldb=8, stats=A, w_block=None, c_block=None, gate=None, ldg=0, w_next=None, random=None, dh=A, lddh=8, dout=A, lddo=8, dr=A, lddr=8, db=A,
            lddb=8, dw_block=None, dc_block=None, dgate=None, lddg=0, dw_next=None, dc_next=None, workspace=A, workspace_bytes=64, stream=0)
DROP = dict(x=A, ldx=8, f32=1, tokens=2, n=8, drop=0.5, random=A, y=A, ldy=8, stream=0)
LOGP = dict(logits=A, ldl=8, logits_f32=1, tokens=2, vocab=8, temperature=1.0, targets=A, logprob=A, entropy=None, stats=None, top=0, top_ids=None, top_logprobs=None, stream=0)
LBACK = dict(logits=A, ldl=8, logits_f32=1, tokens=2, vocab=8, temperature=1.0, targets=A, stats=A, entropy=None, top=0, top_ids=None, dlogprob=A, dentropy=None, dtop=None, dlogits=A, ldd=8,
             dlogits_f32=1, stream=0)

REFUSED = [(B.dbspmspv_join, JOIN, c) for c in (
    dict(opts=None), dict(tokens=-1), dict(n=0), dict(n=-5), dict(opts=opts(norm_block=3)), dict(opts=opts(norm_next=-1)), dict(opts=opts(eps_block=-1.0)), dict(opts=opts(eps_next=float("nan"))),
    dict(opts=opts(eps_next=float("inf"))), dict(opts=opts(scale=float("inf"))), dict(opts=opts(drop=-0.1)), dict(opts=opts(drop=1.5)), dict(opts=opts(drop=float("nan"))), dict(opts=opts(drop=0.5)),
    dict(r=None, b=None), dict(out=None, h=None), dict(w_block=A), dict(c_block=A), dict(opts=opts(norm_next=0), w_next=A), dict(opts=opts(norm_next=0), c_next=A), dict(ldr=7), dict(ldb=7),
    dict(ldo=7), dict(ldh=0), dict(gate=A, ldg=7), dict(gate=A, ldg=-8), dict(r=ODD), dict(b=ODD), dict(out=ODD), dict(h=ODD), dict(opts=opts(stream_f32=1), r=ODD[1:]), dict(opts=opts(block_f32=1), b=ODD[1:]),
    dict(opts=opts(params_f32=1), w_next=ODD[1:]), dict(stats=A[1:]), dict(opts=opts(drop=0.5), random=A[1:]))]
REFUSED += [(B.dbspmspv_join_backward, BACK, c) for c in (
    dict(opts=None), dict(tokens=-1), dict(n=0), dict(workspace_bytes=-1), dict(opts=opts(drop=2.0)), dict(dh=None, dout=None), dict(out=None), dict(stats=None), dict(dw_block=A), dict(dc_block=A),
    dict(w_block=A), dict(opts=opts(norm_next=0), dw_next=A), dict(opts=opts(norm_next=0), w_next=A), dict(dgate=A), dict(opts=opts(norm_block=1), b=None), dict(gate=A, dgate=A, b=None),
    dict(opts=opts(drop=0.1)), dict(dr=None, db=None), dict(ldo=7), dict(ldb=7), dict(lddh=7), dict(lddo=7), dict(lddr=7), dict(lddb=7), dict(gate=A, ldg=7), dict(gate=A, ldg=8, dgate=A, lddg=7),
    dict(dh=ODD), dict(dout=ODD), dict(dr=ODD), dict(db=ODD), dict(opts=opts(dblock_f32=1), db=ODD[1:]), dict(dw_next=ODD[1:]), dict(stats=A[2:]), dict(workspace=A[1:]))]
REFUSED += [(B.dbspmspv_dropout, DROP, c) for c in (
    dict(tokens=-1), dict(n=0), dict(n=1 << 31, ldx=1 << 32, ldy=1 << 32), dict(drop=-0.5), dict(drop=1.01), dict(drop=float("nan")), dict(ldx=7), dict(ldy=7), dict(x=None), dict(y=None), dict(random=None),
    dict(x=ODD[1:]), dict(y=ODD), dict(random=A[1:]), dict(f32=0, x=ODD))]
REFUSED += [(B.dbspmspv_logprobs, LOGP, c) for c in (
    dict(tokens=-1), dict(vocab=0), dict(vocab=-3), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=float("nan")), dict(temperature=float("inf")), dict(temperature=1e-39), dict(top=-1), dict(top=9), dict(vocab=100, ldl=100, top=65, top_ids=A),
    dict(ldl=7), dict(logits=None), dict(targets=None), dict(top=2), dict(logits=ODD[1:]), dict(logits_f32=0, logits=ODD), dict(targets=ODD), dict(logprob=ODD), dict(entropy=ODD), dict(stats=A[1:]),
    dict(top=1, top_ids=ODD), dict(top=1, top_ids=A, top_logprobs=ODD))]
REFUSED += [(B.dbspmspv_logprobs_backward, LBACK, c) for c in (
    dict(tokens=-1), dict(vocab=0), dict(temperature=0.0), dict(temperature=1e-39), dict(top=65, vocab=100, ldl=100, ldd=100), dict(top=9), dict(top=-1), dict(ldl=7), dict(ldd=7), dict(logits=None), dict(dlogits=None), dict(stats=None),
    dict(targets=None), dict(dentropy=A), dict(dtop=A), dict(dtop=A, top=2), dict(logits=ODD), dict(dlogits=ODD[1:]), dict(dlogits_f32=0, dlogits=ODD), dict(stats=A[1:]), dict(dlogprob=ODD))]


@pytest.mark.parametrize("f,ok,change", REFUSED, ids=lambda v: getattr(v, "__name__", None))
def test_refused(f, ok, change):
    assert status(f, **{**ok, **change}) == B.ERR_INVALID_ARG, change


def test_wide_rows_are_not_supported():
    wide = dict(n=32769, **{k: 40000 for k in ("ldr", "ldb", "ldo", "ldh")})
    assert status(B.dbspmspv_join, **{**JOIN, **wide}) == B.ERR_UNSUPPORTED
    assert status(B.dbspmspv_join_workspace, opts(), 1, 32769) == B.ERR_UNSUPPORTED
    assert status(B.dbspmspv_join_backward, **{**BACK, "n": 32769}) == B.ERR_UNSUPPORTED


def test_no_tokens():
    """nothing to do, and no device to do it on"""
    for f, ok in ((B.dbspmspv_join, JOIN), (B.dbspmspv_dropout, DROP), (B.dbspmspv_logprobs, LOGP), (B.dbspmspv_logprobs_backward, LBACK)):
        f(**{**ok, "tokens": 0})
    B.dbspmspv_join_backward(**{**BACK, "tokens": 0})
    B.dbspmspv_join(opts(), 0, 8, None, 0, None, 0, None, None, None, 0, None, None, None, None, 0, None, 0, None, 0)


@pytest.mark.parametrize("f,ok", [(B.dbspmspv_join, JOIN), (B.dbspmspv_join_backward, BACK), (B.dbspmspv_dropout, DROP), (B.dbspmspv_logprobs, LOGP), (B.dbspmspv_logprobs_backward, LBACK)])
def test_names_counts_and_types(f, ok):
    with pytest.raises(TypeError):
        f(**ok, nonsense=1)
    with pytest.raises(TypeError):
        f(**{k: v for k, v in ok.items() if k != "tokens"})
    with pytest.raises(TypeError):
        f(*ok.values(), 0)
    with pytest.raises(TypeError):
        f(**{**ok, "tokens": 1.5})
    for bad in ("opts", "drop", "temperature"):
        if bad in ok:
            with pytest.raises(TypeError):
                f(**{**ok, bad: "0.5"})
    if "opts" in ok:
        for bad in (b"short", 4096, B.default_run_opts()):
            with pytest.raises(TypeError):
                f(**{**ok, "opts": bad})
    f(*{**ok, "tokens": 0}.values())                # (all of them by position)
    for k in ("drop", "temperature"):
        if k in ok:
            f(**{**ok, "tokens": 0, k: ctypes.c_float(0.5)})
            f(**{**ok, "tokens": 0, k: 1})


def test_options():
    o = B.default_join_opts()
    assert (o.norm_block, o.norm_next, o.scale, o.drop, o.stream_f32) == (B.NORM_NONE, B.NORM_RMS, 1.0, 0.0, 0)
    assert ctypes.sizeof(B.JoinOpts) == 48
    assert status(B.dbspmspv_join_workspace, opts(norm_next=7), 1, 8) == B.ERR_INVALID_ARG


def test_layout_of_the_options():
    import os
    import re
    text = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "dbspmspv.h")).read()
    body = re.search(r"typedef struct \{([^}]*)\}\s*dbspmspv_join_opts;", re.sub(r"/\*.*?\*/", "", text, flags=re.S)).group(1)
    names = [re.sub(r"\[.*\]", "", d.split(None, 1)[1]).strip() for d in (x.strip() for x in body.split(";")) if d]
    assert names == [f[0] for f in B.JoinOpts._fields_]


def test_known_answers_of_the_generator():
    """of the published test vectors"""
    assert philox((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    f = 0xFFFFFFFF
    assert philox((f, f, f, f), (f, f)) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]
    assert philox((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0)) == [0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1]
    got = numbers((5 << 32 | 7, 9 << 32 | 11), 3, 21)
    for t, c in ((0, 0), (2, 20), (1, 13)):
        w = philox((c // 8, t, 11, 9), (7, 5))
        assert got[t, c] == w[c % 8 // 2] >> (16 * (c % 2)) & 0xFFFF
