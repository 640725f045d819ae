"""The entry points of linear and gated layers refuse a call without a handle, whatever else it says, and need neither torch nor a
device for that."""
import ctypes
import subprocess
import sys

import pytest

from paper_2608_16308_b200 import binding as B

CALLS = {
    "linear": (B.dbspmspv_linear, dict(h=None, x=None, ldx=0, tokens=0, bias=None, act=0, residual=None, ldr=0, y=None, ldy=0, y_f32=0, z=None, ldz=0, workspace=None, workspace_bytes=0)),
    "gated": (B.dbspmspv_gated, dict(gate=None, up=None, x=None, ldx=0, tokens=0, act=0, y=None, ldy=0, g=None, u=None, ldgu=0, workspace=None, workspace_bytes=0)),
    "linear_backward": (B.dbspmspv_linear_backward, dict(h=None, x=None, ldx=0, tokens=0, act=0, z=None, ldz=0, dy=None, lddy=0, dx=None, lddx=0, dw=None, dbias=None, workspace=None,
                                                         workspace_bytes=0)),
    "gated_backward": (B.dbspmspv_gated_backward, dict(gate=None, up=None, x=None, ldx=0, tokens=0, act=0, g=None, u=None, ldgu=0, dy=None, lddy=0, dx=None, lddx=0, dw_gate=None,
                                                       dw_up=None, workspace=None, workspace_bytes=0)),
}


@pytest.mark.parametrize("name", CALLS)
@pytest.mark.parametrize("change", [dict(), dict(tokens=-1), dict(tokens=5), dict(act=7), dict(workspace_bytes=-1), dict(workspace_bytes=1 << 40)], ids=str)
def test_no_handle(name, change):
    f, kw = CALLS[name]
    for args in ((), tuple({**kw, **change}.values()) + (0,)):
        with pytest.raises(B.DbSpmspvError) as e:
            f(*args) if args else f(**{**kw, **change}, stream=0)
        assert e.value.status == B.ERR_INVALID_ARG and f"dbspmspv_{name}" in str(e.value)


@pytest.mark.parametrize("name", CALLS)
def test_wrong_names_counts_and_types(name):
    f, kw = CALLS[name]
    with pytest.raises(TypeError):
        f(**kw, nonsense=1)
    with pytest.raises(TypeError):
        f(**{k: v for k, v in kw.items() if k != "act"})
    with pytest.raises(TypeError):
        f(*kw.values(), 0, 0)
    with pytest.raises(TypeError):
        f(**{**kw, "tokens": 1.5}, stream=0)
    with pytest.raises((TypeError, AttributeError)):
        f(**{**kw, "x": 4096}, stream=0)                 # (an address is not an array)


def test_workspace():
    for up in (None, ctypes.c_void_p()):
        with pytest.raises(B.DbSpmspvError) as e:
            B.dbspmspv_linear_workspace(None, up, 4, True)
        assert e.value.status == B.ERR_INVALID_ARG


def test_options_and_activations():
    assert B.default_create_opts().linear == 0
    assert (B.ACT_NONE, B.ACT_RELU, B.ACT_SILU, B.ACT_GELU) == (0, 1, 2, 3)


def test_a_named_stream_needs_no_torch():
    code = ("import sys; from paper_2608_16308_b200 import binding as B\n"
            "try: B.dbspmspv_gated(None, None, None, 0, 1, 2, None, 0, None, None, 0, None, 0, 0)\n"
            "except B.DbSpmspvError as e: print(e.status, 'torch' in sys.modules)")
    r = subprocess.run([sys.executable, "-c", code], capture_output=True, text=True, timeout=300)
    assert r.stdout.split() == [str(B.ERR_INVALID_ARG), "False"], r.stdout + r.stderr
