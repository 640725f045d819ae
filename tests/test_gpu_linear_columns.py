"""One and two tokens over the active columns: a thread block per strip and clusters of two, four and eight, lists of a warp that are walked one round and
two rounds at a time, entries of x that are there, thinned out or all zero."""
import pytest

from linear_checks import check_gated, check_linear
from linear_util import Layer

pytestmark = pytest.mark.gpu

# (148 multiprocessors) thread blocks of a strip, and the entries that a warp lists at most
SHAPES = {
    "1 block, 192 entries": (9601, 2101),
    "1 block, 64 entries": (9601, 515),
    "2 blocks, 192 entries": (5003, 4201),
    "2 blocks, 64 entries": (5003, 1001),
    "4 blocks, 128 entries": (3001, 4335),
    "4 blocks, 64 entries": (3001, 2047),
    "8 blocks, 128 entries": (70, 9001),
    "8 blocks, 64 entries": (70, 8191),
}


@pytest.mark.parametrize("shape", SHAPES)
def test_one_layer(shape):
    layer = Layer(*SHAPES[shape], 0.5, seed=1)
    for t in (1, 2):
        for k, zeros in enumerate((0.0, 0.9, 1.0)):
            check_linear(layer, t, ("none", "relu", "gelu")[k], bias=k > 0, residual=True, keep=True, zeros=zeros, seed=k)
            check_linear(layer, t, "silu", 3, 1, f32=True, zeros=zeros, seed=k)
    layer.close()


@pytest.mark.parametrize("shape", SHAPES)
def test_gated(shape):
    gate, up = Layer(*SHAPES[shape], 0.5, seed=1), Layer(*SHAPES[shape], 0.3, seed=2)
    for t in (1, 2):
        for k, zeros in enumerate((0.0, 0.9, 1.0)):
            check_gated(gate, up, t, "silu", keep=True, zeros=zeros, seed=k)
            check_gated(gate, up, t, "gelu", 1, 3, keep=k == 1, zeros=zeros, seed=k)
    gate.close(), up.close()
