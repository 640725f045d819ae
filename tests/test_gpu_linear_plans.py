"""Every cut of the tensor-core products -- tile, pairs, clusters that share K -- at the smallest sizes that take it, odd ones, with rows on 16 bytes and off them."""
import pytest
import torch

import linear_plan_util as plan
from linear_checks import check_backward, check_gated, check_linear
from linear_util import Layer

pytestmark = pytest.mark.gpu

# (thread blocks of a tile, its tokens, thread blocks that share K, rows on 16 bytes): rows, columns, tokens
FORWARD = {
    (1, 16, 1, 1): (104, 101, 9), (1, 16, 2, 1): (104, 193, 16), (1, 16, 4, 1): (104, 451, 5), (1, 16, 8, 1): (104, 1286, 15),
    (1, 64, 1, 1): (104, 101, 54), (1, 64, 2, 1): (104, 321, 121), (1, 64, 4, 1): (104, 779, 21), (1, 64, 8, 1): (104, 2563, 95),
    (1, 256, 1, 1): (1632, 129, 2562), (1, 256, 2, 1): (392, 975, 2399), (1, 256, 4, 1): (136, 2703, 2344), (1, 256, 8, 1): (104, 10158, 2581), (2, 256, 1, 1): (968, 131, 2623),
    (1, 64, 1, 0): (103, 101, 54), (1, 64, 8, 0): (103, 2563, 95), (1, 256, 1, 0): (1597, 895, 2577), (1, 256, 2, 0): (389, 1643, 2559), (1, 256, 4, 0): (131, 3753, 2244),
    (1, 256, 8, 0): (103, 11809, 2445), (2, 256, 1, 0): (955, 733, 2603),
}
GATED = {
    (1, 16, 1, 1): (104, 101, 9), (1, 16, 2, 1): (104, 193, 16), (1, 16, 4, 1): (104, 451, 5), (1, 16, 8, 1): (104, 1286, 15),
    (1, 64, 1, 1): (104, 101, 54), (1, 64, 2, 1): (104, 321, 121), (1, 64, 4, 1): (104, 779, 21), (1, 64, 8, 1): (104, 2563, 95),
    (1, 256, 1, 1): (792, 103, 2642), (1, 256, 2, 1): (200, 863, 2559), (1, 256, 4, 1): (104, 2476, 2500), (1, 256, 8, 1): (104, 10115, 1720), (2, 256, 1, 1): (472, 102, 2579),
    (1, 64, 1, 0): (103, 101, 54), (1, 64, 8, 0): (103, 2563, 95), (1, 256, 1, 0): (781, 325, 2567), (1, 256, 2, 0): (201, 1238, 2325), (1, 256, 4, 0): (103, 2995, 2439),
    (1, 256, 8, 0): (103, 10587, 1672), (2, 256, 1, 0): (453, 328, 2680),
}
# one layer below 256 tokens, two from there on
GRADIENT_OF_X = {
    (1, 16, 1, 1): (101, 104, 9), (1, 16, 2, 1): (193, 104, 5), (1, 16, 4, 1): (449, 104, 7), (1, 16, 8, 1): (1291, 104, 5),
    (1, 64, 1, 1): (101, 104, 54), (1, 64, 2, 1): (321, 104, 96), (1, 64, 4, 1): (779, 104, 20), (1, 64, 8, 1): (2315, 104, 31),
    (1, 256, 1, 1): (105, 1616, 2663), (1, 256, 2, 1): (456, 392, 2590), (1, 256, 4, 1): (1379, 136, 2250), (1, 256, 8, 1): (5012, 104, 2216), (2, 256, 1, 1): (101, 952, 2465),
    (1, 64, 1, 0): (101, 103, 54), (1, 64, 8, 0): (2315, 103, 31), (1, 256, 1, 0): (325, 1611, 2562), (1, 256, 2, 0): (795, 397, 2593), (1, 256, 4, 0): (1915, 131, 2500),
    (1, 256, 8, 0): (5963, 101, 2089), (2, 256, 1, 0): (337, 911, 2407),
}
# clusters that share the tokens: one layer, then two
GRADIENT_OF_WEIGHTS = {(1, 256, 1): (101, 103, 9), (1, 256, 2): (101, 103, 598), (1, 256, 4): (101, 103, 1090), (1, 256, 8): (101, 103, 2235), (2, 256, 1): (1030, 6915, 33)}


def as_planned(got, want):
    if torch.cuda.get_device_properties(0).multi_processor_count == 148:
        assert got == want[:3]


@pytest.mark.parametrize("cut", FORWARD, ids=str)
def test_forward(cut):
    m, n, t = FORWARD[cut]
    aligned = cut[3]
    as_planned(plan.forward(m, n, t, 0, aligned), cut)
    layer = Layer(m, n, 0.5, seed=1)
    pad, lead = (0, 0) if aligned else (2, 1)
    check_linear(layer, t, "silu", pad, lead, bias=True)
    check_linear(layer, t, "none", pad, lead, f32=True)
    check_linear(layer, t, "relu", pad, lead, bias=True, residual=True, keep=True)
    layer.close()


@pytest.mark.parametrize("cut", GATED, ids=str)
def test_gated(cut):
    m, n, t = GATED[cut]
    aligned = cut[3]
    as_planned(plan.gated(m, n, t, 0, aligned), cut)
    gate, up = Layer(m, n, 0.5, seed=1), Layer(m, n, 0.3, seed=2)
    pad, lead = (0, 0) if aligned else (2, 1)
    check_gated(gate, up, t, "silu", pad, lead)
    check_gated(gate, up, t, "gelu", pad, lead, keep=True)
    gate.close(), up.close()


@pytest.mark.parametrize("cut", GRADIENT_OF_X, ids=str)
def test_gradient_of_x(cut):
    m, n, t = GRADIENT_OF_X[cut]
    layers = [Layer(m, n, 0.5, seed=1), Layer(m, n, 0.3, seed=2)][:2 if t >= 256 else 1]
    as_planned(plan.gradient_of_x(m, n, t, len(layers), cut[3]), cut)
    pad, lead = (0, 0) if cut[3] else (2, 1)
    check_backward(layers, t, "silu", pad, lead, want_dw=False)
    for w in layers:
        w.close()


@pytest.mark.parametrize("layers", [1, 2])
@pytest.mark.parametrize("cut", GRADIENT_OF_WEIGHTS, ids=str)
def test_gradient_of_weights(cut, layers):
    m, n, t = GRADIENT_OF_WEIGHTS[cut]
    w = [Layer(m, n, 0.5, seed=1), Layer(m, n, 0.3, seed=2)][:layers]
    as_planned(plan.gradient_of_weights(m, n, t, layers), cut)
    check_backward(w, t, "relu", want_dx=False)
    check_backward(w, t, "none", 3, 1, want_dx=False)
    for v in w:
        v.close()
