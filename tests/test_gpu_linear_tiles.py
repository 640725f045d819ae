"""Linear and gated layers with more tiles than the GPU has thread blocks for: a block takes three and more of them, so both of its accumulators
are written again behind their first tile.  Against plain forms in 64 bits, over pairs of thread blocks and single ones."""
import pytest
import torch

from paper_2608_16308_b200 import binding as B
from linear_checks import check_backward, check_gated, check_linear
from linear_util import DEV, HALF, Layer, near

pytestmark = pytest.mark.gpu


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
