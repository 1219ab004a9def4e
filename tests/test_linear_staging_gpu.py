"""Outputs that leave through two staged blocks by turns (no residual, no kept sums): many tiles per CTA pair,
short contractions, so that a tile's sums are ready while the stores of the one before still read their
blocks, and widths with an odd number of 32-column blocks for a warp (those below 33, 65 to 96, 129 to 160,
193 to 224, and tiles of 160 and 224 columns of wider outputs), after which a tile must not start
on the block that the last one ended on. Every row is compared, and the same bits have to come again.
Bounds as in test_linear_gpu.py."""
import pytest
import torch

from paper_2608_11519_gb300 import flarepp
from test_linear_gpu import U, _device, case, randn, reference, sum_error, within  # noqa: F401

pytestmark = pytest.mark.gpu

T = 210_037
STEP = 1 << 15  # rows compared at a time


@pytest.mark.parametrize("K", [8, 64, 256])
@pytest.mark.parametrize("N", [8, 32, 72, 96, 160, 224, 256, 320, 448])
def test_forward_of_every_row(K, N):
    for act, bias in (("none", False), ("gelu", True)):
        X, W, b, _ = case(T, K, N, act, bias, False, seed=N)
        Y = flarepp.linear_fwd(X, W, b, None, act)
        for a in range(0, T, STEP):
            y, _, by, _ = reference(X[a:a + STEP], W, b, None, act)
            within(Y[a:a + STEP], y, by, f"rows from {a}, {act}")
        for _ in range(3):
            assert torch.equal(Y, flarepp.linear_fwd(X, W, b, None, act))


@pytest.mark.parametrize("N", [8, 64, 200])
@pytest.mark.parametrize("K", [24, 96, 160, 224, 320])
def test_input_gradient_of_every_row(K, N):
    X, W, _, _ = case(T, K, N, "none", False, False, seed=K)
    dY = randn(T, N, seed=4)

    def grad():
        return flarepp.linear_bwd(X, W, dY, bias=False, need=(True, False))[0]

    dX = grad()
    for a in range(0, T, STEP):
        g = dY[a:a + STEP].double()
        ref, err = g @ W.double(), sum_error(N) * (g.abs() @ W.double().abs())
        within(dX[a:a + STEP], ref, U * (ref.abs() + err) + err, f"rows from {a}")
    for _ in range(3):
        assert torch.equal(dX, grad())
