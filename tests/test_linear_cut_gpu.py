"""The forward of long contractions with few output tiles, which is cut into chunks: float32 partial sums
in the workspace, then bias, activation, residual and the kept sums in the kernel that adds them.
Rows and columns that end inside a block, a vector or a word. Bounds as in test_linear_gpu.py."""
import ctypes

import pytest
import torch

from paper_2608_11519_gb300 import flarepp
from test_linear_gpu import _device, case, reference, within  # noqa: F401

pytestmark = pytest.mark.gpu


def lines(n):
    return -(-n // 64) * 64


@pytest.mark.parametrize("T,K,N", [(500, 8192, 256), (300, 4096, 512), (1000, 3000, 300),
                                   (257, 16384, 40), (259, 8200, 77), (300, 5001, 129), (513, 12288, 1)])
def test_forward(T, K, N):
    s = flarepp.LinearShape(T, K, N, flarepp.BF16, 0)
    sums = 2 * T * (-(-N // 4) * 4) * 4  # of two chunks at least
    padded = (T + N) * lines(K) * 2 if K % 8 else 0
    assert flarepp.load().flarepp_linear_workspace_bytes(ctypes.byref(s)) >= sums + padded
    for act in flarepp.ACTIVATIONS:
        for bias, residual in ((True, False), (False, True), (True, True), (False, False)):
            X, W, b, R = case(T, K, N, act, bias, residual, seed=K % 89)
            Y = flarepp.linear_fwd(X, W, b, R, act)
            y, z, by, bz = reference(X, W, b, R, act)
            within(Y, y, by, f"Y {act} bias={bias} residual={residual}")
            Y2, Z = flarepp.linear_fwd_train(X, W, b, R, act)
            assert torch.equal(Y, Y2)
            if act != "none":
                within(Z, z, bz, f"Z {act}")


@pytest.mark.parametrize("N,K", [(257, 72), (264, 136), (300, 80), (1000, 264)])
def test_weight_gradient_of_ragged_outputs(N, K):
    """Outputs are the rows of the partial sums: the last 32 of them end inside a warp."""
    T = 6000
    X, W, _, _ = case(T, K, N, "none", False, False, seed=N)
    dY = X.new_empty(T, N).normal_(generator=torch.Generator(device="cuda").manual_seed(3))
    s = flarepp.LinearShape(T, K, N, flarepp.BF16, 0)
    # dZ, W and the sums of db, at most
    rest = (T * (N % 8 > 0) * lines(N) + N * lines(K)) * 2 + 608 // -(-N // 256) * lines(N) * 4 + 2048
    assert flarepp.load().flarepp_linear_bwd_workspace_bytes(ctypes.byref(s)) >= rest + 2 * N * K * 4
    _, dW, _ = flarepp.linear_bwd(X, W, dY, bias=False, need=(False, True))
    ref = dY.double().t() @ X.double()
    err = 2 * (T / 16 + 8) * 2.0 ** -23 * (dY.double().abs().t() @ X.double().abs())
    u = 2.0 ** -8 * 1.01
    within(dW, ref, u * (ref.abs() + err) + err, "dW")
