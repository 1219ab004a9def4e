"""The kernel that makes dZ on its way to dX, at widths whose half tile is no whole 64-column atom, whose last
32-column block is partial, and at odd numbers of slices of the outputs above one (the two groups of warps
swap stages from tile to tile). That the kernel runs is asked of it: the test hook that lets its waits run
out has to reach the call. Bounds as in test_linear_gpu.py."""
import pytest
import torch

from paper_2608_11519_gb300 import flarepp
from test_linear_gpu import U, _device, case, randn, slope64, sum_error, within  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("T,K,N", [(12345, 200, 504), (20011, 248, 512), (40001, 136, 264), (30001, 40, 136),
                                   (20000, 16, 192), (12000, 232, 320), (11000, 24, 448), (10000, 104, 104)])
def test_gradients(T, K, N, act):
    X, W, b, _ = case(T, K, N, act, True, False, seed=T % 97)
    dY = randn(T, N, seed=77)
    Z = (X.float() @ W.float().t() + b.float()).bfloat16()
    status, lib = torch.zeros(1, dtype=torch.int32, device="cuda"), flarepp.load()
    lib.flarepp_test_wait_fault(18, 0, 1_000_000)
    try:
        flarepp.linear_bwd(X, W, dY, Z, act, status=status)
        torch.cuda.synchronize()
    finally:
        lib.flarepp_test_wait_fault(0, -1, 0)
    assert int(status) == flarepp.ERR_TIMEOUT
    status.zero_()
    dX, dW, db = flarepp.linear_bwd(X, W, dY, Z, act, status=status)
    z = Z.double()
    dz = dY.double() * slope64(z, act)
    off = dY.double().abs() * (1e-6 * (1 + z.abs()) + 2.0 ** -23)
    mag = dz.abs() + off
    dx, dw, dbr = dz @ W.double(), dz.t() @ X.double(), dz.sum(0)
    ex = (U + sum_error(N)) * (mag @ W.double().abs()) + off @ W.double().abs()
    ew = (U + sum_error(T)) * (mag.t() @ X.double().abs()) + off.t() @ X.double().abs()
    eb = T * 2.0 ** -24 * mag.sum(0) + off.sum(0)
    within(dX, dx, U * (dx.abs() + ex) + ex, "dX")
    within(dW, dw, U * (dw.abs() + ew) + ew, "dW")
    within(db, dbr, U * (dbr.abs() + eb) + eb, "db")
    assert int(status) == flarepp.OK
    for x, y in zip(flarepp.linear_bwd(X, W, dY, Z, act), (dX, dW, db)):
        assert torch.equal(x, y)
    a, _, c = flarepp.linear_bwd(X, W, dY, Z, act, need=(True, False))  # dZ is not kept
    assert torch.equal(a, dX)
    within(c, dbr, U * (dbr.abs() + eb) + eb, "db")  # its partial sums are added in another order without dW
