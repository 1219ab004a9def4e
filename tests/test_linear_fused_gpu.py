"""The backward that makes dZ on its way to dX (narrow inputs, many rows), at its edges: the fewest rows,
rows that end inside a tile, one slice and partial slices of outputs, inputs from one vector to a
full tile, outputs left out. Bounds as in test_linear_gpu.py."""
import pytest
import torch

from paper_2608_11519_gb300 import flarepp
from test_linear_gpu import U, _device, case, randn, slope64, sum_error, within  # noqa: F401

pytestmark = pytest.mark.gpu

SHAPES = [(9728, 256, 512), (9729, 8, 64), (12345, 200, 1000), (20011, 256, 1024), (50000, 64, 200),
          (40001, 136, 520), (150001, 256, 72)]


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
@pytest.mark.parametrize("T,K,N", SHAPES)
def test_fused_backward(T, K, N, act):
    X, W, b, _ = case(T, K, N, act, True, False, seed=T % 97)
    dY = randn(T, N, seed=77)
    Z = (X.float() @ W.float().t() + b.float()).bfloat16()
    dX, dW, db = flarepp.linear_bwd(X, W, dY, Z, act)
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
    # what is left out changes nothing of the rest, and the same bits come again
    a, none, c = flarepp.linear_bwd(X, W, dY, Z, act, need=(True, False))
    assert none is None and torch.equal(a, dX)
    assert float((c.double() - dbr).abs().sub(U * (dbr.abs() + eb) + eb).max()) <= 0
    a, w, none = flarepp.linear_bwd(X, W, dY, Z, act, bias=False)
    assert none is None and torch.equal(a, dX) and torch.equal(w, dW)
    for x, y in zip(flarepp.linear_bwd(X, W, dY, Z, act), (dX, dW, db)):
        assert torch.equal(x, y)


def test_special_values_stay_in_their_row():
    T, K, N = 10000, 64, 128
    X, W, b, _ = case(T, K, N, "gelu", True, False)
    dY, Z = randn(T, N, seed=1), randn(T, N, seed=2)
    want, _, db0 = flarepp.linear_bwd(X, W, dY, Z, "gelu")
    dY[5, 3], Z[9000, 100] = float("nan"), float("inf")
    dX, _, db = flarepp.linear_bwd(X, W, dY, Z, "gelu")
    rows = torch.ones(T, dtype=torch.bool, device="cuda")
    rows[5] = rows[9000] = False
    assert torch.equal(dX[rows], want[rows]) and dX[5].isnan().all()
    cols = torch.ones(N, dtype=torch.bool, device="cuda")
    cols[3] = cols[100] = False
    assert db[3].isnan() and torch.equal(db[cols], db0[cols])


def test_bounded_wait_runs_out_and_call_recovers():
    T, K, N = 30000, 128, 512
    X, W, b, _ = case(T, K, N, "silu", True, False)
    dY, Z = randn(T, N, seed=1), randn(T, N, seed=2)
    want = flarepp.linear_bwd(X, W, dY, Z, "silu")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    lib = flarepp.load()
    for item in (0, 9):
        lib.flarepp_test_wait_fault(18, item, 1_000_000)
        try:
            flarepp.linear_bwd(X, W, dY, Z, "silu", status=status)
            torch.cuda.synchronize()
        finally:
            lib.flarepp_test_wait_fault(0, -1, 0)
        assert int(status) == flarepp.ERR_TIMEOUT
        status.zero_()
        got = flarepp.linear_bwd(X, W, dY, Z, "silu", status=status)
        torch.cuda.synchronize()
        assert int(status) == flarepp.OK
        assert all(torch.equal(x, y) for x, y in zip(got, want))
