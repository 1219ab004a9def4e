"""Failure detection of the linear layer without a GPU fault: the test hook withholds one ring item
of CTA 0 and bounds the launch's waits at 1 ms. The kernel must give up, report
FLAREPP_ERR_TIMEOUT in `status` and leave the GPU usable: the next call must be right."""
import pytest
import torch

from paper_2608_11519_gb300 import flarepp

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kernel,T,K,N,item", [(16, 3000, 1280, 512, 0), (16, 3000, 1280, 512, 7),
                                               (16, 70000, 128, 256, 3), (17, 50, 2048, 300, 0),
                                               (17, 200, 4096, 1000, 5)])
def test_bounded_wait_runs_out_and_call_recovers(kernel, T, K, N, item):
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    lib = flarepp.load()
    X = torch.randn(T, K, device="cuda").bfloat16()
    W = (torch.randn(N, K, device="cuda") * K ** -0.5).bfloat16()
    R = torch.randn(T, N, device="cuda").bfloat16()
    want = flarepp.linear_fwd(X, W, None, R, "silu")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    lib.flarepp_test_wait_fault(kernel, item, 1_000_000)
    try:
        flarepp.linear_fwd(X, W, None, R, "silu", status=status)
        torch.cuda.synchronize()
    finally:
        lib.flarepp_test_wait_fault(0, -1, 0)
    assert int(status) == flarepp.ERR_TIMEOUT
    status.zero_()
    again = flarepp.linear_fwd(X, W, None, R, "silu", status=status)
    torch.cuda.synchronize()
    assert int(status) == flarepp.OK and torch.equal(again, want)
