"""Group norm of samples without rows."""
import pytest
import torch

from paper_2608_11519_gb300 import flarepp
from test_group_norm_gpu import _device  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("B,C,G,eps", [(3, 16, 2, 1e-5), (1, 7, 7, 1e-2), (700, 512, 8, 1e-5), (2, 5000, 1, 0.25)])
def test_statistics(dtype, B, C, G, eps):
    """They are those of a sample whose length is 0, bit for bit: mean 0 and 1 / sqrt(eps)."""
    X = torch.zeros(B, 0, C, dtype=dtype, device="cuda")
    stats = torch.full((B, 2, G), float("nan"), device="cuda")
    flarepp.group_norm_fwd_train(X, G, eps=eps, stats=stats)
    none = torch.zeros(B, dtype=torch.int32, device="cuda")
    for N in (1, 9):
        _, want = flarepp.group_norm_fwd_train(torch.zeros(B, N, C, dtype=dtype, device="cuda"), G, eps=eps,
                                               lengths=none)
        assert torch.equal(stats, want)
    assert not bool(stats[:, 0].any())
