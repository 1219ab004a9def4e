"""The table's gradient for wide rows of odd lengths (several narrow vectors per thread, several blocks of
columns) and for tables so long that their marks are cleared apart. Bounds as in test_embedding_gpu.py."""
import pytest
import torch

from paper_2608_11519_gb300 import flarepp
from test_embedding_gpu import _device, check_bwd, make_ids  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind", ["uniform", "same", "skewed", "runs"])
@pytest.mark.parametrize("T,V,C", [(5003, 257, 255), (5003, 257, 346), (3001, 57, 1023), (700, 57, 1023),
                                   (20011, 4001, 129), (9001, 2, 514), (40, 3_000_000, 8), (1500, 8_000_000, 3)])
def test_gradient(T, V, C, kind):
    for k, dt in enumerate((torch.float32, torch.bfloat16)):
        ids = make_ids(kind, T, V, seed=T + k)
        on = ids.to(torch.int64 if k else torch.int32).cuda()
        g = torch.Generator(device="cuda").manual_seed(5)
        buf = torch.full((V * C + 512,), 9.0, dtype=dt, device="cuda")
        grad = buf[256:256 + V * C].view(V, C)
        dY = torch.randn(T, C, generator=g, device="cuda").to(dt)
        flarepp.embedding_bwd(on, dY, V, 0.7, dtable=grad)
        check_bwd(ids, dY, V, 0.7, grad)
        assert (buf[:256] == 9).all() and (buf[256 + V * C:] == 9).all()
        assert torch.equal(grad, flarepp.embedding_bwd(on, dY, V, 0.7))
