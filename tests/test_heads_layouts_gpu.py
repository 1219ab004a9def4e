"""Queries, keys and values as parts of one projection in every order of its sizes: turned in place, and their
gradients written into the parts of another such buffer, bit for bit as between tensors of their own."""
import pytest
import torch

from paper_2608_11519_gb300 import flarepp
from test_decay_gpu import _device, decays, heads, tensor  # noqa: F401

pytestmark = pytest.mark.gpu
ORDERS = {"bphn": (0, 1, 2, 3), "bnph": (0, 2, 3, 1), "bnhp": (0, 3, 2, 1), "bhnp": (0, 3, 1, 2), "bhpn": (0, 2, 1, 3),
          "nbhp": (1, 3, 2, 0)}  # where batch, parts, heads and tokens lie


def parts(buffer, order):
    return [p for p in buffer.permute(*ORDERS[order], 4).unbind(1)]


@pytest.mark.parametrize("order", ORDERS)
@pytest.mark.parametrize("B,H,N", [(2, 4, 150), (1, 3, 40), (3, 1, 200), (2, 2, 1)])
def test_in_place_and_gradients(order, B, H, N):
    D = 64
    sizes = dict(b=B, p=3, h=H, n=N)
    buffer = tensor(1, *(sizes[c] for c in order), D)
    q, k, v = parts(buffer, order)
    assert q.shape == (B, H, N, D)
    own = [t.clone(memory_format=torch.contiguous_format) for t in (q, k, v)]
    pos = torch.arange(N, dtype=torch.int32, device="cuda")[:, None]
    freqs = flarepp.rotary_frequencies([32])
    want = flarepp.rotary_fwd(own[0], own[1], pos, freqs, [32])
    flarepp.rotary_fwd(q, k, pos, freqs, [32], q_out=q, k_out=k)
    assert torch.equal(q, want[0]) and torch.equal(k, want[1]) and torch.equal(v, own[2])
    dy, ld = heads(4, B, H, N, D, std=0.1), decays(H)
    grads = torch.full_like(buffer, float("nan"))
    dq, dk, dv = parts(grads, order)
    flarepp.decay_attention_bwd(q, k, v, ld, dy, dQ=dq, dK=dk, dV=dv)
    for a, b in zip((dq, dk, dv), flarepp.decay_attention_bwd(want[0], want[1], own[2], ld, dy)):
        assert torch.equal(a, b)
