"""Rotary angles of far positions, for frequencies of all 24 bits.

The bound, of a pair's length: its angle is a sum of fractions of turns, each at most a half: four roundings at
magnitudes up to 1, 4 x 2^-25 turns or 7.5e-7 rad; the sine and cosine are good to two units (1.2e-7 each, 1.7e-7
together); two products and their sum are rounded (1.8e-7); and the reference's angle, a product of 31 and 24 bits in
64, is off by 2^-23 (1.2e-7) at most: 1.25e-6."""
import pytest
import torch

from causal_refs import rotary_ref
from paper_2608_11519_gb300 import flarepp
from test_rotary_gpu import _device  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("real", [False, True])
@pytest.mark.parametrize("D,pairing", [(64, "halves"), (80, "halves"), (8, "adjacent"), (20, "axes")])
def test_angles(real, D, pairing):
    """80 channels are rows of pairs that no vector divides, 20 channels take single values."""
    N, P = 4000, D // 2 - 1 if D == 80 else D // 2
    g = torch.Generator().manual_seed(D)
    bits = 40 if real else 31
    pos = torch.exp2(torch.rand(1, N, 1, generator=g, dtype=torch.float64) * (bits - 1) + 1) - 1
    pos = pos * (1 - 2 * torch.randint(0, 2, pos.shape, generator=g))
    pos[0, :4, 0] = torch.tensor([2.0 ** 31 - 1, -2.0 ** 31, 2.0 ** 31 - 129, 16777217.0])
    pos = (pos.float() if real else pos.round().to(torch.int64).int()).cuda()
    freqs = torch.exp2(-6 * torch.rand(P, generator=g)).cuda()
    x = torch.randn(1, 2, N, D, generator=g).cuda()
    got, _ = flarepp.rotary_fwd(x, None, pos, freqs, [P], pairing)
    d = (got.double() - rotary_ref(x, pos, freqs, [P], pairing)).abs()
    for p in range(P):
        i, j = {"halves": (p, p + P), "adjacent": (2 * p, 2 * p + 1), "axes": (p, p + P)}[pairing]
        length = x[..., (i, j)].double().norm(dim=-1, keepdim=True)
        worst = float((d[..., (i, j)] / length).max())
        assert worst <= 1.25e-6, f"pair {p}: {worst:.3g} of its length"
