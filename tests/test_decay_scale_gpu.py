"""The decay attention with scales far from 1: a scale moves every score alike, however small the powers of
the decay are that it meets within a chunk."""
import math

import pytest
import torch

from test_decay_gpu import _device, check, inputs  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [2.0 ** -12, -(2.0 ** -17), 2.0 ** -24, 2.0 ** -90, 2.0 ** 40])
@pytest.mark.parametrize("Dk,Dv", [(64, 64), (72, 128)])
def test_small_and_large_scales(scale, Dk, Dv):
    """Decays of a half and a little more, whose power over 127 tokens is near float32's smallest normal number."""
    q, k, v, _, dy, S, G = inputs(1, 4, 4, 261, Dk, Dv)
    ld = torch.tensor([math.log(g) for g in (0.5, 0.505, 0.6, 0.9)], device="cuda")
    check(q, k, v, ld, dy, S, G, scale)
