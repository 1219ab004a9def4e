"""How exact what the decay attention makes of a state is: two bf16 of it in a product's operand where keys or values
have up to 64 channels, one where both have more; which a bound for all terms at once does not tell."""
import math

import pytest
import torch

from causal_refs import U, walk
from paper_2608_11519_gb300 import flarepp
from test_decay_gpu import _device, tensor  # noqa: F401

pytestmark = pytest.mark.gpu


def beyond(got, ref, most, wide):
    """How many values are further off than the output's own rounding, the state's (U of itself, or U of what the first
    bf16 leaves) and float32 sums' 1e-5 of the terms' magnitudes allow."""
    bound = U * ref.abs() + ((U if wide else U * U) + 1e-5) * (1 + U) * most + 1e-30
    return int(((got.double() - ref).abs() > bound).sum())


@pytest.mark.parametrize("N", [1, 100, 128, 300])
@pytest.mark.parametrize("Dk,Dv", [(64, 64), (32, 16), (128, 64), (64, 128), (40, 104), (128, 128), (72, 72)])
def test_what_a_state_gives(Dk, Dv, N):
    """Nothing is added to the state (keys, queries or dY of zeros), so that outputs are its products alone: Y and dQ
    of the state in front, dK and dV of the gradient behind."""
    B, H = 1, 3
    wide = Dk > 64 and Dv > 64
    ld = torch.tensor([0.0, math.log(0.99), math.log(0.6)], device="cuda")
    g, c = ld.double().exp(), 1 / math.sqrt(Dk)
    q, k, v, dy = (tensor(i, B, H, N, D) for i, D in ((1, Dk), (2, Dk), (3, Dv), (4, Dv)))
    S, G = (tensor(i, B, H, Dk, Dv, dtype=torch.float32) for i in (5, 6))
    zk, zv = torch.zeros_like(k), torch.zeros_like(v)
    t = lambda x: x.transpose(-1, -2)
    got = {"Y": flarepp.decay_attention_fwd(q, zk, zv, ld, state=S)[0],
           "dQ": flarepp.decay_attention_bwd(q, zk, zv, ld, dy, state=S)[0]}
    _, got["dK"], got["dV"], _ = flarepp.decay_attention_bwd(torch.zeros_like(q), k, v, ld, torch.zeros_like(dy),
                                                             dstate_out=G)
    for name, x, da, dv, state, back, s in (("Y", q, Dk, Dv, S, False, c), ("dQ", dy, Dv, Dk, t(S), False, c),
                                            ("dK", v, Dv, Dk, t(G), True, 1.0), ("dV", k, Dk, Dv, G, True, 1.0)):
        a, w = torch.zeros(B, H, N, da, device="cuda").double(), torch.zeros(B, H, N, dv, device="cuda").double()
        x = x.double() * s
        ref, _ = walk(x, a, w, g, state.double(), back)
        most, _ = walk(x.abs(), a, w, g, state.double().abs(), back)
        assert beyond(got[name], ref, most, wide) == 0, name
        if not wide:  # a state of one bf16 would be seen
            one, _ = walk(x, a, w, g, state.bfloat16().double(), back)
            assert beyond(one.bfloat16(), ref, most, wide) > 0, name
