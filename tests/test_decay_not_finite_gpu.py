"""The decay attention with infinities and NaN among its operands: they reach what the recurrence lets them reach,
and nothing else. No earlier token (in the gradients' walks from the end: no later one), no other sequence, and
no further than their own token where nothing is remembered (log_decay -inf). What they do reach is not finite;
all else is within the bounds of causal_refs.py."""
import math

import pytest
import torch

import causal_refs
from paper_2608_11519_gb300 import flarepp
from test_decay_gpu import _device, inputs  # noqa: F401

pytestmark = pytest.mark.gpu
NAMES = ("Y", "state", "dQ", "dK", "dV", "dstate")


def walk(x, a, v, g, S, back=False):
    """causal_refs.walk that forgets, where g is 0, what is not finite too."""
    N = x.shape[-2]
    y = torch.zeros(*x.shape[:-1], v.shape[-1], dtype=x.dtype, device=x.device)
    g = g[..., None, None]
    decayed = lambda S: torch.where(g > 0, S * g, torch.zeros_like(S))
    for t in (reversed(range(N)) if back else range(N)):
        if not back:
            S = decayed(S)
        S = S + a[..., t, :, None] * v[..., t, None, :]
        y[..., t, :] = (x[..., t, :, None] * S).sum(-2)
        if back:
            S = decayed(S)
    return y, S


@pytest.fixture(autouse=True)
def _forgetting(monkeypatch):
    monkeypatch.setattr(causal_refs, "walk", walk)


def compare(got, ref, name):
    value, bound = ref
    finite = torch.isfinite(value)
    assert torch.equal(torch.isfinite(got), finite), (
        f"{name}: {int((torch.isfinite(got) & ~finite).sum())} values are finite that should not be, "
        f"{int((~torch.isfinite(got) & finite).sum())} are not that should be")
    zero = torch.zeros_like(value)
    causal_refs.within(torch.where(finite, got.double(), zero), torch.where(finite, value, zero),
                       torch.where(finite, bound, zero + 1e-30), name)


def run(q, k, v, ld, dy, S, G, offsets=None):
    Y, out = flarepp.decay_attention_fwd(q, k, v, ld, state=S, need_state=True, offsets=offsets)
    grads = flarepp.decay_attention_bwd(q, k, v, ld, dy, state=S, dstate_out=G, need_dstate=True, offsets=offsets)
    return dict(zip(NAMES, (Y, out) + tuple(grads)))


def check(q, k, v, ld, dy, S, G):
    ref = causal_refs.decay_refs(q, k, v, ld, 1 / math.sqrt(q.shape[-1]), S, dy, G)
    got = run(q, k, v, ld, dy, S, G)
    for name in NAMES:
        compare(got[name], ref[name], name)
    return ref


def memory(H, kind):
    """Decays of heads that remember for long and for short, or of ones that remember nothing."""
    if kind == "none":
        return torch.full((H,), -math.inf, device="cuda")
    return torch.tensor([math.log(g) for g in (1.0, 0.97, 0.5, 1e-9)][:H], device="cuda")


@pytest.mark.parametrize("kind", ["none", "some"])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("Dk,Dv", [(64, 64), (128, 64), (40, 128), (128, 128), (16, 32)])
def test_states(kind, bad, Dk, Dv):
    """A state, or its gradient, of which a value is not finite: forgotten with the rest of it, or kept."""
    q, k, v, _, dy, S, G = inputs(1, 3, 3, 300, Dk, Dv)
    ld = memory(3, kind)
    S[0, 1, 2, 5] = bad
    ref = check(q, k, v, ld, dy, S, G)
    assert bool(torch.isfinite(ref["Y"][0]).all()) == (kind == "none")
    G[0, 0, 7, 3], G[0, 2] = bad, bad
    check(q, k, v, ld, dy, S, G)
