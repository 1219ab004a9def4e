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


@pytest.mark.parametrize("kind", ["none", "some"])
@pytest.mark.parametrize("which", ["q", "k", "dy"])
@pytest.mark.parametrize("Dk,Dv", [(64, 64), (40, 128), (128, 128)])
def test_queries_and_keys(kind, which, Dk, Dv):
    """Rows of the other operands; in a walk of the gradients each of them is what is added to the state."""
    t = dict(zip(("q", "k", "v", "ld", "dy", "S", "G"), inputs(1, 3, 3, 300, Dk, Dv)))
    t["ld"] = memory(3, kind)
    at = [(0, 0, 100, 1), (0, 1, 127, 0), (0, 1, 200, 4), (0, 2, 299, 7)]
    for i, place in enumerate(at):
        t[which][place] = (math.nan, math.inf, -math.inf)[i % 3]
    check(*t.values())


@pytest.mark.parametrize("kind", ["none", "some"])
@pytest.mark.parametrize("N", [1, 70, 300])
@pytest.mark.parametrize("Dk,Dv", [(64, 64), (128, 64), (40, 128), (128, 128), (16, 32)])
def test_values(kind, N, Dk, Dv):
    """Values that are no numbers, several of them in one chunk and channel."""
    q, k, v, _, dy, S, G = inputs(2, 3, 3, N, Dk, Dv, last=True)
    places = [(0, 0, 0, 3), (0, 1, N - 1, Dv - 1), (0, 1, N // 2, 0), (1, 1, N // 3, 5), (1, 1, N // 2, 5),
              (1, 2, 2 * N // 3, Dv // 2)]
    for i, place in enumerate(places):
        v[place] = (math.nan, math.inf, -math.inf)[i % 3]
    check(q, k, v, memory(3, kind), dy, S, G)


@pytest.mark.parametrize("kind", ["none", "some"])
def test_cut_shared_and_long(kind):
    """Query heads that share a key head, in a sequence that blocks share; a whole token of no numbers."""
    q, k, v, _, dy, S, G = inputs(1, 4, 2, 1700, 64, 64)
    ld = memory(4, kind)
    v[0, 0, 900], k[0, 1, 1000, 5], dy[0, 1, 130, 2], q[0, 3, 1500, 3] = math.nan, math.inf, math.nan, -math.inf
    check(q, k, v, ld, dy, S, G)


@pytest.mark.parametrize("kind", ["none", "some"])
@pytest.mark.parametrize("count", [1, 60])
def test_packed_sequences_keep_to_themselves(kind, count):
    """Each sequence has values that are no numbers in its first or last token, or in none; with many sequences
    they are cut."""
    lens = [70, 1, 200, 0, 129, 55] * count
    cuts = [3]
    for n in lens:
        cuts.append(cuts[-1] + n)
    q, k, v, _, dy, S, G = inputs(1, 2, 2, cuts[-1] + 5, 64, 64, n=len(lens))
    ld = memory(2, kind)
    ends = [(i, a, b) for i, (a, b) in enumerate(zip(cuts, cuts[1:]))]
    for i, a, b in ends:
        if b > a and i % 4 < 3:
            v[0, 0, b - 1 if i % 2 else a, 5] = math.nan
            k[0, 1, a if i % 2 else b - 1, 7] = math.inf
    off = torch.tensor(cuts, dtype=torch.int32, device="cuda")
    got = run(q, k, v, ld, dy, S, G, off)
    for i, a, b in ends[:12]:
        part = [x[:, :, a:b] for x in (q, k, v)]
        ref = causal_refs.decay_refs(*part, ld, 0.125, S[i:i + 1], dy[:, :, a:b], G[i:i + 1])
        for name in NAMES:
            t = got[name]
            compare(t[i:i + 1] if "state" in name else t[:, :, a:b], ref[name], f"{name} of sequence {i}")


@pytest.mark.parametrize("kind", ["none", "some"])
def test_prompt_and_steps_agree(kind):
    """What a prompt makes of a state that is not finite is what its tokens make of it one by one."""
    B, H, N, D = 2, 3, 130, 64
    q, k, v, _, _, S, _ = inputs(B, H, H, N, D, D)
    ld = memory(H, kind)
    S[0, 0, 3, 3], S[1, 2, 60] = math.inf, math.nan
    v[0, 1, 40, 9] = math.inf
    Y, out = flarepp.decay_attention_fwd(q, k, v, ld, state=S, need_state=True)
    one = S.clone()
    for t in range(N):
        y = flarepp.decay_attention_step(q[:, :, t], k[:, :, t], v[:, :, t], ld, one)
        assert torch.equal(torch.isfinite(y), torch.isfinite(Y[:, :, t])), t
    assert torch.equal(torch.isfinite(one), torch.isfinite(out))
