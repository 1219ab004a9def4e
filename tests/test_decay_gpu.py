"""The decay attention (flarepp_decay_attention_*) against its recurrences in 64 bits; causal_refs.py
derives the bounds."""
import math

import pytest
import torch

from causal_refs import U, decay_refs, walk, within
from paper_2608_11519_gb300 import flarepp

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    yield
    assert flarepp.layers_status() == flarepp.OK


def tensor(seed, *shape, std=1.0, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)


def heads(seed, B, H, N, D, last=False, std=1.0):
    return (tensor(seed, B, N, H, D, std=std).transpose(1, 2) if last else tensor(seed, B, H, N, D, std=std))


def decays(H):
    """From no memory at all to nothing forgotten."""
    ld = torch.log1p(-torch.exp2(-torch.linspace(0.5, 12, max(H, 2), dtype=torch.float64))).float()
    ld[-1] = 0.0
    if H > 2:
        ld[0] = -math.inf
    return ld[:H].cuda()


def inputs(B, Hq, Hk, N, Dk, Dv, last=False, state=True, n=None):
    q, k, v = (heads(i, B, H, N, D, last) for i, H, D in ((1, Hq, Dk), (2, Hk, Dk), (3, Hk, Dv)))
    dy = heads(4, B, Hq, N, Dv, last, std=0.1)
    S = tensor(5, n or B, Hq, Dk, Dv, std=2.0, dtype=torch.float32) if state else None
    G = tensor(6, n or B, Hq, Dk, Dv, std=0.1, dtype=torch.float32) if state else None
    return q, k, v, decays(Hq), dy, S, G


def check(q, k, v, ld, dy, S, G, scale=None):
    c = 1 / math.sqrt(q.shape[-1]) if scale is None else scale
    ref = decay_refs(q, k, v, ld, c, S, dy, G)
    Y, out = flarepp.decay_attention_fwd(q, k, v, ld, scale, S, need_state=True)
    dQ, dK, dV, dS = flarepp.decay_attention_bwd(q, k, v, ld, dy, scale, S, dstate_out=G, need_dstate=True)
    for name, got in (("Y", Y), ("state", out), ("dQ", dQ), ("dK", dK), ("dV", dV), ("dstate", dS)):
        within(got, *ref[name], name)


@pytest.mark.parametrize("N", [1, 2, 31, 33, 127, 128, 129, 300])
def test_lengths(N):
    check(*inputs(2, 3, 3, N, 64, 64))


@pytest.mark.parametrize("Dk,Dv", [(8, 8), (32, 32), (40, 72), (64, 128), (128, 64), (128, 128), (104, 16)])
@pytest.mark.parametrize("last", [False, True])
def test_widths_and_layouts(Dk, Dv, last):
    check(*inputs(2, 4, 4, 200, Dk, Dv, last))


@pytest.mark.parametrize("Hq,Hk", [(4, 1), (6, 2), (8, 8), (1, 1)])
@pytest.mark.parametrize("state", [False, True])
def test_grouped_heads(Hq, Hk, state):
    check(*inputs(1, Hq, Hk, 261, 64, 64, True, state))


def test_scale_zero_and_negative():
    for scale in (0.0, -0.7):
        check(*inputs(1, 2, 2, 140, 32, 32), scale=scale)


@pytest.mark.parametrize("B,H,N,D", [(1, 2, 5000, 64), (1, 1, 9001, 128), (3, 4, 2500, 32)])
def test_long_sequences_are_cut_and_joined(B, H, N, D):
    check(*inputs(B, H, H, N, D, D))


@pytest.mark.parametrize("Dk,Dv", [(64, 128), (128, 64), (40, 104), (96, 24), (128, 128)])
def test_cut_sequences_of_unlike_widths(Dk, Dv):
    """The states in front of the parts of one gradient's walk are those of another's, turned."""
    check(*inputs(1, 2, 1, 1700, Dk, Dv))


@pytest.mark.parametrize("Dk,Dv", [(64, 128), (128, 24)])
def test_packed_and_cut(Dk, Dv):
    """Parts that begin in front of a sequence's first chunk, at it and behind it; empty sequences among them."""
    lens = [0, 1, 700, 0, 0, 128, 129, 3, 900, 256, 0]
    cuts = [5]
    for n in lens:
        cuts.append(cuts[-1] + n)
    q, k, v, ld, dy, S, G = inputs(1, 4, 2, cuts[-1] + 3, Dk, Dv, n=len(lens))
    off = torch.tensor(cuts, dtype=torch.int32, device="cuda")
    Y, out = flarepp.decay_attention_fwd(q, k, v, ld, state=S, offsets=off, need_state=True)
    dQ, dK, dV, dS = flarepp.decay_attention_bwd(q, k, v, ld, dy, state=S, offsets=off, dstate_out=G,
                                                 need_dstate=True)
    for i, (a, b) in enumerate(zip(cuts, cuts[1:])):
        part = [x[:, :, a:b] for x in (q, k, v)]
        ref = decay_refs(*part, ld, 1 / math.sqrt(Dk), S[i:i + 1], dy[:, :, a:b], G[i:i + 1])
        for name, got in (("Y", Y), ("dQ", dQ), ("dK", dK), ("dV", dV)):
            within(got[:, :, a:b], *ref[name], f"{name} of sequence {i}")
        within(out[i:i + 1], *ref["state"], f"state of sequence {i}")
        within(dS[i:i + 1], *ref["dstate"], f"dstate of sequence {i}")


OFFSETS = {"even": [0, 128, 256, 400], "ragged": [3, 4, 4, 131, 133, 389, 390], "one": [0, 400],
           "empty": [7, 7, 7], "tail": [0, 50, 129]}


@pytest.mark.parametrize("kind", OFFSETS)
@pytest.mark.parametrize("Hq,Hk,Dk,Dv", [(3, 3, 64, 64), (4, 2, 32, 128)])
def test_packed_sequences(kind, Hq, Hk, Dk, Dv):
    """Each sequence as by itself; what lies outside all of them is no number, is not met, and is 0 behind."""
    cuts, N = OFFSETS[kind], 400
    n = len(cuts) - 1
    q, k, v, ld, dy, S, G = inputs(1, Hq, Hk, N, Dk, Dv, n=n)
    outside = torch.ones(N, dtype=torch.bool, device="cuda")
    outside[cuts[0]:cuts[-1]] = False
    for t in (q, k, v, dy):
        t[:, :, outside] = math.nan
    off = torch.tensor(cuts, dtype=torch.int32, device="cuda")
    Y, out = flarepp.decay_attention_fwd(q, k, v, ld, state=S, offsets=off, need_state=True)
    dQ, dK, dV, dS = flarepp.decay_attention_bwd(q, k, v, ld, dy, state=S, offsets=off, dstate_out=G,
                                                 need_dstate=True)
    for t in (Y, dQ, dK, dV):
        assert not bool(t[:, :, outside].any())
    for i, (a, b) in enumerate(zip(cuts, cuts[1:])):
        part = [x[:, :, a:b] for x in (q, k, v)]
        ref = decay_refs(*part, ld, 1 / math.sqrt(Dk), S[i:i + 1], dy[:, :, a:b], G[i:i + 1])
        for name, got in (("Y", Y), ("dQ", dQ), ("dK", dK), ("dV", dV)):
            within(got[:, :, a:b], *ref[name], f"{name} of sequence {i}")
        within(out[i:i + 1], *ref["state"], f"state of sequence {i}")
        within(dS[i:i + 1], *ref["dstate"], f"dstate of sequence {i}")


def test_packed_long_and_many():
    """Sequences of several pieces among thousands of short ones (more than one block of the cut)."""
    lens = [3000] + [i % 5 for i in range(2100)] + [1500, 0, 1]
    cuts = [0]
    for n in lens:
        cuts.append(cuts[-1] + n)
    q, k, v, ld, dy, _, _ = inputs(1, 2, 2, cuts[-1] + 9, 64, 64, state=False)
    off = torch.tensor(cuts, dtype=torch.int32, device="cuda")
    Y, out = flarepp.decay_attention_fwd(q, k, v, ld, offsets=off, need_state=True)
    dQ, dK, dV, _ = flarepp.decay_attention_bwd(q, k, v, ld, dy, offsets=off)
    for i in (0, 1, 4, 7, 1027, 2100, 2101, 2102, 2103):
        a, b = cuts[i], cuts[i + 1]
        ref = decay_refs(q[:, :, a:b], k[:, :, a:b], v[:, :, a:b], ld, 0.125, None, dy[:, :, a:b])
        for name, got in (("Y", Y), ("dQ", dQ), ("dK", dK), ("dV", dV)):
            within(got[:, :, a:b], *ref[name], f"{name} of sequence {i}")
        within(out[i:i + 1], *ref["state"], f"state of sequence {i}")


def test_bad_offsets_and_decays_are_recorded():
    q, k, v, ld, _, _, _ = inputs(1, 2, 2, 100, 32, 32, state=False)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    bad = torch.tensor([-5, 60, 40, 2000], dtype=torch.int32, device="cuda")
    Y, _ = flarepp.decay_attention_fwd(q, k, v, ld, offsets=bad, status=status)
    assert int(status) == flarepp.ERR_INVALID_ARGUMENT
    good = torch.tensor([0, 60, 60, 100], dtype=torch.int32, device="cuda")
    assert torch.equal(Y, flarepp.decay_attention_fwd(q, k, v, ld, offsets=good)[0])
    for wrong, taken in ((0.5, 0.0), (math.nan, -math.inf)):
        status.zero_()
        a, b = ld.clone(), ld.clone()
        a[0], b[0] = wrong, taken
        Y, _ = flarepp.decay_attention_fwd(q, k, v, a, status=status)
        assert int(status) == flarepp.ERR_INVALID_ARGUMENT
        assert torch.equal(Y, flarepp.decay_attention_fwd(q, k, v, b)[0])
        S = tensor(9, 1, 2, 32, 32, dtype=torch.float32)
        S2 = S.clone()
        one = (q[:, :, 0], k[:, :, 0], v[:, :, 0])
        status.zero_()
        y = flarepp.decay_attention_step(*one, a, S, status=status)
        assert int(status) == flarepp.ERR_INVALID_ARGUMENT
        assert torch.equal(y, flarepp.decay_attention_step(*one, b, S2)) and torch.equal(S, S2)


def test_parts_of_one_buffer_and_shared_heads():
    """Operands that are parts of one projection, gradients written into parts of one buffer, and heads
    that are one and the same (stride 0)."""
    B, N, H, D = 2, 150, 3, 64
    qkv, ld = tensor(1, B, N, 3, H, D), decays(H)
    q, k, v = (qkv[:, :, i].transpose(1, 2) for i in range(3))
    dy = heads(4, B, H, N, D, True, 0.1)
    grads = torch.full_like(qkv, math.nan)
    parts = [grads[:, :, i].transpose(1, 2) for i in range(3)]
    ref = decay_refs(q, k, v, ld, 0.125, None, dy)
    flarepp.decay_attention_bwd(q, k, v, ld, dy, dQ=parts[0], dK=parts[1], dV=parts[2])
    for name, got in zip(("dQ", "dK", "dV"), parts):
        within(got, *ref[name], name)
    one = k[:, :1].expand(B, H, N, D)
    Y, _ = flarepp.decay_attention_fwd(q, one, v, ld)
    within(Y, *decay_refs(q, one, v, ld, 0.125, None)["Y"], "Y with one key head for all")
    both = q[:1].expand(B, H, N, D)
    Y, _ = flarepp.decay_attention_fwd(both, k, v, ld)
    within(Y, *decay_refs(both, k, v, ld, 0.125, None)["Y"], "Y with one batch element's queries")


def test_cut_sequences_go_on_in_place():
    """40 heads of 29 chunks in parts of 8: blocks that end a sequence, and write its state, are done long before
    the one that begins with it comes to its state."""
    q, k, v, ld, dy, S, G = inputs(1, 40, 40, 29 * 128 - 5, 32, 32)
    Y, out = flarepp.decay_attention_fwd(q, k, v, ld, state=S, need_state=True)
    dQ, dK, dV, dS = flarepp.decay_attention_bwd(q, k, v, ld, dy, state=S, dstate_out=G, need_dstate=True)
    for _ in range(5):
        s, g = S.clone(), G.clone()
        Y1, s1 = flarepp.decay_attention_fwd(q, k, v, ld, state=s, state_out=s)
        grads = flarepp.decay_attention_bwd(q, k, v, ld, dy, state=S, dstate_out=g, dstate=g)
        for a, b in zip((Y, out, dQ, dK, dV, dS), (Y1, s1) + tuple(grads)):
            assert torch.equal(a, b)


def test_a_sequence_in_parts_goes_on_in_place():
    """Prompt, further prompt and single tokens, the state kept in one buffer."""
    B, H, N, D = 2, 4, 330, 64
    q, k, v, ld, _, _, _ = inputs(B, H, H, N, D, D, state=False)
    ref = decay_refs(q, k, v, ld, 0.125, None)
    S = torch.zeros(B, H, D, D, device="cuda")
    for a, b in ((0, 200), (200, 201), (201, 325)):
        part = [x[:, :, a:b] for x in (q, k, v)]
        Y, _ = flarepp.decay_attention_fwd(*part, ld, state=S, state_out=S)
        within(Y, ref["Y"][0][:, :, a:b], ref["Y"][1][:, :, a:b], f"Y of {a} to {b}")
    for t in range(325, N):
        y = flarepp.decay_attention_step(q[:, :, t], k[:, :, t], v[:, :, t], ld, S)
        within(y, ref["Y"][0][:, :, t], ref["Y"][1][:, :, t], f"y of {t}")
    within(S, *ref["state"], "state")


@pytest.mark.parametrize("B,Hq,Hk,Dk,Dv", [(1, 8, 8, 64, 64), (5, 6, 2, 128, 128), (3, 2, 1, 40, 8),
                                           (2, 1, 1, 8, 120)])
def test_step(B, Hq, Hk, Dk, Dv):
    """float32 throughout: 2^-20 of the sums of magnitudes, and Y's rounding."""
    q, k, v = tensor(1, B, Hq, Dk), tensor(2, B, Hk, Dk), tensor(3, B, Hk, Dv)
    S, ld = tensor(5, B, Hq, Dk, Dv, std=3.0, dtype=torch.float32), decays(Hq)
    group = Hq // Hk
    f = lambda t: t.double().repeat_interleave(group, 1)
    g = ld.double().exp()[None, :, None, None]
    add = f(k)[..., None] * f(v)[..., None, :]
    want, most = S.double() * g + add, S.double().abs() * g + add.abs()
    c = Dk ** -0.5
    y = (q.double()[..., None] * want).sum(-2) * c
    ya = (q.double().abs()[..., None] * most).sum(-2) * c
    Y = flarepp.decay_attention_step(q, k, v, ld, S)
    within(S, want, 2.0 ** -20 * most + 1e-30, "state")
    within(Y, y, U * y.abs() + 2.0 ** -20 * ya + 1e-30, "Y")


def test_gradients_are_the_differences():
    """The slope of sum(Y dY) + sum(state dstate) along a random direction of each input, by differences of
    the recurrence in 64 bits (which is bilinear in each input: exact but for rounding), is the
    gradient's product with the direction, within the gradients' bounds."""
    q, k, v, ld, dy, S, G = inputs(1, 4, 2, 150, 32, 64)
    c = 32 ** -0.5
    ref = decay_refs(q, k, v, ld, c, S, dy, G)
    names = ("dQ", "dK", "dV", "dstate")
    got = flarepp.decay_attention_bwd(q, k, v, ld, dy, state=S, dstate_out=G, need_dstate=True)
    g = ld.double().exp()

    def loss(q, k, v, S):
        y, last = walk(q * c, k.repeat_interleave(2, 1), v.repeat_interleave(2, 1), g, S)
        return float((y * dy.double()).sum() + (last * G.double()).sum())

    at = [x.double() for x in (q, k, v, S)]
    for i, name in enumerate(names):
        d = tensor(20 + i, *at[i].shape).double()
        up, down = list(at), list(at)
        up[i], down[i] = at[i] + d / 2, at[i] - d / 2
        slope = loss(*up) - loss(*down)
        bound = float((ref[name][1] * d.abs()).sum()) + 1e-9 * abs(slope)
        assert abs(float((got[i].double() * d).sum()) - slope) <= bound, name


def test_repeats_streams_and_graphs():
    """The same bits again, on another stream, and from a captured graph replayed on new inputs, with a
    workspace of the graph's own."""
    q, k, v, ld, dy, S, G = inputs(1, 2, 2, 3000, 64, 64)
    call = lambda **kw: flarepp.decay_attention_bwd(q, k, v, ld, dy, state=S, dstate_out=G,
                                                    need_dstate=True, **kw)
    fwd = lambda **kw: flarepp.decay_attention_fwd(q, k, v, ld, state=S, need_state=True, **kw)
    first = call() + fwd()
    again = call() + fwd()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    other = call(stream=side) + fwd(stream=side)
    side.synchronize()
    for a, b, c in zip(first, again, other):
        assert torch.equal(a, b) and torch.equal(a, c)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        inside = call() + fwd()
    new = tensor(77, 1, 2, 3000, 64)
    q.copy_(new)
    graph.replay()
    want = call() + fwd()
    torch.cuda.synchronize()
    for a, b in zip(inside, want):
        assert torch.equal(a, b)


@pytest.mark.parametrize("Dk,Dv", [(128, 64), (64, 128), (128, 128), (64, 64)])
def test_runs_agree(Dk, Dv):
    """Walks of many chunks with many others behind them: a wait that returns early shows as a difference."""
    q, k, v, ld, dy, _, _ = inputs(1, 8, 8, 30000, Dk, Dv, state=False)
    first, differ = None, torch.zeros(4, dtype=torch.int64, device="cuda")
    for _ in range(30):
        got = flarepp.decay_attention_bwd(q, k, v, ld, dy)[:3] + flarepp.decay_attention_fwd(q, k, v, ld)[:1]
        first = first or got
        differ += torch.stack([(a != b).any() for a, b in zip(first, got)])
    assert differ.tolist() == [0, 0, 0, 0]


def test_nothing_to_do():
    for B, H, N in ((0, 2, 5), (2, 0, 5), (2, 2, 0)):
        q = torch.zeros(B, H, N, 32, dtype=torch.bfloat16, device="cuda")
        ld = torch.zeros(H, device="cuda")
        S = torch.ones(B, H, 32, 32, device="cuda")
        Y, out = flarepp.decay_attention_fwd(q, q, q, ld, state=S, need_state=True)
        assert Y.shape == q.shape and torch.equal(out, S)
        grads = flarepp.decay_attention_bwd(q, q, q, ld, q, state=S, dstate_out=S, need_dstate=True)
        assert torch.equal(grads[3], S)
        zero, none = flarepp.decay_attention_fwd(q, q, q, ld)
        assert none is None


def test_a_wait_that_runs_out_is_reported():
    """The load warp leaves one of the first chunk's three tiles out (700 tokens of two heads are cut into
    pieces of a chunk): the waits end, the call reports it, and the next call is right."""
    q, k, v, ld, dy, S, G = inputs(1, 2, 2, 700, 64, 64)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    lib = flarepp.load()
    for item in (0, 1, 2):
        status.zero_()
        lib.flarepp_test_wait_fault(19, item, 20_000_000)
        try:
            flarepp.decay_attention_fwd(q, k, v, ld, status=status)
            torch.cuda.synchronize()
        finally:
            lib.flarepp_test_wait_fault(0, -1, 0)
        assert int(status) == flarepp.ERR_TIMEOUT
    check(q, k, v, ld, dy, S, G)
