"""Rotary positions, decay attention and group norm as they are used together: a causal block
    q, k, v = heads of x Win^T, rotary(q, k), y = decay attention, n = silu(group norm by head of y), x + n Wo^T
its training step against autograd in 64 bits, and its prompt against token by token."""
import math

import pytest
import torch

from causal_refs import norm_ref, rotary_ref, walk
from paper_2608_11519_gb300 import flarepp

pytestmark = pytest.mark.gpu
H, D, SECTIONS = 4, 32, [8, 8]
C = H * D


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)
    yield
    assert flarepp.layers_status() == flarepp.OK


def model(seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    normal = lambda *s, std: (torch.randn(*s, generator=g, device="cuda") * std).bfloat16()
    p = {"Win": normal(3 * C, C, std=C ** -0.5), "Wo": normal(C, C, std=C ** -0.5),
         "gamma": (1 + normal(C, std=0.1)).bfloat16(), "beta": normal(C, std=0.1)}
    ld = torch.log1p(-torch.exp2(-torch.linspace(2, 6, H, dtype=torch.float64))).float().cuda()
    return p, ld, flarepp.rotary_frequencies(SECTIONS, base=100.0)


def places(N, width=16):
    t = torch.arange(N, device="cuda")
    return torch.stack((t // width, t % width), 1).int()


def split(z):
    return [z[..., i * C:(i + 1) * C].unflatten(-1, (H, D)).transpose(1, 2) for i in range(3)]


def forward(p, ld, freqs, x, pos, state=None):
    """What a training step keeps, with the output last and the state behind the last token first."""
    B, N, _ = x.shape
    z = flarepp.linear_fwd(x, p["Win"])
    q, k, v = split(z)
    q, k = flarepp.rotary_fwd(q, k, pos, freqs, SECTIONS, q_out=q, k_out=k)  # in place: parts of z
    y, last = flarepp.decay_attention_fwd(q, k, v, ld, state=state, need_state=True)
    rows = y.transpose(1, 2).reshape(B * N, 1, C)
    n, stats = flarepp.group_norm_fwd_train(rows, H, p["gamma"], p["beta"], act="silu")
    out = flarepp.linear_fwd(n.view(B, N, C), p["Wo"], residual=x)
    return last, (q, k, v), rows, stats, n, out


def backward(p, ld, freqs, x, pos, kept, dout):
    _, (q, k, v), rows, stats, n, _ = kept
    B, N, _ = x.shape
    dn, dWo, _ = flarepp.linear_bwd(n.view(B, N, C), p["Wo"], dout, bias=False)
    drows, dgamma, dbeta = flarepp.group_norm_bwd(rows, dn.view(B * N, 1, C), stats, H, p["gamma"], p["beta"],
                                                  act="silu")
    dz = torch.empty(B, N, 3 * C, dtype=x.dtype, device=x.device)
    dq, dk, dv = split(dz)
    flarepp.decay_attention_bwd(q, k, v, ld, drows.view(B, N, H, D).transpose(1, 2), dQ=dq, dK=dk, dV=dv)
    flarepp.rotary_bwd(dq, dk, pos, freqs, SECTIONS, dq_out=dq, dk_out=dk)
    dx, dWin, _ = flarepp.linear_bwd(x, p["Win"], dz, bias=False)
    return {"x": dx + dout, "Win": dWin, "Wo": dWo, "gamma": dgamma, "beta": dbeta}


def reference(p, ld, freqs, x, pos, dout):
    leaf = {k: t.double().requires_grad_() for k, t in dict(p, x=x).items()}
    B, N, _ = x.shape
    q, k, v = split(leaf["x"] @ leaf["Win"].t())
    turn = lambda t: torch.stack([t[..., i] for i in range(D)], -1)
    ang = torch.cat([pos[:, a:a + 1].double() * freqs[8 * a:8 * a + 8].double() for a in range(2)], 1)
    cos, sin = ang.cos(), ang.sin()

    def rot(t):
        a, b, rest = t[..., :16], t[..., 16:32], t[..., 32:]
        return torch.cat((a * cos - b * sin, b * cos + a * sin, rest), -1)

    gap = torch.arange(N, device="cuda").view(-1, 1) - torch.arange(N, device="cuda")
    w = torch.exp(gap.clamp(min=0) * ld.double().view(-1, 1, 1)) * (gap >= 0)
    y = ((rot(q) @ rot(k).transpose(-1, -2)) * w / math.sqrt(D)) @ v
    rows = y.transpose(1, 2).reshape(B * N, H, D)
    h = (rows - rows.mean(-1, keepdim=True)) * (rows.var(-1, correction=0, keepdim=True) + 1e-5).rsqrt()
    z = h.reshape(B, N, C) * leaf["gamma"] + leaf["beta"]
    out = leaf["x"] + (z * torch.sigmoid(z)) @ leaf["Wo"].t()
    grads = torch.autograd.grad((out * dout.double()).sum(), list(leaf.values()))
    return out.detach(), dict(zip(leaf, grads))


def test_training_step():
    """bf16 between the operators: some six stages that round to 2^-8 lie between a weight and the output or its
    gradient, so each agrees to a few per cent of its norm."""
    p, ld, freqs = model()
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(2, 300, C, generator=g, device="cuda").bfloat16()
    dout = torch.randn(2, 300, C, generator=g, device="cuda").bfloat16()
    pos = places(300)
    kept = forward(p, ld, freqs, x, pos)
    grads = backward(p, ld, freqs, x, pos, kept, dout)
    out, want = reference(p, ld, freqs, x, pos, dout)
    assert float((kept[-1].double() - out).norm() / out.norm()) <= 1e-2
    for k, t in want.items():
        off = float((grads[k].double() - t).norm() / t.norm())
        assert off <= 5e-2, f"{k}: {off:.3g}"


def test_step_from_a_captured_graph():
    """A whole training step captured and replayed on new inputs gives what the same calls give."""
    p, ld, freqs = model()
    g = torch.Generator(device="cuda").manual_seed(2)
    x, dout = (torch.randn(1, 2000, C, generator=g, device="cuda").bfloat16() for _ in range(2))
    pos = places(2000)
    forward(p, ld, freqs, x, pos)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = forward(p, ld, freqs, x, pos)
        grads = backward(p, ld, freqs, x, pos, kept, dout)
    x.copy_(torch.randn(1, 2000, C, generator=g, device="cuda"))
    graph.replay()
    want_kept = forward(p, ld, freqs, x, pos)
    want = backward(p, ld, freqs, x, pos, want_kept, dout)
    assert torch.equal(kept[-1], want_kept[-1])
    for k in want:
        assert torch.equal(grads[k], want[k]), k


def test_prompt_then_token_by_token():
    """The block over a prompt, then one token at a time from the state that it leaves, is the block over all of
    them: each token's output agrees to roundings (2^-8) of what goes into it."""
    p, ld, freqs = model()
    g = torch.Generator(device="cuda").manual_seed(3)
    x = torch.randn(2, 150, C, generator=g, device="cuda").bfloat16()
    pos = places(150)
    whole = forward(p, ld, freqs, x, pos)[-1].double()
    state = forward(p, ld, freqs, x[:, :130].contiguous(), pos[:130])[0]
    for t in range(130, 150):
        xt = x[:, t:t + 1].contiguous()
        q, k, v = split(flarepp.linear_fwd(xt, p["Win"]))
        q, k = flarepp.rotary_fwd(q, k, pos[t:t + 1], freqs, SECTIONS)
        y = flarepp.decay_attention_step(q[:, :, 0], k[:, :, 0], v[:, :, 0], ld, state)
        n = flarepp.group_norm_fwd(y.reshape(2, 1, C), H, p["gamma"], p["beta"], act="silu")
        out = flarepp.linear_fwd(n, p["Wo"], residual=xt)
        assert float((out[:, 0].double() - whole[:, t]).norm() / whole[:, t].norm()) <= 1e-2


def test_references_agree():
    """The tests' plain forms against the formulas written another way."""
    g = torch.Generator(device="cuda").manual_seed(4)
    f = lambda *s: torch.randn(*s, generator=g, device="cuda", dtype=torch.float64)
    q, k, v = f(1, 2, 20, 8), f(1, 2, 20, 8), f(1, 2, 20, 4)
    ld = torch.tensor([-0.1, -2.0], dtype=torch.float64, device="cuda")
    gap = torch.arange(20, device="cuda").view(-1, 1) - torch.arange(20, device="cuda")
    w = torch.exp(gap.clamp(min=0) * ld.view(-1, 1, 1)) * (gap >= 0)
    y, _ = walk(q, k, v, ld.exp(), torch.zeros(1, 2, 8, 4, dtype=torch.float64, device="cuda"))
    assert torch.allclose(y, (q @ k.transpose(-1, -2) * w) @ v)
    pos = torch.randint(0, 9, (1, 20, 1), generator=g, device="cuda")
    r = rotary_ref(q, pos, torch.ones(4), [4], "halves")
    z = torch.complex(q[..., :4], q[..., 4:]) * torch.exp(1j * pos.double()).unsqueeze(1)
    assert torch.allclose(r, torch.cat((z.real, z.imag), -1))
    x = f(2, 30, 12)
    want = torch.nn.functional.group_norm(x.transpose(1, 2), 3).transpose(1, 2)
    assert torch.allclose(norm_ref(x, 3, None, None, 1e-5, "none")["Y"], want)
