"""Plain 64-bit forms of the decay attention, rotary positions and group norm, which their tests compare
with (imported by the tests, no tests of its own)."""
import math

import torch

U = 2.0 ** -8 * 1.01  # a rounding to bf16, relative


def within(got, ref, bound, what):
    got = got.double()
    assert bool(torch.isfinite(got).all()), f"{what}: not finite"
    d = (got - ref).abs()
    over = d > bound
    assert not bool(over.any()), (f"{what}: {int(over.sum())} of {d.numel()} beyond the bound, worst "
                                  f"{float((d / bound.clamp(min=1e-300)).max()):.3g} of it")


def walk(x, a, v, g, S, back=False):
    """y_t = x_t S_t, S_t = g S_(t-1) + a_t v_t^T, [.., N, D] and [.., Da, Dv]; backwards S enters undecayed
    and leaves decayed. Returns (y, S)."""
    N = x.shape[-2]
    y = torch.zeros(*x.shape[:-1], v.shape[-1], dtype=x.dtype, device=x.device)
    g = g[..., None, None]
    for t in (reversed(range(N)) if back else range(N)):
        if not back:
            S = S * g
        S = S + a[..., t, :, None] * v[..., t, None, :]
        y[..., t, :] = (x[..., t, None, :] @ S)[..., 0, :]
        if back:
            S = S * g
    return y, S


def decay_refs(Q, K, V, log_decay, scale, state, dY=None, dstate_out=None):
    """{name: (value, bound)} of a forward, and with dY of its gradients, for one batch of sequences. The
    bounds: an operand that is rounded to bf16 is off by U of itself, so by U of the sums of magnitudes
    of the terms that it is in. A term within a chunk has its score rounded once; one through the state has its
    value as two bf16, of which the second is off by U of what the first leaves, U of it, and the state
    the same again or (Dk and Dv above 64) rounded once: at most U + U^2 for either, and 2 U^2 else; then
    the output's own. Sums of float32 terms in chunks of 128 and powers of g from exponentials: 1e-5 of
    the sum of magnitudes."""
    Q, K, V = Q.double(), K.double(), V.double()
    group = Q.shape[1] // K.shape[1]
    g = log_decay.double().exp()
    Kr, Vr = K.repeat_interleave(group, 1), V.repeat_interleave(group, 1)
    zero = torch.zeros(*Q.shape[:2], Q.shape[-1], V.shape[-1], dtype=torch.float64, device=Q.device)
    S0 = zero if state is None else state.double()
    t = lambda x: x.transpose(-1, -2)
    out = {}

    def both(x, a, v, S, back=False, c=1.0):
        y, last = walk(x * c, a, v, g, S, back)
        ya, la = walk(x.abs() * abs(c), a.abs(), v.abs(), g, S.abs(), back)
        return y, (U + U * U) * ya + 1e-5 * ya, last, U * U * la + 1e-5 * la

    def put(name, y, e):
        out[name] = (y, e + U * y.abs() + 1e-30)

    y, e, S, se = both(Q, Kr, Vr, S0, c=scale)
    put("Y", y, e)
    out["state"] = (S, se + 1e-30)
    if dY is None:
        return out
    dY = dY.double()
    G = zero if dstate_out is None else dstate_out.double()
    y, e, _, _ = both(dY, Vr, Kr, t(S0), c=scale)
    put("dQ", y, e)
    heads = lambda x: x.unflatten(1, (-1, group)).sum(2)
    dk, ek, _, _ = both(Vr, dY, Q * scale, t(G), back=True)
    dv, ev, first, fe = both(Kr, Q * scale, dY, G, back=True)
    put("dK", heads(dk), heads(ek))
    put("dV", heads(dv), heads(ev))
    out["dstate"] = (first, fe + 1e-30)
    return out


def pairs(sections, pairing):
    P, at, out = sum(sections), 0, []
    for axis, n in enumerate(sections):
        for i in range(n):
            p = at + i
            out.append((axis, p) + {"halves": (p, p + P), "adjacent": (2 * p, 2 * p + 1),
                                    "axes": (2 * at + i, 2 * at + n + i)}[pairing])
        at += n
    return out


def rotary_ref(x, positions, freqs, sections, pairing, inverse=False):
    y, x = x.double().clone(), x.double()
    for axis, p, i, j in pairs(sections, pairing):
        a = positions[..., axis].double() * float(freqs[p])
        a = (-a if inverse else a).unsqueeze(-2)
        y[..., i] = x[..., i] * a.cos() - x[..., j] * a.sin()
        y[..., j] = x[..., j] * a.cos() + x[..., i] * a.sin()
    return y


def act64(z, act):
    return {"none": lambda: z, "relu": lambda: z.clamp(min=0),
            "gelu": lambda: 0.5 * z * (1 + torch.erf(z / math.sqrt(2))),
            "silu": lambda: z * torch.sigmoid(z)}[act]()


def norm_ref(X, G, gamma, beta, eps, act, lengths=None, dY=None):
    """{name: value} from the definition, the gradients by autograd in 64 bits."""
    B, N, C = X.shape
    x = X.detach().double().requires_grad_(dY is not None)
    one = torch.ones(C, dtype=torch.float64, device=X.device)
    ga = (one if gamma is None else gamma.detach().double()).clone().requires_grad_(dY is not None)
    be = (0 * one if beta is None else beta.detach().double()).clone().requires_grad_(dY is not None)
    rows, stats = [], torch.zeros(B, 2, G, dtype=torch.float64, device=X.device)
    for b in range(B):
        n = N if lengths is None else int(lengths[b])
        xb = x[b, :n].reshape(n, G, C // G)
        if n:
            mean = xb.mean((0, 2), keepdim=True)
            rstd = ((xb - mean).square().mean((0, 2), keepdim=True) + eps).rsqrt()
        else:
            mean = torch.zeros(1, G, 1, dtype=torch.float64, device=X.device)
            rstd = mean + eps ** -0.5
        stats[b, 0], stats[b, 1] = mean.detach()[0, :, 0], rstd.detach()[0, :, 0]
        y = act64(((xb - mean) * rstd).reshape(n, C) * ga + be, act)
        rows.append(torch.cat((y, torch.zeros(N - n, C, dtype=torch.float64, device=X.device))))
    Y = torch.stack(rows) if rows else x.clone()
    out = {"Y": Y.detach(), "stats": stats}
    if dY is not None:
        gx, gg, gb = torch.autograd.grad((Y * dY.double()).sum(), (x, ga, be))
        out.update(dX=gx, dgamma=gg, dbeta=gb)
    return out
