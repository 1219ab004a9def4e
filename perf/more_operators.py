"""Cases that measure the operators of a causal block: linear attention with a decay for each head
(over whole prompts, its gradients, and its single-token step), rotary positions with several axes,
and group norm with an activation, channels last.

`run` computes them plainly (elementary torch operations in 32 bits, angles and long sums in 64,
rounded once at the end), or, where `own` is true, with the framework's kernels. `exact` gives the
same outputs from the definitions in 64 bits."""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ACTS = ("none", "relu", "gelu", "silu")
PAIRINGS = ("halves", "adjacent", "axes")
EPS = 1e-5
CHUNK = 256        # tokens that the plain form of a scan takes at a time
MOST_STEPS = 140000  # tokens that the 64-bit recurrence walks, one after the other


# ------------------------------------------------------------------ cases

def decay(name, mode, B, Hq, Hk, N, Dk, Dv, seqs=0, state=False, heads_last=False):
    """seqs: 0 for B sequences of N tokens each, else N tokens packed from that many sequences."""
    return {"name": name, "op": "decay", "mode": mode, "B": B, "Hq": Hq, "Hk": Hk, "N": N, "Dk": Dk,
            "Dv": Dv, "seqs": seqs, "state": state, "heads_last": heads_last}


def rotary(name, mode, B, Hq, Hk, N, D, sections, pairing, dtype="bf16", real=False, far=0,
           heads_last=False):
    """sections: how many pairs of channels turn with each axis. real: positions are coordinates in 32-bit floats. far: where the positions start."""
    return {"name": name, "op": "rotary", "mode": mode, "B": B, "Hq": Hq, "Hk": Hk, "N": N, "D": D,
            "sections": "-".join(map(str, sections)), "pairing": pairing, "dtype": dtype, "real": real, "far": far,
            "heads_last": heads_last}


def sections_of(case):
    return [int(n) for n in case["sections"].split("-")]


def norm(name, mode, B, N, C, G, act, dtype, affine=True, ragged=False):
    return {"name": name, "op": "norm", "mode": mode, "B": B, "N": N, "C": C, "G": G, "act": act,
            "dtype": dtype, "affine": affine, "ragged": ragged}


def listed():
    return [
        # serving: the next token of one sequence, where latency counts
        decay("decay_step_one", "step", 1, 8, 8, 1, 64, 64),
        # serving: the next tokens of a large batch with grouped heads, where the states' bytes count
        decay("decay_step_batch", "step", 256, 16, 4, 1, 128, 128),
        # serving: a short further prompt of a conversation, from the state that the last one left
        decay("decay_prompt", "fwd", 1, 8, 8, 300, 64, 64, state=True),
        # serving: a batch of prompts through a wide model with grouped heads, projections unsplit
        decay("decay_prefill", "fwd", 4, 32, 8, 8192, 128, 128, heads_last=True),
        # a training step on sequences of many lengths (32 x 4,096 tokens) packed into one
        decay("decay_train_packed", "train", 1, 8, 8, 32 * 4096, 32, 32, seqs=45),
        # the backward of one long sequence with few heads, wider values than keys
        decay("decay_bwd_long", "bwd", 1, 8, 8, 131072, 64, 128),
        # serving: queries and keys of a batch's next tokens, far into their sequences
        rotary("rotary_token", "fwd", 32, 32, 8, 1, 128, [64], "halves", far=1000000),
        # queries and keys on a mesh of a million points with real coordinates, an axis a block
        rotary("rotary_mesh", "fwd", 1, 8, 8, 1 << 20, 32, [6, 5, 5], "axes", real=True),
        # a training step on video (13 x 30 x 52 patches; time, height, width), projections unsplit
        rotary("rotary_video", "train", 2, 16, 16, 20280, 128, [16, 24, 24], "halves",
               heads_last=True),
        # the head norm behind one prompt's decay attention: every token by itself, 8 heads
        norm("norm_heads", "fwd", 300, 1, 512, 8, "silu", "bf16"),
        # training on 2D meshes (4 x 16,384 points, C = 256)
        norm("norm_mesh_train", "train", 4, 16384, 256, 32, "gelu", "bf16"),
        # the backward on a padded batch of large meshes, a width that no vector divides, 32 bits
        norm("norm_ragged_bwd", "bwd", 6, 99991, 250, 10, "silu", "f32", ragged=True),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(("decay", "decay", "rotary", "norm"))
    if op == "decay":
        mode = rng.choice(("step", "fwd", "train", "bwd"))
        Hk, group = rng.choice((1, 2, 4, 8)), rng.choice((1, 1, 2, 4))
        Dk = rng.choice((8, 24, 32, 40, 64, 64, 80, 128))
        Dv = Dk if rng.random() < 0.6 else rng.choice((16, 32, 64, 104, 128))
        Hq = Hk * group
        wide = Hq * max(Dk, Dv)
        if mode == "step":
            return dict(decay("", mode, log(1, max(1, min(512, (1 << 26) // (Hq * Dk * Dv)))), Hq, Hk, 1,
                              Dk, Dv))
        N = log(1, min(65536, (1 << 25) // wide))
        if rng.random() < 0.4:
            c = decay("", mode, 1, Hq, Hk, N, Dk, Dv, seqs=rng.randint(1, min(60, N)),
                      state=rng.random() < 0.3)
        else:
            c = decay("", mode, log(1, max(1, min(16, (1 << 25) // (wide * N)))), Hq, Hk, N, Dk, Dv,
                      state=rng.random() < 0.4, heads_last=rng.random() < 0.5)
    elif op == "rotary":
        D = rng.choice((16, 32, 48, 64, 80, 128))
        axes = rng.randint(1, 3)
        sections = [D // 2 // axes] * axes
        if rng.random() < 0.4:  # some channels are left as they are
            sections[0] = max(1, sections[0] - rng.randint(1, 4))
        dtype = rng.choice(("bf16", "f32"))
        Hk, group = rng.choice((1, 2, 4, 8)), rng.choice((1, 1, 4))
        N = log(1, min(300000, (1 << 27) // (Hk * (group + 1) * D)))
        B = log(1, max(1, min(64, (1 << 27) // (Hk * (group + 1) * D * N))))
        c = rotary("", rng.choice(("fwd", "train")), B, Hk * group, Hk, N, D, sections,
                   rng.choice(PAIRINGS), dtype, rng.random() < 0.3, rng.choice((0, 0, 100000)),
                   rng.random() < 0.5)
    else:
        G = rng.choice((1, 2, 5, 8, 16, 32))
        C = G * log(1, 64)
        N = log(1, min(300000, (1 << 27) // C))
        B = log(1, max(1, min(4096, (1 << 27) // (C * N))))
        c = norm("", rng.choice(("fwd", "train", "bwd")), B, N, C, G, rng.choice(ACTS),
                 rng.choice(("bf16", "f32")), rng.random() < 0.8, rng.random() < 0.3)
    del c["name"]
    return c


# ------------------------------------------------------------------ inputs

def cuts(case, seed):
    """Where the packed sequences begin, and where the last one ends (some rows may be left over)."""
    N, S = case["N"], case["seqs"]
    g = torch.Generator().manual_seed(seed)
    share = torch.rand(S, generator=g) + 0.02
    share = share * share  # a few long ones, many short ones
    ends = (torch.cumsum(share, 0) / share.sum() * (N - N // 200)).long()
    return [0] + ends.tolist()


def spans(case, seed):
    """The sequences of a case as (index in the batch, first token, one past the last)."""
    if case["seqs"]:
        at = cuts(case, seed)
        return [(0, a, b) for a, b in zip(at, at[1:])]
    return [(b, 0, case["N"]) for b in range(case["B"])]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.bfloat16, std=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)

    def heads(B, H, N, D, dtype=torch.bfloat16, std=1.0):  # [B, H, N, D] in either order of memory
        if case["heads_last"]:
            return normal(B, N, H, D, dtype=dtype, std=std).transpose(1, 2)
        return normal(B, H, N, D, dtype=dtype, std=std)

    s = {"case": case}
    if case["op"] == "decay":
        B, Hq, Hk, N, Dk, Dv = (case[k] for k in ("B", "Hq", "Hk", "N", "Dk", "Dv"))
        # decays from a few tokens' memory to thousands'
        power = torch.rand(Hq, generator=g, device="cuda", dtype=torch.float64) * 9 + 1
        s["log_decay"] = torch.log1p(-torch.exp2(-power)).float()
        if case["mode"] == "step":
            s["Q"], s["K"], s["V"] = normal(B, Hq, Dk), normal(B, Hk, Dk), normal(B, Hk, Dv)
            s["state"] = normal(B, Hq, Dk, Dv, dtype=torch.float32, std=4.0)
            return s
        s["Q"], s["K"], s["V"] = heads(B, Hq, N, Dk), heads(B, Hk, N, Dk), heads(B, Hk, N, Dv)
        s["spans"] = spans(case, seed)
        n = len(s["spans"])
        s["offsets"] = None
        if case["seqs"]:
            s["offsets"] = torch.tensor(cuts(case, seed), dtype=torch.int32, device="cuda")
        s["state"] = normal(n, Hq, Dk, Dv, dtype=torch.float32, std=4.0) if case["state"] else None
        if case["mode"] != "fwd":
            s["dY"] = heads(B, Hq, N, Dv, std=1e-2)
            s["dstate"] = None
            if case["state"]:
                s["dstate"] = normal(n, Hq, Dk, Dv, dtype=torch.float32, std=1e-2)
    elif case["op"] == "rotary":
        B, Hq, Hk, N, D = (case[k] for k in ("B", "Hq", "Hk", "N", "D"))
        axes, dtype = len(sections_of(case)), DTYPES[case["dtype"]]
        s["Q"], s["K"] = heads(B, Hq, N, D, dtype), heads(B, Hk, N, D, dtype)
        if case["mode"] == "train":
            s["dQ"], s["dK"] = heads(B, Hq, N, D, dtype, 1e-2), heads(B, Hk, N, D, dtype, 1e-2)
        base = 10000.0
        s["freqs"] = torch.cat([base ** (-torch.arange(n, dtype=torch.float64) / max(n, 1))
                                for n in sections_of(case)]).float().cuda()
        if case["real"]:
            s["positions"] = torch.rand(B, N, axes, generator=g, device="cuda") * 100
        else:
            side = max(1, round(N ** (1 / axes)))
            t = torch.arange(N, device="cuda").unsqueeze(1) // (
                side ** torch.arange(axes - 1, -1, -1, device="cuda"))
            t[:, 1:] %= side
            start = torch.randint(0, 1000, (B, 1, 1), generator=g, device="cuda") + case["far"]
            s["positions"] = (t + start).int().contiguous()
    else:
        B, N, C, G = (case[k] for k in ("B", "N", "C", "G"))
        dtype = DTYPES[case["dtype"]]
        mean = normal(1, 1, C, dtype=torch.float32)
        spread = normal(1, 1, C, dtype=torch.float32).abs() + 0.2
        s["X"] = (torch.randn(B, N, C, generator=g, device="cuda") * spread + mean).to(dtype)
        s["gamma"] = s["beta"] = s["lengths"] = None
        if case["affine"]:
            s["gamma"] = (1 + normal(C, dtype=torch.float32, std=0.2)).to(dtype)
            s["beta"] = normal(C, dtype=dtype, std=0.2)
        if case["ragged"]:
            s["lengths"] = torch.randint(N - N // 2, N + 1, (B,), generator=g, device="cuda",
                                         dtype=torch.int32)
        if case["mode"] != "fwd":
            s["dY"] = normal(B, N, C, dtype=dtype, std=1e-2)
        if case["mode"] == "bwd":  # what a forward pass has kept
            s["stats"] = statistics(s, torch.float64).float()
    return s


# ------------------------------------------------------------------ one pass

def run(s):
    op = s["case"]["op"]
    if own:
        return {"decay": decay_own, "rotary": rotary_own, "norm": norm_own}[op](s)
    return {"decay": decay_plain, "rotary": rotary_plain, "norm": norm_plain}[op](s)


def decay_own(s):
    from paper_2608_11519_gb300 import flarepp
    c, out = s["case"], {}
    args = (s["Q"], s["K"], s["V"], s["log_decay"])
    if c["mode"] == "step":
        out["Y"] = flarepp.decay_attention_step(*args, s["state"])
        return dict(out, state=s["state"])
    if c["mode"] != "bwd":
        out["Y"], state = flarepp.decay_attention_fwd(*args, state=s["state"], offsets=s["offsets"],
                                                      need_state=c["state"])
        if c["state"]:
            out["state"] = state
    if c["mode"] != "fwd":
        out["dQ"], out["dK"], out["dV"], dstate = flarepp.decay_attention_bwd(
            *args, s["dY"], state=s["state"], offsets=s["offsets"], dstate_out=s["dstate"],
            need_dstate=c["state"])
        if c["state"]:
            out["dstate"] = dstate
    return out


def rotary_own(s):
    from paper_2608_11519_gb300 import flarepp
    c, out = s["case"], {}
    how = (s["positions"], s["freqs"], sections_of(c), c["pairing"])
    out["Q"], out["K"] = flarepp.rotary_fwd(s["Q"], s["K"], *how)
    if c["mode"] == "train":
        out["dQ"], out["dK"] = flarepp.rotary_bwd(s["dQ"], s["dK"], *how)
    return out


def norm_own(s):
    from paper_2608_11519_gb300 import flarepp
    c, out = s["case"], {}
    how = {"gamma": s["gamma"], "beta": s["beta"], "act": c["act"], "lengths": s["lengths"]}
    stats = s.get("stats")
    if c["mode"] == "fwd":
        return {"Y": flarepp.group_norm_fwd(s["X"], c["G"], eps=EPS, **how)}
    if c["mode"] == "train":
        out["Y"], stats = flarepp.group_norm_fwd_train(s["X"], c["G"], eps=EPS, **how)
    out["dX"], dgamma, dbeta = flarepp.group_norm_bwd(s["X"], s["dY"], stats, c["G"], **how)
    if c["affine"]:
        out.update(dgamma=dgamma, dbeta=dbeta)
    return out


def scan(q, k, v, log_decay, S, back=False):
    """y_t = q_t S_t with S_t = g S_{t-1} + k_t v_t^T, in chunks, for [H, L, D] in 32 bits; returns
    y and the last state. Backwards, the sequence runs from its end and the state that is handed
    in has not yet been decayed (the one handed out has been)."""
    H, L = q.shape[:2]
    ld = log_decay.double().view(H, 1, 1)
    y = torch.empty(H, L, v.shape[-1], device=q.device)
    starts = range(0, L, CHUNK)
    first = 0 if back else 1
    for a in (reversed(starts) if back else starts):
        b = min(L, a + CHUNK)
        n = b - a
        i = torch.arange(n, device=q.device)
        gap = (i[:, None] - i[None, :]) * (-1 if back else 1)
        weight = (torch.exp(gap.clamp(min=0) * ld) * (gap >= 0)).float()
        since = (n - 1 - i if back else i).view(1, n, 1)
        rest = (n - 1 - since + (1 - first)) * ld
        qa, ka, va = q[:, a:b], k[:, a:b], v[:, a:b]
        y[:, a:b] = ((qa @ ka.transpose(1, 2)) * weight) @ va
        y[:, a:b] += torch.exp((since + first) * ld).float() * (qa @ S)
        S = torch.exp(n * ld).float() * S + ka.transpose(1, 2) @ (va * torch.exp(rest).float())
    return y, S


def decay_plain(s):
    c = s["case"]
    Hq, Hk, Dk, Dv = (c[k] for k in ("Hq", "Hk", "Dk", "Dv"))
    group, scale, ld = Hq // Hk, c["Dk"] ** -0.5, s["log_decay"]

    def spread(x):  # the heads of k and v, once for each head of q
        return x.float().repeat_interleave(group, 1)

    if c["mode"] == "step":
        g = torch.exp(ld.double()).float().view(1, Hq, 1, 1)
        k, v = spread(s["K"]), spread(s["V"])
        s["state"].mul_(g).add_(k.unsqueeze(-1) * v.unsqueeze(-2))
        Y = (s["Q"].float().unsqueeze(-1) * s["state"]).sum(-2) * scale
        return {"Y": Y.to(s["Q"].dtype), "state": s["state"]}
    out = {}
    fwd, bwd = c["mode"] != "bwd", c["mode"] != "fwd"
    B, N, dtype = c["B"], c["N"], s["Q"].dtype

    def blank(H, D):
        return torch.zeros(B, H, N, D, dtype=dtype, device="cuda")

    if fwd:
        out["Y"] = blank(Hq, Dv)
    if bwd:
        out.update(dQ=blank(Hq, Dk), dK=blank(Hk, Dk), dV=blank(Hk, Dv))
    if c["state"]:
        if fwd:
            out["state"] = torch.empty_like(s["state"])
        if bwd:
            out["dstate"] = torch.empty_like(s["state"])
    zero = torch.zeros(Hq, Dk, Dv, device="cuda")
    for n, (b, lo, hi) in enumerate(s["spans"]):
        q = s["Q"][b, :, lo:hi].float() * scale
        k, v = (x[b, :, lo:hi].float().repeat_interleave(group, 0) for x in (s["K"], s["V"]))
        S = s["state"][n] if c["state"] else zero
        if fwd:
            y, last = scan(q, k, v, ld, S)
            out["Y"][b, :, lo:hi] = y
            if c["state"]:
                out["state"][n] = last
        if bwd:
            dy = s["dY"][b, :, lo:hi].float()
            G = s["dstate"][n] if c["state"] else zero
            out["dQ"][b, :, lo:hi] = scan(dy, v, k, ld, S.transpose(1, 2))[0] * scale
            dk, _ = scan(v, dy, q, ld, G.transpose(1, 2), back=True)
            dv, first = scan(k, q, dy, ld, G, back=True)
            out["dK"][b, :, lo:hi] = dk.view(Hk, group, hi - lo, Dk).sum(1)
            out["dV"][b, :, lo:hi] = dv.view(Hk, group, hi - lo, Dv).sum(1)
            if c["state"]:
                out["dstate"][n] = first
    return out


def places(case):
    """The two channels of every pair, and the axis of every pair."""
    sections, first, second, axis, at = sections_of(case), [], [], [], 0
    P = sum(sections)
    for a, n in enumerate(sections):
        for i in range(n):
            p = at + i
            x, y = {"halves": (p, p + P), "adjacent": (2 * p, 2 * p + 1),
                    "axes": (2 * at + i, 2 * at + n + i)}[case["pairing"]]
            first.append(x)
            second.append(y)
            axis.append(a)
        at += n
    return first, second, axis


def rotary_plain(s):
    c, out = s["case"], {}
    first, second, axis = (torch.tensor(x, device="cuda") for x in places(c))
    angle = s["positions"].double()[..., axis] * s["freqs"].double()
    cos, sin = (f(angle).float().unsqueeze(1) for f in (torch.cos, torch.sin))

    def turned(x, sin):
        y = x.clone()
        a, b = x[..., first].float(), x[..., second].float()
        y[..., first] = (a * cos - b * sin).to(x.dtype)
        y[..., second] = (b * cos + a * sin).to(x.dtype)
        return y

    out["Q"], out["K"] = turned(s["Q"], sin), turned(s["K"], sin)
    if c["mode"] == "train":
        out["dQ"], out["dK"] = turned(s["dQ"], -sin), turned(s["dK"], -sin)
    return out


def act_of(z, act):
    if act == "relu":
        return z.clamp(min=0)
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "silu":
        return z * torch.sigmoid(z)
    return z


def slope_of(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return (0.5 * (1 + torch.erf(z * math.sqrt(0.5)))
                + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi)))
    if act == "silu":
        p = torch.sigmoid(z)
        return p * (1 + z * (1 - p))
    return torch.ones_like(z)


def live_rows(s):
    """[B, N, 1] truth values: rows before their sample's length."""
    c = s["case"]
    n = torch.arange(c["N"], device="cuda").view(1, -1, 1)
    lengths = torch.full((c["B"],), c["N"], device="cuda") if s["lengths"] is None else s["lengths"]
    return n < lengths.view(-1, 1, 1)


def statistics(s, dtype):
    """Mean and 1 / deviation of every sample and group, [B, 2, G], over the rows that are live."""
    c = s["case"]
    B, N, C, G = (c[k] for k in ("B", "N", "C", "G"))
    x = s["X"].to(dtype).view(B, N, G, C // G)
    live = live_rows(s).unsqueeze(-1)
    count = (live.sum((1, 2, 3)) * (C // G)).clamp(min=1).view(B, 1).double()
    mean = ((x * live).sum((1, 3), dtype=torch.float64) / count).to(dtype)
    gap = (x - mean.view(B, 1, G, 1)) * live
    var = (gap * gap).sum((1, 3), dtype=torch.float64) / count
    return torch.stack((mean, torch.rsqrt(var + EPS).to(dtype)), 1)


def norm_plain(s):
    c, out, dtype = s["case"], {}, s["X"].dtype
    B, N, C, G = (c[k] for k in ("B", "N", "C", "G"))
    live = live_rows(s)
    stats = s["stats"] if c["mode"] == "bwd" else statistics(s, torch.float32)
    mean, rstd = (stats[:, i].repeat_interleave(C // G, 1).view(B, 1, C) for i in (0, 1))
    xhat = (s["X"].float() - mean) * rstd
    z = xhat
    if c["affine"]:
        z = xhat * s["gamma"].float() + s["beta"].float()
    if c["mode"] != "bwd":
        out["Y"] = torch.where(live, act_of(z, c["act"]), 0.0).to(dtype)
        if c["mode"] == "fwd":
            return out
    dz = torch.where(live, s["dY"].float() * slope_of(z, c["act"]), 0.0)
    g = dz
    if c["affine"]:
        out["dgamma"] = (dz * xhat).sum((0, 1), dtype=torch.float64).to(dtype)
        out["dbeta"] = dz.sum((0, 1), dtype=torch.float64).to(dtype)
        g = dz * s["gamma"].float()
    count = (live.sum((1, 2)) * (C // G)).clamp(min=1).view(B, 1).double()

    def mean_of(x):
        m = x.view(B, N, G, C // G).sum((1, 3), dtype=torch.float64) / count
        return m.float().repeat_interleave(C // G, 1).view(B, 1, C)

    dx = rstd * (g - mean_of(g) - xhat * mean_of(g * xhat))
    out["dX"] = torch.where(live, dx, 0.0).to(dtype)
    return out


# ------------------------------------------------------------------ what one pass costs

def work(case):
    if case["op"] == "decay":
        B, Hq, Hk, N, Dk, Dv = (case[k] for k in ("B", "Hq", "Hk", "N", "Dk", "Dv"))
        n = case["seqs"] or B
        state = n * Hq * Dk * Dv * 4
        q, k, v, y = (2 * B * H * N * D for H, D in ((Hq, Dk), (Hk, Dk), (Hk, Dv), (Hq, Dv)))
        flops = 4.0 * B * Hq * N * Dk * Dv  # a token's state, and its row of it
        if case["mode"] == "step":
            return {"bytes": q + k + v + y + 2 * state, "flops": flops * 1.5}
        fwd = {"bytes": q + k + v + y + 2 * state * case["state"], "flops": flops}
        bwd = {"bytes": 2 * (q + k + v) + y + 3 * state * case["state"], "flops": 2.5 * flops}
        if case["mode"] == "fwd":
            return fwd
        return bwd if case["mode"] == "bwd" else {k: fwd[k] + bwd[k] for k in fwd}
    if case["op"] == "rotary":
        e, passes = (2 if case["dtype"] == "bf16" else 4), (2 if case["mode"] == "train" else 1)
        rows = case["B"] * case["N"]
        n = rows * (case["Hq"] + case["Hk"]) * case["D"]
        return {"bytes": passes * (2 * n * e + rows * len(sections_of(case)) * 4),
                "flops": passes * 3.0 * n}
    e = 2 if case["dtype"] == "bf16" else 4
    n = case["B"] * case["N"] * case["C"]
    passes = {"fwd": 2, "bwd": 3, "train": 5}[case["mode"]]
    return {"bytes": passes * n * e, "flops": 10.0 * passes * n}


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "decay":
        if case["mode"] == "step":
            return exact_step(s)
        if max(hi - lo for _, lo, hi in s["spans"]) > MOST_STEPS:
            return None
        return exact_decay(s)
    return exact_rotary(s) if case["op"] == "rotary" else exact_norm(s)


def exact_step(s):
    c = s["case"]
    kv = torch.arange(c["Hq"], device="cuda") // (c["Hq"] // c["Hk"])
    k, v = s["K"].double()[:, kv], s["V"].double()[:, kv]
    S = s["state"].double() * s["log_decay"].double().exp()[:, None, None]
    S += torch.einsum("bhk,bhv->bhkv", k, v)
    return {"Y": torch.einsum("bhk,bhkv->bhv", s["Q"].double(), S) / math.sqrt(c["Dk"]), "state": S}


def exact_decay(s):
    """The recurrences, token by token; all sequences at once, padded to the longest: tokens in
    front (k, v and dY of zero) where the walk starts, so that all end together."""
    c = s["case"]
    Hq, Hk, Dk, Dv, B, N = (c[k] for k in ("Hq", "Hk", "Dk", "Dv", "B", "N"))
    f64, sp = torch.float64, s["spans"]
    L, n = max(hi - lo for _, lo, hi in sp), len(sp)
    kv = torch.arange(Hq, device="cuda") // (Hq // Hk)
    g = s["log_decay"].double().exp().view(1, Hq, 1, 1)
    sizes = torch.tensor([hi - lo for _, lo, hi in sp], device="cuda")

    def padded(x, heads=None):  # [L, sequences, heads, D], each sequence from its first token on
        x = x if heads is None else x[:, heads]
        out = torch.zeros(L, n, x.shape[1], x.shape[3], dtype=x.dtype, device="cuda")
        for i, (b, lo, hi) in enumerate(sp):
            out[:hi - lo, i] = x[b, :, lo:hi].transpose(0, 1)
        return out

    def put(rows):  # back to [B, H, N, D]
        out = torch.zeros(B, rows.shape[2], N, rows.shape[3], dtype=f64, device="cuda")
        for i, (b, lo, hi) in enumerate(sp):
            out[b, :, lo:hi] = rows[:hi - lo, i].transpose(0, 1)
        return out

    def start(x):
        return torch.zeros(n, Hq, Dk, Dv, dtype=f64, device="cuda") if x is None else x.double()

    scale = 1 / math.sqrt(Dk)
    Q, K, V = padded(s["Q"]), padded(s["K"], kv), padded(s["V"], kv)
    dY = padded(s["dY"]) if c["mode"] != "fwd" else None
    # g for a step inside the sequence, 1 for one behind its end (where k = v = 0)
    ragged = int(sizes.min()) < L
    out, S = {}, start(s["state"])
    rows = [torch.empty(L, n, Hq, D, dtype=f64, device="cuda") for D in (Dv, Dk)]
    for t in range(L):
        S = S * (torch.where((t < sizes).view(n, 1, 1, 1), g, 1.0) if ragged else g)
        S.addcmul_(K[t].double().unsqueeze(-1), V[t].double().unsqueeze(-2))
        if c["mode"] != "bwd":
            torch.sum(Q[t].double().unsqueeze(-1) * S, -2, out=rows[0][t])
        if c["mode"] != "fwd":
            torch.sum(dY[t].double().unsqueeze(-2) * S, -1, out=rows[1][t])
    if c["mode"] != "bwd":
        out["Y"] = put(rows[0] * scale)
        if c["state"]:
            out["state"] = S
    if c["mode"] == "fwd":
        return out
    out["dQ"] = put(rows[1] * scale)
    G = start(s["dstate"])  # what the state behind the last token is worth
    for t in reversed(range(L)):
        G.addcmul_((Q[t].double() * scale).unsqueeze(-1), dY[t].double().unsqueeze(-2))
        torch.sum(K[t].double().unsqueeze(-1) * G, -2, out=rows[0][t])
        torch.sum(V[t].double().unsqueeze(-2) * G, -1, out=rows[1][t])
        G = G * (torch.where((t < sizes).view(n, 1, 1, 1), g, 1.0) if ragged else g)
    for name, x in (("dV", rows[0]), ("dK", rows[1])):
        out[name] = put(x.view(L, n, Hk, Hq // Hk, -1).sum(3))
    if c["state"]:
        out["dstate"] = G
    return out


def exact_rotary(s):
    c, out = s["case"], {}
    turn = []  # [B, 1, N] unit complex numbers, one for each pair
    axis = [a for a, n in enumerate(sections_of(c)) for _ in range(n)]
    for p, a in enumerate(axis):
        angle = s["positions"][..., a].to(torch.float64) * float(s["freqs"][p])
        turn.append(torch.polar(torch.ones_like(angle), angle).unsqueeze(1))
    for name in ("Q", "K", "dQ", "dK"):
        if name not in s:
            continue
        x = s[name].double()
        for p, (i, j) in enumerate(zip(*places(c)[:2])):
            w = turn[p].conj() if name[0] == "d" else turn[p]
            z = torch.complex(s[name][..., i].double(), s[name][..., j].double()) * w
            x[..., i], x[..., j] = z.real, z.imag
        out[name] = x
    return out


def exact_norm(s):
    c, out = s["case"], {}
    B, N, C, G = (c[k] for k in ("B", "N", "C", "G"))
    w = C // G
    phi = torch.distributions.Normal(0.0, 1.0)
    names = ("Y",) * (c["mode"] != "bwd") + ("dX",) * (c["mode"] != "fwd")
    for name in names:
        out[name] = torch.zeros(B, N, C, dtype=torch.float64, device="cuda")
    sums = torch.zeros(2, C, dtype=torch.float64, device="cuda")
    gamma = s["gamma"].double() if c["affine"] else torch.ones(C, dtype=torch.float64, device="cuda")
    beta = s["beta"].double() if c["affine"] else torch.zeros_like(gamma)
    same = s["lengths"] is None  # then all samples go at once
    for b in [slice(None)] if same else [slice(i, i + 1) for i in range(B)]:
        n = N if same else int(s["lengths"][b])
        if n == 0:
            continue
        x = s["X"][b, :n].double().unflatten(-1, (G, w))
        if c["mode"] == "bwd":
            mean, rstd = (s["stats"][b, i].double().view(-1, 1, G, 1) for i in (0, 1))
        else:
            mean = x.mean((1, 3), keepdim=True)
            rstd = (x.var((1, 3), correction=0, keepdim=True) + EPS) ** -0.5
        h = ((x - mean) * rstd).flatten(-2)
        z = h * gamma + beta
        e = torch.exp(-z)
        if "Y" in out:
            out["Y"][b, :n] = {"none": lambda: z, "relu": lambda: torch.where(z > 0, z, 0.0),
                               "gelu": lambda: z * torch.special.ndtr(z),
                               "silu": lambda: z / (1 + e)}[c["act"]]()
        if c["mode"] == "fwd":
            continue
        slope = {"none": lambda: torch.ones_like(z), "relu": lambda: (z > 0).double(),
                 "gelu": lambda: torch.special.ndtr(z) + z * phi.log_prob(z).exp(),
                 "silu": lambda: (1 + e + z * e) / (1 + e) ** 2}[c["act"]]()
        dz = s["dY"][b, :n].double() * slope
        sums[0] += torch.einsum("bnc,bnc->c", dz, h)
        sums[1] += torch.einsum("bnc->c", dz)
        d, h = (dz * gamma).unflatten(-1, (G, w)), h.unflatten(-1, (G, w))
        dx = rstd * (d - d.mean((1, 3), keepdim=True) - h * (d * h).mean((1, 3), keepdim=True))
        out["dX"][b, :n] = dx.flatten(-2)
    if c["mode"] != "fwd" and c["affine"]:
        out["dgamma"], out["dbeta"] = sums[0], sums[1]
    return out
