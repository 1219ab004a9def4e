"""Cases that measure the operators around the token mixer: the linear layer with its epilogue
(bias, activation, residual), its training form and its gradients; the scaled embedding lookup
and the gradient of its table; and the AdamW step over all tensors of a model.

`run` computes them plainly (elementary torch operations in 32 bits, rounded once at the end), or,
where `own` is true, with the framework's kernels. `exact` gives the same outputs from the
definitions in 64 bits."""
import math

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
ACTS = ("none", "relu", "gelu", "silu")
BLOCK = 256       # values that share one scale in an 8-bit state
M_TOP = 256.0     # what the largest |m| of a block is stored as (8-bit float, 3 mantissa bits)
R_TOP = 16384.0   # what the largest sqrt(v) of a block is stored as (8 bits, 4 exponent, 4 mantissa)
TINY = 2.0 ** -100  # a block whose largest value is below this is stored as zeros
HYPER = {"lr": 1e-3, "betas": (0.9, 0.999), "eps": 1e-8, "weight_decay": 1e-2}
STEPS = 100       # steps that the optimiser's state has behind it


# ------------------------------------------------------------------ cases

def linear(name, mode, T, K, N, act="none", bias=True, residual=False):
    return {"name": name, "op": "linear", "mode": mode, "T": T, "K": K, "N": N, "act": act,
            "bias": bias, "residual": residual}


def embedding(name, mode, B, L, V, C, dtype, ids="i64", pad=0.0):
    return {"name": name, "op": "embedding", "mode": mode, "B": B, "L": L, "V": V, "C": C,
            "dtype": dtype, "ids": ids, "pad": pad}


def adamw(name, C, blocks, M, V, dtype, bits, master):
    return {"name": name, "op": "adamw", "C": C, "blocks": blocks, "M": M, "V": V,
            "dtype": dtype, "bits": bits, "master": master}


def listed():
    return [
        # serving: one token through a wide layer, where latency and the weight's bytes count
        linear("linear_one_token", "fwd", 1, 2048, 2048, "gelu"),
        # serving: the logits of a small batch of pooled sequences over an odd number of classes
        linear("linear_logits", "fwd", 48, 4096, 1001),
        # inference on 2D meshes (4 x 16,384 points, C = 256): the MLP's first layer, ratio 2
        linear("linear_mlp_up", "fwd", 4 * 16384, 256, 512, "gelu"),
        # inference on a mesh of a million points: the MLP's second layer with the block's residual
        linear("linear_mlp_down", "fwd", 1 << 20, 512, 256, residual=True),
        # a wide model's square layer: the tensor cores are the bound
        linear("linear_wide", "fwd", 16384, 4096, 4096, "silu", residual=True),
        # a training step of the MLP's first layer on long sequences (32 x 4,096 tokens)
        linear("linear_train", "train", 32 * 4096, 256, 512, "gelu"),
        # the backward alone, on a ragged batch of points and widths that no tile divides
        linear("linear_bwd_ragged", "bwd", 20011, 1000, 1544, "relu"),
        # serving: the lookup of one short sequence
        embedding("embedding_short", "fwd", 1, 257, 32000, 256, "bf16"),
        # training on byte sequences (32 x 4,096, padded): few rows, each met many times
        embedding("embedding_bytes", "train", 32, 4096, 257, 256, "bf16", pad=0.2),
        # the table's gradient for a large vocabulary, most of whose rows are met never or once
        embedding("embedding_vocab", "bwd", 64, 4096, 131072, 512, "f32", ids="i32"),
        # the optimiser of an eight-block model trained in 32 bits
        adamw("adamw_f32", 256, 8, 512, 257, "f32", 32, False),
        # the optimiser of a wide model: bf16 weights, 32-bit masters, states in 8 bits
        adamw("adamw_8bit", 1024, 16, 512, 32000, "bf16", 8, True),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    def width(lo, hi):  # most widths are powers of two or multiples of 8, as a model's are
        w, kind = log(lo, hi), rng.random()
        if kind < 0.25:
            return 2 ** max(3, round(math.log2(w)))
        return w if kind > 0.75 else max(8, w // 8 * 8)

    op = rng.choice(("linear", "linear", "embedding", "adamw"))
    if op == "linear":
        mode = rng.choice(("fwd", "fwd", "train", "bwd"))
        K, N = width(2, 3000), width(1, 3000)
        passes = {"fwd": 1, "bwd": 2, "train": 3}[mode]
        most = min(1 << 20, 5e11 / (2 * K * N * passes), 8e8 / ((K + N) * passes))
        c = linear("", mode, log(1, max(1, most)), K, N, rng.choice(ACTS),
                   rng.random() < 0.7, mode != "bwd" and rng.random() < 0.4)
    elif op == "embedding":
        C = width(16, 1024)
        L, V = log(1, 8192), log(2, 262144)
        V = max(2, min(V, (1 << 26) // C))
        B = log(1, max(1, (1 << 27) // (C * L)))
        c = embedding("", rng.choice(("fwd", "train", "bwd")), B, L, V, C,
                      rng.choice(("bf16", "f32")), rng.choice(("i32", "i64")),
                      rng.choice((0.0, 0.3)))
    else:
        C = width(16, 896)
        dtype = rng.choice(("bf16", "f32"))
        c = adamw("", C, rng.randint(1, 16), log(16, 1024), log(2, 32000), dtype,
                  rng.choice((8, 32)), dtype == "bf16" and rng.random() < 0.6)
    del c["name"]
    return c


def sizes(case):
    """Values in each tensor of a model: an embedding table, blocks of a mixer (input and output
    weights, seeds) and a two-layer MLP with biases, and a head."""
    C = case["C"]
    block = [4 * C * C, C * C, case["M"] * C, 2 * C * C, 2 * C, 2 * C * C, C]
    return [case["V"] * C] + block * case["blocks"] + [C * 10, 10]


def starts(case):
    """Where each tensor starts in a buffer that holds all of them, each at a whole block."""
    at, out = 0, []
    for n in sizes(case):
        out.append(at)
        at += -(-n // BLOCK) * BLOCK
    return out, at


# ------------------------------------------------------------------ inputs

def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, dtype=torch.bfloat16, std=1.0):
        return (torch.randn(*shape, generator=g, device="cuda") * std).to(dtype)

    s = {"case": case}
    if case["op"] == "linear":
        T, K, N = case["T"], case["K"], case["N"]
        s["X"] = normal(T, K)
        s["W"] = normal(N, K, std=K ** -0.5)
        s["b"] = normal(N, std=0.1) if case["bias"] else None
        s["R"] = normal(T, N) if case["residual"] else None
        s["dY"] = normal(T, N, std=1e-3) if case["mode"] != "fwd" else None
        s["Z"] = None
        if case["mode"] == "bwd" and case["act"] != "none":  # what a forward pass has kept
            s["Z"] = torch.matmul(s["X"], s["W"].t())
            if case["bias"]:
                s["Z"] += s["b"]
    elif case["op"] == "embedding":
        B, L, V, C = case["B"], case["L"], case["V"], case["C"]
        dtype = DTYPES[case["dtype"]]
        u = torch.rand(B, L, generator=g, device="cuda", dtype=torch.float64)
        ids = torch.exp(u * math.log(V + 1.0)).floor().long().sub_(1).clamp_(0, V - 1)
        if case["pad"]:  # sequences end early; what follows is -1
            ends = L * (1 - 2 * case["pad"] * torch.rand(B, 1, generator=g, device="cuda"))
            ids[torch.arange(L, device="cuda") >= ends] = -1
        s["ids"] = ids.to(torch.int32 if case["ids"] == "i32" else torch.int64)
        s["scale"] = math.sqrt(C)
        if case["mode"] != "bwd":
            s["table"] = normal(V, C, dtype=dtype, std=C ** -0.5)
        if case["mode"] != "fwd":
            s["dY"] = normal(B, L, C, dtype=dtype, std=1e-3)
    else:
        at, total = starts(case)
        ns = sizes(case)
        dtype = DTYPES[case["dtype"]]
        live = torch.zeros(total, dtype=torch.bool, device="cuda")
        for a, n in zip(at, ns):
            live[a:a + n] = True
        w = torch.randn(total, generator=g, device="cuda") * 0.02 * live
        # gradients differ in size from tensor to tensor and, by a heavy tail, within one
        grad = torch.randn(total, generator=g, device="cuda") * live
        grad = grad * grad.abs() * 1e-3
        r = (torch.randn(total, generator=g, device="cuda").abs() + 0.1) * 1e-3 * live
        m = torch.randn(total, generator=g, device="cuda") * 0.3 * r
        s["p"] = w.to(dtype)
        s["g"] = grad.to(dtype)
        s["w"] = w.clone() if case["master"] else None
        s["step"] = STEPS
        if case["bits"] == 8:
            s["m"], s["ms"] = pack_m(m)
            s["v"], s["vs"] = pack_r(r)
            s["m_out"], s["v_out"] = torch.zeros_like(m), torch.zeros_like(m)
        else:
            s["m"], s["v"], s["ms"], s["vs"] = m, r * r, None, None
        if own:
            s["opt"] = optimiser(s, at, ns)
    return s


def optimiser(s, at, ns):
    from paper_2608_11519_gb300 import flarepp

    def views(t, per=1):
        return None if t is None else [t[a // per:a // per + -(-n // per)] for a, n in zip(at, ns)]

    if s["ms"] is not None:
        s["m_views"], s["v_views"] = views(s["m_out"]), views(s["v_out"])
    return flarepp.AdamW(
        views(s["p"]), views(s["g"]), state_bits=s["case"]["bits"], masters=views(s["w"]),
        state={"m": views(s["m"]), "v": views(s["v"]), "m_scale": views(s["ms"], BLOCK),
               "v_scale": views(s["vs"], BLOCK), "step": s["step"]}, **HYPER)


# ------------------------------------------------------------------ one pass

def run(s):
    c = s["case"]
    if c["op"] == "linear":
        return run_linear_own(s) if own else run_linear(s)
    if c["op"] == "embedding":
        return run_embedding_own(s) if own else run_embedding(s)
    return run_adamw_own(s) if own else run_adamw(s)


def run_linear_own(s):
    from paper_2608_11519_gb300 import flarepp
    c, out = s["case"], {}
    Z = s["Z"]
    if c["mode"] == "fwd":
        return {"Y": flarepp.linear_fwd(s["X"], s["W"], s["b"], s["R"], c["act"])}
    if c["mode"] == "train":
        out["Y"], Z = flarepp.linear_fwd_train(s["X"], s["W"], s["b"], s["R"], c["act"])
        if Z is not None:
            out["Z"] = Z
    dX, dW, db = flarepp.linear_bwd(s["X"], s["W"], s["dY"], Z, c["act"], bias=c["bias"])
    out.update(dX=dX, dW=dW)
    if c["bias"]:
        out["db"] = db
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
    p = torch.sigmoid(z)
    return p * (1 + z * (1 - p))


def run_linear(s):
    c, out, dtype = s["case"], {}, s["X"].dtype
    X, W, Z = s["X"].float(), s["W"].float(), s["Z"]
    if c["mode"] != "bwd":
        z = X @ W.t()
        if s["b"] is not None:
            z = z + s["b"].float()
        Y = act_of(z, c["act"])
        if s["R"] is not None:
            Y = Y + s["R"].float()
        out["Y"] = Y.to(dtype)
        if c["mode"] == "fwd":
            return out
        if c["act"] != "none":
            out["Z"] = Z = z.to(dtype)
    dz = s["dY"].float()
    if c["act"] != "none":
        dz = dz * slope_of(Z.float(), c["act"])
    out["dX"] = (dz @ W).to(dtype)
    out["dW"] = (dz.t() @ X).to(dtype)
    if c["bias"]:
        out["db"] = dz.sum(0).to(dtype)
    return out


def run_embedding_own(s):
    from paper_2608_11519_gb300 import flarepp
    c, out = s["case"], {}
    if c["mode"] != "bwd":
        out["Y"] = flarepp.embedding_fwd(s["ids"], s["table"], s["scale"])
    if c["mode"] != "fwd":
        out["dtable"] = flarepp.embedding_bwd(s["ids"], s["dY"], c["V"], s["scale"])
    return out


def run_embedding(s):
    c, out, dtype = s["case"], {}, DTYPES[s["case"]["dtype"]]
    met = (s["ids"] >= 0).unsqueeze(-1)
    ids = s["ids"].clamp(min=0).long()
    if c["mode"] != "bwd":
        out["Y"] = (s["table"][ids].float() * s["scale"] * met).to(dtype)
    if c["mode"] != "fwd":
        rows = (s["dY"].float() * met).reshape(-1, c["C"])
        sums = torch.zeros(c["V"], c["C"], device=rows.device).index_add_(0, ids.reshape(-1), rows)
        out["dtable"] = (sums * s["scale"]).to(dtype)
    return out


def run_adamw_own(s):
    opt, out = s["opt"], {"p": s["p"]}
    opt.step()
    if s["w"] is not None:
        out["w"] = s["w"]
    if s["ms"] is None:
        return dict(out, m=s["m"], v=s["v"])
    opt.moments(s["m_views"], s["v_views"])
    return dict(out, m=s["m_out"], v=s["v_out"])


def scaled(x, top):
    """x in blocks of BLOCK, each block's largest value becoming `top`, and the largest values.
    A block of (almost) nothing becomes zeros with a scale of zero."""
    x = x.reshape(-1, BLOCK)
    most = x.abs().amax(1, keepdim=True)
    live = ~(most < TINY)  # a block that holds a NaN is not empty
    by = torch.full_like(most, top) / torch.where(live, most, 1.0)
    return x * by * live, torch.where(live, most, 0.0)


def pack_m(m):
    """A first moment as 8-bit floats (4 exponent bits, 3 mantissa bits) with a scale for each block."""
    y, most = scaled(m, M_TOP)
    return y.to(torch.float8_e4m3fn).reshape(-1), (most * (1 / M_TOP)).reshape(-1)


def unpack_m(code, scale):
    return (code.float().reshape(-1, BLOCK) * scale.unsqueeze(1)).reshape(-1)


def pack_r(r):
    """sqrt(v) in 8 bits without a sign: code c stands for c / 16 below 16, and above that for
    (1 + (c % 16) / 16) 2^(c // 16 - 1). A value that is not zero never becomes zero."""
    y, most = scaled(r, R_TOP)
    bits = y.view(torch.int32)
    high = ((bits + 0x3FFFF + ((bits >> 19) & 1)) >> 19) - (126 << 4)
    code = torch.where(y < 1, torch.round(y * 16).int(), high).clamp(0, 255)
    code = torch.where(y > 0, code.clamp(min=1), code)
    return code.to(torch.uint8).reshape(-1), (most * (1 / R_TOP)).reshape(-1)


def unpack_r(code, scale):
    c = code.to(torch.int32)
    y = torch.where(c < 16, c.float() * (1 / 16), ((c + (126 << 4)) << 19).view(torch.float32))
    return (y.reshape(-1, BLOCK) * scale.unsqueeze(1)).reshape(-1)


def run_adamw(s):
    s["step"] += 1
    t, (b1, b2), lr = s["step"], HYPER["betas"], HYPER["lr"]
    small = s["ms"] is not None
    g = s["g"].float()
    w = (s["p"] if s["w"] is None else s["w"]).float()
    m = unpack_m(s["m"], s["ms"]) if small else s["m"]
    v = unpack_r(s["v"], s["vs"]).square() if small else s["v"]
    m = m * b1 + g * (1 - b1)
    v = v * b2 + g * g * (1 - b2)
    r = v.sqrt()
    over = r * (1 / math.sqrt(1 - b2 ** t)) + HYPER["eps"]
    w = w * (1 - lr * HYPER["weight_decay"]) - m / over * (lr / (1 - b1 ** t))
    s["p"].copy_(w)
    out = {"p": s["p"]}
    if s["w"] is not None:
        s["w"].copy_(w)
        out["w"] = s["w"]
    if not small:
        s["m"], s["v"] = m, v
        return dict(out, m=m, v=v)
    s["m"], s["ms"] = pack_m(m)
    s["v"], s["vs"] = pack_r(r)
    return dict(out, m=unpack_m(s["m"], s["ms"]), v=unpack_r(s["v"], s["vs"]).square())


# ------------------------------------------------------------------ what one pass costs

def work(case):
    if case["op"] == "linear":
        T, K, N, e = case["T"], case["K"], case["N"], 2
        x, w, y = T * K * e, N * K * e, T * N * e
        b, kept = N * e * case["bias"], y * (case["act"] != "none")
        fwd = x + w + b + y * (2 if case["residual"] else 1)
        bwd = x + w + y + kept + x + w + b
        flops = 2.0 * T * K * N
        return {"fwd": {"bytes": fwd, "flops": flops}, "bwd": {"bytes": bwd, "flops": 2 * flops},
                "train": {"bytes": fwd + bwd + kept, "flops": 3 * flops}}[case["mode"]]
    if case["op"] == "embedding":
        T, V, C = case["B"] * case["L"], case["V"], case["C"]
        e, i = (2 if case["dtype"] == "bf16" else 4), (4 if case["ids"] == "i32" else 8)
        met = min(V, T)  # the most rows that are read
        fwd, bwd = T * i + met * C * e + T * C * e, T * i + T * C * e + V * C * e
        return {"bytes": {"fwd": fwd, "bwd": bwd, "train": fwd + bwd}[case["mode"]],
                "flops": T * C * {"fwd": 1, "bwd": 1, "train": 2}[case["mode"]]}
    n = sum(sizes(case))
    e = 2 if case["dtype"] == "bf16" else 4
    per = e + (8 if case["master"] else e) + e  # gradient; weights (and masters), both ways
    if case["bits"] == 8:  # states both ways with their scales, and the values they stand for
        return {"bytes": n * (per + 4 + 16.0 / BLOCK + 8), "flops": 20.0 * n}
    return {"bytes": n * (per + 16.0), "flops": 15.0 * n}


# ------------------------------------------------------------------ the definitions in 64 bits

def exact(case, seed):
    if case["op"] == "linear" and 2.0 * case["T"] * case["K"] * case["N"] > 3e12:
        return None
    s = prepare(case, seed)
    return {"linear": exact_linear, "embedding": exact_embedding, "adamw": exact_adamw}[case["op"]](s)


def exact_linear(s):
    c, f = s["case"], {k: v.double() for k, v in s.items() if torch.is_tensor(v)}
    phi = torch.distributions.Normal(0.0, 1.0)
    out = {}
    zeros = torch.zeros((), dtype=torch.float64, device="cuda")
    z = f.get("Z")
    if c["mode"] != "bwd":
        z = torch.einsum("tk,nk->tn", f["X"], f["W"]) + f.get("b", zeros)
        value = {"none": lambda: z, "relu": lambda: torch.where(z > 0, z, 0.0),
                 "gelu": lambda: z * torch.special.ndtr(z), "silu": lambda: z / (1 + torch.exp(-z))}
        out["Y"] = value[c["act"]]() + f.get("R", zeros)
        if c["mode"] == "fwd":
            return out
        if c["act"] != "none":
            out["Z"] = z
    dz = f["dY"]
    if c["act"] == "relu":
        dz = torch.where(z > 0, dz, 0.0)
    elif c["act"] == "gelu":
        dz = dz * (torch.special.ndtr(z) + z * phi.log_prob(z).exp())
    elif c["act"] == "silu":
        e = torch.exp(-z)
        dz = dz * ((1 + e + z * e) / (1 + e) ** 2)
    out["dX"] = torch.einsum("tn,nk->tk", dz, f["W"])
    out["dW"] = torch.einsum("tn,tk->nk", dz, f["X"])
    if c["bias"]:
        out["db"] = torch.einsum("tn->n", dz)
    return out


def exact_embedding(s):
    c, out = s["case"], {}
    ids = s["ids"].long().reshape(-1)
    here = torch.nonzero(ids >= 0).reshape(-1)
    if c["mode"] != "bwd":
        Y = torch.zeros(ids.numel(), c["C"], dtype=torch.float64, device="cuda")
        Y[here] = s["table"].double()[ids[here]] * s["scale"]
        out["Y"] = Y.reshape(c["B"], c["L"], c["C"])
    if c["mode"] != "fwd":
        total = torch.zeros(c["V"], c["C"], dtype=torch.float64, device="cuda")
        rows = s["dY"].reshape(-1, c["C"])[here].double() * s["scale"]
        out["dtable"] = total.index_put_((ids[here],), rows, accumulate=True)
    return out


def nearest(y, bits, low):
    """The float with `bits` mantissa bits next to y; below 2^low the steps stay those of 2^low."""
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** low))) - bits)
    return torch.round(y / step) * step


def exact_adamw(s):
    c, h = s["case"], HYPER
    b1, b2 = h["betas"]
    t = s["step"] + 1
    g = s["g"].double()
    w = (s["w"] if c["master"] else s["p"]).double()
    if c["bits"] == 8:
        m = s["m"].to(torch.float64) * s["ms"].double().repeat_interleave(BLOCK)
        k = s["v"].to(torch.float64)
        r = torch.where(k < 16, k / 16, (1 + (k % 16) / 16) * torch.exp2(torch.floor(k / 16) - 1))
        v = (r * s["vs"].double().repeat_interleave(BLOCK)) ** 2
    else:
        m, v = s["m"].double(), s["v"].double()
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g ** 2
    m_hat, v_hat = m / (1 - b1 ** t), v / (1 - b2 ** t)
    w = w - h["lr"] * (m_hat / (v_hat.sqrt() + h["eps"]) + h["weight_decay"] * w)
    out = {"p": w}
    if c["master"]:
        out["w"] = w
    if c["bits"] == 8:
        by = m.view(-1, BLOCK).abs().amax(1).repeat_interleave(BLOCK).clamp(min=1e-300) / M_TOP
        m = nearest(m / by, 3, -6) * by
        r = v.sqrt()
        by = r.view(-1, BLOCK).amax(1).repeat_interleave(BLOCK).clamp(min=1e-300) / R_TOP
        v = (torch.where(r > 0, nearest(r / by, 4, 0).clamp(min=1 / 16), 0.0) * by) ** 2
    return dict(out, m=m, v=v)
