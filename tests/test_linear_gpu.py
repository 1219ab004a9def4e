"""The linear layer (flarepp_linear_fwd, flarepp_linear_bwd) against its definition in 64 bits.

Tolerances, element by element, from the arithmetic (u = 2^-8 is the rounding of a bf16 result):
  - a product of K terms is summed in float32 in steps of 16 terms, each of which may lose one unit
    of 2^-23 of the sum of magnitudes S so far, and at most 512 partial sums are added after that:
    (K / 16 + 8) 2^-23 S, doubled;
  - the activations and their slopes come from approximations good to 2e-7 and from
    reciprocals and exponentials good to 2^-21: 1e-6 (1 + |z|), and they change a sum's error by
    a factor of 1.13 at most;
  - dZ is rounded to bf16 before the products that make dX and dW: u of every |dZ| in them.
"""
import math

import pytest
import torch

from paper_2608_11519_gb300 import flarepp

pytestmark = pytest.mark.gpu
U = 2.0 ** -8 * 1.01


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def randn(*shape, seed, std=1.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * std).bfloat16()


def act64(z, act):
    return {"none": lambda: z, "relu": lambda: z.clamp(min=0),
            "gelu": lambda: z * torch.special.ndtr(z), "silu": lambda: z * torch.sigmoid(z)}[act]()


def slope64(z, act):
    if act == "none":
        return torch.ones_like(z)
    if act == "relu":
        return (z > 0).double()
    if act == "gelu":
        return torch.special.ndtr(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    s = torch.sigmoid(z)
    return s * (1 + z * (1 - s))


def sum_error(K):
    return 2 * (K / 16 + 8) * 2.0 ** -23


def within(got, ref, bound, what):
    d = (got.double() - ref).abs()
    over = d > bound
    assert not bool(over.any()), \
        f"{what}: {int(over.sum())} of {d.numel()} beyond the bound, worst {float((d / bound).max()):.3g} of it"
    assert torch.isfinite(got.double()).all(), what


def case(T, K, N, act, bias, residual, seed=3):
    X, W = randn(T, K, seed=seed), randn(N, K, seed=seed + 1, std=K ** -0.5)
    b = randn(N, seed=seed + 2) if bias else None
    R = randn(T, N, seed=seed + 3) if residual else None
    return X, W, b, R


def reference(X, W, b, R, act):
    """(Y, Z) in 64 bits and the bounds of their errors"""
    z = X.double() @ W.double().t()
    S = X.double().abs() @ W.double().abs().t()
    if b is not None:
        z, S = z + b.double(), S + b.double().abs()
    y = act64(z, act)
    r = torch.zeros_like(y) if R is None else R.double()
    dz = sum_error(X.shape[1]) * S
    dy = 1.13 * dz + 2.0 ** -23 * (y.abs() + r.abs()) + 1e-6 * (1 + z.abs()) * (act != "none")
    y = y + r
    return y, z, U * (y.abs() + dy) + dy, U * (z.abs() + dz) + dz


# tokens, inputs, outputs: one token; the few-token form's edges; tiles that end inside a
# block, a slice or a vector; widths that are no multiple of 8; several column tiles; cut contractions
SHAPES = [(1, 1, 1), (1, 64, 48), (1, 2048, 2048), (2, 7, 10), (3, 100, 1000), (5, 640, 33),
          (17, 4096, 129), (48, 1000, 1001), (127, 72, 136), (128, 256, 512), (129, 256, 512),
          (200, 8, 16), (256, 64, 64), (257, 2, 256), (300, 1000, 1544), (500, 4096, 40),
          (511, 65, 250), (1000, 256, 10), (1000, 24, 1), (2049, 512, 264), (4097, 40, 520),
          (30000, 256, 512), (40001, 520, 256)]


@pytest.mark.parametrize("T,K,N", SHAPES)
def test_forward(T, K, N):
    for i, act in enumerate(flarepp.ACTIVATIONS):
        for bias, residual in ((True, False), (False, True), (True, True))[i % 2::2]:
            X, W, b, R = case(T, K, N, act, bias, residual, seed=10 * i)
            Y = flarepp.linear_fwd(X, W, b, R, act)
            y, z, by, bz = reference(X, W, b, R, act)
            within(Y, y, by, f"Y {act} bias={bias} residual={residual}")
            Y2, Z = flarepp.linear_fwd_train(X, W, b, R, act)
            assert torch.equal(Y, Y2)
            if act == "none":
                assert Z is None
            else:
                within(Z, z, bz, f"Z {act}")


@pytest.mark.parametrize("T,K,N", SHAPES)
def test_backward(T, K, N):
    for i, act in enumerate(flarepp.ACTIVATIONS):
        X, W, b, _ = case(T, K, N, act, True, False, seed=10 * i)
        dY = randn(T, N, seed=77 + i)
        Z = None if act == "none" else (X.float() @ W.float().t() + b.float()).bfloat16()
        dX, dW, db = flarepp.linear_bwd(X, W, dY, Z, act)
        z = torch.zeros(T, N, dtype=torch.float64, device="cuda") if Z is None else Z.double()
        dz = dY.double() * slope64(z, act)
        off = (dY.double().abs() * (1e-6 * (1 + z.abs()) + 2.0 ** -23) if act != "none" else 0 * dz)
        mag = dz.abs() + off
        # act none multiplies dY as it is; else dZ is rounded first
        u = 0.0 if act == "none" else U
        dx, dw, dbr = dz @ W.double(), dz.t() @ X.double(), dz.sum(0)
        ex = (u + sum_error(N)) * (mag @ W.double().abs()) + off @ W.double().abs()
        ew = (u + sum_error(T)) * (mag.t() @ X.double().abs()) + off.t() @ X.double().abs()
        eb = T * 2.0 ** -24 * mag.sum(0) + off.sum(0)
        within(dX, dx, U * (dx.abs() + ex) + ex, f"dX {act}")
        within(dW, dw, U * (dw.abs() + ew) + ew, f"dW {act}")
        within(db, dbr, U * (dbr.abs() + eb) + eb, f"db {act}")


@pytest.mark.parametrize("act", list(flarepp.ACTIVATIONS))
def test_backward_against_differences(act):
    """The gradients along a direction against central differences of the forward in 64 bits."""
    T, K, N = 40, 72, 56
    X, W, b, _ = case(T, K, N, act, True, False, seed=5)
    dY = randn(T, N, seed=6)
    z0 = X.double() @ W.double().t() + b.double()
    if act == "relu":  # keep clear of the kink, which a difference would straddle
        dY = torch.where(z0.abs() < 1e-2, torch.zeros_like(dY), dY)
    _, Z = flarepp.linear_fwd_train(X, W, b, None, act)
    dX, dW, db = flarepp.linear_bwd(X, W, dY, Z, act)
    h = 1e-5

    def loss(x, w, c):
        return (act64(x @ w.t() + c, act) * dY.double()).sum()

    # Z is kept in bf16: a slope moves by at most 1.2 times Z's rounding (its second derivative
    # stays below 0.8 for gelu, 0.5 for silu), and dZ is rounded once more
    off = dY.double().abs() * (U * (1.2 * z0.abs() + 1.13) + 1e-5)
    args = [X.double(), W.double(), b.double()]
    bounds = [off @ W.double().abs(), off.t() @ X.double().abs(), off.sum(0)]
    for i, (g, slack) in enumerate(zip((dX, dW, db), bounds)):
        V = torch.randn(args[i].shape, generator=torch.Generator().manual_seed(i)).double().cuda()
        lo, hi = list(args), list(args)
        lo[i], hi[i] = args[i] - h * V, args[i] + h * V
        want = float((loss(*hi) - loss(*lo)) / (2 * h))
        got = float((g.double() * V).sum())
        bound = float(((slack + 2 * U * g.double().abs()) * V.abs()).sum()) + 1e-6 * abs(want)
        assert abs(got - want) <= bound, (i, got, want, bound)
        # the bound above is a worst case; rounding errors are independent, so hold the sum also to
        # six times their root of squares
        rms = float((((slack + 2 * U * g.double().abs()) * V) ** 2).sum()) ** 0.5
        assert abs(got - want) <= 6 * rms + 1e-6 * abs(want), (i, got, want, rms)


def test_gradients_left_out():
    X, W, b, _ = case(300, 64, 96, "gelu", True, False)
    dY, Z = randn(300, 96, seed=8), randn(300, 96, seed=9)
    full = flarepp.linear_bwd(X, W, dY, Z, "gelu")
    for need, bias in (((True, False), False), ((False, True), True), ((False, False), True)):
        part = flarepp.linear_bwd(X, W, dY, Z, "gelu", bias=bias, need=need)
        for keep, p, f in zip((*need, bias), part, full):
            assert (p is None) if not keep else torch.equal(p, f)


def test_leading_dimensions_and_empty():
    X, W, b, R = case(6 * 50, 64, 96, "gelu", True, True)
    flat = flarepp.linear_fwd(X, W, b, R, "gelu")
    Y = flarepp.linear_fwd(X.view(6, 50, 64), W, b, R.view(6, 50, 96), "gelu")
    assert Y.shape == (6, 50, 96) and torch.equal(Y.view(300, 96), flat)
    E = X[:0]
    assert flarepp.linear_fwd(E, W, b).shape == (0, 96)
    dW, db = torch.full_like(W, 7), torch.full_like(b, 7)
    dX, dW, db = flarepp.linear_bwd(E, W, E.new_empty(0, 96), dW=dW, db=db)
    assert dX.shape == (0, 64) and not dW.any() and not db.any()


@pytest.mark.parametrize("T", [4, 100, 700])
def test_special_values_stay_in_their_row(T):
    X, W, b, _ = case(T, 128, 200, "gelu", True, False)
    ref = flarepp.linear_fwd(X, W, b, None, "gelu")
    X2 = X.clone()
    X2[1, 5], X2[2, 7] = float("nan"), float("inf")
    Y = flarepp.linear_fwd(X2, W, b, None, "gelu")
    rows = torch.ones(T, dtype=torch.bool, device="cuda")
    rows[1:3] = False
    assert torch.equal(Y[rows], ref[rows])
    assert Y[1].isnan().all() and (~torch.isfinite(Y[2].float())).any()
    # relu keeps a NaN instead of turning it into a zero
    assert flarepp.linear_fwd(X2, W, b, None, "relu")[1].isnan().all()


@pytest.mark.parametrize("act", ["gelu", "silu"])
def test_activation_over_its_range(act):
    """Inputs of 1 x z cross the activation's whole range: tails keep their relative precision."""
    z = torch.linspace(-40, 40, 4001, device="cuda").bfloat16().view(-1, 1)
    one = torch.ones(1, 1, dtype=torch.bfloat16, device="cuda")
    Y = flarepp.linear_fwd(z, one, None, None, act).double()
    y = act64(z.double(), act)
    bound = U * y.abs() + 4e-7 * z.double().abs().clamp(min=1) + 1e-30
    assert bool(((Y - y).abs() <= bound).all())
    dX, _, _ = flarepp.linear_bwd(z, one, torch.ones_like(z), z, act)
    g = slope64(z.double(), act)
    assert bool(((dX.double() - g).abs() <= 2.1 * U * g.abs() + 2e-6).all())


@pytest.mark.parametrize("T,K,N", [(3, 256, 512), (90, 256, 200), (5000, 256, 512), (700, 1000, 100)])
def test_same_bits_again_and_nothing_outside(T, K, N):
    """Two calls give the same bits; the bytes around the outputs stay as they are."""
    X, W, b, R = case(T, K, N, "silu", True, True)
    dY = randn(T, N, seed=21)

    def fenced(*shape):
        n = math.prod(shape)
        buf = torch.full((n + 1024 + (-n) % 8,), 123.0, dtype=torch.bfloat16, device="cuda")
        return buf, buf[512:512 + n].view(*shape)

    outs = [fenced(T, N), fenced(T, N), fenced(T, K), fenced(N, K), fenced(N)]
    (_, Y), (_, Z), (_, dX), (_, dW), (_, db) = outs
    ws = flarepp.Workspace()
    first = None
    for _ in range(3):
        flarepp.linear_fwd_train(X, W, b, R, "silu", Y=Y, Z=Z, workspace=ws)
        flarepp.linear_bwd(X, W, dY, Z, "silu", dX=dX, dW=dW, db=db, workspace=ws)
        now = [t.clone() for _, t in outs]
        assert first is None or all(torch.equal(a, c) for a, c in zip(first, now))
        first = now
    for buf, t in outs:
        assert (buf[:512] == 123).all() and (buf[512 + t.numel():] == 123).all()


def test_on_another_stream():
    X, W, b, R = case(3000, 256, 512, "gelu", True, True)
    want = flarepp.linear_fwd(X, W, b, R, "gelu")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    Y = torch.empty_like(want)
    with torch.cuda.stream(s):
        flarepp.linear_fwd(X, W, b, R, "gelu", Y=Y)
    s.synchronize()
    assert torch.equal(Y, want)
    Y2 = torch.empty_like(want)
    ws = flarepp.Workspace()
    flarepp.linear_fwd(X, W, b, R, "gelu", Y=Y2, workspace=ws, stream=s)
    s.synchronize()
    assert torch.equal(Y2, want)


def test_in_a_graph():
    X, W, b, R = case(64, 512, 640, "gelu", True, True)
    ws, Y = flarepp.Workspace(), torch.empty(64, 640, dtype=torch.bfloat16, device="cuda")
    flarepp.linear_fwd(X, W, b, R, "gelu", Y=Y, workspace=ws)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        flarepp.linear_fwd(X, W, b, R, "gelu", Y=Y, workspace=ws)
    X.copy_(randn(64, 512, seed=99))
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(Y, flarepp.linear_fwd(X, W, b, R, "gelu"))


def test_more_than_2_to_31_values():
    T, K, N = 1_100_003, 8, 2048
    X, W = randn(T, K, seed=1), randn(N, K, seed=2)
    Y = flarepp.linear_fwd(X, W, None, None, "relu")
    for a in (0, T // 2, T - 300):
        y, _, by, _ = reference(X[a:a + 300], W, None, None, "relu")
        within(Y[a:a + 300], y, by, f"rows from {a}")
    dX, _, _ = flarepp.linear_bwd(X, W, Y, Y, "relu", bias=False, need=(True, False))
    dy = Y[-300:].double()
    ref = dy @ W.double()
    err = sum_error(N) * (dy.abs() @ W.double().abs())
    within(dX[-300:], ref, U * (ref.abs() + err) + err, "dX")


def test_refusals():
    X, W, b, R = case(10, 16, 24, "none", True, True)
    with pytest.raises(ValueError):
        flarepp.linear_fwd(X, W, b, act="tanh")
    with pytest.raises(ValueError):
        flarepp.linear_fwd(X, W[:, :8].contiguous())
    with pytest.raises(ValueError):
        flarepp.linear_fwd(X, W, b[:8])
    with pytest.raises(ValueError):
        flarepp.linear_fwd(X.t().contiguous().t(), W)
    with pytest.raises(TypeError):
        flarepp.linear_fwd(X, W.float())
    with pytest.raises(ValueError):
        flarepp.linear_fwd(X, W.cpu())
    with pytest.raises(flarepp.FlareppError) as e:
        flarepp.linear_fwd(X.float(), W.float())
    assert e.value.status == flarepp.ERR_UNSUPPORTED
    with pytest.raises(flarepp.FlareppError) as e:  # in place
        flarepp.linear_fwd(X, W[:16].contiguous(), residual=X, Y=X)
    assert e.value.status == flarepp.ERR_INVALID_ARGUMENT
    X15, W15 = X[:, :15].contiguous(), W[:, :15].contiguous()  # padded in the workspace
    with pytest.raises(flarepp.FlareppError) as e:
        flarepp.linear_fwd(X15, W15, workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))
    assert e.value.status == flarepp.ERR_WORKSPACE
    with pytest.raises(TypeError):
        flarepp.linear_bwd(X, W, R, None, "gelu")
