"""Group norm (flarepp_group_norm_*) against its definition and autograd in 64 bits.

Bounds: float32 sums in chunks leave the mean and the variance off by some 2^-20 of the magnitudes, so
xhat by 2^-18 (1 + |xhat| + |mean| rstd); the activations' approximations by 1e-6 (1 + |z|); the result
is rounded once. A gradient's averages are those of its terms, so they are off by 2^-18 of the
terms' own size; dgamma and dbeta by that of their sums of magnitudes."""
import pytest
import torch

from causal_refs import norm_ref, within
from paper_2608_11519_gb300 import flarepp

pytestmark = pytest.mark.gpu
HALF = {torch.bfloat16: 2.0 ** -8 * 1.01, torch.float32: 2.0 ** -24 * 1.01}
E = 2.0 ** -17


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def tensor(seed, *shape, dtype=torch.bfloat16, std=1.0, mean=0.0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return (torch.randn(*shape, generator=g, device="cuda") * std + mean).to(dtype)


def check(B, N, C, G, act, dtype, affine=True, lengths=None, mean=0.5, param=None, eps=1e-5):
    X, dY = tensor(1, B, N, C, dtype=dtype, std=1.5, mean=mean), tensor(2, B, N, C, dtype=dtype)
    param = param or dtype
    gamma = tensor(3, C, dtype=param, std=0.3, mean=1.0) if affine else None
    beta = tensor(4, C, dtype=param, std=0.3) if affine else None
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    if lengths is not None:  # what does not count is no number
        for b, r in enumerate(lengths):
            X[b, r:], dY[b, r:] = float("nan"), float("nan")
        Xr, dYr = X.nan_to_num(), dY.nan_to_num()
    else:
        Xr, dYr = X, dY
    ref = norm_ref(Xr, G, gamma, beta, eps, act, n, dYr)
    how = dict(gamma=gamma, beta=beta, act=act, lengths=n)
    Y, stats = flarepp.group_norm_fwd_train(X, G, eps=eps, **how)
    assert torch.equal(Y, flarepp.group_norm_fwd(X, G, eps=eps, **how))
    dX, dgamma, dbeta = flarepp.group_norm_bwd(X, dY, stats, G, **how)
    m, r = (ref["stats"][:, i].repeat_interleave(C // G, 1)[:, None] for i in (0, 1))
    xhat = ((Xr.double() - m) * r).abs()
    off = E * (1 + xhat + m.abs() * r)  # of xhat
    ga = 1.0 if gamma is None else gamma.double().abs()
    z = xhat * ga + (0.0 if beta is None else beta.double().abs())
    ez = off * ga + 1e-6 * (1 + z)  # of the activation (slopes of at most 1.13)
    half, ref_y = HALF[dtype], ref["Y"]
    within(Y, ref_y, half * ref_y.abs() + 1.2 * ez + 1e-30, "Y")
    scale = (Xr.double().abs().amax() + 1)
    within(stats[:, 0], ref["stats"][:, 0], E * scale.expand(B, G), "means")
    within(stats[:, 1], ref["stats"][:, 1], E * ref["stats"][:, 1] * (1 + (m.abs() * r)[:, 0, ::C // G]), "rstds")
    # relu's slope jumps at 0, where z's sign may be lost: leave out what is that close
    dz = dYr.double().abs() * (1.2 + ez)
    near = (z < 0) & (z > 0)
    if act == "relu":
        zz = (Xr.double() - m) * r * (1 if gamma is None else gamma.double()) + \
            (0 if beta is None else beta.double())
        near = zz.abs() < ez
    g = dz * ga
    # a value of dz is off by its slope's error (at most ez, slopes' slopes being below 1.2, or all of it
    # where relu's sign is lost), an average of g or g xhat by the averages of that and of 2^-17 g
    eg = (dYr.double().abs() * ga) * (1.2 * ez + E) + g * near
    live = torch.ones(B, N, 1, dtype=torch.bool, device="cuda")
    if n is not None:
        live = torch.arange(N, device="cuda").view(1, -1, 1) < n.view(-1, 1, 1)
    count = (live.sum((1, 2)) * (C // G)).clamp(min=1).view(B, 1, 1).double()

    def avg(t):
        s = (t * live).view(B, N, G, C // G).sum((1, 3)) / count[:, :, 0]
        return s.repeat_interleave(C // G, 1)[:, None]

    e0, e1 = avg(eg + E * g), avg((eg + E * g) * xhat + g * off)
    a1 = avg(g * xhat)
    bound = r * (eg + E * g + e0 + xhat * e1 + off * a1 + E * (avg(g) + xhat * a1))
    within(dX, ref["dX"] * live, half * ref["dX"].abs() + bound * live + 1e-30, "dX")
    assert not bool((dX * ~live).any()) and not bool((Y * ~live).any())
    if affine:
        hp = HALF[param]
        eb = ((dYr.double().abs() * (1.2 * ez + E) + dz * near) * live)
        within(dbeta, ref["dbeta"], hp * ref["dbeta"].abs() + eb.sum((0, 1)) + 1e-30, "dbeta")
        within(dgamma, ref["dgamma"], hp * ref["dgamma"].abs() + (eb * xhat + dz * off * live).sum((0, 1)) + 1e-30,
               "dgamma")
    else:
        assert dgamma is None and dbeta is None


@pytest.mark.parametrize("act", ["none", "relu", "gelu", "silu"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_activations(act, dtype):
    check(3, 100, 64, 8, act, dtype)


@pytest.mark.parametrize("N", [1, 2, 3, 4, 5, 31, 1000])
@pytest.mark.parametrize("C,G", [(64, 1), (64, 64), (512, 8), (30, 5), (250, 10), (7, 1), (96, 4)])
def test_lengths_and_groups(N, C, G):
    check(5, N, C, G, "silu", torch.bfloat16)
    check(2, N, C, G, "gelu", torch.float32, affine=False)


@pytest.mark.parametrize("C,G", [(5000, 1), (4096, 2), (3000, 3000), (2500, 4), (2056, 257), (1029, 3)])
def test_wide(C, G):
    """Channels over several tiles, and groups that cross them."""
    check(3, 17, C, G, "none", torch.bfloat16)
    check(2, 1, C, G, "silu", torch.float32)


@pytest.mark.parametrize("C", [8, 96, 132, 512, 1000, 1024, 1028])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_layer_norm(C, dtype):
    """One group and one row: what one warp holds, and more."""
    check(700, 1, C, 1, "none", dtype)
    check(3, 1, C * 3, 3, "gelu", dtype)


@pytest.mark.parametrize("B,N", [(1, 40000), (700, 20), (5000, 1), (2000, 7)])
def test_many(B, N):
    check(B, N, 48, 3, "gelu", torch.bfloat16)


@pytest.mark.parametrize("N,lengths", [(50, [50, 0, 1, 49]), (3, [3, 0, 1, 2]), (9000, [9000, 17, 0, 8999])])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_padded_batches(N, lengths, dtype):
    check(4, N, 64, 4, "silu", dtype, lengths=lengths)


def test_parameters_of_another_type():
    check(3, 60, 64, 4, "silu", torch.bfloat16, param=torch.float32)
    check(3, 60, 64, 4, "silu", torch.float32, param=torch.bfloat16)


def test_means_far_from_zero_keep_the_variance():
    """Deviations a thousandth of the mean: the bounds grow with mean * rstd only."""
    check(2, 3000, 32, 4, "none", torch.float32, mean=1500.0)


def test_constant_groups():
    """No variance: rstd is 1 / sqrt(eps), Y is beta, and nothing is NaN."""
    X = torch.full((2, 40, 16), 3.0, device="cuda")
    beta = tensor(1, 16, dtype=torch.float32)
    Y, stats = flarepp.group_norm_fwd_train(X, 4, torch.ones(16, device="cuda"), beta, eps=1e-4)
    assert torch.equal(Y, beta.expand_as(Y))
    within(stats[:, 1], torch.full((2, 4), 100.0, dtype=torch.float64, device="cuda"),
           torch.full((2, 4), 1e-4, device="cuda"), "rstd")


def test_a_wrong_length_is_recorded():
    X = tensor(1, 2, 30, 16)
    for N in (30, 3):
        x = X[:, :N].contiguous()
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        bad = torch.tensor([-3, 1000], dtype=torch.int32, device="cuda")
        Y = flarepp.group_norm_fwd(x, 2, lengths=bad, status=status)
        assert int(status) == flarepp.ERR_INVALID_ARGUMENT
        good = torch.tensor([0, N], dtype=torch.int32, device="cuda")
        assert torch.equal(Y, flarepp.group_norm_fwd(x, 2, lengths=good))
    flarepp.group_norm_fwd(X, 2, lengths=bad)
    assert flarepp.layers_status() == flarepp.ERR_INVALID_ARGUMENT
    assert flarepp.layers_status() == flarepp.OK


def test_repeats_streams_and_graphs():
    X, dY = tensor(1, 4, 5000, 64), tensor(2, 4, 5000, 64)
    gamma, beta = tensor(3, 64), tensor(4, 64)

    def call(**kw):
        Y, stats = flarepp.group_norm_fwd_train(X, 8, gamma, beta, act="silu", **kw)
        return (Y, stats) + flarepp.group_norm_bwd(X, dY, stats, 8, gamma, beta, act="silu", **kw)

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    first, again, other = call(), call(), call(stream=side)
    side.synchronize()
    for a, b, c in zip(first, again, other):
        assert torch.equal(a, b) and torch.equal(a, c)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        inside = call()
    X.copy_(tensor(9, 4, 5000, 64))
    graph.replay()
    for a, b in zip(inside, call()):
        assert torch.equal(a, b)


def test_nothing_to_do():
    for B, N in ((0, 5), (3, 0)):
        X = torch.zeros(B, N, 16, device="cuda")
        one = torch.ones(16, device="cuda")
        Y, stats = flarepp.group_norm_fwd_train(X, 2, one, one)
        dX, dgamma, dbeta = flarepp.group_norm_bwd(X, X, stats, 2, one, one)
        assert dX.shape == X.shape and not bool(dgamma.any()) and not bool(dbeta.any())
