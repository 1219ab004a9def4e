"""The embedding lookup and the gradient of its table against their definitions in 64 bits.

Tolerances: a looked-up value is one float32 product, rounded to the table's type: u times its
size (2^-8 for bf16, 2^-23 for float32, which a product and its rounding stay below). A row of
the gradient sums n values in float32, whatever the order: n 2^-24 of the sum of magnitudes,
and two roundings after it."""
import pytest
import torch

from paper_2608_11519_gb300 import flarepp

pytestmark = pytest.mark.gpu
U = {torch.bfloat16: 2.0 ** -8 * 1.01, torch.float32: 2.0 ** -23}


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def make_ids(kind, T, V, seed):
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(0, V, (T,), generator=g)
    if kind == "same":
        ids[:] = V - 1
    elif kind == "empty":
        ids[:] = -1
    elif kind == "skewed":  # half of all positions name one row, some none
        ids[torch.rand(T, generator=g) < 0.5] = V // 2
        ids[torch.rand(T, generator=g) < 0.2] = -5
    elif kind == "runs":  # few rows, each met many times in a row
        ids = (torch.arange(T) * 7 // max(1, T)) % V
    return ids


def check_bwd(ids, dY, V, scale, got):
    C, dt = dY.shape[-1], dY.dtype
    on = (ids >= 0) & (ids < V)
    at = ids[on].long().cuda()
    rows = dY.reshape(-1, C)[on.cuda()].double() * scale
    ref = torch.zeros(V, C, dtype=torch.float64, device="cuda").index_add_(0, at, rows)
    mag = torch.zeros(V, C, dtype=torch.float64, device="cuda").index_add_(0, at, rows.abs())
    n = torch.bincount(at, minlength=V).double().unsqueeze(1)
    err = n * 2.0 ** -24 * mag
    bound = U[dt] * (ref.abs() + err) + err
    d = (got.double() - ref).abs()
    assert bool((d <= bound).all()), f"worst {float((d - bound).max())} beyond"
    assert not got[(n == 0).reshape(-1)].any(), "rows that no id names"


SIZES = [(1, 1, 1), (1, 70000, 8), (2, 3, 2), (31, 5, 16), (64, 257, 256), (65, 257, 3),
         (1000, 2047, 100), (1000, 2048, 24), (4096, 2, 520), (5000, 40000, 64),
         (70001, 257, 32), (70001, 100000, 12), (200000, 7, 8), (3000, 4300000, 2)]


@pytest.mark.parametrize("T,V,C", SIZES)
@pytest.mark.parametrize("kind", ["uniform", "same", "skewed", "runs", "empty"])
def test_both_directions(T, V, C, kind):
    for k, dt in enumerate((torch.float32, torch.bfloat16)):
        ids = make_ids(kind, T, V, seed=T + k)
        it = ids.to(torch.int32 if k else torch.int64).cuda()
        g = torch.Generator(device="cuda").manual_seed(5)
        table = torch.randn(V, C, generator=g, device="cuda").to(dt)
        dY = torch.randn(T, C, generator=g, device="cuda").to(dt)
        scale = 1.7
        Y = flarepp.embedding_fwd(it, table, scale)
        on = (ids >= 0).cuda()
        ref = table.double()[ids.clamp(min=0).cuda()] * scale * on.unsqueeze(1)
        assert bool(((Y.double() - ref).abs() <= U[dt] * ref.abs()).all())
        grad = torch.full((V, C), 9.0, dtype=dt, device="cuda")
        flarepp.embedding_bwd(it, dY, V, scale, dtable=grad)
        check_bwd(ids, dY, V, scale, grad)
        assert torch.equal(grad, flarepp.embedding_bwd(it, dY, V, scale))  # the same bits again


@pytest.mark.parametrize("T", [9727, 9728, 20003])
@pytest.mark.parametrize("C", [15, 17, 18, 33, 255, 346, 1023])
@pytest.mark.parametrize("dt", [torch.float32, torch.bfloat16])
def test_lookup_of_rows_off_16_bytes(T, C, dt):
    """Many rows whose lines start off 16-byte blocks, the table's last ones among them, and nothing is
    written before or behind the output."""
    V = 37
    g = torch.Generator(device="cuda").manual_seed(C)
    ids = torch.randint(-3, V, (T,), generator=g, device="cuda")
    ids[-1] = V - 1
    table = torch.randn(V, C, generator=g, device="cuda").to(dt)
    table[3, 1], table[V - 1, C - 1] = float("inf"), float("nan")
    buf = torch.full((T * C + 256,), 7.0, dtype=dt, device="cuda")
    Y = flarepp.embedding_fwd(ids, table, 0.5, Y=buf[128:128 + T * C].view(T, C))
    rows = torch.where((ids >= 0).unsqueeze(1), table[ids.clamp(min=0)] * 0.5, torch.zeros((), device="cuda"))
    assert torch.equal(Y.nan_to_num(9.0), rows.to(dt).nan_to_num(9.0))  # a factor of 1/2 is exact
    assert (buf[:128] == 7).all() and (buf[128 + T * C:] == 7).all()


def test_gradient_against_differences():
    """The lookup is linear in the table: <dtable, D> is the change of the loss along D."""
    V, C = 50, 24
    ids = make_ids("skewed", 300, V, 1).view(3, 100).cuda()
    g = torch.Generator(device="cuda").manual_seed(2)
    table, D = (torch.randn(V, C, generator=g, device="cuda", dtype=torch.float64) for _ in "ab")
    dY = torch.randn(3, 100, C, generator=g, device="cuda")
    grad = flarepp.embedding_bwd(ids, dY, V, 0.5)

    def loss(t):
        return (torch.where((ids >= 0).unsqueeze(-1), t[ids.clamp(min=0)] * 0.5, 0.0) * dY.double()).sum()

    want = float((loss(table + D) - loss(table - D)) / 2)
    got = float((grad.double() * D).sum())
    assert abs(got - want) <= 300 * 2.0 ** -23 * float(dY.double().abs().sum() * D.abs().max())


def test_ids_beyond_the_table_are_reported():
    table = torch.randn(10, 16, device="cuda")
    ids = torch.tensor([0, 9, 10, -1, 2 ** 40], device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    Y = flarepp.embedding_fwd(ids, table, 2.0, status=status)
    assert int(status) == flarepp.ERR_INVALID_ARGUMENT
    assert torch.equal(Y[:2], table[[0, 9]] * 2) and not Y[2:].any()
    status.zero_()
    grad = flarepp.embedding_bwd(ids, torch.ones(5, 16, device="cuda"), 10, status=status)
    assert int(status) == flarepp.ERR_INVALID_ARGUMENT
    assert (grad[[0, 9]] == 1).all() and not grad[1:9].any()
    status.zero_()
    flarepp.embedding_bwd(ids[:2].clone(), torch.ones(2, 16, device="cuda"), 10, status=status)
    assert int(status) == flarepp.OK


def test_special_values_stay_in_their_row():
    ids = torch.arange(500, device="cuda") % 20
    dY = torch.ones(500, 8, device="cuda")
    dY[7, 3], dY[28, 0] = float("nan"), float("inf")
    grad = flarepp.embedding_bwd(ids, dY, 21)
    want = torch.full((21, 8), 25.0, device="cuda")
    want[20] = 0
    want[7, 3], want[8, 0] = float("nan"), float("inf")
    assert torch.equal(grad.nan_to_num(-1, 1e9), want.nan_to_num(-1, 1e9))


def test_long_table_and_long_output():
    """Offsets beyond 2^31 values: in the table, in Y and in dY."""
    V, C = 2_200_000, 1024
    table = torch.zeros(V, C, dtype=torch.bfloat16, device="cuda")
    table[-1], table[5] = 3.0, 2.0
    T = 2_200_001
    ids = torch.full((T,), 5, dtype=torch.int32, device="cuda")
    ids[-1] = V - 1
    Y = flarepp.embedding_fwd(ids, table)
    assert (Y[-1] == 3).all() and (Y[-2] == 2).all() and (Y[0] == 2).all()
    del table
    Y[:] = 0
    Y[-1], Y[-2] = 1.5, 0.25
    grad = flarepp.embedding_bwd(ids, Y, V)
    assert (grad[-1] == 1.5).all() and (grad[5] == 0.25).all() and not grad[6:-1].any()


def test_on_another_stream_and_fenced():
    ids = make_ids("skewed", 3001, 300, 4).cuda()
    dY = torch.randn(3001, 40, device="cuda")
    want = flarepp.embedding_bwd(ids, dY, 300)
    buf = torch.full((300 * 40 + 512,), 5.0, device="cuda")
    out = buf[256:256 + 12000].view(300, 40)
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        flarepp.embedding_bwd(ids, dY, 300, dtable=out)
    s.synchronize()
    assert torch.equal(out, want) and (buf[:256] == 5).all() and (buf[-256:] == 5).all()


def test_no_positions():
    ids = torch.empty(0, dtype=torch.int64, device="cuda")
    assert flarepp.embedding_fwd(ids, torch.ones(3, 4, device="cuda")).shape == (0, 4)
    grad = torch.ones(3, 4, device="cuda")
    flarepp.embedding_bwd(ids, torch.ones(0, 4, device="cuda"), 3, dtable=grad)
    assert not grad.any()


def test_refusals():
    ids, table = torch.zeros(4, dtype=torch.int64, device="cuda"), torch.ones(3, 8, device="cuda")
    with pytest.raises(TypeError):
        flarepp.embedding_fwd(ids.short(), table)
    with pytest.raises(TypeError):
        flarepp.embedding_fwd(ids, table.half())
    with pytest.raises(ValueError):
        flarepp.embedding_fwd(ids.cpu(), table)
    with pytest.raises(ValueError):
        flarepp.embedding_fwd(ids, table.t())
    with pytest.raises(ValueError):
        flarepp.embedding_bwd(ids, torch.ones(5, 8, device="cuda"), 3)
    for bad in (float("nan"), float("inf")):
        with pytest.raises(flarepp.FlareppError) as e:
            flarepp.embedding_fwd(ids, table, bad)
        assert e.value.status == flarepp.ERR_INVALID_ARGUMENT
    with pytest.raises(flarepp.FlareppError) as e:
        flarepp.embedding_bwd(ids, torch.ones(4, 8, device="cuda"), 3,
                              workspace=torch.empty(8, dtype=torch.uint8, device="cuda"))
    assert e.value.status == flarepp.ERR_WORKSPACE
    with pytest.raises(flarepp.FlareppError):
        flarepp.embedding_bwd(ids, torch.ones(4, 8, device="cuda"), 0)
