"""What the layers' kernels record for calls that pass no status word: a wait that gives up (made by the
test hook, as in test_linear_failure_gpu.py) and an id beyond the table must not go unseen."""
import pytest
import torch

from paper_2608_11519_gb300 import flarepp
from test_linear_gpu import _device, randn  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(autouse=True)
def _asked(_device):  # noqa: F811
    flarepp.layers_status()
    yield
    flarepp.layers_status()


@pytest.mark.parametrize("T", [2, 500, 30000])
@pytest.mark.parametrize("dt", [torch.int32, torch.int64])
def test_an_id_beyond_the_table(T, dt):
    V, C = 100, 32
    table, dY = torch.ones(V, C, device="cuda"), torch.ones(T, C, device="cuda")
    good = (torch.arange(T, device="cuda") % V).to(dt)
    bad = good.clone()
    bad[T // 2] = V
    word = torch.zeros(1, dtype=torch.int32, device="cuda")
    for call in (lambda ids, **k: flarepp.embedding_fwd(ids, table, **k),
                 lambda ids, **k: flarepp.embedding_bwd(ids, dY, V, **k)):
        call(good)
        assert flarepp.layers_status() == flarepp.OK
        call(bad)
        call(good)  # does not take it back
        assert flarepp.layers_status() == flarepp.ERR_INVALID_ARGUMENT
        assert flarepp.layers_status() == flarepp.OK  # told once
        call(bad, status=word)  # a call with a word of its own leaves the library's alone
        assert flarepp.layers_status() == flarepp.OK and int(word) == flarepp.ERR_INVALID_ARGUMENT
        word.zero_()


def test_on_another_stream_and_in_a_graph():
    table, bad = torch.ones(10, 8, device="cuda"), torch.tensor([3, 10], device="cuda")
    Y = torch.empty(2, 8, device="cuda")
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    flarepp.embedding_fwd(bad, table, Y=Y, stream=s)
    assert flarepp.layers_status(torch.device("cuda", 0), stream=s) == flarepp.ERR_INVALID_ARGUMENT
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        flarepp.embedding_fwd(bad, table, Y=Y)
    assert flarepp.layers_status() == flarepp.OK
    g.replay()
    assert flarepp.layers_status("cuda") == flarepp.ERR_INVALID_ARGUMENT
    with pytest.raises(ValueError):
        flarepp.layers_status("cpu")


@pytest.mark.parametrize("kernel,T,K,N", [(16, 3000, 1280, 512), (17, 50, 2048, 304), (18, 30000, 128, 512)])
def test_a_wait_that_gives_up(kernel, T, K, N):
    X, W = randn(T, K, seed=1), randn(N, K, seed=2, std=K ** -0.5)
    dY, Z = randn(T, N, seed=3), randn(T, N, seed=4)

    def call():
        if kernel == 18:
            return flarepp.linear_bwd(X, W, dY, Z, "gelu")
        return (flarepp.linear_fwd(X, W, act="silu"),)

    want = call()
    assert flarepp.layers_status() == flarepp.OK
    flarepp.embedding_fwd(torch.tensor([5], device="cuda"), torch.ones(5, 8, device="cuda"))
    lib = flarepp.load()
    lib.flarepp_test_wait_fault(kernel, 0, 1_000_000)
    try:
        call()
        torch.cuda.synchronize()
    finally:
        lib.flarepp_test_wait_fault(0, -1, 0)
    assert flarepp.layers_status() == flarepp.ERR_TIMEOUT  # counts for more than the id
    assert all(torch.equal(a, b) for a, b in zip(call(), want))
    assert flarepp.layers_status() == flarepp.OK
