"""Calls of the layers on a stream that is not torch's current one: what a call allocates for itself
belongs to the stream that it runs on, so the current stream cannot be handed it meanwhile."""
import pytest
import torch

from paper_2608_11519_gb300 import flarepp

pytestmark = pytest.mark.gpu


def busy(stream):
    with torch.cuda.stream(stream):
        torch.cuda._sleep(40_000_000)  # some 20 ms, in which the host goes on


def overwrite(sizes):
    """Take blocks of these sizes from the current stream's memory and fill them with ones."""
    return [torch.full((n,), 255, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(4)]


def as_handle(stream, kind):
    return stream if kind == "stream" else stream.cuda_stream


@pytest.mark.parametrize("kind", ["stream", "handle"])
def test_linear(kind):
    T, K, N = 3001, 520, 1031
    g = torch.Generator(device="cuda").manual_seed(1)
    X, W, b, dY = (torch.randn(*s, generator=g, device="cuda").bfloat16()
                   for s in ((T, K), (N, K), (N,), (T, N)))
    Y, Z = flarepp.linear_fwd_train(X, W, b, act="silu")
    want = (Y, Z) + flarepp.linear_bwd(X, W, dY, Z, "silu")
    side = torch.cuda.Stream()
    sizes = [flarepp._entry("linear_bwd_workspace_bytes")(
        flarepp.ctypes.byref(flarepp._linear_shape(X, W, "silu")[0])), T * N * 2, T * K * 2, N * K * 2]
    torch.cuda.synchronize()
    busy(side)
    st = as_handle(side, kind)
    Y, Z = flarepp.linear_fwd_train(X, W, b, act="silu", stream=st)
    got = (Y, Z) + flarepp.linear_bwd(X, W, dY, Z, "silu", stream=st)
    assert torch.cuda.current_stream() == torch.cuda.default_stream()
    kept = overwrite(sizes)
    torch.cuda.synchronize()
    for a, w in zip(got, want):
        assert torch.equal(a, w)
    del kept


@pytest.mark.parametrize("kind", ["stream", "handle"])
def test_embedding_and_moments(kind):
    T, V, C = 70001, 257, 64
    g = torch.Generator(device="cuda").manual_seed(2)
    ids = torch.randint(0, V, (T,), generator=g, device="cuda")
    table, dY = (torch.randn(n, C, generator=g, device="cuda") for n in (V, T))
    want = flarepp.embedding_fwd(ids, table, 2.0), flarepp.embedding_bwd(ids, dY, V, 2.0)
    opt = flarepp.AdamW([table], [want[1]], state_bits=8)
    opt.step()
    moments = [t[0] for t in opt.moments()]
    side = torch.cuda.Stream()
    shape = flarepp.EmbeddingShape(T, V, C, flarepp._DTYPES[torch.float32], 8)
    sizes = [flarepp._entry("embedding_bwd_workspace_bytes")(flarepp.ctypes.byref(shape)), T * C * 4,
             V * C * 4]
    table2 = table.clone()
    want2 = flarepp.embedding_fwd(ids, table2, 2.0)
    torch.cuda.synchronize()
    busy(side)
    st = as_handle(side, kind)
    got = (flarepp.embedding_fwd(ids, table2, 2.0, stream=st),
           flarepp.embedding_bwd(ids, dY, V, 2.0, stream=st))
    got_m = [t[0] for t in opt.moments(stream=st)]
    kept = overwrite(sizes)
    torch.cuda.synchronize()
    assert torch.equal(got[0], want2) and torch.equal(got[1], want[1])
    for a, w in zip(got_m, moments):
        assert torch.equal(a, w)
    del kept


def test_the_null_stream_by_its_handle():
    X, W = (torch.randn(64, 64, device="cuda").bfloat16() for _ in "ab")
    want = flarepp.linear_fwd(X, W)
    assert torch.equal(flarepp.linear_fwd(X, W, stream=0), want)
