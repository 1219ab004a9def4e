"""Rotary positions (flarepp_rotary) against the turns in 64 bits.

Bounds: angles are good to some 2^-22 rad (a few 2^-25 turns, and the sine's own 2^-22), two
products and a sum in float32 add 2^-23 of the magnitudes each; then the result is rounded."""
import pytest
import torch

from causal_refs import rotary_ref, within
from paper_2608_11519_gb300 import flarepp

pytestmark = pytest.mark.gpu
HALF = {torch.bfloat16: 2.0 ** -8 * 1.01, torch.float32: 2.0 ** -24 * 1.01}


@pytest.fixture(autouse=True)
def _device():
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    torch.cuda.set_device(0)


def tensor(seed, *shape, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.randn(*shape, generator=g, device="cuda").to(dtype)


def places(B, N, A, real=False, far=0, seed=9):
    g = torch.Generator(device="cuda").manual_seed(seed)
    if real:
        return torch.rand(B, N, A, generator=g, device="cuda") * 200 - 100
    return (torch.randint(0, 4000, (B, N, A), generator=g, device="cuda") + far).int()


def check(got, x, positions, freqs, sections, pairing, inverse=False):
    ref = rotary_ref(x, positions, freqs, sections, pairing, inverse)
    most = x.double().abs().amax(-1, keepdim=True)
    within(got, ref, HALF[x.dtype] * ref.abs() + 2.0 ** -20 * most + 1e-30, "rotary")
    P = sum(sections)
    assert torch.equal(got[..., 2 * P:], x[..., 2 * P:])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("pairing", ["halves", "adjacent", "axes"])
@pytest.mark.parametrize("D,sections", [(64, [32]), (64, [8, 16]), (32, [6, 5, 5]), (128, [16, 24, 24]),
                                        (80, [8, 8]), (24, [1, 0, 3, 7]), (10, [2, 3]), (7, [3]), (16, [0])])
def test_pairings_and_sections(dtype, pairing, D, sections):
    B, N = 2, 37
    freqs, pos = flarepp.rotary_frequencies(sections), places(B, N, len(sections))
    q, k = tensor(1, B, 6, N, D, dtype=dtype), tensor(2, B, 2, N, D, dtype=dtype)
    args = (pos, freqs, sections, pairing)
    q1, k1 = flarepp.rotary_fwd(q, k, *args)
    check(q1, q, *args)
    check(k1, k, *args)
    q2, none = flarepp.rotary_bwd(q, None, *args)
    check(q2, q, *args, inverse=True)
    assert none is None


@pytest.mark.parametrize("real,far", [(True, 0), (False, 0), (False, 2 ** 24), (False, 2 ** 31 - 4001),
                                      (False, -2 ** 31)])
def test_far_positions(real, far):
    B, N, D, sections = 2, 50, 64, [16, 16]
    freqs, pos = flarepp.rotary_frequencies(sections), places(B, N, 2, real, far)
    for dtype in (torch.bfloat16, torch.float32):
        q = tensor(3, B, 4, N, D, dtype=dtype)
        check(flarepp.rotary_fwd(q, None, pos, freqs, sections)[0], q, pos, freqs, sections, "halves")


@pytest.mark.parametrize("D,sections,pairing", [(64, [32], "halves"), (32, [6, 5, 5], "axes"), (12, [5], "halves")])
def test_layouts_and_in_place(D, sections, pairing):
    """Parts of one projection in place, transposed views, a batch that shares positions."""
    B, N, H = 3, 41, 4
    pos, freqs = places(1, N, len(sections))[0], flarepp.rotary_frequencies(sections)
    args = (pos, freqs, sections, pairing)
    qkv = tensor(5, B, N, 3, H, D)
    before = qkv.clone()
    q, k, v = (qkv[:, :, i].transpose(1, 2) for i in range(3))
    q1, k1 = flarepp.rotary_fwd(q, k, *args)
    assert q1.stride(1) < q1.stride(2)  # in the order of q
    out = flarepp.rotary_fwd(q, k, *args, q_out=q, k_out=k)
    assert out[0] is q and torch.equal(q, q1) and torch.equal(k, k1)
    assert torch.equal(v, before[:, :, 2].transpose(1, 2))
    for got, i in ((q1, 0), (k1, 1)):
        check(got, before[:, :, i].transpose(1, 2), *args)
    odd = tensor(6, B, H, N, D + 1)[..., 1:]  # rows that no vector divides
    check(flarepp.rotary_fwd(odd, None, *args)[0], odd, *args)
    one = tensor(7, B, 1, N, D).expand(B, H, N, D)
    check(flarepp.rotary_fwd(one, None, *args)[0], one, *args)


def test_many_tokens_and_one():
    sections = [6, 5, 5]
    freqs = flarepp.rotary_frequencies(sections)
    for B, H, N in ((1, 16, 70001), (32, 40, 1), (1, 1, 1), (2, 3, 0), (0, 3, 4)):
        x, pos = tensor(8, B, H, N, 32), places(B, N, 3, True)
        got = flarepp.rotary_fwd(x, x.clone(), pos, freqs, sections, "axes")
        if x.numel():
            check(got[0], x, pos, freqs, sections, "axes")
            assert torch.equal(got[0], got[1])


def test_backwards_undoes_and_is_the_gradient():
    """A turn keeps products: <turn(x), y> = <x, turn back(y)>, and differences of a linear map are its values."""
    sections, N, D = [10, 22], 300, 64
    freqs, pos = flarepp.rotary_frequencies(sections), places(1, N, 2)
    x, y = (tensor(s, 1, 3, N, D, dtype=torch.float32) for s in (11, 12))
    fx, _ = flarepp.rotary_fwd(x, None, pos, freqs, sections)
    by, _ = flarepp.rotary_bwd(y, None, pos, freqs, sections)
    n = float((x.double().abs() * y.double().abs()).sum())
    assert abs(float((fx.double() * y.double()).sum() - (x.double() * by.double()).sum())) <= 2.0 ** -19 * n
    back, _ = flarepp.rotary_bwd(fx, None, pos, freqs, sections)
    within(back, x.double(), 2.0 ** -18 * x.double().abs().amax(-1, keepdim=True), "undone")


def test_streams_and_graphs():
    sections = [32]
    freqs, pos, x = flarepp.rotary_frequencies(sections), places(1, 500, 1), tensor(4, 1, 8, 500, 64)
    call = lambda **kw: flarepp.rotary_fwd(x, x, pos, freqs, sections, **kw)[0]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a, b = call(), call(stream=side)
    side.synchronize()
    assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        inside = call()
    pos.add_(17)
    graph.replay()
    assert torch.equal(inside, call()) and not torch.equal(inside, a)
