"""Which tensors of heads that share a buffer are taken to be apart, on the host: calls in place without a pair to
turn or without a workspace, which end before anything is launched, so these tests run without a GPU; the
addresses are never dereferenced."""
import ctypes
import itertools
import random

import pytest

from paper_2608_11519_gb300 import flarepp
from test_causal_abi import decay, decay_shape, rotary_shape
from test_layers_abi import INVALID, WORKSPACE, at, lib  # noqa: F401


def in_place(lib, s, q, k, k_out=None):  # noqa: F811
    """Turn no pairs of q and k, each its own output: OK, or what is wrong with the tensors. They are (first value,
    strides); k_out if it is not k."""
    size = 2 if s.dtype == flarepp.BF16 else 4
    v = [ctypes.byref(flarepp.Heads(at(1) + at_ * size, *st)) for at_, st in (q, k, q, k if k_out is None else k_out)]
    return lib.flarepp_rotary(ctypes.byref(s), None, None, *v, None)


def layouts(B, H, N, D, parts):
    """Strides (b, h, n) of a part of a dense buffer, and the distance of two parts, by the order of its sizes."""
    sizes = {"b": B, "p": parts, "h": H, "n": N}
    for order in itertools.permutations("bphn"):
        stride, step = {}, D
        for name in reversed(order):
            stride[name] = step
            step *= sizes[name]
        yield "".join(order), (stride["b"], stride["h"], stride["n"]), stride["p"]


@pytest.mark.parametrize("dtype", [flarepp.F32, flarepp.BF16])
@pytest.mark.parametrize("B,H,N", [(2, 4, 100), (1, 4, 100), (2, 1, 100), (2, 4, 1), (1, 1, 7), (3, 1, 1), (1, 4, 1)])
def test_parts_of_one_buffer(lib, B, H, N, dtype):  # noqa: F811
    """All orders of [B, parts, H, N, D], with the sizes' strides or (a size of 1) any others."""
    D, parts = 64, 3
    s = rotary_shape(B=B, Hq=H, Hk=H, N=N, D=D, sections=(0,), pos=0, dtype=dtype)
    for order, st, part in layouts(B, H, N, D, parts):
        odd = tuple(x if n > 1 else 12345 for x, n in zip(st, (B, H, N)))
        for i, j in itertools.permutations(range(parts), 2):
            for other in (st, odd):
                assert in_place(lib, s, (i * part, st), (j * part, other)) == flarepp.OK, order
        assert in_place(lib, s, (part, st), (part, st)) == INVALID, order
        assert in_place(lib, s, (part, st), (2 * part - 8, st)) == INVALID, order


def test_padded_batches(lib):  # noqa: F811
    """Parts of [B, N, 3, H, D] and of [B, N, H, 3, D] whose batch elements have rows behind them that no row's
    stride divides, and a part that is shifted into the next element's."""
    B, H, N, D = 2, 4, 10, 64
    s = rotary_shape(B=B, Hq=H, Hk=H, N=N, D=D, sections=(0,), pos=0)
    row = 3 * H * D
    for st, part in (((N * row + 88, D, row), H * D), ((N * row + 88, 3 * D, row), D)):
        assert in_place(lib, s, (0, st), (part, st)) == flarepp.OK
        assert in_place(lib, s, (2 * part, st), (0, st)) == flarepp.OK
        assert in_place(lib, s, (0, st), (part + N * row, st)) == INVALID
        assert in_place(lib, s, (0, st), (part + N * row + 88, st)) == flarepp.OK  # (one element on)


def test_unlike_heads(lib):  # noqa: F811
    """Queries and keys of one projection, more heads of the one than of the other."""
    B, Hq, Hk, N, D = 2, 6, 2, 50, 32
    s = rotary_shape(B=B, Hq=Hq, Hk=Hk, N=N, D=D, sections=(0,), pos=0)
    row = (Hq + 2 * Hk) * D
    assert in_place(lib, s, (0, (N * row, D, row)), (Hq * D, (N * row, D, row))) == flarepp.OK
    assert in_place(lib, s, (0, (N * row, D, row)), (Hq * D - D, (N * row, D, row))) == INVALID
    block = (N * row, N * D, D)
    assert in_place(lib, s, (0, block), (Hq * N * D, block)) == flarepp.OK
    assert in_place(lib, s, (0, block), ((Hq + Hk) * N * D, block)) == flarepp.OK
    assert in_place(lib, s, (0, block), (Hq * N * D - D, block)) == INVALID


@pytest.mark.parametrize("B,H,N", [(1, 4, 10), (2, 1, 10), (2, 4, 1), (1, 1, 1)])
def test_an_output_that_is_its_input(lib, B, H, N):  # noqa: F811
    """The same places, whatever the strides of sizes of 1 say."""
    D = 64
    s = rotary_shape(B=B, Hq=H, Hk=0, N=N, D=D, sections=(0,), pos=0)
    st = [H * N * D, N * D, D]
    other = [x if n > 1 else x + 72 for x, n in zip(st, (B, H, N))]
    call = lambda a, b: lib.flarepp_rotary(ctypes.byref(s), None, None, ctypes.byref(flarepp.Heads(at(1), *a)), None,
                                           ctypes.byref(flarepp.Heads(at(1), *b)), None, None)
    assert call(st, st) == call(st, other) == call(other, st) == flarepp.OK
    for i, n in enumerate((B, H, N)):
        if n > 1:
            wrong = list(st)
            wrong[i] += 2 * H * N * D
            assert call(st, wrong) == INVALID


def places(first, strides, B, H, N, D):
    return [first + b * strides[0] + h * strides[1] + n * strides[2] + d
            for b in range(B) for h in range(H) for n in range(N) for d in range(D)]


def test_what_is_accepted_is_apart(lib):  # noqa: F811
    """Small tensors with strides of all kinds, against the sets of their places: none is accepted that shares one
    with the other, or with itself."""
    rng = random.Random(7)
    accepted = refused = 0
    for _ in range(20000):
        B, H, H2, N, D = (rng.randint(1, 3) for _ in range(5))
        s = rotary_shape(B=B, Hq=H, Hk=H2, N=N, D=D, sections=(0,), pos=0, dtype=flarepp.F32)
        if rng.random() < 0.5:  # parts of a buffer, padded perhaps, shifted perhaps
            order, st, part = rng.choice(list(layouts(B, max(H, H2), N, D, 3)))
            st = tuple(x + rng.choice((0, 0, 0, 1, D)) for x in st)
            st2 = st if rng.random() < 0.8 else tuple(rng.choice((1, 2)) * x for x in st)
            q, k = (rng.randint(0, 2) * part, st), (rng.randint(0, 2) * part + rng.choice((0, 0, 1, D, -1)), st2)
        else:
            q, k = ((rng.randint(0, 40), tuple(rng.randint(0, 30) for _ in range(3))) for _ in range(2))
        got = in_place(lib, s, q, k)
        a, b = places(*q, B, H, N, D), places(*k, B, H2, N, D)
        if got == flarepp.OK:
            accepted += 1
            assert len(set(a)) == len(a) and len(set(b)) == len(b) and not set(a) & set(b), (q, k, B, H, H2, N, D)
        else:
            assert got == INVALID
            refused += 1
    assert accepted > 2000 and refused > 2000


@pytest.mark.parametrize("B", [1, 2])
def test_gradients_in_one_buffer(lib, B):  # noqa: F811
    """dQ, dK and dV as parts of [B, heads, N, D] and of [B, N, heads, D] (the call then ends for want of a workspace)."""
    s = decay_shape(B=B, Hq=4, Hk=2, N=300, Dk=64, Dv=64)
    heads, first = 8, (0, 4, 6)
    for st, step in (((heads * 300 * 64, 300 * 64, 64), 300 * 64), ((300 * heads * 64, 64, heads * 64), 64)):
        part = lambda i, more=0: {"data": at(30) + 2 * (first[i] * step + more),
                                  **dict(zip(("stride_b", "stride_h", "stride_n"), st))}
        assert decay(lib, s, True, dQ=part(0), dK=part(1), dV=part(2), workspace=0) == WORKSPACE
        assert decay(lib, s, True, dQ=part(0), dK=part(1, -64), dV=part(2), workspace=0) == INVALID
        assert decay(lib, s, True, dQ=part(0), dK=part(1), dV=part(1, 64), workspace=0) == INVALID
