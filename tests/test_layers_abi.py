"""The entry points of the linear layer, the embedding and AdamW on the host: sizes, no-op shapes
and refusals. Nothing here launches a kernel (every call fails its checks or has nothing to do),
so these tests run without a GPU; the addresses are never dereferenced."""
import ctypes

import pytest

from paper_2608_11519_gb300 import build as lib_build
from paper_2608_11519_gb300 import flarepp

FAKE = 0x7F0000000000
INVALID, UNSUPPORTED, WORKSPACE = (flarepp.ERR_INVALID_ARGUMENT, flarepp.ERR_UNSUPPORTED,
                                   flarepp.ERR_WORKSPACE)


def test_rows_whose_last_tile_would_pass_32_bits(lib):
    for rows in ((1 << 31) - 255, (1 << 31) - 1):
        s = linear_shape(rows=rows, in_=8, out=8)
        assert fwd(lib, s) == bwd(lib, s) == UNSUPPORTED
        assert lib.flarepp_linear_workspace_bytes(ctypes.byref(s)) == 0
    s = linear_shape(rows=(1 << 31) - 256, in_=8, out=8)
    assert fwd(lib, s, X=FAKE + 1) == INVALID  # large enough, refused for its address


@pytest.fixture(scope="module")
def lib():
    lib_build.build()
    return flarepp.load()


def at(i):
    return FAKE + (i << 38)


def linear_shape(rows=100, in_=64, out=96, dtype=flarepp.BF16, act=0):
    return flarepp.LinearShape(rows, in_, out, dtype, act)


def fwd(lib, s, **over):
    names = ("X", "W", "b", "R", "Y", "Z", "workspace")
    v = {n: over.get(n, at(i + 1)) for i, n in enumerate(names)}
    need = lib.flarepp_linear_workspace_bytes(ctypes.byref(s)) if s else 0
    return lib.flarepp_linear_fwd(ctypes.byref(s) if s else None, *(v[n] for n in names),
                                  over.get("ws_bytes", need), over.get("status", 0), None)


def bwd(lib, s, **over):
    names = ("X", "W", "Z", "dY", "dX", "dW", "db", "workspace")
    v = {n: over.get(n, at(i + 1)) for i, n in enumerate(names)}
    need = lib.flarepp_linear_bwd_workspace_bytes(ctypes.byref(s))
    return lib.flarepp_linear_bwd(ctypes.byref(s), *(v[n] for n in names),
                                  over.get("ws_bytes", need), over.get("status", 0), None)


def test_linear_workspace(lib):
    size = lambda s: lib.flarepp_linear_workspace_bytes(ctypes.byref(s))
    bsize = lambda s: lib.flarepp_linear_bwd_workspace_bytes(ctypes.byref(s))
    assert size(linear_shape()) == 0                      # one launch
    assert size(linear_shape(rows=100000, in_=256, out=512)) == 0
    # widths that are no multiple of 8 are padded to whole 128-byte lines
    assert size(linear_shape(in_=63)) >= (100 + 96) * 64 * 2
    assert size(linear_shape(rows=0)) == bsize(linear_shape(rows=0)) == 0
    # dZ in whole lines and the partial sums of db
    assert bsize(linear_shape(act=2)) >= 100 * 128 * 2 + 96 * 4
    for bad in (linear_shape(rows=-1), linear_shape(in_=0), linear_shape(out=0),
                linear_shape(dtype=7), linear_shape(act=4), linear_shape(dtype=flarepp.F32)):
        assert size(bad) == bsize(bad) == 0
    assert lib.flarepp_linear_workspace_bytes(None) == 0
    assert lib.flarepp_linear_bwd_workspace_bytes(None) == 0


def test_linear_refusals(lib):
    s = linear_shape(in_=63)  # one that needs a workspace
    assert fwd(lib, None) == INVALID
    for k in ("rows", "in_", "out"):
        assert fwd(lib, linear_shape(**{k: -1})) == INVALID
    assert fwd(lib, linear_shape(act=-1)) == INVALID
    assert fwd(lib, linear_shape(dtype=2)) == INVALID
    assert fwd(lib, linear_shape(dtype=flarepp.F32)) == UNSUPPORTED
    assert fwd(lib, linear_shape(rows=1 << 31)) == UNSUPPORTED
    assert fwd(lib, linear_shape(in_=(1 << 20) + 1)) == UNSUPPORTED
    for name in ("X", "W", "Y"):
        assert fwd(lib, s, **{name: 0}) == INVALID
    for name in ("X", "W", "b", "R", "Y", "Z"):
        assert fwd(lib, s, **{name: at(9) + 8}) == INVALID
    for name in ("X", "W", "b", "R", "Z", "workspace"):
        assert fwd(lib, s, Y=at(9), **{name: at(9)}) == INVALID
    for name in ("X", "W", "b", "R"):
        assert fwd(lib, s, workspace=at(9), **{name: at(9) + 256}) == INVALID
        assert fwd(lib, s, status=at(9) + 16, **{name: at(9)}) == INVALID
    assert fwd(lib, s, workspace=0) == WORKSPACE
    assert fwd(lib, s, workspace=at(9) + 16) == WORKSPACE
    need = lib.flarepp_linear_workspace_bytes(ctypes.byref(s))
    assert fwd(lib, s, ws_bytes=need - 1) == WORKSPACE
    assert fwd(lib, linear_shape(rows=0), X=0, W=0, Y=0, workspace=0) == flarepp.OK


def test_linear_backward_refusals(lib):
    s = linear_shape(act=2)
    assert bwd(lib, linear_shape(rows=-1)) == INVALID
    for name in ("X", "W", "Z", "dY"):
        assert bwd(lib, s, **{name: 0}) == INVALID
    for name in ("X", "W", "Z", "dY", "dX", "dW", "db"):
        assert bwd(lib, s, **{name: at(11) + 4}) == INVALID
    for out in ("dX", "dW", "db"):
        for other in ("X", "W", "Z", "dY", "workspace"):
            assert bwd(lib, s, **{out: at(11), other: at(11)}) == INVALID
    assert bwd(lib, s, dX=at(11), dW=at(11) + 16) == INVALID
    assert bwd(lib, s, workspace=0) == WORKSPACE
    assert bwd(lib, s, ws_bytes=16) == WORKSPACE
    # nothing to compute and nothing to write
    none = dict(X=0, W=0, Z=0, dY=0, dX=0, dW=0, db=0, workspace=0)
    assert bwd(lib, linear_shape(rows=0), **none) == flarepp.OK


def emb_shape(T=100, V=50, C=16, dtype=flarepp.F32, id_bytes=8):
    return flarepp.EmbeddingShape(T, V, C, dtype, id_bytes)


def emb_fwd(lib, s, ids=at(1), table=at(2), Y=at(3), scale=1.0, status=0):
    return lib.flarepp_embedding_fwd(ctypes.byref(s), ids, table, scale, Y, status, None)


def emb_bwd(lib, s, ids=at(1), dY=at(2), out=at(3), ws=at(4), ws_bytes=None, scale=1.0, status=0):
    need = lib.flarepp_embedding_bwd_workspace_bytes(ctypes.byref(s))
    return lib.flarepp_embedding_bwd(ctypes.byref(s), ids, dY, scale, out, ws,
                                     need if ws_bytes is None else ws_bytes, status, None)


def test_embedding_refusals(lib):
    for bad in (emb_shape(T=-1), emb_shape(V=0), emb_shape(C=0), emb_shape(dtype=3),
                emb_shape(id_bytes=2)):
        assert emb_fwd(lib, bad) == emb_bwd(lib, bad) == INVALID
        assert lib.flarepp_embedding_bwd_workspace_bytes(ctypes.byref(bad)) == 0
    for bad in (emb_shape(T=1 << 31), emb_shape(V=(1 << 31) - 1), emb_shape(C=(1 << 20) + 1)):
        assert emb_fwd(lib, bad) == emb_bwd(lib, bad) == UNSUPPORTED
    s = emb_shape()
    for k in ("ids", "table", "Y"):
        assert emb_fwd(lib, s, **{k: 0}) == emb_fwd(lib, s, **{k: at(5) + 4}) == INVALID
    for k in ("ids", "dY", "out"):
        assert emb_bwd(lib, s, **{k: 0}) == emb_bwd(lib, s, **{k: at(5) + 4}) == INVALID
    for bad in (float("nan"), float("inf")):
        assert emb_fwd(lib, s, scale=bad) == emb_bwd(lib, s, scale=bad) == INVALID
    assert emb_fwd(lib, s, Y=at(2) + 64) == INVALID           # over the table
    assert emb_fwd(lib, s, status=at(1) + 8) == INVALID       # over the ids
    assert emb_bwd(lib, s, out=at(2)) == emb_bwd(lib, s, ws=at(2)) == INVALID
    assert emb_bwd(lib, s, ws=0) == emb_bwd(lib, s, ws=at(4) + 16) == WORKSPACE
    assert emb_bwd(lib, s, ws_bytes=256) == WORKSPACE
    assert emb_fwd(lib, emb_shape(T=0), ids=0, table=0, Y=0) == flarepp.OK
    assert lib.flarepp_embedding_bwd_workspace_bytes(None) == 0
    # keys, positions, counters and the partial sums of runs that cross stretches
    assert lib.flarepp_embedding_bwd_workspace_bytes(ctypes.byref(emb_shape(T=10000))) > 10000 * 16


def tensor(n=1000, **over):
    v = dict(param=at(1), grad=at(2), master=0, m=at(3), v=at(4), m_scale=at(5), v_scale=at(6),
             n=n, param_dtype=flarepp.F32, grad_dtype=flarepp.F32)
    v.update(over)
    return flarepp.AdamwTensor(*(v[f[0]] for f in flarepp.AdamwTensor._fields_))


def step(lib, ts, bits=32, n=None, **over):
    h = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, step=1, state_bits=bits)
    h.update(over)
    hyper = flarepp.AdamwHyper(*(h[f[0]] for f in flarepp.AdamwHyper._fields_))
    table = (flarepp.AdamwTensor * max(1, len(ts)))(*ts)
    return lib.flarepp_adamw_step(table, len(ts) if n is None else n, ctypes.byref(hyper), None)


def test_adamw_refusals(lib):
    assert step(lib, []) == flarepp.OK
    assert step(lib, [tensor(n=0, param=0, grad=0)]) == flarepp.OK
    assert lib.flarepp_adamw_step(None, 1, None, None) == INVALID
    nan, inf = float("nan"), float("inf")
    for bad in (dict(lr=nan), dict(lr=inf), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0),
                dict(beta2=nan), dict(eps=-1e-9), dict(eps=inf), dict(weight_decay=nan),
                dict(step=0), dict(bits=16)):
        assert step(lib, [], **bad) == INVALID, bad
    assert step(lib, [], n=-1) == INVALID
    for bits in (32, 8):
        for k in ("param", "grad", "m", "v"):
            assert step(lib, [tensor(**{k: 0})], bits) == INVALID
            assert step(lib, [tensor(**{k: at(9) + 8})], bits) == INVALID
        assert step(lib, [tensor(n=-1)], bits) == INVALID
        assert step(lib, [tensor(param_dtype=2)], bits) == INVALID
        assert step(lib, [tensor(grad_dtype=-1)], bits) == INVALID
        assert step(lib, [tensor(master=at(8))], bits) == INVALID  # of a float32 parameter
        for k in ("grad", "m", "v"):
            assert step(lib, [tensor(param=at(9), **{k: at(9) + 16})], bits) == INVALID
    for k in ("m_scale", "v_scale"):
        assert step(lib, [tensor(**{k: 0})], 8) == INVALID
        assert step(lib, [tensor(**{k: at(9) + 2})], 8) == INVALID
        assert step(lib, [tensor(**{k: at(3) + 16})], 8) == INVALID  # inside m
    # one bad tensor among good ones: nothing is enqueued
    assert step(lib, [tensor(), tensor(v=0)]) == INVALID
    outs = (ctypes.c_void_p * 1)(at(7))
    table = (flarepp.AdamwTensor * 1)(tensor(m_scale=0))
    assert lib.flarepp_adamw_moments(table, 1, outs, outs, None) == INVALID
    table = (flarepp.AdamwTensor * 1)(tensor())
    assert lib.flarepp_adamw_moments(table, 1, outs, outs, None) == INVALID  # m_out is v_out
    assert lib.flarepp_adamw_moments(table, 1, None, outs, None) == INVALID
    assert lib.flarepp_adamw_moments(None, 0, None, None, None) == flarepp.OK
