"""The entry points of the decay attention, rotary positions and group norm on the host: sizes, no-op shapes
and refusals. Nothing here launches a kernel (every call fails its checks or has nothing to do), so
these tests run without a GPU; the addresses are never dereferenced."""
import ctypes

import pytest
import torch

from paper_2608_11519_gb300 import flarepp
from test_layers_abi import INVALID, UNSUPPORTED, WORKSPACE, at, lib  # noqa: F401


def decay_shape(B=2, Hq=4, Hk=2, N=300, Dk=64, Dv=32, sequences=0, dtype=flarepp.BF16, scale=0.5):
    return flarepp.DecayShape(B, Hq, Hk, N, Dk, Dv, sequences, dtype, scale)


def dense(i, s, H, D, **over):
    h = {"data": at(i), "stride_b": H * s.N * D, "stride_h": s.N * D, "stride_n": D}
    h.update(over)
    return flarepp.Heads(*(h[k] for k in ("data", "stride_b", "stride_h", "stride_n")))


TENSORS = {"Q": ("Hq", "Dk"), "K": ("Hk", "Dk"), "V": ("Hk", "Dv"), "Y": ("Hq", "Dv"), "dY": ("Hq", "Dv"),
           "dQ": ("Hq", "Dk"), "dK": ("Hk", "Dk"), "dV": ("Hk", "Dv")}


def decay(lib, s, back=False, **over):  # noqa: F811
    """Call the forward or the backward with everything given, but for ``over``; heads as dicts of what differs."""
    heads = {}
    for i, (k, (H, D)) in enumerate(TENSORS.items()):
        o = over.get(k, {})
        heads[k] = None if o is None else ctypes.byref(dense(i + 1, s, getattr(s, H), getattr(s, D), **o))
    v = {"log_decay": at(10), "offsets": at(11) if s.sequences else 0, "state": at(12), "state_out": at(13),
         "dstate_out": at(14), "dstate": at(15), "workspace": at(16), "status": 0}
    v.update({k: x for k, x in over.items() if k in v})
    ref = ctypes.byref(s)
    if back:
        need = over.get("ws_bytes", lib.flarepp_decay_attention_bwd_workspace_bytes(ref))
        return lib.flarepp_decay_attention_bwd(
            ref, heads["Q"], heads["K"], heads["V"], v["log_decay"], v["offsets"], v["state"], heads["dY"],
            v["dstate_out"], heads["dQ"], heads["dK"], heads["dV"], v["dstate"], v["workspace"], need,
            v["status"], None)
    need = over.get("ws_bytes", lib.flarepp_decay_attention_workspace_bytes(ref))
    return lib.flarepp_decay_attention_fwd(
        ref, heads["Q"], heads["K"], heads["V"], v["log_decay"], v["offsets"], v["state"], heads["Y"],
        v["state_out"], v["workspace"], need, v["status"], None)


def step(lib, s, **over):  # noqa: F811
    heads = [ctypes.byref(dense(i + 1, s, getattr(s, H), getattr(s, D), **over.get(k, {})))
             for i, (k, (H, D)) in enumerate(list(TENSORS.items())[:4])]
    return lib.flarepp_decay_attention_step(ctypes.byref(s), *heads[:3], over.get("log_decay", at(10)),
                                            over.get("state", at(12)), heads[3], over.get("status", 0), None)


BAD_SHAPES = [(dict(B=-1), INVALID), (dict(N=-1), INVALID), (dict(Hq=3), INVALID), (dict(Hk=0), INVALID),
              (dict(Dk=0), INVALID), (dict(dtype=7), INVALID), (dict(sequences=-1), INVALID),
              (dict(sequences=3), INVALID), (dict(scale=float("nan")), INVALID),
              (dict(scale=float("inf")), INVALID), (dict(dtype=flarepp.F32), UNSUPPORTED),
              (dict(Dk=12), UNSUPPORTED), (dict(Dv=136), UNSUPPORTED), (dict(Hq=1 << 17, Hk=1), UNSUPPORTED),
              (dict(N=(1 << 31) - 1), UNSUPPORTED)]


@pytest.mark.parametrize("over,status", BAD_SHAPES)
def test_decay_shapes(lib, over, status):  # noqa: F811
    s = decay_shape(**over)
    assert decay(lib, s) == decay(lib, s, back=True) == status
    assert lib.flarepp_decay_attention_workspace_bytes(ctypes.byref(s)) == 0
    assert lib.flarepp_decay_attention_bwd_workspace_bytes(ctypes.byref(s)) == 0


def test_decay_workspaces(lib):  # noqa: F811
    size = lambda **o: lib.flarepp_decay_attention_workspace_bytes(ctypes.byref(decay_shape(**o)))
    back = lambda **o: lib.flarepp_decay_attention_bwd_workspace_bytes(ctypes.byref(decay_shape(**o)))
    assert lib.flarepp_decay_attention_workspace_bytes(None) == 0
    assert size() == 0                                   # nothing is cut
    assert size(B=1, N=1 << 17) > 0                      # states between the blocks
    assert size(B=1, sequences=5) >= 2 * 6 * 4           # the cuts
    assert back() >= 2 * 4 * 300 * 64 * 4                # float32 sums of the query heads that share one
    assert back(Hk=4) == 0
    assert size(B=0) == size(N=0) == size(Hq=0, Hk=0) == 0


def test_decay_refusals(lib):  # noqa: F811
    for s in (decay_shape(B=1, N=1 << 16), decay_shape(B=1, N=1 << 12, sequences=3)):  # with a workspace
        assert decay(lib, s, workspace=0) == decay(lib, s, back=True, workspace=0) == WORKSPACE
        assert decay(lib, s, workspace=at(16) + 16) == WORKSPACE
        need = lib.flarepp_decay_attention_workspace_bytes(ctypes.byref(s))
        assert decay(lib, s, ws_bytes=need - 1) == WORKSPACE
        assert decay(lib, s, log_decay=0) == decay(lib, s, log_decay=at(10) + 2) == INVALID
        assert decay(lib, s, offsets=at(11) if not s.sequences else 0) == INVALID
        assert decay(lib, s, status=at(17) + 1) == INVALID
        for back, names in ((False, ("Q", "K", "V", "Y")), (True, ("Q", "K", "V", "dY", "dQ", "dK", "dV"))):
            for k in names:
                assert decay(lib, s, back, **{k: None}) == INVALID
                assert decay(lib, s, back, **{k: {"data": 0}}) == INVALID
                assert decay(lib, s, back, **{k: {"data": at(9) + 8}}) == INVALID
                assert decay(lib, s, back, **{k: {"stride_n": 60}}) == INVALID   # no multiple of 16 bytes
                assert decay(lib, s, back, **{k: {"stride_n": 24}}) == INVALID   # rows that overlap
                assert decay(lib, s, back, **{k: {"stride_h": -64}}) == INVALID
                assert decay(lib, s, back, **{k: {"stride_h": 1 << 39}}) in (INVALID, UNSUPPORTED)
        # an output whose heads are one and the same, outputs on inputs and on each other
        assert decay(lib, s, Y={"stride_h": 0}) == INVALID
        for k in ("Q", "K", "V"):
            assert decay(lib, s, Y={"data": at(9)}, **{k: {"data": at(9)}}) == INVALID
        assert decay(lib, s, True, dK={"data": at(9)}, dV={"data": at(9) + 4096}) == INVALID
        assert decay(lib, s, state_out=at(4) + 256) == decay(lib, s, state=at(13) + 256) == INVALID
        assert decay(lib, s, state_out=at(1)) == decay(lib, s, workspace=at(3)) == INVALID
        assert decay(lib, s, True, dstate=at(12)) == decay(lib, s, True, dstate=at(14) + 256) == INVALID


def test_decay_nothing_to_do(lib):  # noqa: F811
    none = dict(Q={"data": 0}, K={"data": 0}, V={"data": 0}, Y={"data": 0}, workspace=0)
    assert decay(lib, decay_shape(B=0), **none) == flarepp.OK
    assert decay(lib, decay_shape(Hq=0, Hk=0), **none) == flarepp.OK
    assert decay(lib, decay_shape(N=0), state=0, state_out=0, **none) == flarepp.OK
    assert decay(lib, decay_shape(N=0), state=at(12), state_out=at(12), **none) == flarepp.OK


def test_decay_step_refusals(lib):  # noqa: F811
    s = decay_shape(N=1)
    assert step(lib, decay_shape(N=2)) == step(lib, decay_shape(B=1, N=1, sequences=1)) == INVALID
    assert step(lib, s, state=0) == step(lib, s, state=at(12) + 4) == step(lib, s, log_decay=0) == INVALID
    assert step(lib, s, state=at(10)) == step(lib, s, state=at(1)) == INVALID
    assert step(lib, s, Y={"data": at(2)}) == step(lib, s, Q={"stride_h": 7}) == INVALID
    assert step(lib, decay_shape(N=1, B=0)) == flarepp.OK


# ------------------------------------------------------------------ rotary positions
def rotary_shape(B=2, Hq=4, Hk=2, N=30, D=64, dtype=flarepp.BF16, sections=(8, 16), pairing=0, real=0,
                 inverse=0, pos=60, axes=None):
    pad = (ctypes.c_int32 * 4)(*(list(sections) + [0] * 4)[:4])
    return flarepp.RotaryShape(B, Hq, Hk, N, D, dtype, len(sections) if axes is None else axes, pad, pairing,
                               real, inverse, pos)


def rotary(lib, s, **over):  # noqa: F811
    H = {"q": s.Hq, "k": s.Hk, "q_out": s.Hq, "k_out": s.Hk}
    v = [None if over.get(n, {}) is None else ctypes.byref(dense(i + 1, s, H[n], s.D, **over.get(n, {})))
         for i, n in enumerate(H)]
    return lib.flarepp_rotary(ctypes.byref(s), over.get("positions", at(6)), over.get("freqs", at(7)), *v, None)


@pytest.mark.parametrize("over,status", [
    (dict(B=-1), INVALID), (dict(D=0), INVALID), (dict(dtype=2), INVALID), (dict(axes=0), INVALID),
    (dict(axes=5), INVALID), (dict(pairing=3), INVALID), (dict(pairing=-1), INVALID),
    (dict(sections=(20, 13)), INVALID), (dict(sections=(-1, 3)), INVALID), (dict(pos=-1), INVALID),
    (dict(D=1028), UNSUPPORTED), (dict(Hq=70000), UNSUPPORTED), (dict(B=1 << 16, N=1 << 16), UNSUPPORTED)])
def test_rotary_shapes(lib, over, status):  # noqa: F811
    assert rotary(lib, rotary_shape(**over)) == status


def test_rotary_refusals(lib):  # noqa: F811
    s = rotary_shape()
    for k in ("q", "k", "q_out", "k_out"):
        assert rotary(lib, s, **{k: None}) == rotary(lib, s, **{k: {"data": 0}}) == INVALID
        assert rotary(lib, s, **{k: {"data": at(9) + 1}}) == rotary(lib, s, **{k: {"stride_n": -1}}) == INVALID
    for k in ("positions", "freqs"):
        assert rotary(lib, s, **{k: 0}) == rotary(lib, s, **{k: at(9) + 2}) == INVALID
        assert rotary(lib, s, **{k: at(3)}) == INVALID      # what an output goes over
    assert rotary(lib, s, q_out={"stride_h": 0}) == rotary(lib, s, q_out={"stride_n": 32}) == INVALID
    assert rotary(lib, s, q_out={"data": at(2)}) == rotary(lib, s, q_out={"data": at(4) + 128}) == INVALID
    assert rotary(lib, s, q_out={"data": at(1) + 128}) == INVALID  # its own input, but not the same place
    # parts of one buffer [B, N, 3, H, D] that lie between each other's rows are apart; shifted into them not
    row = 3 * 4 * 64
    part = {"stride_b": 30 * row, "stride_h": 64, "stride_n": row}
    s = rotary_shape(Hk=4, N=0)
    assert rotary(lib, s) == flarepp.OK
    s = rotary_shape(Hk=4)
    over = dict(q=dict(part, data=at(20)), q_out=dict(part, data=at(30)), k=dict(part, data=at(20) + 512))
    assert rotary(lib, s, k_out=dict(part, data=at(30) + 256), **over) == INVALID
    assert rotary(lib, s, k_out=dict(part, data=at(30) + 2 * row - 256), **over) == INVALID
    assert rotary(lib, rotary_shape(Hq=0, Hk=0), q=None, k=None, q_out=None, k_out=None) == flarepp.OK


# ------------------------------------------------------------------ group norm
def norm_shape(B=2, N=100, C=64, G=4, dtype=flarepp.BF16, param=flarepp.F32, act=3, eps=1e-5):
    return flarepp.NormShape(B, N, C, G, dtype, param, act, eps)


def norm(lib, s, back=False, **over):  # noqa: F811
    names = ("X", "dY", "gamma", "beta", "lengths", "stats", "dX", "dgamma", "dbeta") if back else \
        ("X", "gamma", "beta", "lengths", "Y", "stats")
    v = [over.get(n, at(i + 1)) for i, n in enumerate(names)]
    size, call = ((lib.flarepp_group_norm_bwd_workspace_bytes, lib.flarepp_group_norm_bwd) if back else
                  (lib.flarepp_group_norm_workspace_bytes, lib.flarepp_group_norm_fwd))
    need = over.get("ws_bytes", size(ctypes.byref(s)))
    return call(ctypes.byref(s), *v, over.get("workspace", at(12)), need, over.get("status", 0), None)


@pytest.mark.parametrize("over,status", [
    (dict(B=-1), INVALID), (dict(N=-1), INVALID), (dict(C=0), INVALID), (dict(G=0), INVALID),
    (dict(G=5), INVALID), (dict(dtype=2), INVALID), (dict(param=-1), INVALID), (dict(act=4), INVALID),
    (dict(eps=0.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(C=1 << 21, G=1), UNSUPPORTED),
    (dict(N=1 << 31), UNSUPPORTED), (dict(B=1 << 30, N=1 << 20), UNSUPPORTED)])
def test_norm_shapes(lib, over, status):  # noqa: F811
    s = norm_shape(**over)
    assert norm(lib, s) == norm(lib, s, True) == status
    assert lib.flarepp_group_norm_workspace_bytes(ctypes.byref(s)) == 0
    assert lib.flarepp_group_norm_bwd_workspace_bytes(ctypes.byref(s)) == 0


def test_norm_refusals(lib):  # noqa: F811
    s = norm_shape()
    assert lib.flarepp_group_norm_workspace_bytes(ctypes.byref(norm_shape(N=1))) == 0  # one launch
    for back in (False, True):
        out = "dX" if back else "Y"
        assert norm(lib, s, back, workspace=0) == norm(lib, s, back, workspace=at(12) + 16) == WORKSPACE
        assert norm(lib, s, back, ws_bytes=8) == WORKSPACE
        for k in ("X", out) + (("dY", "stats") if back else ()):
            assert norm(lib, s, back, **{k: 0}) == INVALID
        for k in ("X", out):
            assert norm(lib, s, back, **{k: at(11) + 8}) == INVALID
        for k in ("gamma", "beta", "lengths", "stats"):
            assert norm(lib, s, back, **{k: at(11) + 2}) == INVALID
            assert norm(lib, s, back, **{k: at(11), out: at(11)}) == INVALID
        assert norm(lib, s, back, X=at(11), **{out: at(11) + 256}) == INVALID
        assert norm(lib, s, back, status=at(11) + 1) == norm(lib, s, back, status=at(1)) == INVALID
    assert norm(lib, s, True, dgamma=at(9) + 64) == norm(lib, s, True, dgamma=at(6)) == INVALID
    assert norm(lib, norm_shape(B=0), X=0, Y=0, stats=0, workspace=0) == flarepp.OK


# ------------------------------------------------------------------ the binding's own refusals
def test_binding_wants_device_tensors():
    q = torch.zeros(1, 2, 3, 8, dtype=torch.bfloat16)
    ld = torch.zeros(2)
    with pytest.raises(ValueError):
        flarepp.decay_attention_fwd(q, q, q, ld)
    with pytest.raises(ValueError):
        flarepp.decay_attention_step(q[:, :, 0], q[:, :, 0], q[:, :, 0], ld, torch.zeros(1, 2, 8, 8))
    with pytest.raises(ValueError):
        flarepp.rotary_fwd(q, q, torch.zeros(3, 1, dtype=torch.int32), torch.zeros(4), [4])
    with pytest.raises(ValueError):
        flarepp.group_norm_fwd(torch.zeros(1, 2, 8), 2)
    with pytest.raises(ValueError):
        flarepp.rotary_fwd(q, q, torch.zeros(3, 1, dtype=torch.int32), torch.zeros(4), [4], pairing="thirds")


def test_rotary_frequencies():
    f = flarepp.rotary_frequencies([4, 2], base=100.0, device="cpu")
    assert f.dtype == torch.float32
    assert torch.equal(f, torch.tensor([1.0, 100 ** -0.25, 0.1, 100 ** -0.75, 1.0, 0.1]))
