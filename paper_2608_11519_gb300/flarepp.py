"""Python binding of libflarepp (ctypes): argument marshalling only.

Every step of the routing chain runs in the library's CUDA kernels. PyTorch provides the
device memory and the stream. There is no fallback: if the library is not built, every
call raises.

    from paper_2608_11519_gb300 import flarepp
    Y = flarepp.route_fwd(seeds, Kt, Vt, K, V)              # device tensors
    Y, Q, Z = flarepp.route_fwd_debug(seeds, Kt, Vt, K, V)  # plus the intermediates
    Y = flarepp.route_fwd_host(seeds, Kt, Vt, K, V)         # host tensors in, host Y out
"""
import ctypes
import functools
import inspect
import math
import os

import torch

from . import build as _build

F32, BF16 = 0, 1
OK, ERR_INVALID_ARGUMENT, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_CUDA, ERR_TIMEOUT = range(6)
_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}

EXPORTED = ("flarepp_route_workspace_bytes", "flarepp_route_fwd", "flarepp_route_fwd_debug",
            "flarepp_route_fwd_profiled", "flarepp_route_fwd_noalloc",
            "flarepp_flare_fwd", "flarepp_route_host_buffer_bytes", "flarepp_route_fwd_host",
            "flarepp_flare_fwd_host",
            "flarepp_mixer_workspace_bytes", "flarepp_mixer_fwd", "flarepp_mixer_fwd_profiled",
            "flarepp_mixer_saved_bytes", "flarepp_mixer_fwd_train",
            "flarepp_mixer_bwd_workspace_bytes", "flarepp_mixer_bwd",
            "flarepp_route_saved_bytes", "flarepp_route_fwd_train",
            "flarepp_route_bwd_workspace_bytes", "flarepp_route_bwd",
            "flarepp_route_device_status", "flarepp_status_string", "flarepp_version",
            "flarepp_linear_workspace_bytes", "flarepp_linear_fwd",
            "flarepp_linear_bwd_workspace_bytes", "flarepp_linear_bwd",
            "flarepp_embedding_fwd", "flarepp_embedding_bwd_workspace_bytes",
            "flarepp_embedding_bwd", "flarepp_adamw_step", "flarepp_adamw_moments",
            "flarepp_layers_device_status", "flarepp_adamw_step_unbiased")
N_STAGE_EVENTS = 6
STAGES = ("encode1", "combine1", "encode2", "combine2", "decode")


class Shape(ctypes.Structure):
    """Mirror of ``flarepp_shape`` in include/flarepp.h."""
    _fields_ = [("B", ctypes.c_int64), ("H", ctypes.c_int64), ("N", ctypes.c_int64),
                ("M", ctypes.c_int64), ("D", ctypes.c_int64), ("dtype", ctypes.c_int32)]


class LinearShape(ctypes.Structure):
    """Mirror of ``flarepp_linear_shape`` in include/flarepp.h."""
    _fields_ = [("rows", ctypes.c_int64), ("in_", ctypes.c_int64), ("out", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("act", ctypes.c_int32)]


class EmbeddingShape(ctypes.Structure):
    """Mirror of ``flarepp_embedding_shape`` in include/flarepp.h."""
    _fields_ = [("T", ctypes.c_int64), ("V", ctypes.c_int64), ("C", ctypes.c_int64),
                ("dtype", ctypes.c_int32), ("id_bytes", ctypes.c_int32)]


class AdamwTensor(ctypes.Structure):
    """Mirror of ``flarepp_adamw_tensor`` in include/flarepp.h."""
    _fields_ = [("param", ctypes.c_void_p), ("grad", ctypes.c_void_p),
                ("master", ctypes.c_void_p), ("m", ctypes.c_void_p), ("v", ctypes.c_void_p),
                ("m_scale", ctypes.c_void_p), ("v_scale", ctypes.c_void_p),
                ("n", ctypes.c_int64), ("param_dtype", ctypes.c_int32),
                ("grad_dtype", ctypes.c_int32)]


class AdamwHyper(ctypes.Structure):
    """Mirror of ``flarepp_adamw_hyper`` in include/flarepp.h."""
    _fields_ = [("lr", ctypes.c_double), ("beta1", ctypes.c_double), ("beta2", ctypes.c_double),
                ("eps", ctypes.c_double), ("weight_decay", ctypes.c_double),
                ("step", ctypes.c_int64), ("state_bits", ctypes.c_int32)]


class FlareppError(RuntimeError):
    def __init__(self, status: int, what: str):
        super().__init__(f"{what}: status {status} ({status_string(status)})")
        self.status = status


_LIB = None


def lib_path() -> str:
    return _build.lib_path()


def load(path: str = None):
    """Load libflarepp.so (built by ``build.build()``); raises if it is missing."""
    global _LIB
    if _LIB is not None and path is None:
        return _LIB
    path = path or lib_path()
    if not os.path.exists(path):
        raise RuntimeError(f"libflarepp is not built ({path} missing); run "
                           "`python -c 'import __graft_entry__ as g; g.build()'` first")
    lib = ctypes.CDLL(path)
    vp, sz = ctypes.c_void_p, ctypes.c_size_t
    sp = ctypes.POINTER(Shape)
    lib.flarepp_route_workspace_bytes.restype = sz
    lib.flarepp_route_workspace_bytes.argtypes = [sp]
    lib.flarepp_route_fwd.restype = ctypes.c_int
    lib.flarepp_route_fwd.argtypes = [sp, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, sz, vp]
    lib.flarepp_route_fwd_debug.restype = ctypes.c_int
    lib.flarepp_route_fwd_debug.argtypes = [sp, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, sz,
                                            vp, vp, vp]
    lib.flarepp_route_fwd_profiled.restype = ctypes.c_int
    lib.flarepp_route_fwd_profiled.argtypes = [sp, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, sz,
                                               vp, ctypes.POINTER(ctypes.c_void_p), ctypes.c_int]
    lib.flarepp_test_wait_fault.restype = None
    lib.flarepp_test_wait_fault.argtypes = [ctypes.c_int, ctypes.c_int64, ctypes.c_uint64]
    lib.flarepp_route_fwd_noalloc.restype = ctypes.c_int
    lib.flarepp_route_fwd_noalloc.argtypes = [sp, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp]
    lib.flarepp_flare_fwd.restype = ctypes.c_int
    lib.flarepp_flare_fwd.argtypes = [sp, vp, vp, vp, ctypes.c_float, vp, vp, sz, vp, vp]
    lib.flarepp_route_host_buffer_bytes.restype = sz
    lib.flarepp_route_host_buffer_bytes.argtypes = [sp]
    lib.flarepp_route_fwd_host.restype = ctypes.c_int
    lib.flarepp_route_fwd_host.argtypes = [sp, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, sz, vp]
    lib.flarepp_flare_fwd_host.restype = ctypes.c_int
    lib.flarepp_flare_fwd_host.argtypes = [sp, vp, vp, vp, ctypes.c_float, vp, vp, sz, vp]
    lib.flarepp_mixer_workspace_bytes.restype = sz
    lib.flarepp_mixer_workspace_bytes.argtypes = [sp, ctypes.c_int]
    lib.flarepp_mixer_fwd.restype = ctypes.c_int
    lib.flarepp_mixer_fwd.argtypes = [sp, ctypes.c_int, vp, vp, vp, vp, ctypes.c_float, vp, vp,
                                      sz, vp]
    lib.flarepp_mixer_fwd_profiled.restype = ctypes.c_int
    lib.flarepp_mixer_fwd_profiled.argtypes = [sp, ctypes.c_int, vp, vp, vp, vp, ctypes.c_float,
                                               vp, vp, sz, vp, ctypes.POINTER(ctypes.c_void_p),
                                               ctypes.c_int]
    lib.flarepp_mixer_saved_bytes.restype = sz
    lib.flarepp_mixer_saved_bytes.argtypes = [sp, ctypes.c_int]
    lib.flarepp_mixer_fwd_train.restype = ctypes.c_int
    lib.flarepp_mixer_fwd_train.argtypes = [sp, ctypes.c_int, vp, vp, vp, vp, ctypes.c_float, vp,
                                            vp, sz, vp, sz, vp]
    lib.flarepp_mixer_bwd_workspace_bytes.restype = sz
    lib.flarepp_mixer_bwd_workspace_bytes.argtypes = [sp, ctypes.c_int]
    lib.flarepp_mixer_bwd.restype = ctypes.c_int
    lib.flarepp_mixer_bwd.argtypes = [sp, ctypes.c_int, vp, vp, vp, vp, ctypes.c_float, vp, sz,
                                      vp, vp, vp, vp, vp, vp, sz, vp]
    lib.flarepp_route_saved_bytes.restype = sz
    lib.flarepp_route_saved_bytes.argtypes = [sp]
    lib.flarepp_route_fwd_train.restype = ctypes.c_int
    lib.flarepp_route_fwd_train.argtypes = [sp, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, sz,
                                            vp, sz, vp]
    lib.flarepp_route_bwd_workspace_bytes.restype = sz
    lib.flarepp_route_bwd_workspace_bytes.argtypes = [sp]
    lib.flarepp_route_bwd.restype = ctypes.c_int
    lib.flarepp_route_bwd.argtypes = [sp, vp, vp, vp, vp, vp, ctypes.c_float, vp, vp, vp, sz,
                                      vp, vp, vp, vp, vp, vp, sz, vp]
    lib.flarepp_route_device_status.restype = ctypes.c_int
    lib.flarepp_route_device_status.argtypes = [sp, vp, vp, ctypes.POINTER(ctypes.c_int32)]
    lp, ep = ctypes.POINTER(LinearShape), ctypes.POINTER(EmbeddingShape)
    tp, hp = ctypes.POINTER(AdamwTensor), ctypes.POINTER(AdamwHyper)
    for name, args in (
            ("linear_workspace_bytes", [lp]), ("linear_bwd_workspace_bytes", [lp]),
            ("embedding_bwd_workspace_bytes", [ep])):
        getattr(lib, "flarepp_" + name).restype = sz
        getattr(lib, "flarepp_" + name).argtypes = args
    for name, args in (
            ("linear_fwd", [lp] + [vp] * 7 + [sz, vp, vp]),
            ("linear_bwd", [lp] + [vp] * 8 + [sz, vp, vp]),
            ("embedding_fwd", [ep, vp, vp, ctypes.c_float, vp, vp, vp]),
            ("embedding_bwd", [ep, vp, vp, ctypes.c_float, vp, vp, sz, vp, vp]),
            ("adamw_step", [tp, ctypes.c_int64, hp, vp]),
            ("adamw_step_unbiased", [tp, ctypes.c_int64, hp, vp]),
            ("adamw_moments", [tp, ctypes.c_int64, vp, vp, vp]),
            ("layers_device_status", [vp, ctypes.POINTER(ctypes.c_int32)])):
        getattr(lib, "flarepp_" + name).restype = ctypes.c_int
        getattr(lib, "flarepp_" + name).argtypes = args
    lib.flarepp_status_string.restype = ctypes.c_char_p
    lib.flarepp_status_string.argtypes = [ctypes.c_int]
    lib.flarepp_version.restype = ctypes.c_char_p
    if path == lib_path():
        _LIB = lib
    return lib


def status_string(status: int) -> str:
    return load().flarepp_status_string(int(status)).decode()


def version() -> str:
    return load().flarepp_version().decode()


def make_shape(B, H, N, M, D, dtype) -> Shape:
    if isinstance(dtype, torch.dtype):
        dtype = _DTYPES[dtype]
    return Shape(int(B), int(H), int(N), int(M), int(D), int(dtype))


def workspace_bytes(B, H, N, M, D, dtype) -> int:
    return int(load().flarepp_route_workspace_bytes(ctypes.byref(make_shape(B, H, N, M, D, dtype))))


def _ptr(t):
    return None if t is None else ctypes.c_void_p(t.data_ptr())


def _shape_of(seeds, Kt, Vt, K, V) -> Shape:
    for t in (seeds, Kt, Vt, K, V):
        if not isinstance(t, torch.Tensor):
            raise TypeError("inputs must be torch tensors")
        if not t.is_contiguous():
            raise ValueError("inputs must be contiguous (D innermost)")
        if t.dtype != K.dtype:
            raise TypeError("all inputs must share one dtype")
    if K.dtype not in _DTYPES:
        raise TypeError(f"unsupported dtype {K.dtype}; use float32 or bfloat16")
    if K.dim() != 4 or seeds.dim() != 3:
        raise ValueError("expected seeds [H,M,D] and Kt, Vt, K, V [B,H,N,D]")
    B, H, N, D = K.shape
    M = seeds.shape[1]
    if tuple(seeds.shape) != (H, M, D):
        raise ValueError(f"seeds shape {tuple(seeds.shape)} != {(H, M, D)}")
    for t in (Kt, Vt, V):
        if tuple(t.shape) != (B, H, N, D):
            raise ValueError(f"input shape {tuple(t.shape)} != {(B, H, N, D)}")
    return make_shape(B, H, N, M, D, K.dtype)


def _nbytes(t):
    return 0 if t is None else t.numel() * t.element_size()


def _check_out(t, like, name):
    """A caller-supplied output: a contiguous tensor of ``like``'s shape and dtype (the kernels
    write every element of it, so a smaller buffer would be written past its end)."""
    if not isinstance(t, torch.Tensor) or tuple(t.shape) != tuple(like.shape) or \
            t.dtype != like.dtype or not t.is_contiguous():
        raise ValueError(f"{name} must be a contiguous {like.dtype} tensor of shape "
                         f"{tuple(like.shape)}")
    return t


def _check_device(what, device, **tensors):
    """Every tensor a device-side call touches sits on ``device``, a CUDA device: the library
    takes raw pointers and cannot tell a host address, or another GPU's, from its own."""
    if device.type != "cuda":
        raise ValueError(f"{what} takes device tensors (the *_host entries take host tensors)")
    for name, t in tensors.items():
        if isinstance(t, torch.Tensor) and t.device != device:
            raise ValueError(f"{what}: {name} is on {t.device}, expected {device}")


def _on_device(arg):
    """Run the wrapped entry with the CUDA device of argument ``arg`` current. The library
    works on the current device (the no-allocation entry looks its scratch array up there,
    and launches go to the current device's context), so a call on tensors of another GPU
    must make that GPU current first. ``arg`` names a device tensor, or the ``device``
    argument of a host entry."""
    def wrap(fn):
        sig = inspect.signature(fn)

        @functools.wraps(fn)
        def call(*a, **kw):
            v = sig.bind_partial(*a, **kw).arguments.get(arg)
            if v is None and arg in sig.parameters:
                v = sig.parameters[arg].default
            dev = v.device if isinstance(v, torch.Tensor) else (
                torch.device(v) if isinstance(v, (str, torch.device)) else None)
            if dev is None or dev.type != "cuda" or dev.index is None:
                return fn(*a, **kw)
            with torch.cuda.device(dev):
                return fn(*a, **kw)
        return call
    return wrap


class Workspace:
    """A reusable device workspace, grown on demand (one per stream at a time)."""

    def __init__(self, device=None):
        self.device = device
        self.buf = None

    def get(self, nbytes: int, device):
        if nbytes == 0:
            return None
        if self.buf is None or self.buf.numel() < nbytes or self.buf.device != device:
            self.buf = torch.empty(nbytes + 256, dtype=torch.uint8, device=device)
        # the library wants 256-byte alignment; torch allocations are at least that aligned
        if self.buf.data_ptr() % 256 != 0:
            raise RuntimeError("workspace allocation is not 256-byte aligned")
        return self.buf


def _call(debug, seeds, Kt, Vt, K, V, scale, Y, workspace, stream, Q_out, Z_out, events=None):
    lib = load()
    shape = _shape_of(seeds, Kt, Vt, K, V)
    if Y is not None:
        _check_out(Y, K, "Y")
    _check_device("route_fwd", K.device, seeds=seeds, Kt=Kt, Vt=Vt, V=V, Y=Y, Q_out=Q_out,
                  Z_out=Z_out, workspace=workspace)
    if scale is None:
        scale = 1.0 / math.sqrt(shape.D)
    if Y is None:
        Y = torch.empty_like(K)
    nbytes = int(lib.flarepp_route_workspace_bytes(ctypes.byref(shape)))
    if isinstance(workspace, Workspace):
        ws = workspace.get(nbytes, K.device)
    elif workspace is None:
        ws = torch.empty(nbytes, dtype=torch.uint8, device=K.device) if nbytes else None
    else:
        ws = workspace
    ws_bytes = 0 if ws is None else ws.numel() * ws.element_size()
    if stream is None:
        stream = torch.cuda.current_stream(K.device)
    st = ctypes.c_void_p(stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream))
    if events is not None:
        arr = (ctypes.c_void_p * len(events))(*[ctypes.c_void_p(e) for e in events])
        rc = lib.flarepp_route_fwd_profiled(ctypes.byref(shape), _ptr(seeds), _ptr(Kt), _ptr(Vt),
                                            _ptr(K), _ptr(V), float(scale), _ptr(Y), _ptr(ws),
                                            ws_bytes, st, arr, len(events))
        if rc != OK:
            raise FlareppError(rc, "flarepp_route_fwd_profiled")
        return Y
    if debug:
        rc = lib.flarepp_route_fwd_debug(ctypes.byref(shape), _ptr(seeds), _ptr(Kt), _ptr(Vt),
                                         _ptr(K), _ptr(V), float(scale), _ptr(Y), _ptr(ws),
                                         ws_bytes, st, _ptr(Q_out), _ptr(Z_out))
    else:
        rc = lib.flarepp_route_fwd(ctypes.byref(shape), _ptr(seeds), _ptr(Kt), _ptr(Vt), _ptr(K),
                                   _ptr(V), float(scale), _ptr(Y), _ptr(ws), ws_bytes, st)
    if rc != OK:
        raise FlareppError(rc, "flarepp_route_fwd" + ("_debug" if debug else ""))
    return Y


def device_status(shape_or_tensors, workspace, stream=None) -> int:
    """The device status word the last call left in ``workspace`` (synchronises ``stream``):
    OK, or ERR_TIMEOUT when a bounded wait inside a kernel gave up."""
    shape = (shape_or_tensors if isinstance(shape_or_tensors, Shape)
             else _shape_of(*shape_or_tensors))
    buf = workspace.buf if isinstance(workspace, Workspace) else workspace
    dev = buf.device if isinstance(buf, torch.Tensor) and buf.is_cuda else None
    with torch.cuda.device(dev):
        if stream is None:
            stream = torch.cuda.current_stream()
        out = ctypes.c_int32(-1)
        rc = load().flarepp_route_device_status(ctypes.byref(shape), _ptr(buf),
                                                ctypes.c_void_p(stream.cuda_stream),
                                                ctypes.byref(out))
    if rc != OK:
        raise FlareppError(rc, "flarepp_route_device_status")
    return int(out.value)


@_on_device("K")
def route_fwd(seeds, Kt, Vt, K, V, scale=None, Y=None, workspace=None, stream=None):
    """Y = routing chain (Sec. 3.2) on device tensors; returns Y [B,H,N,D] (enqueued on
    ``stream``, default torch's current stream)."""
    return _call(False, seeds, Kt, Vt, K, V, scale, Y, workspace, stream, None, None)


class StageEvents:
    """Six timing events the library records around its stages (flarepp_route_fwd_profiled)."""

    def __init__(self, stream=None):
        stream = stream or torch.cuda.current_stream()
        self.events = [torch.cuda.Event(enable_timing=True) for _ in range(N_STAGE_EVENTS)]
        for e in self.events:  # create the underlying cudaEvent_t
            e.record(stream)
        self.handles = [int(e.cuda_event) for e in self.events]

    def stage_ms(self):
        """Milliseconds of each stage of the last recorded call (synchronises on the events)."""
        self.events[-1].synchronize()
        return {name: self.events[i].elapsed_time(self.events[i + 1])
                for i, name in enumerate(STAGES)}


@_on_device("K")
def route_fwd_profiled(seeds, Kt, Vt, K, V, events: StageEvents, scale=None, Y=None,
                       workspace=None, stream=None):
    """``route_fwd`` that records ``events`` around each stage on the launching stream."""
    return _call(False, seeds, Kt, Vt, K, V, scale, Y, workspace, stream, None, None,
                 events.handles)


@_on_device("K")
def route_fwd_noalloc(seeds, Kt, Vt, K, V, scale=None, Y=None, stream=None):
    """``route_fwd`` through flarepp_route_fwd_noalloc: for callers that cannot allocate
    device memory at call time, the library uses its own fixed 64 MiB scratch array instead
    of a workspace (larger shapes raise ERR_WORKSPACE). Calls that overlap on the GPU share
    that array and race; the first call on a device should come before any stream capture.
    Y is allocated here only when not given."""
    lib = load()
    shape = _shape_of(seeds, Kt, Vt, K, V)
    if Y is not None:
        _check_out(Y, K, "Y")
    _check_device("route_fwd_noalloc", K.device, seeds=seeds, Kt=Kt, Vt=Vt, V=V, Y=Y)
    if scale is None:
        scale = 1.0 / math.sqrt(shape.D)
    if Y is None:
        Y = torch.empty_like(K)
    if stream is None:
        stream = torch.cuda.current_stream(K.device)
    rc = lib.flarepp_route_fwd_noalloc(ctypes.byref(shape), _ptr(seeds), _ptr(Kt), _ptr(Vt),
                                       _ptr(K), _ptr(V), float(scale), _ptr(Y),
                                       ctypes.c_void_p(stream.cuda_stream))
    if rc != OK:
        raise FlareppError(rc, "flarepp_route_fwd_noalloc")
    return Y


@_on_device("K")
def route_fwd_debug(seeds, Kt, Vt, K, V, scale=None, Y=None, workspace=None, stream=None):
    """Like ``route_fwd``, also returning the float32 intermediates Q and Z [B,H,M,D]."""
    B, H, N, D = K.shape
    M = seeds.shape[1]
    Q = torch.empty(B, H, M, D, dtype=torch.float32, device=K.device)
    Z = torch.empty_like(Q)
    Y = _call(True, seeds, Kt, Vt, K, V, scale, Y, workspace, stream, Q, Z)
    return Y, Q, Z


@_on_device("K")
def flare_fwd(Q, K, V, scale=None, Y=None, workspace=None, stream=None, Z_out=None):
    """FLARE with learned queries (Sec. 3, eq. prelim_flare_sdpa) on device tensors:
    Z = SDPA(Q_h, K, V), Y = SDPA(K, Q_h, Z). Q [H, M, D] is shared by the batch; K, V
    [B, H, N, D]. Returns Y; ``Z_out`` (float32 [B, H, M, D], device) receives Z if given."""
    lib = load()
    shape = _shape_of(Q, K, V, K, V)
    if Y is not None:
        _check_out(Y, K, "Y")
    if Z_out is not None and (Z_out.dtype != torch.float32 or not Z_out.is_contiguous() or
                              tuple(Z_out.shape) != (shape.B, shape.H, shape.M, shape.D)):
        raise ValueError("Z_out must be a contiguous float32 [B, H, M, D] tensor")
    _check_device("flare_fwd", K.device, Q=Q, V=V, Y=Y, Z_out=Z_out)
    if scale is None:
        scale = 1.0 / math.sqrt(shape.D)
    if Y is None:
        Y = torch.empty_like(K)
    nbytes = int(lib.flarepp_route_workspace_bytes(ctypes.byref(shape)))
    ws = (workspace if isinstance(workspace, Workspace) else Workspace()).get(nbytes, K.device)
    st = stream if stream is not None else torch.cuda.current_stream(K.device)
    rc = lib.flarepp_flare_fwd(ctypes.byref(shape), _ptr(Q), _ptr(K), _ptr(V), float(scale),
                               _ptr(Y), None if ws is None else ctypes.c_void_p(ws.data_ptr()),
                               nbytes, ctypes.c_void_p(st.cuda_stream), _ptr(Z_out))
    if rc != OK:
        raise FlareppError(rc, "flarepp_flare_fwd")
    return Y


MIXER_STAGES = ("projection", "chain", "output")


class MixerEvents:
    """Four timing events the library records around the mixer's stages
    (flarepp_mixer_fwd_profiled)."""

    def __init__(self, stream=None):
        stream = stream or torch.cuda.current_stream()
        self.events = [torch.cuda.Event(enable_timing=True) for _ in range(4)]
        for e in self.events:  # create the underlying cudaEvent_t
            e.record(stream)
        self.handles = (ctypes.c_void_p * 4)(*[ctypes.c_void_p(int(e.cuda_event))
                                               for e in self.events])

    def stage_ms(self):
        """Milliseconds of each stage of the last recorded call (synchronises on the events)."""
        self.events[-1].synchronize()
        return {s: self.events[i].elapsed_time(self.events[i + 1])
                for i, s in enumerate(MIXER_STAGES)}


@_on_device("X")
def mixer_fwd(X, W_in, Wo, seeds, scale=None, O=None, workspace=None, stream=None, events=None):
    """The FLARE++ mixer layer (Fig. 1) on device tensors: X [B, N, C], W_in [P*C, C] (P = 4:
    K, V, K~, V~; P = 2: shared projection), Wo [C, C] (both out x in), seeds [H, M, D].
    Returns O [B, N, C]."""
    lib = load()
    shape, P = _mixer_shape(X, W_in, Wo, seeds)
    if O is not None:
        _check_out(O, X, "O")
    _check_device("mixer_fwd", X.device, W_in=W_in, Wo=Wo, seeds=seeds, O=O)
    if scale is None:
        scale = 1.0 / math.sqrt(shape.D)
    if O is None:
        O = torch.empty_like(X)
    nbytes = int(lib.flarepp_mixer_workspace_bytes(ctypes.byref(shape), P))
    ws = (workspace if isinstance(workspace, Workspace) else Workspace()).get(nbytes, X.device)
    st = stream if stream is not None else torch.cuda.current_stream(X.device)
    args = (ctypes.byref(shape), P, _ptr(X), _ptr(W_in), _ptr(Wo), _ptr(seeds), float(scale),
            _ptr(O), None if ws is None else ctypes.c_void_p(ws.data_ptr()), nbytes,
            ctypes.c_void_p(st.cuda_stream))
    if events is None:
        rc = lib.flarepp_mixer_fwd(*args)
    else:
        rc = lib.flarepp_mixer_fwd_profiled(*args, events.handles, 4)
    if rc != OK:
        raise FlareppError(rc, "flarepp_mixer_fwd")
    return O


def _mixer_shape(X, W_in, Wo, seeds):
    for t in (X, W_in, Wo, seeds):
        if not isinstance(t, torch.Tensor) or not t.is_contiguous():
            raise ValueError("inputs must be contiguous torch tensors")
        if t.dtype != torch.bfloat16:
            raise TypeError("the mixer takes bfloat16 tensors")
    if X.dim() != 3 or W_in.dim() != 2 or Wo.dim() != 2 or seeds.dim() != 3:
        raise ValueError("expected X [B,N,C], W_in [P*C,C], Wo [C,C], seeds [H,M,D], C = H*D")
    B, N, C = X.shape
    H, M, D = seeds.shape
    if H * D != C or tuple(Wo.shape) != (C, C) or W_in.shape[1] != C or \
            W_in.shape[0] not in (2 * C, 4 * C):
        raise ValueError("expected X [B,N,C], W_in [P*C,C], Wo [C,C], seeds [H,M,D], C = H*D")
    return make_shape(B, H, N, M, D, torch.bfloat16), W_in.shape[0] // C


@_on_device("X")
def mixer_fwd_train(X, W_in, Wo, seeds, scale=None, O=None, saved=None, workspace=None,
                    stream=None):
    """The mixer layer's forward that keeps its backward's state. Returns (O, saved)."""
    lib = load()
    shape, P = _mixer_shape(X, W_in, Wo, seeds)
    if O is not None:
        _check_out(O, X, "O")
    _check_device("mixer_fwd_train", X.device, W_in=W_in, Wo=Wo, seeds=seeds, O=O, saved=saved)
    if scale is None:
        scale = 1.0 / math.sqrt(shape.D)
    if O is None:
        O = torch.empty_like(X)
    sbytes = int(lib.flarepp_mixer_saved_bytes(ctypes.byref(shape), P))
    if saved is None or _nbytes(saved) < sbytes:
        saved = torch.empty(max(sbytes, 1), dtype=torch.uint8, device=X.device)
    nbytes = int(lib.flarepp_mixer_workspace_bytes(ctypes.byref(shape), P))
    ws = (workspace if isinstance(workspace, Workspace) else Workspace()).get(nbytes, X.device)
    st = stream if stream is not None else torch.cuda.current_stream(X.device)
    rc = lib.flarepp_mixer_fwd_train(ctypes.byref(shape), P, _ptr(X), _ptr(W_in), _ptr(Wo),
                                     _ptr(seeds), float(scale), _ptr(O), _ptr(saved), sbytes,
                                     None if ws is None else ctypes.c_void_p(ws.data_ptr()),
                                     nbytes, ctypes.c_void_p(st.cuda_stream))
    if rc != OK:
        raise FlareppError(rc, "flarepp_mixer_fwd_train")
    return O, saved


@_on_device("X")
def mixer_bwd(X, W_in, Wo, seeds, saved, dO, scale=None, grads=None, workspace=None,
              stream=None):
    """The mixer layer's backward from :func:`mixer_fwd_train`'s ``saved``: returns
    (dX, dW_in, dWo, dseeds) in bf16; ``grads`` may supply those four output tensors."""
    lib = load()
    shape, P = _mixer_shape(X, W_in, Wo, seeds)
    if tuple(dO.shape) != tuple(X.shape) or dO.dtype != X.dtype or not dO.is_contiguous():
        raise ValueError("dO must be a contiguous tensor of X's shape and dtype")
    if grads is not None:
        if len(grads) != 4:
            raise ValueError("grads must hold four tensors: dX, dW_in, dWo, dseeds")
        grads = tuple(_check_out(g, like, name) for g, like, name in
                      zip(grads, (X, W_in, Wo, seeds), ("dX", "dW_in", "dWo", "dseeds")))
    _check_device("mixer_bwd", X.device, W_in=W_in, Wo=Wo, seeds=seeds, saved=saved, dO=dO,
                  **({} if grads is None else dict(zip(("dX", "dW_in", "dWo", "dseeds"), grads))))
    if scale is None:
        scale = 1.0 / math.sqrt(shape.D)
    if grads is None:
        grads = (torch.empty_like(X), torch.empty_like(W_in), torch.empty_like(Wo),
                 torch.empty_like(seeds))
    nbytes = int(lib.flarepp_mixer_bwd_workspace_bytes(ctypes.byref(shape), P))
    ws = (workspace if isinstance(workspace, Workspace) else Workspace()).get(nbytes, X.device)
    st = stream if stream is not None else torch.cuda.current_stream(X.device)
    rc = lib.flarepp_mixer_bwd(ctypes.byref(shape), P, _ptr(X), _ptr(W_in), _ptr(Wo),
                               _ptr(seeds), float(scale), _ptr(saved),
                               _nbytes(saved), _ptr(dO),
                               *(_ptr(g) for g in grads),
                               None if ws is None else ctypes.c_void_p(ws.data_ptr()), nbytes,
                               ctypes.c_void_p(st.cuda_stream))
    if rc != OK:
        raise FlareppError(rc, "flarepp_mixer_bwd")
    return grads


@_on_device("K")
def route_fwd_train(seeds, Kt, Vt, K, V, scale=None, Y=None, saved=None, workspace=None,
                    stream=None):
    """The chain's forward that also keeps the state its backward needs (App. A.5).
    Returns (Y, saved): ``saved`` is an opaque uint8 device tensor for :func:`route_bwd`."""
    lib = load()
    shape = _shape_of(seeds, Kt, Vt, K, V)
    if Y is not None:
        _check_out(Y, K, "Y")
    _check_device("route_fwd_train", K.device, seeds=seeds, Kt=Kt, Vt=Vt, V=V, Y=Y, saved=saved)
    if scale is None:
        scale = 1.0 / math.sqrt(shape.D)
    if Y is None:
        Y = torch.empty_like(K)
    sbytes = int(lib.flarepp_route_saved_bytes(ctypes.byref(shape)))
    if saved is None or _nbytes(saved) < sbytes:
        saved = torch.empty(max(sbytes, 1), dtype=torch.uint8, device=K.device)
    nbytes = int(lib.flarepp_route_workspace_bytes(ctypes.byref(shape)))
    ws = (workspace if isinstance(workspace, Workspace) else Workspace()).get(nbytes, K.device)
    st = stream if stream is not None else torch.cuda.current_stream(K.device)
    rc = lib.flarepp_route_fwd_train(ctypes.byref(shape), _ptr(seeds), _ptr(Kt), _ptr(Vt),
                                     _ptr(K), _ptr(V), float(scale), _ptr(Y), _ptr(saved),
                                     sbytes, None if ws is None else ctypes.c_void_p(ws.data_ptr()),
                                     nbytes, ctypes.c_void_p(st.cuda_stream))
    if rc != OK:
        raise FlareppError(rc, "flarepp_route_fwd_train")
    return Y, saved


@_on_device("K")
def route_bwd(seeds, Kt, Vt, K, V, Y, dY, saved, scale=None, grads=None, workspace=None,
              stream=None):
    """Backward of the chain (App. A.5) from :func:`route_fwd_train`'s ``Y`` and ``saved``.
    Returns (dseeds [H, M, D], dKt, dVt, dK, dV [B, H, N, D]) in the input dtype; ``grads``
    may supply those five output tensors."""
    lib = load()
    shape = _shape_of(seeds, Kt, Vt, K, V)
    for t in (Y, dY):
        if tuple(t.shape) != tuple(K.shape) or t.dtype != K.dtype or not t.is_contiguous():
            raise ValueError("Y and dY must be contiguous tensors of K's shape and dtype")
    names = ("dseeds", "dKt", "dVt", "dK", "dV")
    if grads is not None:
        if len(grads) != 5:
            raise ValueError("grads must hold five tensors: dseeds, dKt, dVt, dK, dV")
        grads = tuple(_check_out(g, like, name) for g, like, name in
                      zip(grads, (seeds, Kt, Vt, K, V), names))
    _check_device("route_bwd", K.device, seeds=seeds, Kt=Kt, Vt=Vt, V=V, Y=Y, dY=dY,
                  saved=saved, **({} if grads is None else dict(zip(names, grads))))
    if scale is None:
        scale = 1.0 / math.sqrt(shape.D)
    if grads is None:
        grads = (torch.empty_like(seeds), torch.empty_like(Kt), torch.empty_like(Vt),
                 torch.empty_like(K), torch.empty_like(V))
    sbytes = int(lib.flarepp_route_saved_bytes(ctypes.byref(shape)))
    nbytes = int(lib.flarepp_route_bwd_workspace_bytes(ctypes.byref(shape)))
    ws = (workspace if isinstance(workspace, Workspace) else Workspace()).get(nbytes, K.device)
    st = stream if stream is not None else torch.cuda.current_stream(K.device)
    rc = lib.flarepp_route_bwd(ctypes.byref(shape), _ptr(seeds), _ptr(Kt), _ptr(Vt), _ptr(K),
                               _ptr(V), float(scale), _ptr(Y), _ptr(dY), _ptr(saved),
                               _nbytes(saved),
                               *(_ptr(g) for g in grads),
                               None if ws is None else ctypes.c_void_p(ws.data_ptr()), nbytes,
                               ctypes.c_void_p(st.cuda_stream))
    if rc != OK:
        raise FlareppError(rc, "flarepp_route_bwd")
    return grads


@_on_device("device")
def route_fwd_host(seeds, Kt, Vt, K, V, scale=None, Y_host=None, device="cuda", workspace=None,
                   stream=None, dev_bufs=None):
    """End-to-end call on host tensors through ``flarepp_route_fwd_host``: the library copies
    the inputs to the device, runs the chain and copies Y back into ``Y_host`` (allocated
    pinned here if not given), overlapping the copies with the computation by head groups.
    Pass pinned host tensors for the copies to overlap. Returns Y_host once the copy has
    completed. ``workspace`` (a :class:`Workspace`) holds the device buffer between calls;
    ``dev_bufs`` is accepted for compatibility and unused."""
    del dev_bufs
    lib = load()
    shape = _shape_of(seeds, Kt, Vt, K, V)
    for t in (seeds, Kt, Vt, K, V):
        if t.is_cuda:
            raise ValueError("route_fwd_host takes host tensors")
    if scale is None:
        scale = 1.0 / math.sqrt(shape.D)
    if Y_host is None:
        Y_host = torch.empty(K.shape, dtype=K.dtype, pin_memory=True)
    elif tuple(Y_host.shape) != tuple(K.shape) or Y_host.dtype != K.dtype or Y_host.is_cuda:
        raise ValueError("Y_host must be a host tensor of K's shape and dtype")
    dev = torch.device(device)
    if dev.index is None:
        dev = torch.device("cuda", torch.cuda.current_device())
    nbytes = int(lib.flarepp_route_host_buffer_bytes(ctypes.byref(shape)))
    ws = workspace if workspace is not None else Workspace()
    buf = ws.get(nbytes, dev) if nbytes else None
    st = stream if stream is not None else torch.cuda.current_stream(dev)
    rc = lib.flarepp_route_fwd_host(ctypes.byref(shape), _ptr(seeds), _ptr(Kt), _ptr(Vt), _ptr(K),
                                    _ptr(V), float(scale), _ptr(Y_host),
                                    None if buf is None else ctypes.c_void_p(buf.data_ptr()),
                                    nbytes, ctypes.c_void_p(st.cuda_stream))
    if rc != 0:
        raise FlareppError(rc, "flarepp_route_fwd_host")
    st.synchronize()
    return Y_host


@_on_device("device")
def flare_fwd_host(Q, K, V, scale=None, Y_host=None, device="cuda", workspace=None, stream=None):
    """FLARE with learned queries Q [H, M, D] on host tensors through
    ``flarepp_flare_fwd_host``: copies in, FLARE, Y copied back into ``Y_host`` (allocated
    pinned here if not given), overlapped by head groups. Returns Y_host once it is filled."""
    lib = load()
    shape = _shape_of(Q, K, V, K, V)
    for t in (Q, K, V):
        if t.is_cuda:
            raise ValueError("flare_fwd_host takes host tensors")
    if scale is None:
        scale = 1.0 / math.sqrt(shape.D)
    if Y_host is None:
        Y_host = torch.empty(K.shape, dtype=K.dtype, pin_memory=True)
    elif tuple(Y_host.shape) != tuple(K.shape) or Y_host.dtype != K.dtype or Y_host.is_cuda:
        raise ValueError("Y_host must be a host tensor of K's shape and dtype")
    dev = torch.device(device)
    if dev.index is None:
        dev = torch.device("cuda", torch.cuda.current_device())
    nbytes = int(lib.flarepp_route_host_buffer_bytes(ctypes.byref(shape)))
    ws = workspace if workspace is not None else Workspace()
    buf = ws.get(nbytes, dev) if nbytes else None
    st = stream if stream is not None else torch.cuda.current_stream(dev)
    rc = lib.flarepp_flare_fwd_host(ctypes.byref(shape), _ptr(Q), _ptr(K), _ptr(V),
                                    float(scale), _ptr(Y_host),
                                    None if buf is None else ctypes.c_void_p(buf.data_ptr()),
                                    nbytes, ctypes.c_void_p(st.cuda_stream))
    if rc != 0:
        raise FlareppError(rc, "flarepp_flare_fwd_host")
    st.synchronize()
    return Y_host


# ---------------------------------------------------------------- layers around the mixer
# As the chain's entry points, these record no autograd graph: what they return requires no gradient,
# whatever their inputs do, and linear_bwd and embedding_bwd write gradients (they add to nothing).
ACTIVATIONS = {"none": 0, "relu": 1, "gelu": 2, "silu": 3}
STATE_BLOCK = 256  # values that share one scale in an 8-bit optimiser state


def _need(t, what, shape, dtype, device, optional=False):
    """A contiguous tensor of this shape, dtype and CUDA device; returns its address (0 for an
    optional one that is missing)."""
    if isinstance(t, torch.Tensor):
        if t.dtype is dtype and t.shape == shape and t.device == device and t.is_contiguous():
            return t.data_ptr()
    elif t is None and optional:
        return 0
    else:
        raise TypeError(f"{what} must be a torch tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{what} has dtype {t.dtype}, expected {dtype}")
    if t.shape != shape:
        raise ValueError(f"{what} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if t.device != device:
        raise ValueError(f"{what} is on {t.device}, expected {device}")
    raise ValueError(f"{what} must be contiguous")


def _cuda_device(t, what):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{what} must be a torch tensor")
    if t.device.type != "cuda":
        raise ValueError(f"{what} must be a device tensor")
    return t.device


_ENTRIES = {}  # name -> entry point


def _entry(name):
    fn = _ENTRIES.get(name)
    if fn is None:
        fn = _ENTRIES[name] = getattr(load(), "flarepp_" + name)
    return fn


def _current_stream(device):
    """The handle of torch's current stream on ``device``."""
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)  # spares building a Stream object
    return raw(device.index) if raw else torch.cuda.current_stream(device).cuda_stream


def _current(stream, device):
    """``stream`` (a torch stream, one with ``cuda_stream``, or a handle) as torch's current one: what
    a call allocates is then that stream's, and not another stream's to have while the call runs."""
    if not isinstance(stream, torch.cuda.Stream):
        handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
        stream = (torch.cuda.ExternalStream(handle, device) if handle
                  else torch.cuda.default_stream(device))
    if stream.device != device:
        raise ValueError(f"stream is on {stream.device}, the call's tensors on {device}")
    return torch.cuda.stream(stream)


def _enqueue(name, device, stream, *args):
    """Call entry ``flarepp_<name>`` with the device current, the stream as last argument."""
    fn = _entry(name)
    if stream is None:
        handle = _current_stream(device)
    else:
        handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
    if torch.cuda.current_device() == device.index:
        rc = fn(*args, handle)
    else:
        with torch.cuda.device(device):
            rc = fn(*args, handle)
    if rc != OK:
        raise FlareppError(rc, "flarepp_" + name)


def _scratch(workspace, nbytes, device):
    """(tensor to keep until the call is enqueued, its address, its bytes)"""
    if nbytes == 0 and workspace is None:
        return None, 0, 0
    if isinstance(workspace, Workspace):
        buf = workspace.get(nbytes, device)
    elif workspace is None:
        buf = torch.empty(nbytes, dtype=torch.uint8, device=device)
    else:
        _check_device("the call", device, workspace=workspace)
        buf = workspace
    return buf, 0 if buf is None else buf.data_ptr(), _nbytes(buf)


def _status_word(status, device):
    return 0 if status is None else _need(status, "status", (1,), torch.int32, device)


def layers_status(device=None, stream=None) -> int:
    """What the kernels of ``linear_*`` and ``embedding_*`` calls without ``status`` recorded on
    ``device`` (default: torch's current one) since this was last asked: OK, ERR_TIMEOUT (a bounded
    wait gave up: outputs are invalid) or ERR_INVALID_ARGUMENT (an id beyond the table). Waits for
    ``stream`` (default: torch's current one there)."""
    dev = torch.device("cuda", torch.cuda.current_device()) if device is None else torch.device(device)
    if dev.type != "cuda":
        raise ValueError(f"the layers run on CUDA devices, not {dev}")
    with torch.cuda.device(dev):
        if stream is None:
            stream = torch.cuda.current_stream()
        handle = stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)
        out = ctypes.c_int32(-1)
        rc = _entry("layers_device_status")(handle, ctypes.byref(out))
    if rc != OK:
        raise FlareppError(rc, "flarepp_layers_device_status")
    return int(out.value)


def _linear_shape(X, W, act):
    """(shape, address of X, address of W) of a linear layer on device tensors X and W."""
    code = ACTIVATIONS.get(act)
    if code is None:
        raise ValueError(f"act must be one of {tuple(ACTIVATIONS)}")
    dev = _cuda_device(X, "X")
    dt = X.dtype
    if dt not in _DTYPES:
        raise TypeError(f"unsupported dtype {dt}; the linear layer takes bfloat16")
    if not isinstance(W, torch.Tensor):
        raise TypeError("W must be a torch tensor")
    if W.dim() != 2 or X.dim() < 1 or X.shape[-1] != W.shape[1]:
        raise ValueError(f"expected X [..., in] and W [out, in], got {tuple(X.shape)} and "
                         f"{tuple(W.shape)}")
    out, in_ = W.shape
    wp = _need(W, "W", W.shape, dt, dev)
    if not X.is_contiguous():
        raise ValueError("X must be contiguous")
    s = LinearShape(X.numel() // in_ if in_ else 0, in_, out, _DTYPES[dt], code)
    return s, X.data_ptr(), wp


def _linear(X, W, b, residual, act, Y, Z, keep, workspace, status, stream):
    s, xp, wp = _linear_shape(X, W, act)
    dev, dt, out = X.device, X.dtype, W.shape[0]
    if stream is not None:
        with _current(stream, dev):
            return _linear(X, W, b, residual, act, Y, Z, keep, workspace, status, None)
    shape = (*X.shape[:-1], out)
    bp = 0 if b is None else _need(b, "b", (out,), dt, dev)
    rp = 0 if residual is None else _need(residual, "residual", shape, dt, dev)
    if Y is None:
        Y = torch.empty(shape, dtype=dt, device=dev)
        yp = Y.data_ptr()
    else:
        yp = _need(Y, "Y", shape, dt, dev)
    if keep and Z is None:
        Z = torch.empty(shape, dtype=dt, device=dev)
    zp = 0 if Z is None else _need(Z, "Z", shape, dt, dev)
    ref = ctypes.byref(s)
    buf, wsp, wsn = _scratch(workspace, _entry("linear_workspace_bytes")(ref), dev)
    _enqueue("linear_fwd", dev, None, ref, xp, wp, bp, rp, yp, zp, wsp, wsn,
             _status_word(status, dev))
    return Y, Z


def linear_fwd(X, W, b=None, residual=None, act="none", Y=None, workspace=None, status=None,
               stream=None):
    """Y = act(X W^T + b) + residual [..., out] for X [..., in], W [out, in], b [out], in bf16;
    ``act`` one of ``ACTIVATIONS``. ``status``: a device int32 [1] that a timeout sets (without one,
    ``layers_status`` tells)."""
    return _linear(X, W, b, residual, act, Y, None, False, workspace, status, stream)[0]


def linear_fwd_train(X, W, b=None, residual=None, act="none", Y=None, Z=None, workspace=None,
                     status=None, stream=None):
    """``linear_fwd`` that also returns Z = X W^T + b, which ``linear_bwd`` takes (None for
    ``act="none"``, whose backward does not need it)."""
    if act == "none" and Z is not None:
        raise ValueError("act='none' keeps no Z")
    return _linear(X, W, b, residual, act, Y, Z, act != "none", workspace, status, stream)


def linear_bwd(X, W, dY, Z=None, act="none", bias=True, dX=None, dW=None, db=None,
               need=(True, True), workspace=None, status=None, stream=None):
    """(dX, dW, db), the gradients of ``linear_fwd_train`` for the output gradient dY [..., out]
    (the residual's gradient is dY). ``bias=False`` leaves db out, ``need`` dX or dW; what is left
    out is returned as None."""
    s, xp, wp = _linear_shape(X, W, act)
    dev, dt = X.device, X.dtype
    if stream is not None:
        with _current(stream, dev):
            return linear_bwd(X, W, dY, Z, act, bias, dX, dW, db, need, workspace, status)
    shape = (*X.shape[:-1], s.out)
    gp = _need(dY, "dY", shape, dt, dev)
    zp = _need(Z, "Z", shape, dt, dev, optional=act == "none")
    if need[0] and dX is None:
        dX = torch.empty_like(X)
    if need[1] and dW is None:
        dW = torch.empty_like(W)
    if bias and db is None:
        db = torch.empty(s.out, dtype=dt, device=dev)
    dX, dW, db = dX if need[0] else None, dW if need[1] else None, db if bias else None
    dxp = _need(dX, "dX", X.shape, dt, dev, optional=True)
    dwp = _need(dW, "dW", W.shape, dt, dev, optional=True)
    dbp = _need(db, "db", (s.out,), dt, dev, optional=True)
    ref = ctypes.byref(s)
    buf, wsp, wsn = _scratch(workspace, _entry("linear_bwd_workspace_bytes")(ref), dev)
    _enqueue("linear_bwd", dev, None, ref, xp, wp, zp, gp, dxp, dwp, dbp, wsp, wsn,
             _status_word(status, dev))
    return dX, dW, db


def _ids_of(ids):
    dev = _cuda_device(ids, "ids")
    if ids.dtype not in (torch.int32, torch.int64):
        raise TypeError(f"ids have dtype {ids.dtype}, expected int32 or int64")
    if not ids.is_contiguous():
        raise ValueError("ids must be contiguous")
    return dev, ids.data_ptr(), 4 if ids.dtype is torch.int32 else 8


def _float_dtype(t, what):
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{what} must be a torch tensor")
    if t.dtype not in _DTYPES:
        raise TypeError(f"unsupported dtype {t.dtype}; use float32 or bfloat16")
    return t.dtype


def embedding_fwd(ids, table, scale=1.0, Y=None, status=None, stream=None):
    """Y [..., C] = scale * table[ids] for ids [...] (int32 or int64) and table [V, C] (float32 or
    bf16). A negative id gives a row of zeros; one of V or more too, and sets ``status`` (a device
    int32 [1]; without one, ``layers_status`` tells) to ERR_INVALID_ARGUMENT."""
    dev, ip, size = _ids_of(ids)
    if stream is not None:
        with _current(stream, dev):
            return embedding_fwd(ids, table, scale, Y, status)
    dt = _float_dtype(table, "table")
    if table.dim() != 2:
        raise ValueError("expected table [V, C]")
    V, C = table.shape
    tp = _need(table, "table", (V, C), dt, dev)
    shape = (*ids.shape, C)
    if Y is None:
        Y = torch.empty(shape, dtype=dt, device=dev)
        yp = Y.data_ptr()
    else:
        yp = _need(Y, "Y", shape, dt, dev)
    s = EmbeddingShape(ids.numel(), V, C, _DTYPES[dt], size)
    _enqueue("embedding_fwd", dev, None, ctypes.byref(s), ip, tp, float(scale), yp,
             _status_word(status, dev))
    return Y


def embedding_bwd(ids, dY, V, scale=1.0, dtable=None, workspace=None, status=None, stream=None):
    """dtable [V, C], the gradient of ``embedding_fwd``'s table for dY [..., C]: the rows of dY
    summed by id in a fixed order, times ``scale``; rows that no id names are 0."""
    dev, ip, size = _ids_of(ids)
    if stream is not None:
        with _current(stream, dev):
            return embedding_bwd(ids, dY, V, scale, dtable, workspace, status)
    dt = _float_dtype(dY, "dY")
    if dY.dim() != ids.dim() + 1:
        raise ValueError("expected dY of the ids' shape and one more dimension")
    C = dY.shape[-1]
    gp = _need(dY, "dY", (*ids.shape, C), dt, dev)
    if dtable is None:
        dtable = torch.empty((V, C), dtype=dt, device=dev)
    s = EmbeddingShape(ids.numel(), V, C, _DTYPES[dt], size)
    ref = ctypes.byref(s)
    buf, wsp, wsn = _scratch(workspace, _entry("embedding_bwd_workspace_bytes")(ref), dev)
    _enqueue("embedding_bwd", dev, None, ref, ip, gp, float(scale),
             _need(dtable, "dtable", (V, C), dt, dev), wsp, wsn, _status_word(status, dev))
    return dtable


def _check_apart(spans):
    """Refuse spans (begin, end, whether it is written, name) of which one that is written overlaps
    another."""
    most, written = (0, None), (0, None)  # the largest ends so far, of all and of those written
    for begin, end, writes, name in sorted(x for x in spans if x[0] < x[1]):
        other = most if writes else written
        if begin < other[0]:
            raise FlareppError(ERR_INVALID_ARGUMENT, f"AdamW: {name} overlaps {other[1]}")
        most = max(most, (end, name), key=lambda x: x[0])
        if writes:
            written = max(written, (end, name), key=lambda x: x[0])


class AdamW:
    """AdamW over fixed buffers: parameters, their gradients, and the state it keeps.

        opt = flarepp.AdamW(params, grads, lr=1e-3, state_bits=8, masters=True)
        ...                      # a step's gradients are written into ``grads``
        opt.step()

    params, grads: lists of contiguous CUDA tensors of the same shapes, float32 or bf16 each.
    masters: True makes a float32 master of every bf16 parameter (whose rounded copy it then is), a
    list gives them (None where there is none); masters that ``state`` holds are used before any is
    made, and with ``masters=None`` too (False: none). state_bits: 32, or 8 (the moments in 8 bits with
    a scale for every ``STATE_BLOCK`` values: a quarter of the memory; include/flarepp.h says how).
    state_rounding: of 8-bit states, "nearest", or "unbiased" (by a hash of place and step), without
    which the second moment of a long run with a large beta2 stops following its average.
    state: the state to go on from, as ``state_dict`` returns it (its tensors are used, not
    copied). The optimiser works on the buffers that it was given, whose storage it keeps alive:
    a parameter or gradient that moves to another buffer needs a new optimiser (give it
    ``state_dict()``); no two buffers of which one is written may overlap. ``lr`` and ``weight_decay`` are attributes that a schedule may change."""

    def __init__(self, params, grads, lr=1e-3, betas=(0.9, 0.999), eps=1e-8, weight_decay=1e-2,
                 state_bits=32, masters=None, state=None, state_rounding="nearest"):
        params, grads = [p.detach() for p in params], [g.detach() for g in grads]
        if len(params) != len(grads):
            raise ValueError(f"{len(params)} parameters, {len(grads)} gradients")
        if state_bits not in (8, 32):
            raise ValueError("state_bits must be 8 or 32")
        if state_rounding not in ("nearest", "unbiased"):
            raise ValueError("state_rounding must be 'nearest' or 'unbiased'")
        if state_rounding == "unbiased" and state_bits != 8:
            raise ValueError("only 8-bit states are rounded without bias")
        self.state_rounding = state_rounding
        self.lr, self.betas, self.eps = lr, betas, eps
        self.weight_decay, self.state_bits = weight_decay, state_bits
        self.params, self.grads = params, grads
        self.device = _cuda_device(params[0], "params[0]") if params else None
        kept = state.get("masters") if state else None
        if masters is None:
            masters = kept
        elif masters is True:
            masters = [p.float() if p.dtype == torch.bfloat16 and k is None else k
                       for p, k in zip(params, kept or [None] * len(params))]

        def own(ts):  # aliases, which keep the storage whatever becomes of the caller's tensors
            return [None if t is None else t.detach() for t in ts or [None] * len(params)]

        self.masters = own(masters)
        made = self._zero_state() if state is None else state
        self.m, self.v = own(made["m"]), own(made["v"])
        self.m_scale, self.v_scale = own(made.get("m_scale")), own(made.get("v_scale"))
        self.steps = int(made.get("step", 0))
        self._table = (AdamwTensor * max(1, len(params)))()
        lists = (grads, self.masters, self.m, self.v, self.m_scale, self.v_scale)
        if any(len(x) != len(params) for x in lists):
            raise ValueError("the lists of tensors differ in length")
        for i, p in enumerate(params):
            self._fill(i, p)
        _check_apart([(t.data_ptr(), t.data_ptr() + t.numel() * t.element_size(), ts is not grads,
                       f"{name}[{i}]")
                      for name, ts in zip(("params", "grads", "masters", "m", "v", "m_scale", "v_scale"),
                                          (params, *lists))
                      for i, t in enumerate(ts) if t is not None])

    def _zero_state(self):
        def zeros(n, dtype):
            return torch.zeros(n, dtype=dtype, device=self.device)
        if self.state_bits == 32:
            return {k: [zeros(p.shape, torch.float32) for p in self.params] for k in "mv"}
        ns = [p.numel() for p in self.params]
        blocks = [-(-n // STATE_BLOCK) for n in ns]
        return {"m": [zeros(n, torch.float8_e4m3fn) for n in ns],
                "v": [zeros(n, torch.uint8) for n in ns],
                "m_scale": [zeros(b, torch.float32) for b in blocks],
                "v_scale": [zeros(b, torch.float32) for b in blocks]}

    def _fill(self, i, p):
        dev, f32, e = self.device, torch.float32, self._table[i]
        dt = _float_dtype(p, f"params[{i}]")
        g = self.grads[i]
        n = p.numel()
        e.param = _need(p, f"params[{i}]", p.shape, dt, dev)
        e.grad = _need(g, f"grads[{i}]", p.shape, _float_dtype(g, f"grads[{i}]"), dev)
        e.master = _need(self.masters[i], f"masters[{i}]", p.shape, f32, dev, optional=True)
        e.n, e.param_dtype, e.grad_dtype = n, _DTYPES[dt], _DTYPES[g.dtype]
        if self.state_bits == 32:
            for k in ("m", "v"):
                t = getattr(self, k)[i]
                setattr(e, k, _need(t.view(p.shape), f"{k}[{i}]", p.shape, f32, dev))
            return
        blocks = -(-n // STATE_BLOCK)
        e.m = _need(self.m[i].view(-1), f"m[{i}]", (n,), torch.float8_e4m3fn, dev)
        e.v = _need(self.v[i].view(-1), f"v[{i}]", (n,), torch.uint8, dev)
        e.m_scale = _need(self.m_scale[i], f"m_scale[{i}]", (blocks,), f32, dev)
        e.v_scale = _need(self.v_scale[i], f"v_scale[{i}]", (blocks,), f32, dev)

    def step(self, stream=None):
        """One step from what the gradients hold now."""
        if not self.params:
            return
        h = AdamwHyper(self.lr, self.betas[0], self.betas[1], self.eps, self.weight_decay,
                       self.steps + 1, self.state_bits)
        _enqueue("adamw_step_unbiased" if self.state_rounding == "unbiased" else "adamw_step",
                 self.device, stream, self._table, len(self.params), ctypes.byref(h))
        self.steps += 1

    def moments(self, m_out=None, v_out=None, stream=None):
        """The moments as lists of float32 tensors: the state itself with 32 bits, the values that
        it stands for with 8 (written into m_out and v_out where they are given)."""
        if self.state_bits == 32:
            if m_out is not None or v_out is not None:
                raise ValueError("32-bit moments are the state itself: m_out and v_out are not used")
            return self.m, self.v
        if stream is not None and self.params:
            with _current(stream, self.device):
                return self.moments(m_out, v_out)
        outs = []
        for given, name in ((m_out, "m_out"), (v_out, "v_out")):
            if given is None:
                given = [torch.empty(p.shape, device=self.device) for p in self.params]
            if len(given) != len(self.params):
                raise ValueError(f"{name} has {len(given)} tensors, expected {len(self.params)}")
            ptrs = [_need(t, name, p.shape, torch.float32, self.device)
                    for t, p in zip(given, self.params)]
            outs.append((given, (ctypes.c_void_p * max(1, len(ptrs)))(*ptrs)))
        if self.params:
            _enqueue("adamw_moments", self.device, None, self._table, len(self.params),
                     outs[0][1], outs[1][1])
        return outs[0][0], outs[1][0]

    def state_dict(self):
        """The state to save and to go on from, masters among it; its tensors are the optimiser's own."""
        return {"m": self.m, "v": self.v, "m_scale": self.m_scale, "v_scale": self.v_scale,
                "masters": self.masters, "step": self.steps}
