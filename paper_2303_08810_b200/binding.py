"""ctypes binding of libbra_b200.so: same names as the C boundary (include/bra.h).

Argument marshalling only.  PyTorch provides device memory and the CUDA
stream; every step of the path runs inside the library's kernels.  If the
library has not been built, or there is no CUDA device, calls raise: there is
no fallback.  `stream` (a torch stream or a handle; None: the current one) is
where a call runs, and what it is not given (outputs, ws) is allocated there, as
inside `with torch.cuda.stream(stream)`.
"""
from __future__ import annotations

import ctypes
import math
import os
from ctypes import byref, c_double, c_float, c_int32, c_int64, c_size_t, c_void_p

_LIB = None
_TORCH = None            # torch, once it has shown a CUDA device
_RAW_STREAM = None       # () -> address of the current stream
_LIB_NAME = "libbra_b200.so"

IMPL_AUTO, IMPL_SIMT, IMPL_MMA, IMPL_TC, IMPL_IMG, IMPL_TC_FUSED = 0, 1, 2, 3, 4, 5
F32, BF16 = 0, 1


class BraProblem(ctypes.Structure):
    """Mirror of `bra_problem` (Algorithm 1 notation: H, W, C, S, k, plus batch and heads)."""

    _fields_ = [
        ("B", c_int32), ("H", c_int32), ("W", c_int32), ("C", c_int32),
        ("heads", c_int32), ("S", c_int32), ("topk", c_int32), ("dtype", c_int32),
        ("scale", c_float), ("shared_routing", c_int32), ("lce_ksize", c_int32), ("impl", c_int32),
        ("inject", c_int32),
    ]

    @property
    def R(self):
        return self.S * self.S

    @property
    def heads_i(self):
        return 1 if self.shared_routing else self.heads


class BraRopeProblem(ctypes.Structure):
    """Mirror of `bra_rope_problem`."""

    _fields_ = [
        ("B", c_int32), ("N", c_int32), ("heads", c_int32), ("kv_heads", c_int32), ("head_dim", c_int32),
        ("rot_dim", c_int32), ("layout", c_int32), ("axes", c_int32), ("width", c_int32), ("first", c_int32),
        ("dtype", c_int32), ("magnitude", c_float), ("q_stride", c_int64), ("k_stride", c_int64),
    ]


class BraCrossProblem(ctypes.Structure):
    """Mirror of `bra_cross_problem`."""

    _fields_ = [
        ("B", c_int32), ("Nq", c_int32), ("Nk", c_int32), ("heads", c_int32), ("kv_heads", c_int32),
        ("head_dim", c_int32), ("dtype", c_int32), ("scale", c_float),
        ("q_stride", c_int64), ("k_stride", c_int64), ("v_stride", c_int64),
    ]


class BraNormProblem(ctypes.Structure):
    """Mirror of `bra_norm_problem`."""

    _fields_ = [
        ("B", c_int32), ("N", c_int32), ("C", c_int32), ("pre", c_int32), ("post", c_int32), ("gate", c_int32),
        ("per_image", c_int32), ("dtype", c_int32), ("eps", c_float), ("alpha", c_float),
    ]


class BraError(RuntimeError):
    def __init__(self, code, where):
        self.code = int(code)
        super().__init__(f"{where}: {status_string(code)} (bra_status {int(code)})")


def library_path() -> str:
    """The built library next to this file, or the file BRA_LIBRARY_PATH names (to try another build)."""
    return os.environ.get("BRA_LIBRARY_PATH") or os.path.join(os.path.dirname(os.path.abspath(__file__)), _LIB_NAME)


def load_library():
    """Load the built library (never builds it; see build.py / __graft_entry__.build)."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = library_path()
    if not os.path.exists(path):
        raise RuntimeError(
            f"{path} is missing: build it with `python -m paper_2303_08810_b200.build` "
            "(there is no CPU fallback)")
    lib = ctypes.CDLL(path)
    P = ctypes.POINTER(BraProblem)
    v = c_void_p
    lib.bra_workspace_bytes.restype = c_size_t
    lib.bra_workspace_bytes.argtypes = [P]
    lib.bra_workspace_init.restype = c_int32
    lib.bra_workspace_init.argtypes = [P, v, c_size_t, v]
    lib.bra_route.restype = c_int32
    lib.bra_route.argtypes = [P, v, v, v, v, v, v, c_size_t, v]
    lib.bra_route_static.restype = c_int32
    lib.bra_route_static.argtypes = [P, v, v, v, v]
    lib.bra_attend.restype = c_int32
    lib.bra_attend.argtypes = [P, v, v, v, v, v, v, v, v, v, c_size_t, v]
    lib.bra_forward.restype = c_int32
    lib.bra_forward.argtypes = [P, v, v, v, v, v, v, v, v, v, c_size_t, v]
    lib.bra_backward.restype = c_int32
    lib.bra_backward.argtypes = [P] + [v] * 12 + [v, c_size_t, v]
    lib.bra_rope_frequencies.restype = c_int32
    lib.bra_rope_frequencies.argtypes = [c_int32, c_int32, c_double, c_int32, c_double, c_double, c_double, c_double, v]
    lib.bra_rope.restype = c_int32
    lib.bra_rope.argtypes = [ctypes.POINTER(BraRopeProblem), v, v, v, v, c_int32, v, v, v]
    PC = ctypes.POINTER(BraCrossProblem)
    lib.bra_cross_workspace_bytes.restype = c_size_t
    lib.bra_cross_workspace_bytes.argtypes = [PC]
    lib.bra_cross_attend.restype = c_int32
    lib.bra_cross_attend.argtypes = [PC] + [v] * 8 + [c_size_t, v]
    lib.bra_cross_backward.restype = c_int32
    lib.bra_cross_backward.argtypes = [PC] + [v] * 12 + [c_size_t, v]
    PN = ctypes.POINTER(BraNormProblem)
    lib.bra_norm_workspace_bytes.restype = c_size_t
    lib.bra_norm_workspace_bytes.argtypes = [PN]
    lib.bra_residual_norm.restype = c_int32
    lib.bra_residual_norm.argtypes = [PN] + [v] * 10
    lib.bra_residual_norm_backward.restype = c_int32
    lib.bra_residual_norm_backward.argtypes = [PN] + [v] * 16 + [c_size_t, v]
    lib.bra_device_status.restype = c_int32
    lib.bra_device_status.argtypes = [v, v]
    lib.bra_last_launch_count.restype = c_int32
    lib.bra_last_launch_count.argtypes = []
    lib.bra_status_string.restype = ctypes.c_char_p
    lib.bra_status_string.argtypes = [c_int32]
    lib.bra_version.restype = c_int32
    lib.bra_version.argtypes = []
    _LIB = lib
    return lib


def status_string(code) -> str:
    return load_library().bra_status_string(int(code)).decode()


def version() -> int:
    return load_library().bra_version()


def last_launch_count() -> int:
    return load_library().bra_last_launch_count()


def make_problem(B, H, W, C, heads, S, topk, dtype="bf16", scale=0.0, shared_routing=False,
                 lce=True, impl=IMPL_AUTO, inject=0) -> BraProblem:
    dt = {"f32": F32, "bf16": BF16, F32: F32, BF16: BF16}[dtype]
    return BraProblem(B, H, W, C, heads, S, topk, dt, float(scale), int(bool(shared_routing)),
                      5 if lce else 0, int(impl), int(inject))


def workspace_bytes(p: BraProblem) -> int:
    return int(load_library().bra_workspace_bytes(ctypes.byref(p)))


# What follows is on the way of every call: of small problems, whose kernels take less time than their marshalling, it is the
# bound.  The current stream cost 3.2 us a call through torch.cuda, the device check 0.7 at each use.  Without them a forward +
# backward pass at 1 x 16 x 16 x 32 takes 40.5 us among others instead of 52.8, bra_forward of one 56 x 56 image into the caller's
# tensor 10.8 instead of 15.9.
def _torch():
    global _TORCH
    if _TORCH is None:
        import torch
        if not torch.cuda.is_available():
            raise RuntimeError("paper_2303_08810_b200 needs a CUDA device (no CPU fallback)")
        _TORCH = torch
    return _TORCH


def workspace(p: BraProblem, device="cuda"):
    """Zero-filled scratch tensor of bra_workspace_bytes(p) bytes."""
    torch = _torch()
    n = workspace_bytes(p)
    if n == 0:
        raise BraError(2, "bra_workspace_bytes")
    return torch.zeros(n, dtype=torch.uint8, device=device)


def workspace_init(p: BraProblem, ws, stream=None):
    """bra_workspace_init: status block, job counters and flags of `ws` set to zero."""
    _check(load_library().bra_workspace_init(ctypes.byref(p), _ptr(ws), ws.numel(), _stream(stream)),
           "bra_workspace_init")
    return ws


def _ptr(t):
    if t is None or isinstance(t, int):
        return t
    return t.data_ptr()


def _raw_stream_getter():
    """The cheapest way this torch has to name the current stream of the current device."""
    global _RAW_STREAM
    torch = _torch()
    slow = lambda: torch.cuda.current_stream().cuda_stream           # noqa: E731
    _RAW_STREAM = slow
    raw, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
    if slow() is not None and raw and device and raw(device()) == slow():
        _RAW_STREAM = lambda: raw(device())                          # noqa: E731
    return _RAW_STREAM


def _stream(stream):
    if stream is None:
        return (_RAW_STREAM or _raw_stream_getter())()
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def _on(stream):
    """The context in which torch's current stream is `stream`.  What a call makes itself (outputs, scratch and its zeros) has to belong to
    the stream that the call runs on: from another stream's pool it could be memory that this one still uses, the zeros could come late,
    and scratch that is let go at the end of the call could be handed out while the kernels count in it."""
    torch = _torch()
    if isinstance(stream, torch.cuda.Stream):
        return torch.cuda.stream(stream)
    handle = _stream(stream)                                 # 0 and 1 name the default stream in CUDA's interface
    return torch.cuda.stream(torch.cuda.ExternalStream(handle) if handle > 1 else torch.cuda.default_stream())


def _tdtype(p):
    torch = _torch()
    return torch.bfloat16 if p.dtype == BF16 else torch.float32


def _check(code, where):
    if code != 0:
        raise BraError(code, where)


def bra_route(p, Q, K, q_mean=None, k_mean=None, index=None, ws=None, stream=None, want_means=True):
    """bra_route: Q, K -> (q_mean, k_mean, index)."""
    if stream is not None and (ws is None or index is None or (want_means and (q_mean is None or k_mean is None))):
        with _on(stream):
            return bra_route(p, Q, K, q_mean, k_mean, index, ws, None, want_means)
    torch = _torch()
    lib = load_library()
    ws = workspace(p, Q.device) if ws is None else ws
    if want_means:
        q_mean = torch.empty(p.B, p.R, p.C, dtype=torch.float32, device=Q.device) if q_mean is None else q_mean
        k_mean = torch.empty(p.B, p.R, p.C, dtype=torch.float32, device=Q.device) if k_mean is None else k_mean
    if index is None:
        index = torch.empty(p.B, p.heads_i, p.R, p.topk, dtype=torch.int32, device=Q.device)
    _check(lib.bra_route(ctypes.byref(p), _ptr(Q), _ptr(K), _ptr(q_mean), _ptr(k_mean), _ptr(index),
                         _ptr(ws), ws.numel(), _stream(stream)), "bra_route")
    return q_mean, k_mean, index


ROUTE_STATIC_MAX_MEAN_FLOATS = 512 * 1024


def bra_route_static(p, Q, K, index=None, stream=None):
    """bra_route_static: Q, K -> index, for callers that have no scratch buffer to give.

    The region means stay inside the library (a fixed array of
    2 x ROUTE_STATIC_MAX_MEAN_FLOATS floats per GPU); the C call allocates
    nothing.  Pass a preallocated `index` to keep the whole call allocation-free:
    only when `index` is None does this wrapper ask torch for one.  Calls on
    one device share the array, so keep them ordered on a stream.
    """
    if stream is not None and index is None:
        with _on(stream):
            return bra_route_static(p, Q, K)
    torch = _torch()
    lib = load_library()
    if index is None:
        index = torch.empty(p.B, p.heads_i, p.R, p.topk, dtype=torch.int32, device=Q.device)
    _check(lib.bra_route_static(ctypes.byref(p), _ptr(Q), _ptr(K), _ptr(index), _stream(stream)),
           "bra_route_static")
    return index


def bra_attend(p, Q, K, V, index, lce_w=None, lce_b=None, O=None, lse=None, ws=None, stream=None,
               want_lse=True):
    """bra_attend: Q, K, V, index -> (O, lse)."""
    if stream is not None and (ws is None or O is None or (lse is None and want_lse)):
        with _on(stream):
            return bra_attend(p, Q, K, V, index, lce_w, lce_b, O, lse, ws, None, want_lse)
    torch = _torch()
    lib = load_library()
    ws = workspace(p, Q.device) if ws is None else ws
    O = torch.empty_like(Q) if O is None else O
    if lse is None and want_lse:
        lse = torch.empty(p.B, p.heads, p.H * p.W, dtype=torch.float32, device=Q.device)
    _check(lib.bra_attend(ctypes.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(index), _ptr(lce_w),
                          _ptr(lce_b), _ptr(O), _ptr(lse), _ptr(ws), ws.numel(), _stream(stream)),
           "bra_attend")
    return O, lse


def bra_forward(p, Q, K, V, lce_w=None, lce_b=None, O=None, index=None, lse=None, ws=None,
                stream=None, want_index=True, want_lse=True):
    """bra_forward: Q, K, V -> (O, index, lse)."""
    if stream is not None and (ws is None or O is None or (index is None and want_index) or (lse is None and want_lse)):
        with _on(stream):
            return bra_forward(p, Q, K, V, lce_w, lce_b, O, index, lse, ws, None, want_index, want_lse)
    torch = _torch()
    lib = load_library()
    ws = workspace(p, Q.device) if ws is None else ws
    O = torch.empty_like(Q) if O is None else O
    if index is None and want_index:
        index = torch.empty(p.B, p.heads_i, p.R, p.topk, dtype=torch.int32, device=Q.device)
    if lse is None and want_lse:
        lse = torch.empty(p.B, p.heads, p.H * p.W, dtype=torch.float32, device=Q.device)
    _check(lib.bra_forward(ctypes.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(lce_w), _ptr(lce_b),
                           _ptr(O), _ptr(index), _ptr(lse), _ptr(ws), ws.numel(), _stream(stream)),
           "bra_forward")
    return O, index, lse


def bra_backward(p, Q, K, V, index, lce_w, lse, dO, dQ=None, dK=None, dV=None, d_lce_w=None,
                 d_lce_b=None, ws=None, stream=None, want_bias_grad=False):
    """bra_backward: -> (dQ, dK, dV, d_lce_w, d_lce_b)."""
    if stream is not None and (ws is None or dQ is None or dK is None or dV is None or (d_lce_w is None and p.lce_ksize) or
                               (d_lce_b is None and want_bias_grad)):
        with _on(stream):
            return bra_backward(p, Q, K, V, index, lce_w, lse, dO, dQ, dK, dV, d_lce_w, d_lce_b, ws, None, want_bias_grad)
    torch = _torch()
    lib = load_library()
    ws = workspace(p, Q.device) if ws is None else ws
    dQ = torch.empty_like(Q) if dQ is None else dQ
    dK = torch.empty_like(K) if dK is None else dK
    dV = torch.empty_like(V) if dV is None else dV
    if d_lce_w is None and p.lce_ksize:
        d_lce_w = torch.empty(p.C, 5, 5, dtype=torch.float32, device=Q.device)
    if d_lce_b is None and want_bias_grad:
        d_lce_b = torch.empty(p.C, dtype=torch.float32, device=Q.device)
    _check(lib.bra_backward(ctypes.byref(p), _ptr(Q), _ptr(K), _ptr(V), _ptr(index), _ptr(lce_w),
                            _ptr(lse), _ptr(dO), _ptr(dQ), _ptr(dK), _ptr(dV), _ptr(d_lce_w),
                            _ptr(d_lce_b), _ptr(ws), ws.numel(), _stream(stream)), "bra_backward")
    return dQ, dK, dV, d_lce_w, d_lce_b


def bra_device_status(ws, stream=None) -> int:
    """Synchronise the stream and return (and clear) the first device-detected error in ws."""
    return int(load_library().bra_device_status(_ptr(ws), _stream(stream)))


# ---------------------------------------------------------------- what stands around the attention of a block
# These calls take tensors of a program's own making (slices of fused projections, masks, positions), so what a wrong one would
# make the kernels read is checked here: element type, shape, order in memory, device.
_DTYPES = {"f32": F32, "bf16": BF16, F32: F32, BF16: BF16}
_GET_DEVICE = None


def _device_getter():
    global _GET_DEVICE
    torch = _torch()
    _GET_DEVICE = getattr(torch._C, "_cuda_getDevice", None) or torch.cuda.current_device
    return _GET_DEVICE


class _Shape(set):
    """The axes `of` a dense tensor as the kernels count them, and the shapes seen so far that lay its elements out in that order."""

    def __init__(self, *of):
        super().__init__((of,))
        self.of = of
        self.numel = math.prod(of)


def _lays_out(shape, axes):
    """Whether a dense tensor of `shape` has its elements in the order of `axes`: whole axes may be merged and an axis may be split, but none
    lies elsewhere ([B, heads, N, D] is not [B, N, heads, D], though it has as many elements)."""
    edges = [1]
    for n in axes:
        edges.append(edges[-1] * n)
    at = 1
    for n in shape:
        if n == 1:
            continue
        to = at * n
        if not (at in edges and to in edges):                # else: within one axis
            end = min((e for e in edges if e > at), default=0)
            if not to or to > end or end % to:
                return False
        at = to
    return at == edges[-1]


def _at(t, name, where, dtype, shape, device):
    """Address of a dense tensor of `shape` (a _Shape) on the current device."""
    if t is not None and t.dtype is dtype and t.shape in shape and t.get_device() == device and t.is_contiguous():
        return t.data_ptr()
    return _look(t, name, where, dtype, shape, device)


def _look(t, name, where, dtype, shape, device):
    if t is None:
        raise BraError(1, f"{where}: {name}")
    if t.dtype is not dtype:
        raise BraError(4, f"{where}: {name} is {t.dtype}, not {dtype}")
    if t.get_device() != device:
        raise ValueError(f"{where}: {name} is on {t.device}, the current device is cuda:{device}")
    if t.numel() != shape.numel:
        raise BraError(2, f"{where}: {name} has {t.numel()} elements, not {shape.numel}")
    if not t.is_contiguous():
        raise BraError(2, f"{where}: {name} is not contiguous")
    if not _lays_out(t.shape, shape.of):
        raise BraError(2, f"{where}: {name} is {list(t.shape)}, not {list(shape.of)}")
    shape.add(tuple(t.shape))
    return t.data_ptr()


def _ws_at(ws, where, device):
    if ws.dtype is _TORCH.uint8 and ws.get_device() == device and ws.is_contiguous():
        return ws.data_ptr()
    return _look(ws, "ws", where, _TORCH.uint8, _Shape(ws.numel()), device)


def _rows_at(t, name, where, dtype, device, tokens):
    """Address of a tensor of tokens = (images, tokens, channels, stride, shape): dense, or a [images, tokens, channels] view whose
    tokens lie `stride` elements apart."""
    B, N, C, stride, shape = tokens
    if stride == C:
        if t is not None and t.dtype is dtype and t.shape in shape and t.get_device() == device and t.is_contiguous():      # _at, a call less
            return t.data_ptr()
        return _look(t, name, where, dtype, shape, device)
    if t is None or t.dtype is not dtype or t.get_device() != device:
        return _look(t, name, where, dtype, shape, device)
    if t.dim() != 3 or tuple(t.shape) != (B, N, C) or (C > 1 and t.stride(2) != 1) or (N > 1 and t.stride(1) != stride) or \
            (B > 1 and t.stride(0) != N * stride):
        raise BraError(2, f"{where}: {name} is not a [{B}, {N}, {C}] view with {stride} elements from token to token")
    return t.data_ptr()


# What a call derives from its problem, by the problem's bytes: small calls are bound by their marshalling.
_DERIVED = {}


def _derived(p, make):
    key = make, bytes(p)
    try:
        return _DERIVED[key]
    except KeyError:
        pass
    if len(_DERIVED) > 4096:
        _DERIVED.clear()
    d = _DERIVED[key] = make(p)
    return d


def _like(t, tokens):
    """A new tensor laid out as `t` (a slice of channels of a wider tensor stays one)."""
    torch = _torch()
    B, N, C, stride, _ = tokens
    if stride == C:
        return torch.empty_like(t)
    return torch.empty(B, N, stride, dtype=t.dtype, device=t.device)[..., :C]


def _scratch(nbytes, where, device):
    if nbytes == 0:
        raise BraError(2, where)
    return _torch().zeros(nbytes, dtype=_torch().uint8, device=device)


def make_rope_problem(B, N, heads, head_dim, kv_heads=None, rot_dim=None, layout="interleaved", axes=1, width=0, first=0,
                      dtype="bf16", magnitude=1.0, q_stride=0, k_stride=0) -> BraRopeProblem:
    return BraRopeProblem(B, N, heads, heads if kv_heads is None else kv_heads, head_dim,
                          head_dim if rot_dim is None else rot_dim, {"interleaved": 0, "half": 1}[layout], axes, width, first,
                          _DTYPES[dtype], float(magnitude), q_stride, k_stride)


def rope_frequencies(rot_dim, axes=1, base=10000.0, scaling="none", factor=1.0, original_length=0.0, low=1.0, high=32.0,
                     device="cuda"):
    """bra_rope_frequencies, on the device: fp64 [rot_dim / axes / 2].  Made once and kept with the layer."""
    torch = _torch()
    out = torch.empty(max(0, rot_dim // axes // 2), dtype=torch.float64)
    _check(load_library().bra_rope_frequencies(rot_dim, axes, float(base), {"none": 0, "linear": 1, "base": 2, "parts": 3}[scaling],
                                               float(factor), float(original_length), float(low), float(high), _ptr(out)),
           "bra_rope_frequencies")
    return out.to(device)


def _rope_derived(p):
    q, k = p.heads * p.head_dim, p.kv_heads * p.head_dim
    return (_tdtype(p), (p.B, p.N, q, p.q_stride or q, _Shape(p.B, p.N, p.heads, p.head_dim)),
            (p.B, p.N, k, p.k_stride or k, _Shape(p.B, p.N, p.kv_heads, p.head_dim)),
            _Shape(p.rot_dim // p.axes // 2 if p.axes else 0), _Shape(p.B, p.N, p.axes))


def bra_rope(p, Q, K, freq, positions=None, Qo=None, Ko=None, inverse=False, stream=None):
    """bra_rope: Q, K -> (Qo, Ko).  Pass Q and K as Qo and Ko to rotate in place; inverse=True is the gradient's rotation."""
    if stream is not None and (Qo is None or (Ko is None and K is not None)):
        with _on(stream):
            return bra_rope(p, Q, K, freq, positions, Qo, Ko, inverse)
    torch, dev, where = _TORCH or _torch(), (_GET_DEVICE or _device_getter())(), "bra_rope"
    t, q, k, pairs, places = _derived(p, _rope_derived)
    q_at = _rows_at(Q, "Q", where, t, dev, q)
    k_at = _rows_at(K, "K", where, t, dev, k) if k[2] or K is not None else None
    f_at = _at(freq, "freq", where, torch.float64, pairs, dev)
    at = None if positions is None else _at(positions, "positions", where, torch.int32, places, dev)
    if Qo is None:
        Qo = _like(Q, q)
        qo_at = Qo.data_ptr()
    else:
        qo_at = _rows_at(Qo, "Qo", where, t, dev, q)
    if k_at is None:
        ko_at = None
    elif Ko is None:
        Ko = _like(K, k)
        ko_at = Ko.data_ptr()
    else:
        ko_at = _rows_at(Ko, "Ko", where, t, dev, k)
    code = (_LIB or load_library()).bra_rope(byref(p), q_at, k_at, at, f_at, 1 if inverse else 0, qo_at, ko_at, _stream(stream))
    if code:
        raise BraError(code, where)
    return Qo, Ko


def make_cross_problem(B, Nq, Nk, heads, head_dim, kv_heads=None, dtype="bf16", scale=0.0, q_stride=0, k_stride=0,
                       v_stride=0) -> BraCrossProblem:
    return BraCrossProblem(B, Nq, Nk, heads, heads if kv_heads is None else kv_heads, head_dim, _DTYPES[dtype], float(scale),
                           q_stride, k_stride, v_stride)


def cross_workspace_bytes(p: BraCrossProblem) -> int:
    return int(load_library().bra_cross_workspace_bytes(ctypes.byref(p)))


def cross_workspace(p: BraCrossProblem, device="cuda"):
    """Zero-filled scratch tensor of bra_cross_workspace_bytes(p) bytes."""
    return _scratch(cross_workspace_bytes(p), "bra_cross_workspace_bytes", device)


def _cross_derived(p):
    C, Ck = p.heads * p.head_dim, p.kv_heads * p.head_dim
    q, k = _Shape(p.B, p.Nq, p.heads, p.head_dim), _Shape(p.B, p.Nk, p.kv_heads, p.head_dim)
    return (_tdtype(p), (p.B, p.Nq, C, p.q_stride or C, q), (p.B, p.Nk, Ck, p.k_stride or Ck, k), (p.B, p.Nk, Ck, p.v_stride or Ck, k),
            q, _Shape(p.B), _Shape(p.B, p.Nk), _Shape(p.B, p.heads, p.Nq))


def _cross_mask(key_len, key_mask, where, torch, images, keys, dev):
    return (None if key_len is None else _at(key_len, "key_len", where, torch.int32, images, dev),
            None if key_mask is None else
            _at(key_mask, "key_mask", where, torch.bool if key_mask.dtype is torch.bool else torch.uint8, keys, dev))


def bra_cross_attend(p, Q, K, V, key_len=None, key_mask=None, O=None, lse=None, ws=None, stream=None, want_lse=True):
    """bra_cross_attend: Q, K, V -> (O, lse).  key_len int32 [B], key_mask bool or uint8 [B, Nk]."""
    if stream is not None and (ws is None or O is None or (lse is None and want_lse)):
        with _on(stream):
            return bra_cross_attend(p, Q, K, V, key_len, key_mask, O, lse, ws, None, want_lse)
    torch, dev, where = _TORCH or _torch(), (_GET_DEVICE or _device_getter())(), "bra_cross_attend"
    t, q, k, v, dense, images, keys, stats = _derived(p, _cross_derived)
    q_at, k_at, v_at = _rows_at(Q, "Q", where, t, dev, q), _rows_at(K, "K", where, t, dev, k), _rows_at(V, "V", where, t, dev, v)
    len_at, mask_at = _cross_mask(key_len, key_mask, where, torch, images, keys, dev)
    if ws is None:
        ws = cross_workspace(p, Q.device)
    if O is None:
        O = torch.empty(Q.shape, dtype=t, device=Q.device)
        o_at = O.data_ptr()
    else:
        o_at = _at(O, "O", where, t, dense, dev)
    if lse is None and want_lse:
        lse = torch.empty(stats.of, dtype=torch.float32, device=Q.device)
    n_ws = ws.numel()
    code = (_LIB or load_library()).bra_cross_attend(
        byref(p), q_at, k_at, v_at, len_at, mask_at, o_at, None if lse is None else _at(lse, "lse", where, torch.float32, stats, dev),
        _ws_at(ws, where, dev), n_ws, _stream(stream))
    if code:
        raise BraError(code, where)
    return O, lse


def bra_cross_backward(p, Q, K, V, O, lse, dO, key_len=None, key_mask=None, dQ=None, dK=None, dV=None, ws=None, stream=None):
    """bra_cross_backward: -> (dQ, dK, dV)."""
    if stream is not None and (ws is None or dQ is None or dK is None or dV is None):
        with _on(stream):
            return bra_cross_backward(p, Q, K, V, O, lse, dO, key_len, key_mask, dQ, dK, dV, ws)
    torch, dev, where = _TORCH or _torch(), (_GET_DEVICE or _device_getter())(), "bra_cross_backward"
    t, q, k, v, dense, images, keys, stats = _derived(p, _cross_derived)
    ins = (_rows_at(Q, "Q", where, t, dev, q), _rows_at(K, "K", where, t, dev, k), _rows_at(V, "V", where, t, dev, v),
           *_cross_mask(key_len, key_mask, where, torch, images, keys, dev), _at(O, "O", where, t, dense, dev),
           _at(lse, "lse", where, torch.float32, stats, dev), _at(dO, "dO", where, t, dense, dev))
    if ws is None:
        ws = cross_workspace(p, Q.device)
    dQ = _like(Q, q) if dQ is None else dQ
    dK = _like(K, k) if dK is None else dK
    dV = _like(V, v) if dV is None else dV
    n_ws = ws.numel()
    code = (_LIB or load_library()).bra_cross_backward(
        byref(p), *ins, _rows_at(dQ, "dQ", where, t, dev, q), _rows_at(dK, "dK", where, t, dev, k), _rows_at(dV, "dV", where, t, dev, v),
        _ws_at(ws, where, dev), n_ws, _stream(stream))
    if code:
        raise BraError(code, where)
    return dQ, dK, dV


_NORMS, _GATES = {"none": 0, "rms": 1, "layer": 2}, {"none": 0, "channel": 1, "image": 2}


def make_norm_problem(B, N, C, pre="layer", post="none", gate="none", per_image=False, alpha=1.0, eps=1e-6,
                      dtype="bf16") -> BraNormProblem:
    return BraNormProblem(B, N, C, _NORMS[pre], _NORMS[post], _GATES[gate], int(bool(per_image)), _DTYPES[dtype], float(eps), float(alpha))


def norm_workspace_bytes(p: BraNormProblem) -> int:
    return int(load_library().bra_norm_workspace_bytes(ctypes.byref(p)))


def norm_workspace(p: BraNormProblem, device="cuda"):
    """Scratch tensor of bra_norm_workspace_bytes(p) bytes (for the gradients)."""
    return _scratch(norm_workspace_bytes(p), "bra_norm_workspace_bytes", device)


def _norm_derived(p):
    # which image a token belongs to matters only where weights are an image's
    rows = _Shape(p.B, p.N, p.C) if p.gate == 2 or p.per_image else _Shape(p.B * p.N, p.C)
    return (_tdtype(p), rows, _Shape(p.C), _Shape(p.B, p.C) if p.gate == 2 else _Shape(p.C), _Shape(p.B, p.C) if p.per_image else _Shape(p.C),
            p.pre != 0)


def _weight(t, name, where, shape, dev):
    return None if t is None else _at(t, name, where, _TORCH.float32, shape, dev)


def bra_residual_norm(p, x, y=None, gate=None, post_w=None, post_b=None, w=None, b=None, h=None, n=None, stream=None, want_h=True):
    """bra_residual_norm: x, y -> (h, n): the residual stream behind the block, and what the next block reads."""
    if stream is not None and ((h is None and want_h) or (n is None and p.pre)):
        with _on(stream):
            return bra_residual_norm(p, x, y, gate, post_w, post_b, w, b, h, n, None, want_h)
    torch, dev, where = _TORCH or _torch(), (_GET_DEVICE or _device_getter())(), "bra_residual_norm"
    t, rows, C, gates, affine, normed = _derived(p, _norm_derived)
    x_at = _at(x, "x", where, t, rows, dev)
    y_at = None if y is None else _at(y, "y", where, t, rows, dev)
    if h is None and want_h:
        h = torch.empty_like(x)
        h_at = h.data_ptr()
    else:
        h_at = None if h is None else _at(h, "h", where, t, rows, dev)
    if n is None and normed:
        n = torch.empty_like(x)
        n_at = n.data_ptr()
    else:
        n_at = None if n is None else _at(n, "n", where, t, rows, dev)
    code = (_LIB or load_library()).bra_residual_norm(
        byref(p), x_at, y_at, _weight(gate, "gate", where, gates, dev), _weight(post_w, "post_w", where, C, dev),
        _weight(post_b, "post_b", where, C, dev), _weight(w, "w", where, affine, dev), _weight(b, "b", where, affine, dev), h_at, n_at,
        _stream(stream))
    if code:
        raise BraError(code, where)
    return h, n


def bra_residual_norm_backward(p, x, y, dh, dn, gate=None, post_w=None, post_b=None, w=None, b=None, dx=None, dy=None, ws=None,
                               stream=None):
    """bra_residual_norm_backward: -> {"dx", "dy", and of the weights that are given "dgate", "d_post_w", "d_post_b", "dw", "db"}."""
    if stream is not None:                                   # the weights' gradients are always its own
        with _on(stream):
            return bra_residual_norm_backward(p, x, y, dh, dn, gate, post_w, post_b, w, b, dx, dy, ws)
    torch, dev, where = _TORCH or _torch(), (_GET_DEVICE or _device_getter())(), "bra_residual_norm_backward"
    t, rows, C, gates, affine, _ = _derived(p, _norm_derived)
    ins = (_at(x, "x", where, t, rows, dev), None if y is None else _at(y, "y", where, t, rows, dev), _weight(gate, "gate", where, gates, dev),
           _weight(post_w, "post_w", where, C, dev), _weight(post_b, "post_b", where, C, dev), _weight(w, "w", where, affine, dev),
           None if dh is None else _at(dh, "dh", where, t, rows, dev), None if dn is None else _at(dn, "dn", where, t, rows, dev))
    _weight(b, "b", where, affine, dev)
    if ws is None:
        ws = norm_workspace(p, x.device)
    out = {"dx": torch.empty_like(x) if dx is None else dx}
    if y is not None:
        out["dy"] = torch.empty_like(y) if dy is None else dy
    for name, weight in (("dgate", gate), ("d_post_w", post_w), ("d_post_b", post_b), ("dw", w), ("db", b)):
        if weight is not None:
            out[name] = torch.empty_like(weight)
    n_ws = ws.numel()
    code = (_LIB or load_library()).bra_residual_norm_backward(
        byref(p), *ins, _at(out["dx"], "dx", where, t, rows, dev), None if y is None else _at(out["dy"], "dy", where, t, rows, dev),
        *(_ptr(out.get(name)) for name in ("dgate", "d_post_w", "d_post_b", "dw", "db")),
        _ws_at(ws, where, dev), n_ws, _stream(stream))
    if code:
        raise BraError(code, where)
    return out
