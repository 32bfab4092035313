"""Python binding of libosoftmax (online-normalizer softmax, fused softmax +
top-k, sampling, log probabilities, expert routing and balance on MI355X).
Argument marshalling only: every step of the computation runs in the library's
HIP kernels, reached through its C ABI (``include/osoftmax.h``).  PyTorch
supplies device memory and the current stream.  There is no fallback: if the
library is missing, every call raises.
"""
from __future__ import annotations

import ctypes
import functools
import os
from typing import NamedTuple

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libosoftmax.so")

F32, BF16 = 0, 1
NAIVE, SAFE, ONLINE, RESIDENT = 0, 1, 2, 3
RESIDENT_MAX_VEC = 16384
KERNEL_AUTO, KERNEL_ROWS, KERNEL_SPLIT = 0, 1, 2
OK, EINVAL, EUNSUPPORTED, EHIP, ENOMEM, ESCRATCH = 0, 1, 2, 3, 4, 5
NOALLOC_SCRATCH_BYTES = 1 << 20
TOPK_KMAX = 64
PROJ_KMAX = 16
ROUTE_EMAX, ROUTE_GMAX = 1024, 64
LOGPROB_TMAX = 64
SCORES = {"softmax": 0, "sigmoid": 1}
TOPK_ONLINE_FUSED, TOPK_SAFE_FUSED, TOPK_SAFE_UNFUSED, TOPK_ONLINE_UNFUSED, TOPK_VALUES = range(5)
TOPK_ALGOS = {"online_fused": TOPK_ONLINE_FUSED, "safe_fused": TOPK_SAFE_FUSED,
              "safe_unfused": TOPK_SAFE_UNFUSED, "online_unfused": TOPK_ONLINE_UNFUSED,
              "values": TOPK_VALUES}
UNFUSED = (TOPK_SAFE_UNFUSED, TOPK_ONLINE_UNFUSED)

MODES = {"naive": NAIVE, "safe": SAFE, "online": ONLINE, "resident": RESIDENT}
_DTYPES = {torch.float32: F32, torch.bfloat16: BF16}

_lib = None


class SampleParams(ctypes.Structure):
    """``osm_sample_params``."""
    _fields_ = [("temperature", ctypes.c_void_p), ("top_k", ctypes.c_void_p),
                ("top_p", ctypes.c_void_p), ("min_p", ctypes.c_void_p),
                ("temperature_all", ctypes.c_float), ("top_k_all", ctypes.c_int32),
                ("top_p_all", ctypes.c_float), ("min_p_all", ctypes.c_float)]


class Route(ctypes.Structure):
    """``osm_route``."""
    _fields_ = [("score", ctypes.c_int), ("groups", ctypes.c_int), ("top_groups", ctypes.c_int),
                ("group_top", ctypes.c_int), ("renorm", ctypes.c_int), ("scale", ctypes.c_float)]


class Logprob(ctypes.Structure):
    """``osm_logprob``."""
    _fields_ = [("tokens", ctypes.c_void_p), ("logp", ctypes.c_void_p),
                ("entropy", ctypes.c_void_p), ("stats", ctypes.c_void_p),
                ("top_logp", ctypes.c_void_p), ("top_idx", ctypes.c_void_p),
                ("T", ctypes.c_int), ("K", ctypes.c_int), ("temperature", ctypes.c_float)]


class Logprobs(NamedTuple):
    """What logprob_fwd returns; None for what it was not asked for."""
    logp: torch.Tensor | None
    entropy: torch.Tensor | None
    stats: torch.Tensor | None
    top_vals: torch.Tensor | None
    top_idx: torch.Tensor | None


class Balance(NamedTuple):
    """What balance_fwd returns."""
    loss: torch.Tensor
    counts: torch.Tensor
    probs: torch.Tensor
    rows: torch.Tensor


class OsmError(RuntimeError):
    def __init__(self, status: int, what: str):
        self.status = status
        super().__init__(f"{what}: {status_string(status)} (status {status})")


def lib() -> ctypes.CDLL:
    """The loaded C library (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is not built; run __graft_entry__.build() "
                           "(or python paper_1805_02867_amd/build.py)")
    L = ctypes.CDLL(LIB_PATH)
    vp, i64, i32 = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int
    L.softmax_fwd.argtypes = [vp, vp, i64, i64, i32, i32, vp]
    L.softmax_fwd.restype = i32
    L.softmax_fwd_ex.argtypes = [vp, vp, i64, i64, i32, i32, i32, i64, vp]
    L.softmax_fwd_ex.restype = i32
    L.softmax_topk.argtypes = [vp, vp, vp, i64, i64, i32, vp]
    L.softmax_topk.restype = i32
    L.softmax_topk_dt.argtypes = [vp, vp, vp, i64, i64, i32, i32, vp]
    L.softmax_topk_dt.restype = i32
    L.softmax_topk_ex.argtypes = [vp, vp, vp, i64, i64, i32, i32, i32, i64, vp]
    L.softmax_topk_ex.restype = i32
    L.softmax_topk_ex_noalloc.argtypes = [vp, vp, vp, i64, i64, i32, i32, i32, i64, vp]
    L.softmax_topk_ex_noalloc.restype = i32
    L.softmax_topk_algo.argtypes = [vp, vp, vp, vp, i64, i64, i32, i32, i32, i32, i64, vp]
    L.softmax_topk_algo.restype = i32
    L.topk_fwd.argtypes = [vp, vp, vp, i64, i64, i32, i32, vp]
    L.topk_fwd.restype = i32
    L.osm_topk_plan.argtypes = [i64, i64, i32, i32, ctypes.POINTER(i32), ctypes.POINTER(i64)]
    L.osm_topk_plan.restype = i32
    L.proj_fwd.argtypes = [vp, vp, vp, i64, i64, i64, vp]
    L.proj_fwd.restype = i32
    L.proj_softmax_topk.argtypes = [vp, vp, vp, vp, i64, i64, i64, i32, vp]
    L.proj_softmax_topk.restype = i32
    L.softmax_sample.argtypes = [vp, i64, vp, vp, vp, vp, i64, i64, i32, vp]
    L.softmax_sample.restype = i32
    L.softmax_sample_ws.argtypes = [vp, i64, vp, vp, vp, vp, i64, i64, i32, vp, ctypes.c_size_t,
                                    vp]
    L.softmax_sample_ws.restype = i32
    L.osm_sample_workspace.argtypes = [i64, i64, i32, ctypes.POINTER(ctypes.c_size_t)]
    L.osm_sample_workspace.restype = i32
    L.route_fwd.argtypes = [vp, vp, vp, vp, i64, i64, i32, i32, vp, vp]
    L.route_fwd.restype = i32
    L.route_bwd.argtypes = [vp, vp, vp, vp, i64, i64, i32, i32, vp, vp]
    L.route_bwd.restype = i32
    size_t, f32 = ctypes.c_size_t, ctypes.c_float
    L.logprob_fwd.argtypes = [vp, i64, vp, i64, i64, i32, vp]
    L.logprob_fwd.restype = i32
    L.logprob_fwd_ws.argtypes = [vp, i64, vp, i64, i64, i32, vp, size_t, vp]
    L.logprob_fwd_ws.restype = i32
    L.osm_logprob_workspace.argtypes = [i64, i64, i32, i32, ctypes.POINTER(size_t)]
    L.osm_logprob_workspace.restype = i32
    L.logprob_bwd.argtypes = [vp, i64, vp, vp, vp, vp, vp, vp, i64, i64, i64, i32, i32, f32, vp]
    L.logprob_bwd.restype = i32
    L.balance_fwd.argtypes = [vp] * 7 + [i64, i64, i32, i64, i32, i32, f32, vp]
    L.balance_fwd.restype = i32
    L.balance_fwd_ws.argtypes = [vp] * 7 + [i64, i64, i32, i64, i32, i32, f32, vp, size_t, vp]
    L.balance_fwd_ws.restype = i32
    L.osm_balance_workspace.argtypes = [i64, i64, i64, ctypes.POINTER(size_t)]
    L.osm_balance_workspace.restype = i32
    L.balance_bwd.argtypes = [vp] * 7 + [i64, i64, i32, i64, i32, i32, f32, vp]
    L.balance_bwd.restype = i32
    L.osm_plan.argtypes = [i64, i64, i32, i32, ctypes.POINTER(i32), ctypes.POINTER(i64)]
    L.osm_plan.restype = i32
    L.osm_stream_release.argtypes = [vp]
    L.osm_stream_release.restype = i32
    L.osm_ref_stream.argtypes = [i32, vp, vp, i64, vp]
    L.osm_ref_stream.restype = i32
    L.osm_status_string.argtypes = [i32]
    L.osm_status_string.restype = ctypes.c_char_p
    _lib = L
    return L


def status_string(status: int) -> str:
    return lib().osm_status_string(int(status)).decode()


# torch's current device and stream handle, asked for directly (None where a
# torch release has no such entry)
_device = getattr(torch._C, "_cuda_getDevice", None)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) if _device else None


def _stream(stream) -> int:
    """The HIP stream handle of `stream`, or of torch's current stream.  The
    handle is asked for directly: torch.cuda.current_stream() builds a stream
    object for it, 2.8 us of the ~8.5 a small call took (0.2 this way)."""
    if stream is None:
        if _raw_stream is None:
            return torch.cuda.current_stream().cuda_stream
        return _raw_stream(_device())
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _batch(x: torch.Tensor, name: str = "x"):
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise ValueError(f"{name} must be a CUDA (HIP) tensor")
    if x.dtype not in _DTYPES:
        raise ValueError(f"{name} must be float32 or bfloat16, got {x.dtype}")
    if not x.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    shape = x.shape
    if len(shape) == 2:
        return shape
    if len(shape) != 1:
        raise ValueError(f"{name} must be 1-D or 2-D (N x V)")
    return 1, shape[0]


def _like(y, x: torch.Tensor) -> bool:
    """Whether y is a contiguous tensor of x's shape, dtype and device."""
    return (isinstance(y, torch.Tensor) and y.shape == x.shape and y.dtype is x.dtype
            and y.get_device() == x.get_device() and y.is_contiguous())


def _mode(mode) -> int:
    if isinstance(mode, str):
        if mode not in MODES:
            raise ValueError(f"mode must be one of {sorted(MODES)}")
        return MODES[mode]
    return int(mode)


def softmax_fwd(x: torch.Tensor, y: torch.Tensor | None = None, mode="online",
                stream=None, kernel: int = KERNEL_AUTO, param: int = 0) -> torch.Tensor:
    """y = Softmax(x) per row via ``softmax_fwd`` / ``softmax_fwd_ex``."""
    N, V = _batch(x)
    if y is None:
        y = torch.empty_like(x)
    elif not _like(y, x):
        Ny, Vy = _batch(y, "y")
        if (Ny, Vy) != (N, V) or y.dtype != x.dtype or y.device != x.device:
            raise ValueError("y must match x in shape, dtype and device")
    dt = _DTYPES[x.dtype]
    if kernel == KERNEL_AUTO:
        rc = lib().softmax_fwd(x.data_ptr(), y.data_ptr(), N, V, dt, _mode(mode),
                               _stream(stream))
    else:
        rc = lib().softmax_fwd_ex(x.data_ptr(), y.data_ptr(), N, V, dt, _mode(mode),
                                  int(kernel), int(param), _stream(stream))
    if rc != OK:
        raise OsmError(rc, "softmax_fwd")
    return y


def _topk_outputs(x, N, K, vals, idx):
    if vals is None:
        vals = torch.empty((N, K), dtype=torch.float32, device=x.device)
    if idx is None:
        idx = torch.empty((N, K), dtype=torch.int32, device=x.device)
    if not _holds(vals, torch.float32, x, N * K):
        raise ValueError("vals must be a contiguous torch.float32 tensor of N*K elements on "
                         "x's device")
    if not _holds(idx, torch.int32, x, N * K):
        raise ValueError("idx must be a contiguous torch.int32 tensor of N*K elements on "
                         "x's device")
    return vals, idx


def _holds(t: torch.Tensor, dtype, x: torch.Tensor, n: int) -> bool:
    return (t.dtype is dtype and t.is_contiguous() and t.numel() == n
            and t.get_device() == x.get_device())


def _algo(algo) -> int:
    if isinstance(algo, str):
        if algo not in TOPK_ALGOS:
            raise ValueError(f"algo must be one of {sorted(TOPK_ALGOS)}")
        return TOPK_ALGOS[algo]
    return int(algo)


def softmax_topk(x: torch.Tensor, K: int, vals: torch.Tensor | None = None,
                 idx: torch.Tensor | None = None, stream=None, kernel: int = KERNEL_AUTO,
                 param: int = 0, algo="online_fused", y: torch.Tensor | None = None):
    """(vals, idx) = softmax + top-k per row.

    The default (Alg. 4, one pass) goes through ``softmax_topk`` (binary32
    rows), ``softmax_topk_dt`` (bfloat16 rows) or, with an explicit kernel,
    ``softmax_topk_ex``.  Another ``algo`` (see ``TOPK_ALGOS``) goes through
    ``softmax_topk_algo``; the unfused ones write the softmax into ``y``
    (allocated here when not given)."""
    N, V = _batch(x)
    vals, idx = _topk_outputs(x, N, K, vals, idx)
    a = _algo(algo)
    dt = _DTYPES[x.dtype]
    if a != TOPK_ONLINE_FUSED:
        if a in UNFUSED:
            if y is None:
                y = torch.empty_like(x)
            elif (tuple(_batch(y, "y")) != (N, V) or y.dtype != x.dtype or y.device != x.device):
                raise ValueError("y must match x in shape, dtype and device")
        yp = y.data_ptr() if (a in UNFUSED) else None
        rc = lib().softmax_topk_algo(x.data_ptr(), yp, vals.data_ptr(), idx.data_ptr(), N, V,
                                     int(K), dt, a, int(kernel), int(param), _stream(stream))
    elif kernel != KERNEL_AUTO:
        rc = lib().softmax_topk_ex(x.data_ptr(), vals.data_ptr(), idx.data_ptr(), N, V,
                                   int(K), dt, int(kernel), int(param), _stream(stream))
    elif x.dtype == torch.float32:
        rc = lib().softmax_topk(x.data_ptr(), vals.data_ptr(), idx.data_ptr(), N, V, int(K),
                                _stream(stream))
    else:
        rc = lib().softmax_topk_dt(x.data_ptr(), vals.data_ptr(), idx.data_ptr(), N, V,
                                   int(K), dt, _stream(stream))
    if rc != OK:
        raise OsmError(rc, "softmax_topk")
    return vals, idx


softmax_topk_dt = softmax_topk


def softmax_topk_noalloc(x: torch.Tensor, K: int, vals: torch.Tensor | None = None,
                         idx: torch.Tensor | None = None, stream=None,
                         kernel: int = KERNEL_AUTO, param: int = 0):
    """(vals, idx) as softmax_topk, through ``softmax_topk_ex_noalloc``: the
    library allocates nothing (split partials in its fixed per-device scratch
    array).  Calls that can overlap on one device race on that array."""
    N, V = _batch(x)
    vals, idx = _topk_outputs(x, N, K, vals, idx)
    rc = lib().softmax_topk_ex_noalloc(x.data_ptr(), vals.data_ptr(), idx.data_ptr(), N, V,
                                       int(K), _DTYPES[x.dtype], int(kernel), int(param),
                                       _stream(stream))
    if rc != OK:
        raise OsmError(rc, "softmax_topk_ex_noalloc")
    return vals, idx


def topk(x: torch.Tensor, K: int, vals: torch.Tensor | None = None,
         idx: torch.Tensor | None = None, stream=None):
    """(vals, idx) = the K largest elements of each row and their indices
    (``topk_fwd``); larger first, equal values in increasing index order."""
    N, V = _batch(x)
    vals, idx = _topk_outputs(x, N, K, vals, idx)
    rc = lib().topk_fwd(x.data_ptr(), vals.data_ptr(), idx.data_ptr(), N, V, int(K),
                        _DTYPES[x.dtype], _stream(stream))
    if rc != OK:
        raise OsmError(rc, "topk_fwd")
    return vals, idx


def stream_release(stream=None) -> None:
    """Frees the scratch the library keeps for `stream` (``osm_stream_release``),
    in stream order; call before destroying a stream that used the library."""
    if stream is None:
        torch.cuda.init()  # the current stream may be asked for before any tensor was made
    rc = lib().osm_stream_release(_stream(stream))
    if rc != OK:
        raise OsmError(rc, "osm_stream_release")


def topk_plan(N: int, V: int, K: int, dtype=torch.float32):
    """(kernel, param) that the top-k entry points use for this shape."""
    k = ctypes.c_int()
    p = ctypes.c_int64()
    dt = _DTYPES[dtype] if isinstance(dtype, torch.dtype) else int(dtype)
    rc = lib().osm_topk_plan(int(N), int(V), dt, int(K), ctypes.byref(k), ctypes.byref(p))
    if rc != OK:
        raise OsmError(rc, "osm_topk_plan")
    return k.value, p.value


def plan(N: int, V: int, dtype=torch.float32, mode="online"):
    """(kernel, param) that softmax_fwd uses for this shape (``osm_plan``)."""
    k = ctypes.c_int()
    p = ctypes.c_int64()
    dt = _DTYPES[dtype] if isinstance(dtype, torch.dtype) else int(dtype)
    rc = lib().osm_plan(int(N), int(V), dt, _mode(mode), ctypes.byref(k), ctypes.byref(p))
    if rc != OK:
        raise OsmError(rc, "osm_plan")
    return k.value, p.value


def _proj_inputs(h: torch.Tensor, w: torch.Tensor):
    for t, nm in ((h, "h"), (w, "w")):
        if not isinstance(t, torch.Tensor) or not t.is_cuda or t.dtype != torch.bfloat16:
            raise ValueError(f"{nm} must be a bfloat16 CUDA (HIP) tensor")
        if t.dim() != 2 or not t.is_contiguous():
            raise ValueError(f"{nm} must be a contiguous 2-D tensor")
    if h.shape[1] != w.shape[1]:
        raise ValueError("h (N x H) and w (V x H) must have the same H")
    return h.shape[0], h.shape[1], w.shape[0]


def ref_stream(op: str, x: torch.Tensor, y: torch.Tensor, stream=None) -> None:
    """Reference streaming kernel for measurement (``osm_ref_stream``):
    op "read" reads all of x (y: a sink of at least 1 KB), "copy" copies x
    to y (same size).  Nothing of the method; the plain rates the other
    kernels are judged against."""
    if op not in ("read", "copy"):
        raise ValueError("op must be 'read' or 'copy'")
    n = x.numel() * x.element_size()
    if op == "copy" and y.numel() * y.element_size() < n:
        raise ValueError("y is smaller than x")
    rc = lib().osm_ref_stream(0 if op == "read" else 1, x.data_ptr(), y.data_ptr(), n,
                              _stream(stream))
    if rc != OK:
        raise OsmError(rc, "osm_ref_stream")


def proj(h: torch.Tensor, w: torch.Tensor, out: torch.Tensor | None = None, stream=None):
    """logits = h . w^T (``proj_fwd``): h N x H and w V x H bfloat16, binary32 out."""
    N, H, V = _proj_inputs(h, w)
    if out is None:
        out = torch.empty((N, V), dtype=torch.float32, device=h.device)
    elif (out.dtype != torch.float32 or not out.is_contiguous() or out.numel() != N * V):
        raise ValueError("out must be a contiguous float32 tensor of N*V elements")
    rc = lib().proj_fwd(h.data_ptr(), w.data_ptr(), out.data_ptr(), N, H, V, _stream(stream))
    if rc != OK:
        raise OsmError(rc, "proj_fwd")
    return out


def proj_softmax_topk(h: torch.Tensor, w: torch.Tensor, K: int, vals: torch.Tensor | None = None,
                      idx: torch.Tensor | None = None, stream=None):
    """(vals, idx) = top-k of softmax(h . w^T) per row without writing the
    logits (``proj_softmax_topk``)."""
    N, H, V = _proj_inputs(h, w)
    vals, idx = _topk_outputs(h, N, K, vals, idx)
    rc = lib().proj_softmax_topk(h.data_ptr(), w.data_ptr(), vals.data_ptr(), idx.data_ptr(),
                                 N, H, V, int(K), _stream(stream))
    if rc != OK:
        raise OsmError(rc, "proj_softmax_topk")
    return vals, idx


def _on_current_device(x: torch.Tensor, name: str) -> None:
    """The library launches on the current device and its stream."""
    current = torch.cuda.current_device() if _device is None else _device()
    if x.get_device() != current:
        raise ValueError(f"{name} must be on the current device")


def _rows(x: torch.Tensor):
    """(N, V, elements from row to row) of a batch whose rows are contiguous."""
    if not isinstance(x, torch.Tensor) or not x.is_cuda:
        raise ValueError("x must be a CUDA (HIP) tensor")
    if x.dtype not in _DTYPES:
        raise ValueError(f"x must be float32 or bfloat16, got {x.dtype}")
    if x.dim() == 1:
        x = x.unsqueeze(0)
    if x.dim() != 2:
        raise ValueError("x must be 1-D or 2-D (N x V)")
    N, V = x.shape
    ld = x.stride(0) if N > 1 else V
    if V > 1 and x.stride(1) != 1 or ld < V:
        raise ValueError("the rows of x must be contiguous and must not overlap")
    return N, V, ld


def _vector(t, dtype, x: torch.Tensor, n: int, name: str) -> torch.Tensor:
    if not isinstance(t, torch.Tensor) or not _holds(t, dtype, x, n):
        raise ValueError(f"{name} must be a contiguous {dtype} tensor of {n} elements on x's "
                         "device")
    return t


def _output(t, shape, dtype, x: torch.Tensor, name: str) -> torch.Tensor:
    """The caller's output, or a new one (which needs no checks: they take 0.5 us)."""
    if t is None:
        return x.new_empty(shape, dtype=dtype)
    n = shape[0] * shape[1] if len(shape) == 2 else shape[0]
    return _vector(t, dtype, x, n, name)


def _setting(v, dtype, x: torch.Tensor, N: int, name: str):
    """(pointer, value for all rows) of a setting given as a tensor or a number."""
    if isinstance(v, torch.Tensor):
        return _vector(v, dtype, x, N, name).data_ptr(), 0
    if dtype is not torch.int32:
        return None, float(v)
    return None, max(-1 << 31, min(int(v), (1 << 31) - 1))  # (a field would take the low 32 bits)


def softmax_sample(x: torch.Tensor, u: torch.Tensor, temperature=1.0, top_k=0, top_p=1.0,
                   min_p=0.0, vals: torch.Tensor | None = None, idx: torch.Tensor | None = None,
                   workspace: torch.Tensor | None = None, stream=None):
    """(vals, idx) = one element sampled from each row's softmax, with its probability
    among the elements that the filters keep (``softmax_sample``).

    ``u``: N random numbers in [0, 1), float32.  ``temperature``, ``top_p`` and
    ``min_p`` (float32) and ``top_k`` (int32) are numbers or tensors of N.  Rows may
    be apart (``x[:, :V]`` of a padded batch).  ``workspace``: uint8, at least
    ``sample_workspace(N, V, dtype)`` bytes, used instead of the library's scratch
    (``softmax_sample_ws``); while the current stream is being captured into a graph,
    one is taken from the graph's own memory, which is in order on that stream alone: a
    call on another ``stream`` then has to bring its workspace."""
    N, V, ld = _rows(x)
    _on_current_device(x, "x")
    capturing = workspace is None and torch.cuda.is_current_stream_capturing()
    if capturing and _stream(stream) != _stream(None):
        raise ValueError("a captured call on another stream than the current one needs a "
                         "workspace")
    _vector(u, torch.float32, x, N, "u")
    t, t_all = _setting(temperature, torch.float32, x, N, "temperature")
    k, k_all = _setting(top_k, torch.int32, x, N, "top_k")
    p, p_all = _setting(top_p, torch.float32, x, N, "top_p")
    q, q_all = _setting(min_p, torch.float32, x, N, "min_p")
    vals = _output(vals, (N,), torch.float32, x, "vals")
    idx = _output(idx, (N,), torch.int32, x, "idx")
    params = SampleParams(t, k, p, q, t_all, k_all, p_all, q_all)
    if capturing:
        workspace = torch.empty(sample_workspace(N, V, x.dtype), dtype=torch.uint8,
                                device=x.device)
    if workspace is None:
        rc = lib().softmax_sample(x.data_ptr(), ld, u.data_ptr(), ctypes.byref(params),
                                  vals.data_ptr(), idx.data_ptr(), N, V, _DTYPES[x.dtype],
                                  _stream(stream))
    else:
        _vector(workspace, torch.uint8, x, workspace.numel(), "workspace")
        rc = lib().softmax_sample_ws(x.data_ptr(), ld, u.data_ptr(), ctypes.byref(params),
                                     vals.data_ptr(), idx.data_ptr(), N, V, _DTYPES[x.dtype],
                                     workspace.data_ptr(), workspace.numel(), _stream(stream))
    if rc != OK:
        raise OsmError(rc, "softmax_sample")
    return vals, idx


def sample_workspace(N: int, V: int, dtype=torch.float32) -> int:
    """Bytes of workspace of softmax_sample for this shape (``osm_sample_workspace``)."""
    n = ctypes.c_size_t()
    dt = _DTYPES[dtype] if isinstance(dtype, torch.dtype) else int(dtype)
    rc = lib().osm_sample_workspace(int(N), int(V), dt, ctypes.byref(n))
    if rc != OK:
        raise OsmError(rc, "osm_sample_workspace")
    return n.value


@functools.lru_cache(maxsize=256)
def _made_route(score, groups, top_groups, group_top, renorm, scale):
    """A reference to an ``osm_route`` of these values (building one takes 0.9 us)."""
    for v in (score, groups, top_groups, group_top):
        if not -1 << 31 <= v < 1 << 31:  # (a field would take the low 32 bits)
            raise ValueError(f"{v} is no option of a router")
    return ctypes.byref(Route(score, groups, top_groups, group_top, renorm, scale))


def _route(score, groups, top_groups, group_top, renorm, scale):
    # (0.0 and -0.0 are one key)
    make = _made_route if scale else _made_route.__wrapped__
    return make(score, groups, top_groups, group_top, renorm, scale)


def _score(score) -> int:
    if isinstance(score, str):
        if score not in SCORES:
            raise ValueError(f"score must be one of {sorted(SCORES)}")
        return SCORES[score]
    return int(score)


def route_fwd(x: torch.Tensor, K: int, bias: torch.Tensor | None = None, score="softmax",
              groups: int = 1, top_groups: int = 1, group_top: int = 1, renorm: bool = True,
              scale: float = 1.0, vals: torch.Tensor | None = None,
              idx: torch.Tensor | None = None, stream=None):
    """(vals, idx) = weights and indices of each row's K experts (``route_fwd``): N x K
    float32 and int32, best first."""
    N, E = _batch(x)
    _on_current_device(x, "x")
    if bias is not None:
        _vector(bias, torch.float32, x, E, "bias")
    vals = _output(vals, (N, K), torch.float32, x, "vals")
    idx = _output(idx, (N, K), torch.int32, x, "idx")
    rc = lib().route_fwd(x.data_ptr(), None if bias is None else bias.data_ptr(),
                         vals.data_ptr(), idx.data_ptr(), N, E, int(K), _DTYPES[x.dtype],
                         _route(_score(score), int(groups), int(top_groups), int(group_top),
                                bool(renorm), float(scale)),
                         _stream(stream))
    if rc != OK:
        raise OsmError(rc, "route_fwd")
    return vals, idx


def route_bwd(x: torch.Tensor, idx: torch.Tensor, dvals: torch.Tensor, score="softmax",
              renorm: bool = True, scale: float = 1.0, dx: torch.Tensor | None = None,
              stream=None) -> torch.Tensor:
    """dx = gradient with respect to x of route_fwd's weights, whose own gradient is
    ``dvals`` (N x K) at the experts ``idx`` (``route_bwd``)."""
    N, E = _batch(x)
    _on_current_device(x, "x")
    K = idx.shape[-1]
    _vector(idx, torch.int32, x, N * K, "idx")
    _vector(dvals, torch.float32, x, N * K, "dvals")
    if dx is None:
        dx = torch.empty_like(x)
    elif not _like(dx, x):
        raise ValueError("dx must be a contiguous tensor like x")
    rc = lib().route_bwd(x.data_ptr(), idx.data_ptr(), dvals.data_ptr(), dx.data_ptr(), N, E, K,
                         _DTYPES[x.dtype],
                         _route(_score(score), 1, 1, 1, bool(renorm), float(scale)),
                         _stream(stream))
    if rc != OK:
        raise OsmError(rc, "route_bwd")
    return dx


_capturing = getattr(torch._C, "_cuda_isCurrentStreamCapturing", None)


def _own_workspace(workspace, x: torch.Tensor, stream, need, *shape):
    """The workspace that a call is given: the caller's, or while the current stream is being
    captured one of need(*shape) bytes from the graph's own memory (None: the library's
    scratch)."""
    if workspace is not None:
        return _vector(workspace, torch.uint8, x, workspace.numel(), "workspace")
    if not (_capturing or torch.cuda.is_current_stream_capturing)():
        return None
    if _stream(stream) != _stream(None):
        raise ValueError("a captured call on another stream than the current one needs a "
                         "workspace")
    return torch.empty(need(*shape), dtype=torch.uint8, device=x.device)


def _tokens(tokens, x: torch.Tensor, N: int, name: str = "tokens") -> int:
    """T of a tensor of T given tokens for each of x's N rows: N, N x T, or T of a row."""
    if not isinstance(tokens, torch.Tensor):
        raise ValueError(f"{name} must be a tensor")
    shape = tokens.shape
    T = shape[-1] if len(shape) == 2 or (len(shape) == 1 and x.dim() == 1) else 1
    rows = shape[0] if len(shape) == 2 or x.dim() == 2 and len(shape) == 1 else 1
    if len(shape) not in (1, 2) or rows != N:
        raise ValueError(f"{name} must have a row for each of x's")
    return T


def _asked(t, shape, x: torch.Tensor, name: str):
    """An output that is given, asked for (True) or not wanted (False, None)."""
    if not isinstance(t, torch.Tensor) and not t:
        return None
    return _output(None if t is True else t, shape, torch.float32, x, name)


def logprob_fwd(x: torch.Tensor, tokens: torch.Tensor | None = None, K: int = 0, entropy=False,
                stats=False, temperature: float = 1.0, logp: torch.Tensor | None = None,
                top_vals: torch.Tensor | None = None, top_idx: torch.Tensor | None = None,
                workspace: torch.Tensor | None = None, stream=None) -> Logprobs:
    """Log probabilities of each row's given tokens, its entropy and its K best alternatives,
    as far as they are asked for (``logprob_fwd``).

    ``tokens``: int32, N or N x T (T up to ``LOGPROB_TMAX``); one outside [0, V) is ignored, its
    logp is 0.  ``entropy`` and ``stats`` (what logprob_bwd takes, N x 2) are True or the
    tensor to write.  Rows may be apart (``x[:, :V]`` of a padded batch).  ``workspace``: uint8,
    at least ``logprob_workspace(N, V, K, dtype)`` bytes, used instead of the library's
    scratch (``logprob_fwd_ws``); under graph capture as in softmax_sample."""
    N, V, ld = _rows(x)
    _on_current_device(x, "x")
    K, T, tp, lp, vp, ip = int(K), 0, None, None, None, None
    if tokens is not None:
        T = _tokens(tokens, x, N)
        tp = _vector(tokens, torch.int32, x, N * T, "tokens").data_ptr()
        if logp is None:
            logp = x.new_empty((N, T) if tokens.dim() == 2 else (N * T,), dtype=torch.float32)
        else:
            _vector(logp, torch.float32, x, N * T, "logp")
        lp = logp.data_ptr()
    elif logp is not None:
        raise ValueError("logp needs tokens")
    if K > 0:
        top_vals = _output(top_vals, (N, K), torch.float32, x, "top_vals")
        top_idx = _output(top_idx, (N, K), torch.int32, x, "top_idx")
        vp, ip = top_vals.data_ptr(), top_idx.data_ptr()
    elif top_vals is not None or top_idx is not None:
        raise ValueError("top_vals and top_idx need K")
    entropy = _asked(entropy, (N,), x, "entropy")
    stats = _asked(stats, (N, 2), x, "stats")
    p = Logprob(tp, lp, None if entropy is None else entropy.data_ptr(),
                None if stats is None else stats.data_ptr(), vp, ip, T, _int32(K, "K"),
                float(temperature))
    workspace = _own_workspace(workspace, x, stream, logprob_workspace, N, V, K, x.dtype)
    if workspace is None:
        rc = lib().logprob_fwd(x.data_ptr(), ld, ctypes.byref(p), N, V, _DTYPES[x.dtype],
                               _stream(stream))
    else:
        rc = lib().logprob_fwd_ws(x.data_ptr(), ld, ctypes.byref(p), N, V, _DTYPES[x.dtype],
                                  workspace.data_ptr(), workspace.numel(), _stream(stream))
    if rc != OK:
        raise OsmError(rc, "logprob_fwd")
    return Logprobs(logp, entropy, stats, top_vals, top_idx)


def _int32(v, name: str) -> int:
    v = int(v)
    if not -1 << 31 <= v < 1 << 31:  # (a field would take the low 32 bits)
        raise ValueError(f"{name} is out of range")
    return v


def logprob_workspace(N: int, V: int, K: int = 0, dtype=torch.float32) -> int:
    """Bytes of workspace of logprob_fwd for this shape (``osm_logprob_workspace``)."""
    n = ctypes.c_size_t()
    dt = _DTYPES[dtype] if isinstance(dtype, torch.dtype) else int(dtype)
    rc = lib().osm_logprob_workspace(int(N), int(V), _int32(K, "K"), dt, ctypes.byref(n))
    if rc != OK:
        raise OsmError(rc, "osm_logprob_workspace")
    return n.value


def logprob_bwd(x: torch.Tensor, stats: torch.Tensor, tokens: torch.Tensor | None = None,
                dlogp: torch.Tensor | None = None, entropy: torch.Tensor | None = None,
                dentropy: torch.Tensor | None = None, temperature: float = 1.0,
                dx: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """dx = gradient with respect to x of logprob_fwd's logp and entropy, whose own gradients are
    ``dlogp`` (as ``tokens``) and ``dentropy`` (N); either pair may be left out (``logprob_bwd``).
    ``stats`` and ``entropy`` are what logprob_fwd gave for this x and temperature.  dx has
    x's shape; its rows are contiguous, and may be apart if it is given."""
    N, V, ld = _rows(x)
    _on_current_device(x, "x")
    if (tokens is None) != (dlogp is None) or (dentropy is not None and entropy is None):
        raise ValueError("dlogp goes with tokens, and dentropy with entropy")
    T, tp, gp, hp, ep = 0, None, None, None, None
    _vector(stats, torch.float32, x, 2 * N, "stats")
    if tokens is not None:
        T = _tokens(tokens, x, N)
        tp = _vector(tokens, torch.int32, x, N * T, "tokens").data_ptr()
        gp = _vector(dlogp, torch.float32, x, N * T, "dlogp").data_ptr()
    if dentropy is not None:
        hp = _vector(dentropy, torch.float32, x, N, "dentropy").data_ptr()
        ep = _vector(entropy, torch.float32, x, N, "entropy").data_ptr()
    if dx is None:
        dx = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        ldd = V
    else:
        if not isinstance(dx, torch.Tensor) or dx.shape != x.shape or dx.dtype != x.dtype or \
                dx.get_device() != x.get_device():
            raise ValueError("dx must match x in shape, dtype and device")
        ldd = _rows(dx)[2]
    rc = lib().logprob_bwd(x.data_ptr(), ld, tp, stats.data_ptr(), ep, gp, hp, dx.data_ptr(), ldd,
                           N, V, T, _DTYPES[x.dtype], float(temperature), _stream(stream))
    if rc != OK:
        raise OsmError(rc, "logprob_bwd")
    return dx


def _sequences(x: torch.Tensor, idx, starts):
    """(N, E, K, S, pointers of idx and starts) of a packed batch's routing."""
    N, E = _batch(x)
    _on_current_device(x, "x")
    K = _tokens(idx, x, N, "idx")
    _vector(idx, torch.int32, x, N * K, "idx")
    if starts is None:
        return N, E, K, 1, idx.data_ptr(), None
    if not isinstance(starts, torch.Tensor) or starts.dim() != 1 or starts.numel() < 2:
        raise ValueError("starts must have one more element than there are sequences")
    S = starts.numel() - 1
    return N, E, K, S, idx.data_ptr(), _vector(starts, torch.int32, x, S + 1, "starts").data_ptr()


def balance_fwd(x: torch.Tensor, idx: torch.Tensor, starts: torch.Tensor | None = None,
                score="softmax", scale: float = 1.0, loss: torch.Tensor | None = None,
                counts: torch.Tensor | None = None, probs: torch.Tensor | None = None,
                rows: torch.Tensor | None = None, workspace: torch.Tensor | None = None,
                stream=None) -> Balance:
    """The balance loss of each packed sequence of router logits, with the counts of its experts
    and their mean shares (``balance_fwd``): loss S, counts S x E int32, probs S x E and rows S
    int32.

    ``idx``: N x K int32, as route_fwd gave them; a row without any in [0, E) takes no part.
    ``starts``: S + 1 int32, the rows where the sequences begin and where the last one ends
    (None: one sequence, the whole batch).  ``workspace``: uint8, at least
    ``balance_workspace(N, E, S)`` bytes, used instead of the library's scratch
    (``balance_fwd_ws``); under graph capture as in softmax_sample."""
    N, E, K, S, ip, sp = _sequences(x, idx, starts)
    loss = _output(loss, (S,), torch.float32, x, "loss")
    counts = _output(counts, (S, E), torch.int32, x, "counts")
    probs = _output(probs, (S, E), torch.float32, x, "probs")
    rows = _output(rows, (S,), torch.int32, x, "rows")
    workspace = _own_workspace(workspace, x, stream, balance_workspace, N, E, S)
    args = (x.data_ptr(), ip, sp, loss.data_ptr(), counts.data_ptr(), probs.data_ptr(),
            rows.data_ptr(), N, E, K, S, _DTYPES[x.dtype], _int32(_score(score), "score"),
            float(scale))
    if workspace is None:
        rc = lib().balance_fwd(*args, _stream(stream))
    else:
        rc = lib().balance_fwd_ws(*args, workspace.data_ptr(), workspace.numel(),
                                  _stream(stream))
    if rc != OK:
        raise OsmError(rc, "balance_fwd")
    return Balance(loss, counts, probs, rows)


def balance_workspace(N: int, E: int, S: int = 1) -> int:
    """Bytes of workspace of balance_fwd for this shape (``osm_balance_workspace``)."""
    n = ctypes.c_size_t()
    rc = lib().osm_balance_workspace(int(N), int(E), int(S), ctypes.byref(n))
    if rc != OK:
        raise OsmError(rc, "osm_balance_workspace")
    return n.value


def balance_bwd(x: torch.Tensor, idx: torch.Tensor, counts: torch.Tensor, rows: torch.Tensor,
                dloss: torch.Tensor, starts: torch.Tensor | None = None, score="softmax",
                scale: float = 1.0, dx: torch.Tensor | None = None, stream=None) -> torch.Tensor:
    """dx = gradient with respect to x of balance_fwd's losses, whose own gradient is ``dloss``
    (S); ``counts`` and ``rows`` are what it gave, or their sums over the ranks that share the
    loss (``balance_bwd``)."""
    N, E, K, S, ip, sp = _sequences(x, idx, starts)
    _vector(counts, torch.int32, x, S * E, "counts")
    _vector(rows, torch.int32, x, S, "rows")
    _vector(dloss, torch.float32, x, S, "dloss")
    if dx is None:
        dx = torch.empty_like(x)
    elif not _like(dx, x):
        raise ValueError("dx must be a contiguous tensor like x")
    rc = lib().balance_bwd(x.data_ptr(), ip, sp, counts.data_ptr(), rows.data_ptr(),
                           dloss.data_ptr(), dx.data_ptr(), N, E, K, S, _DTYPES[x.dtype],
                           _int32(_score(score), "score"), float(scale),
                           _stream(stream))
    if rc != OK:
        raise OsmError(rc, "balance_bwd")
    return dx
