"""Python binding of libga.so: argument marshalling only.

Every function takes torch CUDA tensors, allocates outputs (and a cached
workspace) with torch, and calls the C ABI declared in include/ga.h on the
current torch stream.  All computation happens in the HIP kernels; there is no
CPU fallback: if the library is missing the call raises.
"""
from __future__ import annotations

import ctypes
import functools
import math
import os

import torch

# GA_LIB lets the sanitizer test load an instrumented build of the same sources.
_LIB_PATH = os.environ.get("GA_LIB") or os.path.join(os.path.dirname(os.path.abspath(__file__)), "libga.so")

GA_F32, GA_BF16 = 0, 1
STATUS = {0: "GA_OK", 1: "GA_ERR_INVALID_ARG", 2: "GA_ERR_UNSUPPORTED", 3: "GA_ERR_WORKSPACE", 4: "GA_ERR_HIP"}
SYMBOLS = ("ga_workspace_bytes", "ga_cluster", "ga_aggregate", "ga_attend", "ga_forward",
           "ga_block_workspace_bytes", "ga_project_qkv", "ga_project_out", "ga_attention_block",
           "ga_merge_plan", "ga_next_group_count", "ga_backward_workspace_bytes", "ga_backward",
           "ga_timing_enable", "ga_timing_collect", "ga_status_string", "ga_last_error", "ga_workspace_check",
           "ga_forward_noalloc",
           "ga_linear_workspace_bytes", "ga_linear_attend", "ga_linear_backward_workspace_bytes",
           "ga_linear_backward", "ga_linear_step", "ga_rotary", "ga_norm_residual",
           "ga_norm_backward_workspace_bytes", "ga_norm_residual_backward")


class Shape(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("H", ctypes.c_int32), ("n", ctypes.c_int32),
                ("d", ctypes.c_int32), ("dtype", ctypes.c_int32)]


class Norm(ctypes.Structure):
    _fields_ = [("B", ctypes.c_int32), ("n", ctypes.c_int32), ("D", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("kind", ctypes.c_int32), ("gate_batches", ctypes.c_int32), ("eps", ctypes.c_float),
                ("residual_scale", ctypes.c_float), ("branch_scale", ctypes.c_float)]


class KernelTime(ctypes.Structure):
    _fields_ = [("name", ctypes.c_char * 32), ("launches", ctypes.c_int32), ("total_ms", ctypes.c_double)]


class GAError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS.get(status, status)}: {message}")
        self.status = status


_lib = None


def lib() -> ctypes.CDLL:
    """The loaded libga.so (raises if it has not been built)."""
    global _lib
    if _lib is None:
        if not os.path.exists(_LIB_PATH):
            raise RuntimeError(f"{_LIB_PATH} is missing: build it with __graft_entry__.build()")
        L = ctypes.CDLL(_LIB_PATH)
        P, i32 = ctypes.c_void_p, ctypes.c_int32
        L.ga_workspace_bytes.argtypes = [Shape, i32]
        L.ga_workspace_bytes.restype = ctypes.c_size_t
        L.ga_cluster.argtypes = [Shape, P, i32, i32, P, P, P, P, P, ctypes.c_size_t, P]
        L.ga_aggregate.argtypes = [Shape, P, P, i32, P, P, ctypes.c_size_t, P]
        L.ga_attend.argtypes = [Shape, P, P, P, P, i32, ctypes.c_float, P, P, ctypes.c_size_t, P]
        L.ga_forward.argtypes = [Shape, P, P, P, i32, i32, ctypes.c_float, P, P, P, P, P, ctypes.c_size_t, P]
        L.ga_forward_noalloc.argtypes = [Shape, P, P, P, i32, i32, ctypes.c_float, P, P, P, P, P]
        L.ga_block_workspace_bytes.argtypes = [Shape, i32]
        L.ga_block_workspace_bytes.restype = ctypes.c_size_t
        L.ga_project_qkv.argtypes = [Shape, P, P, P, P, P, P]
        L.ga_project_out.argtypes = [Shape, P, P, P, P]
        L.ga_attention_block.argtypes = [Shape, P, P, P, i32, i32, ctypes.c_float, P, P, ctypes.c_size_t, P]
        L.ga_merge_plan.argtypes = [Shape, P, P, P, P, P, i32, ctypes.c_float, ctypes.c_double, P, P, P, P, P]
        L.ga_backward_workspace_bytes.argtypes = [Shape, i32]
        L.ga_backward_workspace_bytes.restype = ctypes.c_size_t
        L.ga_backward.argtypes = [Shape, P, P, P, P, P, P, i32, ctypes.c_float, P, P, P, P, ctypes.c_size_t, P]
        L.ga_next_group_count.argtypes = [i32, P, ctypes.c_int64, ctypes.c_double]
        L.ga_next_group_count.restype = i32
        for f in ("ga_cluster", "ga_aggregate", "ga_attend", "ga_forward", "ga_forward_noalloc", "ga_project_qkv",
                  "ga_project_out",
                  "ga_attention_block", "ga_merge_plan", "ga_backward"):
            getattr(L, f).restype = ctypes.c_int
        f32, size = ctypes.c_float, ctypes.c_size_t
        L.ga_linear_workspace_bytes.argtypes = [Shape, i32]
        L.ga_linear_workspace_bytes.restype = size
        L.ga_linear_attend.argtypes = [Shape, i32, P, P, P, P, P, P, f32, P, P, P, size, P]
        L.ga_linear_backward_workspace_bytes.argtypes = [Shape, i32]
        L.ga_linear_backward_workspace_bytes.restype = size
        L.ga_linear_backward.argtypes = [Shape, i32, P, P, P, P, P, P, P, P, f32, P, P, P, P, P, size, P]
        L.ga_linear_step.argtypes = [Shape, i32, P, P, P, P, P, i32, P, f32, P, P, P]
        L.ga_rotary.argtypes = [Shape, i32, P, P, P, i32, i32, P, ctypes.c_double, i32, P, P, P]
        L.ga_norm_residual.argtypes = [Norm, P, P, P, P, P, P, P, P, P, P]
        L.ga_norm_backward_workspace_bytes.argtypes = [Norm]
        L.ga_norm_backward_workspace_bytes.restype = size
        L.ga_norm_residual_backward.argtypes = [Norm] + [P] * 17 + [size, P]
        for f in ("ga_linear_attend", "ga_linear_backward", "ga_linear_step", "ga_rotary", "ga_norm_residual",
                  "ga_norm_residual_backward"):
            getattr(L, f).restype = ctypes.c_int
        L.ga_workspace_check.argtypes = [Shape, i32, P, ctypes.c_size_t, P]
        L.ga_workspace_check.restype = ctypes.c_int
        L.ga_timing_enable.argtypes = [ctypes.c_int]
        L.ga_timing_enable.restype = ctypes.c_int
        L.ga_timing_collect.argtypes = [ctypes.POINTER(KernelTime), i32, ctypes.POINTER(i32)]
        L.ga_timing_collect.restype = ctypes.c_int
        L.ga_status_string.argtypes = [ctypes.c_int]
        L.ga_status_string.restype = ctypes.c_char_p
        L.ga_last_error.argtypes = []
        L.ga_last_error.restype = ctypes.c_char_p
        _lib = L
    return _lib


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return GA_BF16
    if t.dtype == torch.float32:
        return GA_F32
    raise TypeError(f"unsupported dtype {t.dtype} (bf16 or fp32)")


def shape_of(X: torch.Tensor) -> Shape:
    if X.dim() != 4:
        raise ValueError("expected a [B, H, n, d] tensor")
    B, H, n, d = X.shape
    return Shape(B, H, n, d, _dtype_code(X))


def _p(t):
    if t is None:
        return None
    if not t.is_contiguous():
        raise ValueError("tensors must be contiguous")
    return ctypes.c_void_p(t.data_ptr())


def _expect(t, name: str, device, dtype, shape=None, optional: bool = False):
    """Check a tensor handed to the C ABI, which cannot check buffer sizes:
    it must live on `device` (a CUDA device), have `dtype`, be contiguous and
    (if given) have exactly `shape`.  Raises ValueError otherwise, before any
    pointer reaches a kernel."""
    if t is None:
        if optional:
            return
        raise ValueError(f"{name} is required")
    if not isinstance(t, torch.Tensor):
        raise ValueError(f"{name} must be a torch tensor")
    if t.device.type != "cuda" or t.device != device:
        raise ValueError(f"{name} is on {t.device}, expected {device}")
    if t.dtype != dtype:
        raise ValueError(f"{name} has dtype {t.dtype}, expected {dtype}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {tuple(shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _device_of(X: torch.Tensor):
    if X.device.type != "cuda":
        raise ValueError(f"tensors must be on a CUDA device (got {X.device})")
    return X.device


def _qkv_like(X: torch.Tensor, name: str):
    """Shape [B, H, n, d] and the device of the first operand of a call."""
    if not isinstance(X, torch.Tensor) or X.dim() != 4:
        raise ValueError(f"{name} must be a [B, H, n, d] tensor")
    return _device_of(X)


def _check(rc: int):
    if rc != 0:
        raise GAError(rc, lib().ga_last_error().decode())


# torch's handle of the current stream without a Stream object (3 us less per
# lookup, and every call needs one or two: the smallest calls are bound by the
# host); a torch without it takes the public way.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_device = getattr(torch._C, "_cuda_getDevice", torch.cuda.current_device)  # (the tensors are there already)


def _stream_handle(device) -> int:
    if _raw_stream is None or device.index is None:
        return torch.cuda.current_stream(device).cuda_stream
    return _raw_stream(device.index)


def _stream(device) -> ctypes.c_void_p:
    return ctypes.c_void_p(_stream_handle(device))


_ws_cache: dict = {}


def workspace_bytes(shape: Shape, N: int) -> int:
    return int(lib().ga_workspace_bytes(shape, int(N)))


def workspace(shape: Shape, N: int, device, stream=None) -> tuple:
    """A cached device workspace (uint8 tensor) large enough for (shape, N).

    One buffer per (device, stream): the workspace carries state between the
    launches of one call, and calls on one stream run one after another, so
    calls without ws on different streams never share a buffer.  The buffer
    is allocated on (and its memory ordered by) that stream.
    """
    if not isinstance(device, torch.device):
        device = torch.device(device)
    nbytes = max(workspace_bytes(shape, N), 256)
    key = (device, _stream_handle(device) if stream is None else stream.cuda_stream)
    ws = _ws_cache.get(key)
    if ws is None or ws.numel() < nbytes:
        with torch.cuda.stream(torch.cuda.current_stream(device) if stream is None else stream):
            ws = torch.empty(nbytes, dtype=torch.uint8, device=device)
        _ws_cache[key] = ws
    return ws, ws.numel()


def _ws_args(shape, N, device, ws):
    if ws is None:
        ws, nb = workspace(shape, N, device)
    else:
        _expect(ws, "ws", device, torch.uint8)
        nb = ws.numel() * ws.element_size()
    return _p(ws), nb


def cluster(K: torch.Tensor, N: int, iters: int, init: torch.Tensor | None = None, ws=None):
    """Grouping of the keys: returns (belong [B,H,n] int32, count [B,H,N] int32,
    centroid [B,H,N,d] fp32)."""
    dev = _qkv_like(K, "K")
    s = shape_of(K)
    B, H, n, d = K.shape
    _expect(init, "init", dev, torch.float32, (B, H, N, d), optional=True)
    belong = torch.empty(K.shape[:3], dtype=torch.int32, device=dev)
    count = torch.empty((*K.shape[:2], N), dtype=torch.int32, device=dev)
    centroid = torch.empty((*K.shape[:2], N, K.shape[3]), dtype=torch.float32, device=dev)
    wp, nb = _ws_args(s, N, dev, ws)
    _check(lib().ga_cluster(s, _p(K), int(N), int(iters), _p(init), _p(belong), _p(count), _p(centroid),
                            wp, nb, _stream(dev)))
    return belong, count, centroid


def aggregate(V: torch.Tensor, belong: torch.Tensor, N: int, ws=None) -> torch.Tensor:
    """Per-group fp32 sums of the values (fp64 accumulation)."""
    dev = _qkv_like(V, "V")
    s = shape_of(V)
    _expect(belong, "belong", dev, torch.int32, V.shape[:3])
    vsum = torch.empty((*V.shape[:2], N, V.shape[3]), dtype=torch.float32, device=dev)
    wp, nb = _ws_args(s, N, dev, ws)
    _check(lib().ga_aggregate(s, _p(V), _p(belong), int(N), _p(vsum), wp, nb, _stream(dev)))
    return vsum


def attend(Q: torch.Tensor, centroid: torch.Tensor, count: torch.Tensor, vsum: torch.Tensor, N: int,
           scale: float | None = None, ws=None) -> torch.Tensor:
    """Group softmax and combine; returns O [B,H,n,d] in Q's dtype."""
    dev = _qkv_like(Q, "Q")
    s = shape_of(Q)
    B, H, n, d = Q.shape
    _expect(centroid, "centroid", dev, torch.float32, (B, H, N, d))
    _expect(count, "count", dev, torch.int32, (B, H, N))
    _expect(vsum, "vsum", dev, torch.float32, (B, H, N, d))
    scale = 1.0 / math.sqrt(Q.shape[3]) if scale is None else float(scale)
    O = torch.empty_like(Q)
    wp, nb = _ws_args(s, N, dev, ws)
    _check(lib().ga_attend(s, _p(Q), _p(centroid), _p(count), _p(vsum), int(N), scale, _p(O), wp, nb,
                           _stream(dev)))
    return O


def forward(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, N: int, iters: int,
            scale: float | None = None, return_groups: bool = False, out: torch.Tensor | None = None,
            ws=None):
    """Whole group-attention forward; optionally also (belong, count, centroid)."""
    dev = _qkv_like(Q, "Q")
    s = shape_of(Q)
    for t, nm in ((K, "K"), (V, "V"), (out, "out")):
        _expect(t, nm, dev, Q.dtype, Q.shape, optional=nm == "out")
    scale = 1.0 / math.sqrt(Q.shape[3]) if scale is None else float(scale)
    O = torch.empty_like(Q) if out is None else out
    belong = count = centroid = None
    if return_groups:
        belong = torch.empty(K.shape[:3], dtype=torch.int32, device=dev)
        count = torch.empty((*K.shape[:2], N), dtype=torch.int32, device=dev)
        centroid = torch.empty((*K.shape[:2], N, K.shape[3]), dtype=torch.float32, device=dev)
    wp, nb = _ws_args(s, N, dev, ws)
    _check(lib().ga_forward(s, _p(Q), _p(K), _p(V), int(N), int(iters), scale, _p(O), _p(belong), _p(count),
                            _p(centroid), wp, nb, _stream(dev)))
    return (O, belong, count, centroid) if return_groups else O


def forward_noalloc(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, N: int, iters: int,
                    scale: float | None = None, return_groups: bool = False, out: torch.Tensor | None = None):
    """forward() through ga_forward_noalloc: no workspace, the library's static
    scratch instead (bf16, shapes of the one-launch grouping only).  Calls that
    overlap in time on one GPU share that scratch and race."""
    dev = _qkv_like(Q, "Q")
    s = shape_of(Q)
    for t, nm in ((K, "K"), (V, "V"), (out, "out")):
        _expect(t, nm, dev, Q.dtype, Q.shape, optional=nm == "out")
    scale = 1.0 / math.sqrt(Q.shape[3]) if scale is None else float(scale)
    O = torch.empty_like(Q) if out is None else out
    belong = count = centroid = None
    if return_groups:
        belong = torch.empty(K.shape[:3], dtype=torch.int32, device=dev)
        count = torch.empty((*K.shape[:2], N), dtype=torch.int32, device=dev)
        centroid = torch.empty((*K.shape[:2], N, K.shape[3]), dtype=torch.float32, device=dev)
    _check(lib().ga_forward_noalloc(s, _p(Q), _p(K), _p(V), int(N), int(iters), scale, _p(O), _p(belong),
                                    _p(count), _p(centroid), _stream(dev)))
    return (O, belong, count, centroid) if return_groups else O


def block_shape(X: torch.Tensor, H: int) -> Shape:
    """Shape of the attention block for token embeddings X [B, n, 64 H]."""
    if X.dim() != 3 or X.shape[2] != 64 * H:
        raise ValueError(f"expected X of shape [B, n, {64 * H}]")
    return Shape(X.shape[0], H, X.shape[1], 64, _dtype_code(X))


def project_qkv(X: torch.Tensor, Wqkv: torch.Tensor, H: int):
    """(Q, K, V) [B, H, n, 64] = per-head slices of X Wqkv^T (Wqkv [3D, D], rows = outputs)."""
    s = block_shape(X, H)
    dev = _device_of(X)
    B, n, D = X.shape
    _expect(Wqkv, "Wqkv", dev, X.dtype, (3 * D, D))
    Q, K, V = (torch.empty((B, H, n, 64), dtype=X.dtype, device=X.device) for _ in range(3))
    _check(lib().ga_project_qkv(s, _p(X), _p(Wqkv), _p(Q), _p(K), _p(V), _stream(X.device)))
    return Q, K, V


def project_out(O: torch.Tensor, Wo: torch.Tensor) -> torch.Tensor:
    """Y [B, n, D] = heads of O [B, H, n, 64] concatenated, times Wo^T (Wo [D, D])."""
    dev = _qkv_like(O, "O")
    B, H, n, d = O.shape
    _expect(Wo, "Wo", dev, O.dtype, (H * d, H * d))
    Y = torch.empty((B, n, H * d), dtype=O.dtype, device=O.device)
    _check(lib().ga_project_out(Shape(B, H, n, d, _dtype_code(O)), _p(O), _p(Wo), _p(Y), _stream(O.device)))
    return Y


def block_workspace_bytes(shape: Shape, N: int) -> int:
    return int(lib().ga_block_workspace_bytes(shape, int(N)))


def attention_block(X: torch.Tensor, Wqkv: torch.Tensor, Wo: torch.Tensor, H: int, N: int, iters: int,
                    scale: float | None = None, out: torch.Tensor | None = None, ws=None) -> torch.Tensor:
    """Attention block: projections, group-attention forward, output projection.
    ws: a uint8 device tensor of block_workspace_bytes(shape, N) (allocated if None)."""
    s = block_shape(X, H)
    dev = _device_of(X)
    D = X.shape[2]
    _expect(Wqkv, "Wqkv", dev, X.dtype, (3 * D, D))
    _expect(Wo, "Wo", dev, X.dtype, (D, D))
    _expect(out, "out", dev, X.dtype, X.shape, optional=True)
    scale = 1.0 / 8.0 if scale is None else float(scale)
    Y = torch.empty_like(X) if out is None else out
    if ws is None:
        ws = torch.empty(max(block_workspace_bytes(s, N), 256), dtype=torch.uint8, device=X.device)
    _expect(ws, "ws", dev, torch.uint8)
    _check(lib().ga_attention_block(s, _p(X), _p(Wqkv), _p(Wo), int(N), int(iters), scale, _p(Y), _p(ws),
                                    ws.numel(), _stream(dev)))
    return Y


def merge_plan(Q: torch.Tensor, K: torch.Tensor, belong: torch.Tensor, centroid: torch.Tensor,
               count: torch.Tensor, N: int, scale: float | None = None, eps: float = 2.0) -> dict:
    """Merge plan of the adaptive group count (Lemma 1 threshold, Eq. 5 rule):
    dict(radius [B,H,N] fp64, dthr [B,H] fp64, partner [B,H,N] int32, merges [B,H] int32)."""
    dev = _qkv_like(K, "K")
    s = shape_of(K)
    B, H, n, d = K.shape
    _expect(Q, "Q", dev, K.dtype, K.shape)
    _expect(belong, "belong", dev, torch.int32, (B, H, n))
    _expect(centroid, "centroid", dev, torch.float32, (B, H, N, d))
    _expect(count, "count", dev, torch.int32, (B, H, N))
    scale = 1.0 / math.sqrt(K.shape[3]) if scale is None else float(scale)
    radius = torch.empty((B, H, N), dtype=torch.float64, device=dev)
    dthr = torch.empty((B, H), dtype=torch.float64, device=dev)
    partner = torch.empty((B, H, N), dtype=torch.int32, device=dev)
    merges = torch.empty((B, H), dtype=torch.int32, device=dev)
    _check(lib().ga_merge_plan(s, _p(Q), _p(K), _p(belong), _p(centroid), _p(count), int(N), scale, float(eps),
                               _p(radius), _p(dthr), _p(partner), _p(merges), _stream(dev)))
    return dict(radius=radius, dthr=dthr, partner=partner, merges=merges)


def next_group_count(N: int, merges, alpha: float) -> int:
    """Momentum update of N from per-slice merge counts (copied to the host)."""
    m = torch.as_tensor(merges).to("cpu", torch.int32).contiguous().reshape(-1)
    r = lib().ga_next_group_count(int(N), ctypes.c_void_p(m.data_ptr()) if m.numel() else None, m.numel(),
                                  float(alpha))
    if r == 0:
        raise GAError(1, lib().ga_last_error().decode())
    return int(r)


def backward_workspace_bytes(shape: Shape, N: int) -> int:
    return int(lib().ga_backward_workspace_bytes(shape, int(N)))


def backward(Q: torch.Tensor, dO: torch.Tensor, belong: torch.Tensor, centroid: torch.Tensor, count: torch.Tensor,
             vsum: torch.Tensor, N: int, scale: float | None = None, ws=None):
    """Gradient of the forward with the grouping fixed: (dQ, dK, dV) [B,H,n,d] bf16."""
    dev = _qkv_like(Q, "Q")
    s = shape_of(Q)
    B, H, n, d = Q.shape
    _expect(dO, "dO", dev, Q.dtype, Q.shape)
    _expect(belong, "belong", dev, torch.int32, (B, H, n))
    _expect(centroid, "centroid", dev, torch.float32, (B, H, N, d))
    _expect(count, "count", dev, torch.int32, (B, H, N))
    _expect(vsum, "vsum", dev, torch.float32, (B, H, N, d))
    scale = 1.0 / math.sqrt(Q.shape[3]) if scale is None else float(scale)
    dQ, dK, dV = (torch.empty_like(Q) for _ in range(3))
    if ws is None:
        ws = torch.empty(max(backward_workspace_bytes(s, N), 256), dtype=torch.uint8, device=dev)
    _expect(ws, "ws", dev, torch.uint8)
    _check(lib().ga_backward(s, _p(Q), _p(dO), _p(belong), _p(centroid), _p(count), _p(vsum), int(N), scale, _p(dQ),
                             _p(dK), _p(dV), _p(ws), ws.numel(), _stream(dev)))
    return dQ, dK, dV


def _launch(dev, call, *args) -> None:
    """One entry point on the current stream of `dev`, with that device current."""
    if dev.index == _current_device() or dev.index is None:
        rc = call(*args, _stream_handle(dev))
    else:
        with torch.cuda.device(dev):
            rc = call(*args, _stream_handle(dev))
    if rc:
        _check(rc)


def _at(t, name: str, dev, dtype, shape):
    """Address of a tensor that _expect accepts (which says what is wrong with another one).  The smallest calls are
    bound by the host: each check is made once, in one expression."""
    if not (isinstance(t, torch.Tensor) and t.dtype is dtype and t.device == dev and t.shape == shape
            and t.is_contiguous()):
        _expect(t, name, dev, dtype, shape)
    return t.data_ptr()


def _maybe(t, name: str, dev, dtype, shape):
    """_at, or NULL for None."""
    return None if t is None else _at(t, name, dev, dtype, shape)


def _scratch(nbytes: int, dev, ws):
    """(tensor, address, bytes) of a workspace: the caller's, or one of this call's own (so that captured graphs and
    streams never share one).  The tensor is to live until the launch is enqueued."""
    if ws is None:
        if nbytes == 0:
            return None, None, 0
        ws = torch.empty(nbytes, dtype=torch.uint8, device=dev)
    else:
        _expect(ws, "ws", dev, torch.uint8)
    return ws, ws.data_ptr(), ws.numel()


@functools.lru_cache(maxsize=1024)
def _linear_shape(B: int, H: int, Hk: int, n: int, d: int, dtype):
    """(shape, forward workspace, backward workspace, default scale) of a call, which depend on nothing else."""
    if dtype not in (torch.bfloat16, torch.float32):
        raise TypeError(f"unsupported dtype {dtype} (bf16 or fp32)")
    s = Shape(B, H, n, d, GA_BF16 if dtype is torch.bfloat16 else GA_F32)
    return (s, int(lib().ga_linear_workspace_bytes(s, Hk)), int(lib().ga_linear_backward_workspace_bytes(s, Hk)),
            1.0 / math.sqrt(max(d, 1)))


def _heads(Q, K, name: str):
    """(B, H, Hk, n, d, device, dtype) of queries [B,H,n,d] and keys [B,Hk,n,d]."""
    if not isinstance(Q, torch.Tensor) or not isinstance(K, torch.Tensor) or len(qs := Q.shape) != 4 or \
            len(ks := K.shape) != 4:
        raise ValueError(f"Q must be a [B, H, n, d] and {name} a [B, Hk, n, d] tensor")
    dev = Q.device
    if dev.type != "cuda":
        _device_of(Q)
    B, H, n, d = qs
    return B, H, ks[1], n, d, dev, Q.dtype


def linear_workspace_bytes(shape: Shape, Hk: int) -> int:
    return int(lib().ga_linear_workspace_bytes(shape, int(Hk)))


def linear_attend(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, log_decay: torch.Tensor,
                  scale: float | None = None, lengths: torch.Tensor | None = None, state: torch.Tensor | None = None,
                  return_state: bool = False, out: torch.Tensor | None = None, out_state: torch.Tensor | None = None,
                  ws=None):
    """Causal linear attention with a decay per head: O [B,H,n,64], or (O, state [B,H,64,64] fp32) if return_state.
    K, V [B,Hk,n,64]; log_decay [H] fp32; lengths [B] int32; state: the state before the first token (out_state may
    be that tensor itself)."""
    B, H, Hk, n, d, dev, dt = _heads(Q, K, "K")
    q, kv, states = (B, H, n, d), (B, Hk, n, d), (B, H, d, d)
    pointers = (_at(Q, "Q", dev, dt, q), _at(K, "K", dev, dt, kv), _at(V, "V", dev, dt, kv),
                _at(log_decay, "log_decay", dev, torch.float32, (H,)),
                _maybe(lengths, "lengths", dev, torch.int32, (B,)),
                _maybe(state, "state", dev, torch.float32, states))
    O = torch.empty_like(Q) if out is None else out
    if return_state and out_state is None:
        out_state = torch.empty(states, dtype=torch.float32, device=dev)
    s, nbytes, _, usual = _linear_shape(B, H, Hk, n, d, dt)
    ws, wp, nb = _scratch(nbytes, dev, ws)
    _launch(dev, lib().ga_linear_attend, s, Hk, *pointers, usual if scale is None else float(scale),
            O.data_ptr() if out is None else _at(O, "out", dev, dt, q),
            _maybe(out_state, "out_state", dev, torch.float32, states), wp, nb)
    return (O, out_state) if return_state else O


def linear_backward_workspace_bytes(shape: Shape, Hk: int) -> int:
    return int(lib().ga_linear_backward_workspace_bytes(shape, int(Hk)))


def linear_backward(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, dO: torch.Tensor, log_decay: torch.Tensor,
                    scale: float | None = None, lengths: torch.Tensor | None = None,
                    state: torch.Tensor | None = None, dstate: torch.Tensor | None = None,
                    return_dstate: bool = False, ws=None):
    """Gradient of linear_attend: (dQ, dK, dV), and the initial state's gradient if return_dstate.  dstate: the
    gradient that reaches the final state."""
    B, H, Hk, n, d, dev, dt = _heads(Q, K, "K")
    q, kv, states = (B, H, n, d), (B, Hk, n, d), (B, H, d, d)
    pointers = (_at(Q, "Q", dev, dt, q), _at(K, "K", dev, dt, kv), _at(V, "V", dev, dt, kv), _at(dO, "dO", dev, dt, q),
                _at(log_decay, "log_decay", dev, torch.float32, (H,)),
                _maybe(lengths, "lengths", dev, torch.int32, (B,)),
                _maybe(state, "state", dev, torch.float32, states),
                _maybe(dstate, "dstate", dev, torch.float32, states))
    dQ, dK, dV = torch.empty_like(Q), torch.empty_like(K), torch.empty_like(V)
    out = torch.empty(states, dtype=torch.float32, device=dev) if return_dstate else None
    s, _, nbytes, usual = _linear_shape(B, H, Hk, n, d, dt)
    ws, wp, nb = _scratch(nbytes, dev, ws)
    _launch(dev, lib().ga_linear_backward, s, Hk, *pointers, usual if scale is None else float(scale),
            dQ.data_ptr(), dK.data_ptr(), dV.data_ptr(), None if out is None else out.data_ptr(), wp, nb)
    return (dQ, dK, dV, out) if return_dstate else (dQ, dK, dV)


def linear_step(Q: torch.Tensor, K: torch.Tensor, V: torch.Tensor, log_decay: torch.Tensor, state: torch.Tensor,
                scale: float | None = None, slots: torch.Tensor | None = None, out: torch.Tensor | None = None,
                out_state: torch.Tensor | None = None):
    """One token per sequence (Q [B,H,1,64]) on kept states [states,H,64,64] fp32, updated in place unless out_state
    is given: (O, the updated states).  slots [B] int32: the state of each batch row (outside the states: padding)."""
    B, H, Hk, n, d, dev, dt = _heads(Q, K, "K")
    if not isinstance(state, torch.Tensor) or len(state.shape) != 4:
        raise ValueError("state must be a [states, H, 64, 64] tensor")
    many = state.shape[0]
    q, kv, states = (B, H, n, d), (B, Hk, n, d), (many, H, d, d)
    s, _, _, usual = _linear_shape(B, H, Hk, n, d, dt)
    O = torch.empty_like(Q) if out is None else out
    at = _at(state, "state", dev, torch.float32, states)
    if out_state is None:
        out_state = state
    _launch(dev, lib().ga_linear_step, s, Hk, _at(Q, "Q", dev, dt, q), _at(K, "K", dev, dt, kv),
            _at(V, "V", dev, dt, kv), _at(log_decay, "log_decay", dev, torch.float32, (H,)),
            _maybe(slots, "slots", dev, torch.int32, (B,)), many, at, usual if scale is None else float(scale),
            O.data_ptr() if out is None else _at(O, "out", dev, dt, q),
            at if out_state is state else _at(out_state, "out_state", dev, torch.float32, states))
    return O, out_state


ROTARY_INTERLEAVED, ROTARY_SHARED, ROTARY_INVERSE, ROTARY_FLOAT_POS = 1, 2, 4, 8


@functools.lru_cache(maxsize=64)
def _pairs(pairs: tuple):
    return (ctypes.c_int32 * max(1, len(pairs)))(*pairs)


def rotary(Q: torch.Tensor, K: torch.Tensor | None, pos: torch.Tensor, pairs, base: float = 10000.0,
           interleaved: bool = False, shared: bool = False, inverse: bool = False, out=None):
    """Rotary positions with several axes: (Q', K') for Q [B,H,n,64], K [B,Hk,n,64] (Q' alone if K is None).
    pos [axes, B or 1, n] int32 or fp32; pairs: the feature pairs of each axis; shared: one ladder of frequencies over
    all pairs instead of one per axis; inverse: the opposite turn, which is the gradient.  out: (Q', K') to write,
    which may be Q and K themselves."""
    B, H, Hk, n, d, dev, dt = _heads(Q, Q if K is None else K, "K")
    pairs = tuple(int(p) for p in pairs)
    if not isinstance(pos, torch.Tensor) or pos.dim() != 3 or pos.shape[1] not in (1, B):
        raise ValueError(f"pos must be an [axes, 1 or {B}, n] tensor")
    floats = pos.dtype is torch.float32
    if not floats and pos.dtype is not torch.int32:
        raise ValueError(f"pos has dtype {pos.dtype}, expected int32 or float32")
    q, k, many = (B, H, n, d), (B, Hk, n, d), pos.shape[1]
    Qo, Ko = (torch.empty_like(Q), None if K is None else torch.empty_like(K)) if out is None else out
    flags = (ROTARY_INTERLEAVED * bool(interleaved) + ROTARY_SHARED * bool(shared) + ROTARY_INVERSE * bool(inverse)
             + ROTARY_FLOAT_POS * floats)
    _launch(dev, lib().ga_rotary, _linear_shape(B, H, Hk, n, d, dt)[0], Hk, _at(Q, "Q", dev, dt, q),
            None if K is None else _at(K, "K", dev, dt, k), _at(pos, "pos", dev, pos.dtype, (len(pairs), many, n)),
            many, len(pairs), _pairs(pairs), float(base), flags, _at(Qo, "out[0]", dev, dt, q),
            None if K is None else _at(Ko, "out[1]", dev, dt, k))
    return Qo if K is None else (Qo, Ko)


NORMS = {"rms": 0, "layer": 1}


_norm_shape = functools.lru_cache(maxsize=1024)(Norm)  # (0.7 us less than a new one)


def _norm_args(X, F, norm, eps, post_weight, post_bias, gate, pre_weight, pre_bias, residual_scale, branch_scale):
    """Checks shared by the norm's calls; (ga_norm_t, device, dtype, the tensors' addresses)."""
    if not isinstance(X, torch.Tensor) or X.dim() != 3:
        raise ValueError("X must be a [B, n, D] tensor")
    if norm not in NORMS:
        raise ValueError(f"norm must be one of {sorted(NORMS)} (got {norm!r})")
    dev, dt, code = _device_of(X), X.dtype, _dtype_code(X)
    B, n, D = X.shape
    batches, g = 0, None
    if gate is not None:
        if not isinstance(gate, torch.Tensor) or gate.dim() not in (1, 2):
            raise ValueError("gate must be a [D] or [B, D] tensor")
        batches = 1 if gate.dim() == 1 else B
        g = _at(gate, "gate", dev, dt, (D,) if gate.dim() == 1 else (B, D))
    # (+ 0.0: of two equal zeros one is kept)
    s = _norm_shape(B, n, D, code, NORMS[norm], batches, eps, residual_scale + 0.0, branch_scale + 0.0)
    w = (D,)
    return s, dev, dt, (_at(X, "X", dev, dt, (B, n, D)), _maybe(F, "F", dev, dt, (B, n, D)),
                        _maybe(post_weight, "post_weight", dev, dt, w), _maybe(post_bias, "post_bias", dev, dt, w), g,
                        _maybe(pre_weight, "pre_weight", dev, dt, w), _maybe(pre_bias, "pre_bias", dev, dt, w))


def norm_residual(X: torch.Tensor, F: torch.Tensor | None = None, norm: str = "rms", eps: float = 1e-6,
                  post_weight=None, post_bias=None, gate=None, pre_weight=None, pre_bias=None,
                  residual_scale: float = 1.0, branch_scale: float = 1.0, return_sum: bool = True):
    """Y = residual_scale X + branch_scale gate * post_norm(F) and, with pre_weight, H = pre_norm(Y): returns Y,
    (Y, H), or H alone without return_sum.  X, F [B,n,D]; weights and biases [D]; gate [D] or [B,D]; norm "rms" or
    "layer"; no post_weight: F itself; no F: the residual stream alone."""
    s, dev, _, tensors = _norm_args(X, F, norm, eps, post_weight, post_bias, gate, pre_weight, pre_bias,
                                    residual_scale, branch_scale)
    Y = torch.empty_like(X) if return_sum else None
    H = torch.empty_like(X) if pre_weight is not None else None
    _launch(dev, lib().ga_norm_residual, s, *tensors, None if Y is None else Y.data_ptr(),
            None if H is None else H.data_ptr())
    return H if Y is None else Y if H is None else (Y, H)


def norm_backward_workspace_bytes(s: Norm) -> int:
    return int(lib().ga_norm_backward_workspace_bytes(s))


def norm_residual_backward(X: torch.Tensor, F: torch.Tensor | None, dY: torch.Tensor | None,
                           dH: torch.Tensor | None = None, norm: str = "rms", eps: float = 1e-6, post_weight=None,
                           post_bias=None, gate=None, pre_weight=None, pre_bias=None, residual_scale: float = 1.0,
                           branch_scale: float = 1.0, ws=None) -> dict:
    """Gradient of norm_residual from those of Y and H (each may be None): a dict of dX, dF (X's dtype) and, for what
    the call has, dpost_w, dpost_b, dgate, dpre_w, dpre_b (fp32 sums over the tokens)."""
    s, dev, dt, tensors = _norm_args(X, F, norm, eps, post_weight, post_bias, gate, pre_weight, pre_bias,
                                     residual_scale, branch_scale)
    dYp, dHp = (_maybe(t, name, dev, dt, X.shape) for t, name in ((dY, "dY"), (dH, "dH")))
    B, _, D = X.shape
    empty = torch.empty if B else torch.zeros  # no tokens: nothing is enqueued, every sum is zero

    def sums(wanted, *shape):
        return empty(shape, dtype=torch.float32, device=dev) if wanted else None

    got = dict(dX=torch.empty_like(X), dF=None if F is None else torch.empty_like(F),
               dpost_w=sums(post_weight is not None, D), dpost_b=sums(post_bias is not None, D),
               dgate=None if gate is None else sums(True, *gate.shape),
               dpre_w=sums(dH is not None, D), dpre_b=sums(dH is not None and pre_bias is not None, D))
    ws, wp, nb = _scratch(lib().ga_norm_backward_workspace_bytes(s), dev, ws)
    _launch(dev, lib().ga_norm_residual_backward, s, *tensors, dYp, dHp,
            *(None if t is None else t.data_ptr() for t in got.values()), wp, nb)
    return {k: t for k, t in got.items() if t is not None}


def workspace_check(X: torch.Tensor, N: int, ws=None) -> None:
    """Wait for the current stream and raise GAError if the last grouping
    launch that used this workspace (the cached one if ws is None) gave up a
    cross-workgroup wait."""
    dev = _qkv_like(X, "X")
    s = shape_of(X)
    wp, nb = _ws_args(s, N, dev, ws)
    _check(lib().ga_workspace_check(s, int(N), wp, nb, _stream(dev)))


def timing_enable(on: bool = True) -> None:
    """Bracket every kernel launch (this thread) with hipEvents on its stream."""
    _check(lib().ga_timing_enable(1 if on else 0))


def timing_collect() -> dict:
    """{kernel: (launches, total_ms)} since the last collect; waits for the events."""
    buf = (KernelTime * 64)()
    n = ctypes.c_int32(0)
    _check(lib().ga_timing_collect(buf, 64, ctypes.byref(n)))
    return {buf[i].name.decode(): (int(buf[i].launches), float(buf[i].total_ms)) for i in range(n.value)}
