"""Python binding of libusp.so: argument marshalling only.

Every function here forwards to the C entry point of the same name declared in
``include/usp.h``; all computation happens in the library's host encoder and
gfx950 kernels. PyTorch supplies device buffers and the current HIP stream.
There is no fallback: if the library is not built, loading it raises.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np
import torch  # imported first so libusp.so binds to the HIP runtime torch already loaded

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libusp.so")

USP_OK = 0
_STATUS = {0: "USP_OK", 1: "USP_ERR_INVALID_ARG", 2: "USP_ERR_UNSUPPORTED", 3: "USP_ERR_OOM",
           4: "USP_ERR_HIP", 5: "USP_ERR_INTERNAL"}

EXPORTED = ("usp_encode", "usp_encode_q", "usp_workspace_size", "usp_spmm", "usp_spmm_ex", "usp_spmm_noalloc", "usp_spmm_q",
            "usp_quantize", "usp_plan", "usp_group_create", "usp_group_free", "usp_group_workspace_size", "usp_group_plan",
            "usp_spmm_grouped", "usp_norm", "usp_decode_q", "usp_densify", "usp_decode", "usp_info", "usp_free", "usp_last_error")

# Bytes of the per-GPU device scratch usp_spmm_noalloc uses (USP_NOALLOC_SCRATCH_BYTES).
NOALLOC_SCRATCH_BYTES = 32 << 20

# Most columns of an 8-bit weight and of a group's experts (USP_MAX_K_Q).
MAX_K_Q = 129024

# usp_norm_kind and usp_gate_activation
NORMS = {"none": 0, "rms": 1, "layer": 2}
GATES = {"none": 0, "sigmoid": 1, "tanh": 2, "silu": 3}

# usp_activation
ACTIVATIONS = {"none": 0, "relu": 1, "gelu_tanh": 2, "silu": 3}


class UspError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"{_STATUS.get(status, status)}: {msg}")
        self.status = status


class usp_info_t(ctypes.Structure):
    _fields_ = [("M", ctypes.c_int64), ("K", ctypes.c_int64), ("nnz", ctypes.c_int64),
                ("device_bytes", ctypes.c_size_t), ("table_bytes", ctypes.c_size_t),
                ("format_version", ctypes.c_int32), ("tile_rows", ctypes.c_int32),
                ("tile_k", ctypes.c_int32), ("device", ctypes.c_int32)]


class usp_norm_args(ctypes.Structure):
    _fields_ = ([(f, ctypes.c_void_p) for f in ("residual", "y", "gate", "post_weight", "post_bias", "pre_weight",
                                                "pre_bias", "residual_out", "out", "out_q", "out_scale")] +
                [(f, ctypes.c_int64) for f in ("ld_residual", "ld_y", "ld_gate", "ld_residual_out", "ld_out", "ld_out_q")] +
                [("scale", ctypes.c_float), ("eps", ctypes.c_float), ("post_kind", ctypes.c_int),
                 ("pre_kind", ctypes.c_int), ("gate_activation", ctypes.c_int)])


_lib = None

# (M, K) of the live handles and groups made here. The C calls are given row strides alone: a product whose operands are
# narrower than that would read or write beside them.
_shapes: dict[int, tuple[int, int]] = {}

# Live handles whose owners are gone while a group held them: freed with the last of their groups.
_ownerless: set[int] = set()


def load_library(path: str = LIB_PATH) -> ctypes.CDLL:
    """Loads libusp.so (raises when it has not been built)."""
    global _lib
    if _lib is not None and path == LIB_PATH:
        return _lib
    if not os.path.exists(path):
        raise ImportError(f"{path} is not built: run paper_2607_08786_amd/build.py "
                          "(or __graft_entry__.build()) first")
    lib = ctypes.CDLL(path)
    p, i64, sz = ctypes.c_void_p, ctypes.c_int64, ctypes.c_size_t
    st = ctypes.c_int
    lib.usp_encode.argtypes = [p, i64, p, i64, i64, i64, ctypes.c_int, ctypes.POINTER(p)]
    lib.usp_encode.restype = st
    lib.usp_workspace_size.argtypes = [p, i64]
    lib.usp_workspace_size.restype = sz
    lib.usp_spmm.argtypes = [p, p, i64, p, i64, i64, p, sz, p]
    lib.usp_spmm.restype = st
    lib.usp_spmm_ex.argtypes = [p, p, i64, p, i64, i64, p, p, i64, ctypes.c_int, p, sz, p]
    lib.usp_spmm_ex.restype = st
    lib.usp_spmm_noalloc.argtypes = [p, p, i64, p, i64, i64, p]
    lib.usp_spmm_noalloc.restype = st
    lib.usp_plan.argtypes = [p, i64, ctypes.c_char_p, sz]
    lib.usp_plan.restype = st
    lib.usp_densify.argtypes = [p, p, i64, p]
    lib.usp_densify.restype = st
    lib.usp_decode.argtypes = [p, p, p]
    lib.usp_decode.restype = st
    lib.usp_info.argtypes = [p, ctypes.POINTER(usp_info_t)]
    lib.usp_info.restype = st
    lib.usp_free.argtypes = [p]
    lib.usp_free.restype = st
    lib.usp_encode_q.argtypes = [p, i64, p, i64, p, i64, i64, ctypes.c_int, ctypes.POINTER(p)]
    lib.usp_decode_q.argtypes = [p, p, p, p]
    lib.usp_quantize.argtypes = [p, i64, i64, i64, p, i64, p, ctypes.c_int, p]
    lib.usp_spmm_q.argtypes = [p, p, i64, p, p, i64, i64, p, p, i64, ctypes.c_int, p, sz, p]
    lib.usp_group_create.argtypes = [ctypes.POINTER(p), i64, ctypes.POINTER(p)]
    lib.usp_group_free.argtypes = [p]
    lib.usp_spmm_grouped.argtypes = [p, p, i64, i64, p, p, p, i64, p, i64, i64, p, i64, p, ctypes.c_int, p, sz, p]
    lib.usp_norm.argtypes = [ctypes.POINTER(usp_norm_args), i64, i64, ctypes.c_int, p]
    for name in ("usp_encode_q", "usp_decode_q", "usp_quantize", "usp_spmm_q", "usp_group_create", "usp_group_free",
                 "usp_spmm_grouped", "usp_norm", "usp_group_plan"):
        getattr(lib, name).restype = st
    lib.usp_group_workspace_size.argtypes = [p, i64]
    lib.usp_group_plan.argtypes = [p, i64, ctypes.c_char_p, sz]
    lib.usp_group_workspace_size.restype = sz
    lib.usp_last_error.argtypes = []
    lib.usp_last_error.restype = ctypes.c_char_p
    if path == LIB_PATH:
        _lib = lib
    return lib


def usp_last_error() -> str:
    return load_library().usp_last_error().decode()


def _check(status: int):
    if status != USP_OK:
        raise UspError(status, usp_last_error())


def _torch_stream(stream):
    """The torch stream a call is enqueued on: the current one, a torch.cuda.Stream, or a raw
    hipStream_t handle wrapped as an external stream."""
    if stream is None:
        return torch.cuda.current_stream()
    if isinstance(stream, torch.cuda.Stream):
        return stream
    return torch.cuda.ExternalStream(int(stream))


def current_stream_handle(device: int | None = None) -> int:
    """The hipStream_t of torch's current stream (of the current device, or of `device`), without
    the Stream object of torch.cuda.current_stream()."""
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device() if device is None else device)


def _stream_handle(stream) -> int | None:
    if stream is None:
        return current_stream_handle()
    if isinstance(stream, torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def usp_encode(W: np.ndarray, mask: np.ndarray, device: int = 0) -> int:
    """W: (M, K) fp16 bit patterns (uint16 or float16); mask: (M, K), nonzero = kept."""
    W = np.ascontiguousarray(W)
    if W.dtype == np.float16:
        W = W.view(np.uint16)
    if W.dtype != np.uint16 or W.ndim != 2:
        raise TypeError("W must be a 2-D uint16 (fp16 bits) or float16 array")
    mask = np.ascontiguousarray(mask)
    if mask.dtype == np.bool_:
        mask = mask.view(np.uint8)
    if mask.dtype != np.uint8 or mask.shape != W.shape:
        raise TypeError("mask must be a uint8/bool array of W's shape")
    M, K = W.shape
    h = ctypes.c_void_p()
    _check(load_library().usp_encode(W.ctypes.data, K, mask.ctypes.data, K, M, K, device, ctypes.byref(h)))
    _shapes[h.value] = (M, K)
    return h.value


def usp_workspace_size(handle: int, N: int) -> int:
    return int(load_library().usp_workspace_size(handle, N))


def usp_plan(handle: int, N: int) -> str:
    """The kernel usp_spmm (usp_spmm_q on 8-bit tokens) runs for this handle and N (X aligned, ldx = K), as text."""
    buf = ctypes.create_string_buffer(128)
    _check(load_library().usp_plan(handle, N, buf, len(buf)))
    return buf.value.decode()


def usp_spmm(handle: int, X: torch.Tensor, Y: torch.Tensor, workspace: torch.Tensor | None = None,
             stream=None) -> None:
    """Y[N, M] = X[N, K] @ W^T, i.e. Y = W X with token-major X and Y (fp16 device tensors)."""
    if X.dtype != torch.float16 or Y.dtype != torch.float16:
        raise TypeError("X and Y must be float16")
    if X.dim() != 2 or Y.dim() != 2 or X.stride(1) != 1 or Y.stride(1) != 1:
        raise TypeError("X and Y must be 2-D with unit inner stride")
    N = X.shape[0]
    if Y.shape[0] != N:
        raise ValueError("X and Y must have the same number of tokens")
    ws_ptr, ws_bytes = None, 0
    if workspace is not None:
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _check(load_library().usp_spmm(handle, X.data_ptr(), X.stride(0), Y.data_ptr(), Y.stride(0), N,
                                   ws_ptr, ws_bytes, _stream_handle(stream)))


def usp_spmm_ex(handle: int, X: torch.Tensor, Y: torch.Tensor, workspace: torch.Tensor | None = None,
                bias: torch.Tensor | None = None, residual: torch.Tensor | None = None,
                activation: str | int = "none", stream=None) -> None:
    """Y = act(X @ W^T + bias) + residual (token-major fp16 device tensors; bias [M],
    residual [N, M] with unit inner stride, or None; residual may be Y itself)."""
    if X.dtype != torch.float16 or Y.dtype != torch.float16:
        raise TypeError("X and Y must be float16")
    if X.dim() != 2 or Y.dim() != 2 or X.stride(1) != 1 or Y.stride(1) != 1:
        raise TypeError("X and Y must be 2-D with unit inner stride")
    N = X.shape[0]
    if Y.shape[0] != N:
        raise ValueError("X and Y must have the same number of tokens")
    act = ACTIVATIONS[activation] if isinstance(activation, str) else int(activation)
    b_ptr = r_ptr = None
    ldr = 0
    if bias is not None:
        if bias.dtype != torch.float16 or bias.dim() != 1 or bias.stride(0) != 1 or bias.shape[0] != Y.shape[1]:
            raise TypeError("bias must be a contiguous float16 vector of M entries")
        b_ptr = bias.data_ptr()
    if residual is not None:
        if residual.dtype != torch.float16 or residual.dim() != 2 or residual.stride(1) != 1 \
                or tuple(residual.shape) != tuple(Y.shape):
            raise TypeError("residual must be a float16 [N, M] tensor with unit inner stride")
        r_ptr, ldr = residual.data_ptr(), residual.stride(0)
    ws_ptr, ws_bytes = None, 0
    if workspace is not None:
        ws_ptr, ws_bytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    _check(load_library().usp_spmm_ex(handle, X.data_ptr(), X.stride(0), Y.data_ptr(), Y.stride(0), N,
                                      b_ptr, r_ptr, ldr, act, ws_ptr, ws_bytes, _stream_handle(stream)))


def usp_spmm_noalloc(handle: int, X: torch.Tensor, Y: torch.Tensor, stream=None) -> None:
    """usp_spmm with the library's per-GPU device scratch as its workspace (no allocation;
    calls overlapping on one GPU must be serialized by the caller)."""
    if X.dtype != torch.float16 or Y.dtype != torch.float16:
        raise TypeError("X and Y must be float16")
    if X.dim() != 2 or Y.dim() != 2 or X.stride(1) != 1 or Y.stride(1) != 1:
        raise TypeError("X and Y must be 2-D with unit inner stride")
    N = X.shape[0]
    if Y.shape[0] != N:
        raise ValueError("X and Y must have the same number of tokens")
    _check(load_library().usp_spmm_noalloc(handle, X.data_ptr(), X.stride(0), Y.data_ptr(), Y.stride(0), N,
                                           _stream_handle(stream)))


def usp_densify(handle: int, Wd: torch.Tensor, stream=None) -> None:
    if Wd.dtype != torch.float16 or Wd.dim() != 2 or Wd.stride(1) != 1:
        raise TypeError("Wd must be a 2-D float16 tensor with unit inner stride")
    _check(load_library().usp_densify(handle, Wd.data_ptr(), Wd.stride(0), _stream_handle(stream)))


def usp_info(handle: int) -> dict:
    info = usp_info_t()
    _check(load_library().usp_info(handle, ctypes.byref(info)))
    return {f: getattr(info, f) for f, _ in usp_info_t._fields_}


def usp_decode(handle: int):
    info = usp_info(handle)
    M, K = info["M"], info["K"]
    W = np.empty((M, K), dtype=np.uint16)
    mask = np.empty((M, K), dtype=np.uint8)
    _check(load_library().usp_decode(handle, W.ctypes.data, mask.ctypes.data))
    return W, mask


def usp_free(handle: int) -> None:
    shape, ownerless = _shapes.pop(handle, None), handle in _ownerless
    _ownerless.discard(handle)  # all before the number can be another handle's
    status = load_library().usp_free(handle)
    if status != USP_OK:
        if shape is not None:
            _shapes[handle] = shape
        if ownerless:
            _ownerless.add(handle)
        _check(status)


def usp_encode_q(W: np.ndarray, mask: np.ndarray, scale: np.ndarray, device: int = 0) -> int:
    """W: (M, K) int8; mask: (M, K), nonzero = kept; scale: (M,) float32, one per row."""
    W = np.ascontiguousarray(W)
    if W.dtype != np.int8 or W.ndim != 2:
        raise TypeError("W must be a 2-D int8 array")
    mask = np.ascontiguousarray(mask)
    if mask.dtype == np.bool_:
        mask = mask.view(np.uint8)
    if mask.dtype != np.uint8 or mask.shape != W.shape:
        raise TypeError("mask must be a uint8/bool array of W's shape")
    scale = np.ascontiguousarray(scale)
    if scale.dtype != np.float32 or scale.shape != W.shape[:1]:
        raise TypeError("scale must be a float32 array of one value per row of W")
    M, K = W.shape
    h = ctypes.c_void_p()
    _check(load_library().usp_encode_q(W.ctypes.data, K, mask.ctypes.data, K, scale.ctypes.data, M, K, device,
                                       ctypes.byref(h)))
    _shapes[h.value] = (M, K)
    return h.value


def usp_decode_q(handle: int):
    info = usp_info(handle)
    M, K = info["M"], info["K"]
    W, mask, scale = np.empty((M, K), np.int8), np.empty((M, K), np.uint8), np.empty(M, np.float32)
    _check(load_library().usp_decode_q(handle, W.ctypes.data, mask.ctypes.data, scale.ctypes.data))
    return W, mask, scale


def _matrix(t: torch.Tensor, dtype: torch.dtype, shape, dev: int, name: str):
    """(address, row stride) of a 2-D operand after its checks. The stride of a single row is not looked at."""
    if t.dtype is not dtype or len(shape) != 2 or t.dim() != 2:
        raise TypeError(f"{name} must be a 2-D {dtype} tensor")
    if t.get_device() != dev:
        raise ValueError(f"{name} must be on GPU {dev}")
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}")
    ld, inner = t.stride()
    if inner != 1 and shape[1] > 1:
        raise TypeError(f"{name} must have unit inner stride")
    return t.data_ptr(), ld if shape[0] > 1 else max(ld, shape[1])


def _vector(t: torch.Tensor | None, dtype: torch.dtype, n: int, dev: int, name: str) -> int | None:
    """The address of a contiguous vector of n values after its checks; None for None."""
    if t is None:
        return None
    if t.dtype is not dtype or t.shape != (n,) or (n > 1 and t.stride(0) != 1):
        raise TypeError(f"{name} must be a contiguous {dtype} vector of {n} values")
    if t.get_device() != dev:
        raise ValueError(f"{name} must be on GPU {dev}")
    return t.data_ptr()


def _shape_of(handle: int) -> tuple[int, int]:
    """(M, K) of a matrix; an error for one that is not alive."""
    shape = _shapes.get(handle)
    if shape is None:
        info = usp_info(handle)
        shape = info["M"], info["K"]
    return shape


def _check_widths(shape, M: int, K: int) -> None:
    if shape != (M, K):
        raise UspError(1, f"the weight is {shape[0]} x {shape[1]}: X must have {shape[1]} columns (has {K}) and Y {shape[0]} (has {M})")


def _stream_of(stream, dev: int) -> int:
    """The stream of a call on GPU `dev`: its current one, unless one is given."""
    return current_stream_handle(dev) if stream is None else _stream_handle(stream)


def _workspace(ws: torch.Tensor | None, dev: int):
    if ws is None:
        return None, 0
    if ws.get_device() != dev or not ws.is_contiguous():
        raise ValueError(f"the workspace must be a contiguous tensor on GPU {dev}")
    return ws.data_ptr(), ws.nbytes


def _gpu(t: torch.Tensor, name: str) -> int:
    dev = t.get_device()
    if dev < 0:
        raise ValueError(f"{name} must be on a GPU")
    return dev


def usp_quantize(X: torch.Tensor, Xq: torch.Tensor, x_scale: torch.Tensor, stream=None) -> None:
    """Tokens in 8 bits: X [N, K] fp16 into Xq [N, K] int8 and x_scale [N] fp32."""
    dev = _gpu(X, "X")
    shape = X.shape
    x, ldx = _matrix(X, torch.float16, shape, dev, "X")
    q, ldq = _matrix(Xq, torch.int8, shape, dev, "Xq")
    _check((_lib or load_library()).usp_quantize(x, ldx, shape[0], shape[1], q, ldq,
                                                 _vector(x_scale, torch.float32, shape[0], dev, "x_scale"), dev,
                                                 _stream_of(stream, dev)))


def usp_spmm_q(handle: int, Xq: torch.Tensor, x_scale: torch.Tensor | None, Y: torch.Tensor,
               workspace: torch.Tensor | None = None, bias: torch.Tensor | None = None,
               residual: torch.Tensor | None = None, activation: str | int = "none", stream=None) -> None:
    """Y = act(W X + bias) + residual with 8-bit weights and tokens (Xq [N, K] int8 and x_scale [N] fp32, or fp16
    Xq and None, which is quantised first; Y, bias, residual as usp_spmm_ex). Xq and Y must have the weight's widths."""
    dev = _gpu(Xq, "Xq")
    y, ldy = _matrix(Y, torch.float16, Y.shape, dev, "Y")
    N, M = Y.shape
    if Xq.dim() != 2 or Xq.shape[0] != N:
        raise ValueError("Xq and Y must have the same number of tokens")
    _check_widths(_shapes.get(handle) or _shape_of(handle), M, Xq.shape[1])
    act = ACTIVATIONS[activation] if isinstance(activation, str) else int(activation)
    x, ldx = _matrix(Xq, torch.float16 if x_scale is None else torch.int8, Xq.shape, dev, "Xq")
    r, ldr = (None, 0) if residual is None else _matrix(residual, torch.float16, Y.shape, dev, "residual")
    ws, ws_bytes = _workspace(workspace, dev)
    _check((_lib or load_library()).usp_spmm_q(
        handle, x, ldx, _vector(x_scale, torch.float32, N, dev, "x_scale"), y, ldy, N,
        _vector(bias, torch.float16, M, dev, "bias"), r, ldr, act, ws, ws_bytes, _stream_of(stream, dev)))


def usp_group_create(handles) -> int:
    arr = (ctypes.c_void_p * len(handles))(*handles)
    g = ctypes.c_void_p()
    _check(load_library().usp_group_create(arr, len(handles), ctypes.byref(g)))
    _shapes[g.value] = _shape_of(handles[0])
    return g.value


def usp_group_free(group: int) -> None:
    _shapes.pop(group, None)
    _check(load_library().usp_group_free(group))
    _free_ownerless(list(_ownerless))


def _free_ownerless(handles) -> None:
    """Frees those of the ownerless handles that no group holds any more."""
    for h in handles:
        try:
            _ownerless.remove(h)
        except KeyError:  # another thread has it
            continue
        try:
            usp_free(h)
        except UspError:
            if _alive(h):
                _ownerless.add(h)


def _alive(handle: int) -> bool:
    try:
        usp_info(handle)
    except UspError:
        return False
    return True


def _owner_gone(handle: int) -> None:
    """For a handle that could not be freed at its owner's end: the collector takes an owner and the group in any order."""
    if _alive(handle):
        _ownerless.add(handle)
        _free_ownerless([handle])  # the group may be gone by now


def usp_group_workspace_size(group: int, T: int) -> int:
    return int(load_library().usp_group_workspace_size(group, T))


def usp_group_plan(group: int, T: int) -> str:
    """The kernel usp_spmm_grouped runs for this group and T rows, as text."""
    buf = ctypes.create_string_buffer(128)
    _check(load_library().usp_group_plan(group, T, buf, len(buf)))
    return buf.value.decode()


def usp_spmm_grouped(group: int, X: torch.Tensor, offsets: torch.Tensor, Y: torch.Tensor,
                     workspace: torch.Tensor | None = None, x_scale: torch.Tensor | None = None,
                     rows: torch.Tensor | None = None, bias: torch.Tensor | None = None,
                     row_weight: torch.Tensor | None = None, activation: str | int = "none", stream=None) -> None:
    """Y[t] = row_weight[t] * act(W_e X[rows[t]] + bias[e]) for the rows offsets[e] <= t < offsets[e + 1] of
    expert e. X [*, K] fp16, or int8 with x_scale; offsets [E + 1] and rows [T] int32; bias [E, M] fp16;
    row_weight [T] fp32; Y [T, M] fp16. X and Y must have the experts' widths."""
    dev = _gpu(X, "X")
    y, ldy = _matrix(Y, torch.float16, Y.shape, dev, "Y")
    T, M = Y.shape
    act = ACTIVATIONS[activation] if isinstance(activation, str) else int(activation)
    x, ldx = _matrix(X, torch.float16 if x_scale is None else torch.int8, X.shape, dev, "X")
    shape = _shapes.get(group)
    if shape is not None:  # else the call refuses the group, or it was made without this binding
        _check_widths(shape, M, X.shape[1])
    E = offsets.shape[0] - 1
    b, ldb = (None, 0) if bias is None else _matrix(bias, torch.float16, (E, M), dev, "bias")
    ws, ws_bytes = _workspace(workspace, dev)
    _check((_lib or load_library()).usp_spmm_grouped(
        group, x, ldx, X.shape[0], _vector(x_scale, torch.float32, X.shape[0], dev, "x_scale"),
        _vector(rows, torch.int32, T, dev, "rows"), _vector(offsets, torch.int32, E + 1, dev, "offsets"), E, y, ldy, T, b,
        ldb, _vector(row_weight, torch.float32, T, dev, "row_weight"), act, ws, ws_bytes, _stream_of(stream, dev)))


def usp_norm(residual: torch.Tensor, y: torch.Tensor | None = None, gate: torch.Tensor | None = None,
             scale: float = 1.0, post: str = "none", post_weight: torch.Tensor | None = None,
             post_bias: torch.Tensor | None = None, pre: str = "none", pre_weight: torch.Tensor | None = None,
             pre_bias: torch.Tensor | None = None, eps: float = 1e-5, gate_activation: str = "none",
             residual_out: torch.Tensor | None = None, out: torch.Tensor | None = None,
             out_q: torch.Tensor | None = None, out_scale: torch.Tensor | None = None, stream=None) -> None:
    """r = residual + scale * act(gate) * post(y) into residual_out and h = pre(r) into out (fp16) and / or
    out_q, out_scale (8-bit tokens). All [N, K] fp16 but out_q (int8); gate [N, K], or [K] for all tokens; weights
    and biases [K]; out_scale [N] fp32. residual_out may be residual or y, out may be y."""
    dev = _gpu(residual, "residual")
    shape = residual.shape
    f16 = torch.float16
    none = (None, 0)
    res, ld_res = _matrix(residual, f16, shape, dev, "residual")
    N, K = shape
    yp, ld_y = none if y is None else _matrix(y, f16, shape, dev, "y")
    if gate is None:
        gp, ld_g = none
    elif gate.dim() == 1:
        gp, ld_g = _vector(gate, f16, K, dev, "gate"), 0
    else:
        gp, ld_g = _matrix(gate, f16, shape, dev, "gate")
    ro, ld_ro = none if residual_out is None else _matrix(residual_out, f16, shape, dev, "residual_out")
    op, ld_o = none if out is None else _matrix(out, f16, shape, dev, "out")
    qp, ld_q = none if out_q is None else _matrix(out_q, torch.int8, shape, dev, "out_q")
    a = usp_norm_args(res, yp, gp, _vector(post_weight, f16, K, dev, "post_weight"),
                      _vector(post_bias, f16, K, dev, "post_bias"), _vector(pre_weight, f16, K, dev, "pre_weight"),
                      _vector(pre_bias, f16, K, dev, "pre_bias"), ro, op, qp,
                      _vector(out_scale, torch.float32, N, dev, "out_scale"), ld_res, ld_y, ld_g, ld_ro, ld_o, ld_q,
                      scale, eps, NORMS[post], NORMS[pre], GATES[gate_activation])
    _check((_lib or load_library()).usp_norm(ctypes.byref(a), N, K, dev, _stream_of(stream, dev)))


def _zeros(n: int, device: int, stream) -> torch.Tensor | None:
    """n zero bytes, allocated and cleared on `stream`; None for none."""
    if n == 0:
        return None
    with torch.cuda.stream(_torch_stream(stream)):
        return torch.zeros(n, dtype=torch.uint8, device=f"cuda:{device}")


# The part of a workspace that usp_spmm expects cleared; usp_spmm_q and usp_spmm_grouped leave it alone and need nothing
# cleared.
_COUNTER_BYTES = 256 << 10


def _space(n: int, device: int, stream) -> torch.Tensor | None:
    """n bytes for the products that need nothing cleared, allocated on `stream`, the counters' part cleared; None for none."""
    if n == 0:
        return None
    with torch.cuda.stream(_torch_stream(stream)):
        ws = torch.empty(n, dtype=torch.uint8, device=f"cuda:{device}")
        ws[:_COUNTER_BYTES].zero_()
        return ws


class SparseMatrix:
    """Owns one encoded weight matrix (a usp_matrix handle)."""

    def __init__(self, W: np.ndarray, mask: np.ndarray, device: int = 0):
        self._own(usp_encode(W, mask, device), device)

    def _own(self, handle: int, device: int) -> None:
        self.handle = handle
        info = usp_info(self.handle)
        self.M, self.K, self.nnz = info["M"], info["K"], info["nnz"]
        self.device = device
        self.device_bytes = info["device_bytes"] + info["table_bytes"]

    def workspace_size(self, N: int) -> int:
        return usp_workspace_size(self.handle, N)

    def plan(self, N: int) -> str:
        return usp_plan(self.handle, N)

    def make_workspace(self, N: int, stream=None) -> torch.Tensor | None:
        """A zero-filled workspace for N tokens, allocated and cleared on `stream` (default: the
        current stream), so calls enqueued on that stream are ordered after the clear."""
        return _zeros(self.workspace_size(N), self.device, stream)

    def spmm(self, X: torch.Tensor, Y: torch.Tensor | None = None, workspace=None, stream=None,
             bias: torch.Tensor | None = None, residual: torch.Tensor | None = None,
             activation: str | int = "none") -> torch.Tensor:
        """Y = W X (token-major), or act(W X + bias) + residual when any of those is given.

        A Y or workspace this call creates is allocated on `stream`, the stream the product is
        enqueued on, so the caching allocator only reuses that memory in that stream's order."""
        N = X.shape[0]
        if Y is None or workspace is None:
            with torch.cuda.stream(_torch_stream(stream)):
                if Y is None:
                    Y = torch.empty((N, self.M), dtype=torch.float16, device=X.device)
                if workspace is None:
                    workspace = self.make_workspace(N)
        if bias is None and residual is None and activation in ("none", 0):
            usp_spmm(self.handle, X, Y, workspace, stream)
        else:
            usp_spmm_ex(self.handle, X, Y, workspace, bias, residual, activation, stream)
        return Y

    def densify(self, stream=None) -> torch.Tensor:
        Wd = torch.empty((self.M, self.K), dtype=torch.float16, device=f"cuda:{self.device}")
        usp_densify(self.handle, Wd, stream)
        return Wd

    def decode(self):
        return usp_decode(self.handle)

    def info(self) -> dict:
        return usp_info(self.handle)

    def free(self) -> None:
        if self.handle:
            usp_free(self.handle)
            self.handle = None

    def __del__(self):
        try:
            try:
                self.free()
            except UspError:
                _owner_gone(self.handle)
        except Exception:
            pass


class SparseMatrixQ(SparseMatrix):
    """Owns one encoded weight matrix of 8-bit values with a scale per row."""

    def __init__(self, W: np.ndarray, mask: np.ndarray, scale: np.ndarray, device: int = 0):
        self._own(usp_encode_q(W, mask, scale, device), device)

    def make_workspace(self, N: int, stream=None) -> torch.Tensor | None:
        """A workspace for N tokens, allocated on `stream` (default: the current one). Only the part that usp_spmm expects
        cleared is."""
        return _space(self.workspace_size(N), self.device, stream)

    def spmm(self, Xq: torch.Tensor, x_scale: torch.Tensor | None = None, Y: torch.Tensor | None = None, workspace=None, stream=None,
             bias: torch.Tensor | None = None, residual: torch.Tensor | None = None,
             activation: str | int = "none") -> torch.Tensor:
        """act(W X + bias) + residual of 8-bit tokens (usp_quantize), or of fp16 tokens without x_scale; what the call creates is allocated as in
        SparseMatrix.spmm."""
        N = Xq.shape[0]
        if Y is None or workspace is None:
            with torch.cuda.stream(_torch_stream(stream)):
                if Y is None:
                    Y = torch.empty((N, self.M), dtype=torch.float16, device=Xq.device)
                if workspace is None:
                    workspace = self.make_workspace(N)
        usp_spmm_q(self.handle, Xq, x_scale, Y, workspace, bias, residual, activation, stream)
        return Y

    def decode(self):
        return usp_decode_q(self.handle)


class ExpertGroup:
    """Encoded experts of one shape and value type (a usp_group handle); keeps them alive."""

    def __init__(self, experts):
        self.experts = list(experts)
        self.handle = None
        self.handle = usp_group_create([m.handle for m in self.experts])
        self.M, self.K, self.device = self.experts[0].M, self.experts[0].K, self.experts[0].device

    def workspace_size(self, T: int) -> int:
        return usp_group_workspace_size(self.handle, T)

    def plan(self, T: int) -> str:
        return usp_group_plan(self.handle, T)

    def make_workspace(self, T: int, stream=None) -> torch.Tensor | None:
        """A workspace for T rows, allocated on `stream` (default: the current one), cleared as SparseMatrixQ's."""
        return _space(self.workspace_size(T), self.device, stream)

    def spmm(self, X: torch.Tensor, offsets: torch.Tensor, T: int | None = None, Y: torch.Tensor | None = None,
             workspace=None, stream=None, **operands) -> torch.Tensor:
        """usp_spmm_grouped into Y, or into a new tensor of T rows (default: those of `rows`, or of X), of which
        the rows that no expert has are zeros."""
        with torch.cuda.stream(_torch_stream(stream)):
            if Y is None:
                rows = operands.get("rows")
                T = (X if rows is None else rows).shape[0] if T is None else T
                Y = torch.zeros((T, self.M), dtype=torch.float16, device=X.device)
            if workspace is None:
                workspace = self.make_workspace(Y.shape[0])
        usp_spmm_grouped(self.handle, X, offsets, Y, workspace, stream=stream, **operands)
        return Y

    def free(self) -> None:
        if self.handle:
            usp_group_free(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.free()
        except Exception:
            pass
