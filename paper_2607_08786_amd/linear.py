"""Sparse drop-in for ``torch.nn.Linear`` (with a fused activation) on decode
steps: the pruned weight is encoded once and every call is one ``usp_spmm_ex``
(product, bias, activation and residual add in one kernel launch).

``torch.ops.usp.sparse_linear`` is the custom operator; ``SparseLinear`` is the
module around it. Inputs are fp16 CUDA (HIP) tensors whose last dimension is
``in_features``; leading dimensions are flattened into the token count N.

``SparseLinearQ`` is the same with 8-bit weights and tokens, ``SparseExperts`` a linear
layer with a weight for each expert on rows sorted by expert, and ``BlockNorm`` the norms
around a block with its gate and residual scale, whose output may be the 8-bit tokens that
the two read (operators ``usp::sparse_linear_q``, ``usp::sparse_experts``, ``usp::block_norm``).
All of it is for inference: nothing here has a backward pass.
"""
from __future__ import annotations

from typing import Optional, Tuple, Union

import numpy as np
import torch

from . import usp


@torch.library.custom_op("usp::sparse_linear", mutates_args=("workspace",))
def sparse_linear(x: torch.Tensor, handle: int, out_features: int, bias: Optional[torch.Tensor],
                  residual: Optional[torch.Tensor], activation: int,
                  workspace: Optional[torch.Tensor]) -> torch.Tensor:
    """act(x @ W^T + bias) + residual for the encoded W behind ``handle``; x is
    [N, in_features], residual [N, out_features]. The workspace (zero-filled
    once) is left zero again by every call."""
    y = torch.empty((x.shape[0], out_features), dtype=torch.float16, device=x.device)
    usp.usp_spmm_ex(handle, x, y, workspace, bias, residual, activation)
    return y


@sparse_linear.register_fake
def _(x, handle, out_features, bias, residual, activation, workspace):
    return x.new_empty((x.shape[0], out_features))


class Workspaces:
    """The workspaces of a module's calls. Every completed call leaves a workspace ready for the next one of any size, so
    each stream has one buffer for all its calls, replaced when one needs more bytes; it is allocated and used on that
    stream alone, so its memory is reused in that stream's order.

    A captured graph records the buffer's address. A capture takes a buffer that an earlier call (its
    warm-up) left, which from then on belongs to the graphs, is kept as long as the module and is no
    longer given to other calls. Without one of the size, the buffer is allocated and cleared in the
    graph itself."""

    def _no_workspaces(self) -> None:
        self._ws: dict[int, torch.Tensor] = {}  # stream -> the workspace of the calls enqueued on it
        self._graph_ws: list[torch.Tensor] = []  # workspaces whose addresses captured graphs hold

    def _workspace(self, need: int, make) -> Optional[torch.Tensor]:
        """A buffer of at least `need` bytes for a call on the current stream, or what `make` gives; None for none."""
        if need == 0:
            return None
        if torch.cuda.is_current_stream_capturing():
            ws = next((w for w in self._graph_ws if w.numel() >= need), None)
            if ws is not None:
                return ws
            for stream, ws in list(self._ws.items()):  # another thread's call may add its stream meanwhile
                if ws.numel() >= need and self._ws.pop(stream, None) is not None:
                    self._graph_ws.append(ws)
                    return ws
            return make()
        stream = self._stream()
        ws = self._ws.get(stream)
        if ws is None or ws.numel() < need:
            ws = self._ws[stream] = make()
        return ws


def _operand(workspace: Optional[torch.Tensor], x: torch.Tensor) -> Optional[torch.Tensor]:
    """A workspace as an operator's operand. A compiled program has an empty tensor for none: inductor takes no None for an
    operand that the operator writes."""
    return x.new_empty(0, dtype=torch.uint8) if workspace is None and torch.compiler.is_compiling() else workspace


class SparseLinear(Workspaces, torch.nn.Module):
    """``act(x W^T + b) (+ residual)`` with W pruned by ``mask`` (kept where nonzero).

    weight: [out_features, in_features] tensor (converted to fp16); mask: array or
    tensor of the same shape; bias: [out_features] or None; activation: one of
    "none", "relu", "gelu_tanh", "silu".

    Calls on different streams may overlap, also from several threads (one stream each). Graphs that hold
    calls of one module share a workspace: their replays must not overlap each other."""

    def __init__(self, weight: torch.Tensor, mask, bias: Optional[torch.Tensor] = None,
                 activation: str = "none", device: Optional[int] = None):
        super().__init__()
        if activation not in usp.ACTIVATIONS:
            raise ValueError(f"activation must be one of {sorted(usp.ACTIVATIONS)}")
        dev = torch.cuda.current_device() if device is None else int(device)
        w = weight.detach().to(torch.float16).cpu().contiguous().numpy().view(np.uint16)
        m = mask.detach().cpu().numpy() if isinstance(mask, torch.Tensor) else np.asarray(mask)
        m = np.ascontiguousarray(m != 0, dtype=np.uint8)
        if m.shape != w.shape:
            raise ValueError("mask must have the weight's shape")
        self.matrix = usp.SparseMatrix(w, m, dev)
        self._set_up(w.shape, bias, activation, dev)

    def _set_up(self, shape, bias, activation, dev) -> None:
        self.out_features, self.in_features = shape
        self.activation = activation
        self.register_buffer(
            "bias", None if bias is None else bias.detach().to(device=f"cuda:{dev}", dtype=torch.float16).contiguous())
        self._no_workspaces()

    @classmethod
    def from_linear(cls, linear: torch.nn.Linear, mask, activation: str = "none") -> "SparseLinear":
        dev = linear.weight.device.index if linear.weight.is_cuda else None
        return cls(linear.weight, mask, linear.bias, activation, dev)

    def _stream(self) -> int:
        """The stream that forward enqueues its calls on."""
        return usp.current_stream_handle()

    def workspace(self, N: int) -> Optional[torch.Tensor]:
        """A zero-filled workspace of at least usp_workspace_size(N) bytes for a call enqueued on the
        current stream (Workspaces says which)."""
        return self._workspace(self.matrix.workspace_size(N), lambda: self.matrix.make_workspace(N))

    def forward(self, x: torch.Tensor, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
        lead = x.shape[:-1]
        x2 = x.reshape(-1, self.in_features)
        if x2.dtype != torch.float16 or not x2.is_contiguous():
            x2 = x2.to(torch.float16).contiguous()
        N = x2.shape[0]
        r2 = None
        if residual is not None:
            r2 = residual.reshape(N, self.out_features)
            if r2.dtype != torch.float16 or not r2.is_contiguous():
                r2 = r2.to(torch.float16).contiguous()
        y = torch.ops.usp.sparse_linear(x2, self.matrix.handle, self.out_features, self.bias, r2,
                                        usp.ACTIVATIONS[self.activation], _operand(self.workspace(N), x2))
        return y.reshape(*lead, self.out_features)

    def extra_repr(self) -> str:
        return (f"in_features={self.in_features}, out_features={self.out_features}, "
                f"nnz={self.matrix.nnz}, bias={self.bias is not None}, activation={self.activation}")


# ---- 8-bit layers, experts and the norms around a block


def quantize_rows(weight: torch.Tensor, mask) -> Tuple[torch.Tensor, torch.Tensor]:
    """A weight in 8 bits, symmetric per row over the kept entries: (codes int8, scale fp32 [rows])."""
    m = torch.as_tensor(mask, device=weight.device) != 0
    w = torch.where(m, weight.detach().float(), torch.zeros((), device=weight.device))
    scale = w.abs().amax(1) / 127
    safe = torch.where(scale > 0, scale, torch.ones_like(scale))
    return (w / safe[:, None]).round().clamp(-127, 127).to(torch.int8), scale


def _int8_tokens(N: int, K: int, device) -> torch.Tensor:
    """An [N, K] int8 tensor whose rows start at multiples of 16 bytes, as the products read them in place."""
    return torch.empty((N, (K + 15) // 16 * 16), dtype=torch.int8, device=device)[:, :K]


def _tokens(x: torch.Tensor, x_scale: Optional[torch.Tensor]) -> Tuple[torch.Tensor, torch.Tensor]:
    """8-bit tokens and scales: x and x_scale themselves, or fp16 x quantised."""
    if x_scale is not None:
        return x, x_scale
    xq = _int8_tokens(*x.shape, x.device)
    x_scale = torch.empty(x.shape[0], dtype=torch.float32, device=x.device)
    usp.usp_quantize(x, xq, x_scale)
    return xq, x_scale


def _linear_q(x: torch.Tensor, x_scale: Optional[torch.Tensor], handle: int, out_features: int,
              bias: Optional[torch.Tensor], residual: Optional[torch.Tensor], activation: int,
              workspace: Optional[torch.Tensor]) -> torch.Tensor:
    """act(x @ W^T + bias) + residual for the 8-bit weight behind ``handle``; x is [N, in_features], fp16, or int8
    with the tokens' scales."""
    y = x.new_empty((x.shape[0], out_features), dtype=torch.float16)
    usp.usp_spmm_q(handle, x, x_scale, y, workspace, bias, residual, activation)
    return y


def _experts(x: torch.Tensor, x_scale: Optional[torch.Tensor], offsets: torch.Tensor, rows: Optional[torch.Tensor],
             row_weight: Optional[torch.Tensor], group: int, out_features: int, eight_bit: bool,
             bias: Optional[torch.Tensor], activation: int, workspace: Optional[torch.Tensor]) -> torch.Tensor:
    """usp_spmm_grouped into a new tensor; zeros in the rows that no expert has."""
    if eight_bit:
        x, x_scale = _tokens(x, x_scale)
    T = x.shape[0] if rows is None else rows.shape[0]
    y = torch.zeros((T, out_features), dtype=torch.float16, device=x.device)
    usp.usp_spmm_grouped(group, x, offsets, y, workspace, x_scale, rows, bias, row_weight, activation)
    return y


def _block_norm(residual: torch.Tensor, y: Optional[torch.Tensor], gate: Optional[torch.Tensor], scale: float,
                post: str, post_weight: Optional[torch.Tensor], post_bias: Optional[torch.Tensor], pre: str,
                pre_weight: Optional[torch.Tensor], pre_bias: Optional[torch.Tensor], eps: float, gate_activation: str,
                quantize: bool) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """The residual's update, the norm of it (int8 if quantize) and the tokens' scales (empty if not)."""
    N, K = residual.shape
    r = residual.new_empty((N, K))
    h = _int8_tokens(N, K, r.device) if quantize else torch.empty_like(r)
    h_scale = r.new_empty(N if quantize else 0, dtype=torch.float32)
    usp.usp_norm(residual, y, gate, scale, post, post_weight, post_bias, pre, pre_weight, pre_bias, eps, gate_activation,
                 residual_out=r, **(dict(out_q=h, out_scale=h_scale) if quantize else dict(out=h)))
    return r, h, h_scale


sparse_linear_q = torch.library.custom_op("usp::sparse_linear_q", _linear_q, mutates_args=("workspace",))
sparse_experts = torch.library.custom_op("usp::sparse_experts", _experts, mutates_args=("workspace",))
block_norm = torch.library.custom_op("usp::block_norm", _block_norm, mutates_args=())


@sparse_linear_q.register_fake
def _(x, x_scale, handle, out_features, bias, residual, activation, workspace):
    return x.new_empty((x.shape[0], out_features), dtype=torch.float16)


@sparse_experts.register_fake
def _(x, x_scale, offsets, rows, row_weight, group, out_features, eight_bit, bias, activation, workspace):
    return x.new_empty(((x if rows is None else rows).shape[0], out_features), dtype=torch.float16)


@block_norm.register_fake
def _(residual, y, gate, scale, post, post_weight, post_bias, pre, pre_weight, pre_bias, eps, gate_activation, quantize):
    N, K = residual.shape
    h = residual.new_empty((N, (K + 15) // 16 * 16), dtype=torch.int8)[:, :K] if quantize else torch.empty_like(residual)
    return residual.new_empty((N, K)), h, residual.new_empty(N if quantize else 0, dtype=torch.float32)


# What a thread's dispatch keys are where nothing stands between a call and its kernel (the second under inference_mode):
# tracers, dispatch modes and function transforms each add theirs.
_NOTHING_BETWEEN = {
    torch._C.DispatchKeySet(torch._C.DispatchKey.BackendSelect).raw_repr(),
    (torch._C.DispatchKeySet(torch._C.DispatchKey.BackendSelect) |
     torch._C.DispatchKeySet(torch._C.DispatchKey.ADInplaceOrView)).raw_repr(),
}
_PLAIN_VALUES = {type(None), bool, int, float, str}
_PLAIN_TENSORS = {torch.Tensor, torch.nn.Parameter}


def _seen(args) -> bool:
    """Whether anything has to see the call as an operator: a compiler, a tracer, a mode, a transform, a tensor subclass,
    autograd, or a view that only the dispatcher resolves. The function itself writes memory that none of them knows of."""
    if (torch.compiler.is_compiling() or torch._C._dispatch_tls_local_include_set().raw_repr() not in _NOTHING_BETWEEN
            or torch._C._len_torch_function_stack()):
        return True
    grad = torch.is_grad_enabled()
    for a in args:
        t = type(a)
        if t not in _PLAIN_VALUES and (t not in _PLAIN_TENSORS or a.is_neg() or (grad and a.requires_grad)):
            return True
    return False


def _call(op, plain, *args):
    """The operator where anything has to see it; else the function itself, which spares an eager decode step the
    dispatcher (a small layer's kernels take less time than it)."""
    return op(*args) if _seen(args) else plain(*args)


def _rows_of(x: torch.Tensor, width: int) -> torch.Tensor:
    """x [*, width] as fp16 [N, width] with unit inner stride and rows apart from each other."""
    if x.shape[-1] != width:
        raise ValueError(f"expected {width} features, got {x.shape[-1]}")
    if x.dim() != 2:
        x = x.reshape(-1, width)
    ld, inner = x.stride()
    if x.dtype is not torch.float16 or inner != 1 or (ld < width and x.shape[0] > 1):
        x = x.to(torch.float16).contiguous()
    return x


def _codes_of(x: torch.Tensor, width: int) -> torch.Tensor:
    """8-bit tokens [N, width]: rows are padded in memory, so a wrong width would not show by their stride."""
    if x.dim() != 2 or x.shape[1] != width:
        raise ValueError(f"expected 8-bit tokens [N, {width}], got {tuple(x.shape)}")
    return x


Tokens = Union[torch.Tensor, Tuple[torch.Tensor, torch.Tensor]]


class SparseLinearQ(SparseLinear):
    """``act(x W^T + b) (+ residual)`` with W pruned by ``mask`` and held in 8 bits with a scale per output feature,
    x quantised to 8 bits with a scale per token.

    weight: int8 [out_features, in_features]; scale: fp32 [out_features]; the rest as SparseLinear. The input is an
    fp16 tensor, or the pair of int8 tokens [N, in_features] and their scales [N] that BlockNorm gives. Calls and
    captured graphs may overlap as SparseLinear's may."""

    def __init__(self, weight: torch.Tensor, mask, scale: torch.Tensor, bias: Optional[torch.Tensor] = None,
                 activation: str = "none", device: Optional[int] = None):
        torch.nn.Module.__init__(self)
        if activation not in usp.ACTIVATIONS:
            raise ValueError(f"activation must be one of {sorted(usp.ACTIVATIONS)}")
        if weight.dtype != torch.int8:
            raise TypeError("weight must be int8 (quantize_rows makes it from a float weight)")
        dev = torch.cuda.current_device() if device is None else int(device)
        m = mask.detach().cpu().numpy() if isinstance(mask, torch.Tensor) else np.asarray(mask)
        self.matrix = usp.SparseMatrixQ(weight.detach().cpu().contiguous().numpy(), np.ascontiguousarray(m != 0),
                                        scale.detach().float().cpu().numpy(), dev)
        self._set_up(weight.shape, bias, activation, dev)

    @classmethod
    def from_linear(cls, linear: torch.nn.Linear, mask, activation: str = "none") -> "SparseLinearQ":
        dev = linear.weight.device.index if linear.weight.is_cuda else None
        codes, scale = quantize_rows(linear.weight, mask)
        return cls(codes, mask, scale, linear.bias, activation, dev)

    def _stream(self) -> int:
        return usp.current_stream_handle(self.matrix.device)

    def forward(self, x: Tokens, residual: Optional[torch.Tensor] = None) -> torch.Tensor:
        x, x_scale = x if isinstance(x, tuple) else (x, None)
        x2 = _rows_of(x, self.in_features) if x_scale is None else _codes_of(x, self.in_features)
        N = x2.shape[0]
        if N == 0:
            return x.new_empty((*x.shape[:-1], self.out_features), dtype=torch.float16)
        r2 = None if residual is None else _rows_of(residual, self.out_features)
        if r2 is not None and r2.shape[0] != N:
            raise ValueError("residual must have one row per token")
        y = _call(sparse_linear_q, _linear_q, x2, x_scale, self.matrix.handle, self.out_features, self._buffers["bias"],
                  r2, usp.ACTIVATIONS[self.activation], _operand(self.workspace(N), x2))
        return y if x.dim() == 2 else y.reshape(*x.shape[:-1], self.out_features)


class SparseExperts(SparseLinear):
    """A linear layer with a pruned weight for each expert, on rows that are sorted by expert.

    weights: E tensors [out_features, in_features], fp16, or int8 with ``scales`` (E fp32 vectors [out_features]);
    masks: E arrays of that shape; bias: [E, out_features] or None; activation as SparseLinear."""

    def __init__(self, weights, masks, scales=None, bias: Optional[torch.Tensor] = None, activation: str = "none",
                 device: Optional[int] = None):
        torch.nn.Module.__init__(self)
        if activation not in usp.ACTIVATIONS:
            raise ValueError(f"activation must be one of {sorted(usp.ACTIVATIONS)}")
        if len(masks) != len(weights) or (scales is not None and len(scales) != len(weights)):
            raise ValueError("weights, masks and scales must have one entry per expert")
        if bias is not None and tuple(bias.shape) != (len(weights), weights[0].shape[0]):
            raise ValueError("bias must be [experts, out_features]")
        dev = torch.cuda.current_device() if device is None else int(device)
        experts = []
        for e, w in enumerate(weights):
            m = masks[e].detach().cpu().numpy() if isinstance(masks[e], torch.Tensor) else np.asarray(masks[e])
            m = np.ascontiguousarray(m != 0)
            if scales is None:
                w16 = w.detach().to(torch.float16).cpu().contiguous().numpy().view(np.uint16)
                experts.append(usp.SparseMatrix(w16, m, dev))
            else:
                if w.dtype != torch.int8:
                    raise TypeError("weights with scales must be int8 (quantize_rows makes them from float weights)")
                experts.append(usp.SparseMatrixQ(w.detach().cpu().contiguous().numpy(), m,
                                                 scales[e].detach().float().cpu().numpy(), dev))
        self.matrix = usp.ExpertGroup(experts)
        self.eight_bit = scales is not None
        self._set_up(weights[0].shape, bias, activation, dev)

    @classmethod
    def from_linear(cls, linear, mask, activation: str = "none"):
        raise TypeError("SparseExperts is made from the experts' weights")

    def _stream(self) -> int:
        return usp.current_stream_handle(self.matrix.device)

    def forward(self, x: Tokens, offsets: torch.Tensor, rows: Optional[torch.Tensor] = None,
                row_weight: Optional[torch.Tensor] = None) -> torch.Tensor:
        """x: [*, in_features] fp16 (or 8-bit tokens and scales, for 8-bit experts); offsets: int32 [E + 1] on the
        GPU; rows: int32 [T], x's row for each row of the result (default: its own); row_weight: fp32 [T]. Rows
        outside the offsets' range are zeros."""
        x, x_scale = x if isinstance(x, tuple) else (x, None)
        if x_scale is not None and not self.eight_bit:
            raise TypeError("8-bit tokens need 8-bit experts")
        if offsets.shape[0] != len(self.matrix.experts) + 1:
            raise ValueError("offsets must have one entry more than there are experts")
        x2 = _rows_of(x, self.in_features) if x_scale is None else _codes_of(x, self.in_features)
        T = x2.shape[0] if rows is None else rows.shape[0]
        if T == 0 or x2.shape[0] == 0:
            return x2.new_zeros((T, self.out_features), dtype=torch.float16)
        return _call(sparse_experts, _experts, x2, x_scale, offsets, rows, row_weight, self.matrix.handle,
                     self.out_features, self.eight_bit, self._buffers["bias"], usp.ACTIVATIONS[self.activation],
                     _operand(self.workspace(T), x2))

    def extra_repr(self) -> str:
        return (f"experts={len(self.matrix.experts)}, in_features={self.in_features}, "
                f"out_features={self.out_features}, eight_bit={self.eight_bit}, bias={self.bias is not None}, "
                f"activation={self.activation}")


class BlockNorm(torch.nn.Module):
    """The norms around a block: ``r = residual + scale * act(gate) * post(y)`` and ``h = pre(r)``.

    post, pre: "none", "rms" or "layer"; weights and biases are fp16 buffers of ``features`` entries (ones and zeros
    until loaded; biases for "layer" only); gate_activation: "none", "sigmoid", "tanh" or "silu"."""

    def __init__(self, features: int, post: str = "none", pre: str = "rms", scale: float = 1.0, eps: float = 1e-5,
                 gate_activation: str = "none", device=None):
        super().__init__()
        if post not in usp.NORMS or pre not in usp.NORMS:
            raise ValueError(f"post and pre must be one of {sorted(usp.NORMS)}")
        if gate_activation not in usp.GATES:
            raise ValueError(f"gate_activation must be one of {sorted(usp.GATES)}")
        self.features, self.post, self.pre = features, post, pre
        self.scale, self.eps, self.gate_activation = scale, eps, gate_activation
        dev = "cuda" if device is None else f"cuda:{device}" if isinstance(device, int) else device
        for side, kind in (("post", post), ("pre", pre)):
            make = lambda on, fill: torch.full((features,), fill, dtype=torch.float16, device=dev) if on else None  # noqa: E731
            self.register_buffer(side + "_weight", make(kind != "none", 1.0))
            self.register_buffer(side + "_bias", make(kind == "layer", 0.0))

    def forward(self, residual: torch.Tensor, y: Optional[torch.Tensor] = None, gate: Optional[torch.Tensor] = None,
                quantize: bool = False):
        """(r, h): both as residual, or with quantize h as the pair of int8 tokens [N, features] and scales [N].
        Without y (the first block's norm) r is residual and post is not applied. gate: [features], or a row for each of
        residual's."""
        shape = residual.shape
        r2 = _rows_of(residual, self.features)
        y2 = None if y is None else _rows_of(y, self.features)
        g2 = gate
        if gate is not None and gate.dim() != 1:
            g2 = _rows_of(gate, self.features)
        elif gate is not None and (gate.dtype is not torch.float16 or gate.stride(0) != 1):
            g2 = gate.to(torch.float16).contiguous()
        if g2 is not None and g2.shape[-1] != self.features:
            raise ValueError(f"expected a gate of {self.features} features, got {g2.shape[-1]}")
        if r2.shape[0] == 0:
            h = (r2.to(torch.int8), r2.new_empty(0, dtype=torch.float32)) if quantize else r2.reshape(shape)
            return r2.reshape(shape), h
        v = self._buffers  # each attribute of a module costs a search
        r, h, h_scale = _call(block_norm, _block_norm, r2, y2, g2, self.scale, "none" if y is None else self.post,
                              v["post_weight"], v["post_bias"], self.pre, v["pre_weight"], v["pre_bias"], self.eps,
                              self.gate_activation, quantize)
        if len(shape) != 2:
            r, h = r.reshape(shape), h if quantize else h.reshape(shape)
        return r, (h, h_scale) if quantize else h

    def extra_repr(self) -> str:
        return (f"{self.features}, post={self.post}, pre={self.pre}, scale={self.scale}, eps={self.eps}, "
                f"gate_activation={self.gate_activation}")
