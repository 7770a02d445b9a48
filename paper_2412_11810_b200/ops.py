"""Sequence-model operators on torch tensors: argument checks, buffers and streams around the C ABI of include/snn.h.

    h, last, kept = gated_scan(x, gate, state, keep="int8")     # recurrence with learned gates, [T][B][N]
    dx, dgate, dstate = gated_scan_backward(kept, dh, dlast)
    h, state = gated_scan_step(x, gate, state)                  # one token
    packed = pack_activation(x, "int8"); x = unpack_activation(packed)
    loss, row_loss, lse = vocab_loss(x, w_out, targets)         # soft-max cross entropy of x w_out, logits never stored
    dx, dw = vocab_loss_backward(x, w_out, targets, lse)

Gradients are explicit, as in the training step: nothing is recorded for autograd.  Work is launched on the current torch
stream of the tensors' device and the calls return without waiting; they can be captured into a CUDA graph.  Arguments
that do not fit raise ValueError before anything is launched; a status of the library raises `binding.SnnError`.
"""
from __future__ import annotations

import contextlib
from dataclasses import dataclass
from typing import Optional, Tuple

import torch

from . import binding as sb

SCAN_CHUNK = sb.SNN_SCAN_CHUNK   # steps between kept states
KEEP_GROUP = sb.SNN_KEEP_GROUP   # values that share a scale
_DTYPES = {torch.float32: sb.SNN_DTYPE_FP32, torch.bfloat16: sb.SNN_DTYPE_BF16, torch.float16: sb.SNN_DTYPE_FP16}
_MODES = {"sigmoid": sb.SNN_SCAN_SIGMOID, "direct": sb.SNN_SCAN_DIRECT}
_FORMATS = {"int8": sb.SNN_KEEP_INT8, "e4m3": sb.SNN_KEEP_E4M3}
_INT32_MAX = 2 ** 31 - 1


def _need(ok: bool, message: str) -> None:
    if not ok:
        raise ValueError(message)


def _need_values(t: torch.Tensor, name: str, dim: int) -> None:
    _need(isinstance(t, torch.Tensor) and t.is_cuda, f"{name}: a CUDA tensor is required")
    _need(t.dtype in _DTYPES, f"{name}: dtype {t.dtype} is not fp32, bf16 or fp16")
    _need(t.dim() == dim, f"{name}: {dim} dimensions are required, got {t.dim()}")
    _need(t.shape[-1] <= 1 or t.stride(-1) == 1, f"{name}: the last dimension has to be contiguous")


def _need_like(t: torch.Tensor, name: str, like: torch.Tensor, shape, dtype, dense: bool = True) -> None:
    _need(isinstance(t, torch.Tensor) and t.device == like.device, f"{name}: a tensor on {like.device} is required")
    _need(t.dtype == dtype, f"{name}: dtype {t.dtype} instead of {dtype}")
    _need(tuple(t.shape) == tuple(shape), f"{name}: shape {tuple(t.shape)} instead of {tuple(shape)}")
    if dense:
        _need(t.is_contiguous(), f"{name}: has to be contiguous")
    else:
        _need(t.shape[-1] <= 1 or t.stride(-1) == 1, f"{name}: the last dimension has to be contiguous")


def _on(device: torch.device):
    """The library launches on the current device."""
    return contextlib.nullcontext() if device.index == torch.cuda.current_device() else torch.cuda.device(device)


def _stream(device: torch.device) -> int:
    return torch.cuda.current_stream(device).cuda_stream


def _ptr(t: Optional[torch.Tensor]):
    return None if t is None else t.data_ptr()


# ---- activations in 8 bits -----------------------------------------------------------------------------------
@dataclass(frozen=True)
class PackedActivation:
    """Values in 8 bits: `codes` uint8 of the values' shape, `scales` uint8 with one byte per group of 64 values of the
    last dimension (the power of two 2^(byte - 127); 255 marks a group with an infinity or a NaN)."""
    codes: torch.Tensor
    scales: torch.Tensor
    format: str
    dtype: torch.dtype


def _empty_codes(shape, device) -> Tuple[torch.Tensor, torch.Tensor]:
    groups = -(-shape[-1] // KEEP_GROUP)
    return (torch.empty(shape, dtype=torch.uint8, device=device),
            torch.empty((*shape[:-1], groups), dtype=torch.uint8, device=device))


def pack_activation(x: torch.Tensor, format: str = "int8") -> PackedActivation:
    """Encodes a tensor [..., N] to 8 bits ("int8" or "e4m3").  The leading dimensions have to collapse into one without a
    copy, the last one has to be contiguous."""
    _need(isinstance(x, torch.Tensor) and x.is_cuda, "x: a CUDA tensor is required")
    _need(x.dtype in _DTYPES, f"x: dtype {x.dtype} is not fp32, bf16 or fp16")
    _need(x.dim() >= 1, "x: at least one dimension is required")
    _need(format in _FORMATS, f"format: {format!r} is not one of {sorted(_FORMATS)}")
    n = x.shape[-1]
    _need(n <= _INT32_MAX, "x: the last dimension is too long")
    try:
        rows = x.view(-1, n) if x.numel() else x.reshape(0, max(n, 1))
    except RuntimeError:
        raise ValueError("x: the leading dimensions have to collapse into one without a copy") from None
    _need(n <= 1 or rows.numel() == 0 or rows.stride(1) == 1, "x: the last dimension has to be contiguous")
    with _on(x.device):
        codes, scales = _empty_codes(x.shape, x.device)
        if x.numel():
            sb.snn_activation_pack(rows.data_ptr(), _DTYPES[x.dtype], rows.shape[0], n, rows.stride(0), _FORMATS[format],
                                   codes.data_ptr(), scales.data_ptr(), _stream(x.device))
    return PackedActivation(codes, scales, format, x.dtype)


def unpack_activation(packed: PackedActivation, dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """The values that `packed` stands for, in `dtype` (that of the packed tensor by default)."""
    dtype = packed.dtype if dtype is None else dtype
    _need(dtype in _DTYPES, f"dtype: {dtype} is not fp32, bf16 or fp16")
    _need(packed.format in _FORMATS, f"format: {packed.format!r} is not one of {sorted(_FORMATS)}")
    codes, n = packed.codes, packed.codes.shape[-1]
    _need(codes.is_cuda, "codes: a CUDA tensor is required")
    _need_like(codes, "codes", codes, codes.shape, torch.uint8)
    _need_like(packed.scales, "scales", codes, (*codes.shape[:-1], -(-n // KEEP_GROUP)), torch.uint8)
    with _on(codes.device):
        out = torch.empty(codes.shape, dtype=dtype, device=codes.device)
        if codes.numel():
            sb.snn_activation_unpack(codes.data_ptr(), packed.scales.data_ptr(), _FORMATS[packed.format],
                                     codes.numel() // n, n, out.data_ptr(), _DTYPES[dtype], n, _stream(codes.device))
    return out


# ---- gated linear recurrence ---------------------------------------------------------------------------------
@dataclass(frozen=True)
class ScanKept:
    """What a forward pass of `gated_scan` kept for the backward pass: the state before every 64th step and the inputs,
    each as the caller's own tensor (do not change it before the backward pass) or in 8 bits."""
    shape: Tuple[int, int, int]
    dtype: torch.dtype
    mode: str
    states: torch.Tensor
    lengths: Optional[torch.Tensor]
    x: object                      # torch.Tensor or PackedActivation
    gate: object


def _scan_args(shape, dtype: torch.dtype, mode: str, lengths: Optional[torch.Tensor]) -> sb.snn_scan_args:
    a = sb.snn_scan_args()
    a.T, a.B, a.N = shape
    a.dtype, a.mode, a.lengths = _DTYPES[dtype], _MODES[mode], _ptr(lengths)
    return a


def _scan_workspace(a: sb.snn_scan_args, backward: bool, device: torch.device) -> Optional[torch.Tensor]:
    n = sb.snn_scan_workspace(a, backward)
    if n == 0:
        return None
    ws = torch.empty(n, dtype=torch.uint8, device=device)
    a.workspace, a.workspace_bytes = ws.data_ptr(), n
    return ws


def _set_strided(a, name: str, t: torch.Tensor) -> None:
    setattr(a, name, t.data_ptr())
    s = getattr(a, name + "_stride")
    s[0], s[1] = t.stride(0), t.stride(1)


def gated_scan(x: torch.Tensor, gate: torch.Tensor, state: Optional[torch.Tensor] = None, *,
               lengths: Optional[torch.Tensor] = None, mode: str = "sigmoid", keep: Optional[str] = None,
               keep_gate: Optional[str] = None):
    """The gated linear recurrence over x, gate [T][B][N] (fp32, bf16 or fp16; any strides with contiguous channels):

        mode "sigmoid":  h_t = a_t h_{t-1} + (1 - a_t) x_t,  a_t = sigmoid(gate_t)
        mode "direct":   h_t = gate_t h_{t-1} + x_t

    state: fp32 [B][N], the state before the first step (zero if None).  lengths: int32 [B], sample b ends after
    lengths[b] steps (clamped to [0, T]); h is zero behind that and nothing there is read.
    keep: None keeps nothing; "raw" keeps references to x and gate, "int8" and "e4m3" an 8-bit copy of each, made in the
    same pass; keep_gate overrides the format of the gate.  In mode "direct" the gate, a decay close to one, is kept raw.
    Returns (h [T][B][N], last state fp32 [B][N], what was kept for `gated_scan_backward` or None)."""
    _need_values(x, "x", 3)
    _need_values(gate, "gate", 3)
    _need_like(gate, "gate", x, x.shape, x.dtype, dense=False)
    _need(mode in _MODES, f"mode: {mode!r} is not one of {sorted(_MODES)}")
    for name, f in (("keep", keep), ("keep_gate", keep_gate)):
        _need(f is None or f == "raw" or f in _FORMATS, f"{name}: {f!r} is not None, 'raw' or one of {sorted(_FORMATS)}")
    _need(keep is not None or keep_gate is None, "keep_gate: needs keep")
    T, B, N = x.shape
    _need(T < 2 ** 30 and B <= _INT32_MAX and N <= _INT32_MAX, "x: too large")
    if keep_gate is None:
        keep_gate = "raw" if mode == "direct" else keep
    _need(mode != "direct" or keep_gate in (None, "raw"), "keep_gate: the gate of mode 'direct' can only be kept raw")
    if state is not None:
        _need_like(state, "state", x, (B, N), torch.float32)
    if lengths is not None:
        _need_like(lengths, "lengths", x, (B,), torch.int32)
    with _on(x.device):
        h = torch.empty((T, B, N), dtype=x.dtype, device=x.device)
        last = torch.empty((B, N), dtype=torch.float32, device=x.device)
        a = _scan_args((T, B, N), x.dtype, mode, lengths)
        _set_strided(a, "x", x)
        _set_strided(a, "gate", gate)
        _set_strided(a, "h", h)
        a.state, a.last = _ptr(state), last.data_ptr()
        kept = None
        if keep is not None:
            states = torch.empty((-(-T // SCAN_CHUNK), B, N), dtype=torch.float32, device=x.device)
            a.states = states.data_ptr()
            held = {}
            for name, t, f in (("x", x, keep), ("gate", gate, keep_gate)):
                if f == "raw":
                    held[name] = t
                    continue
                codes, scales = _empty_codes((T, B, N), x.device)
                held[name] = PackedActivation(codes, scales, f, x.dtype)
                setattr(a, name + "_format", _FORMATS[f])
                setattr(a, name + "_codes", codes.data_ptr())
                setattr(a, name + "_scales", scales.data_ptr())
            kept = ScanKept((T, B, N), x.dtype, mode, states, lengths, held["x"], held["gate"])
        ws = _scan_workspace(a, False, x.device)  # noqa: F841  (held until the launch)
        sb.snn_scan_forward(a, _stream(x.device))
    return h, last, kept


def gated_scan_step(x: torch.Tensor, gate: torch.Tensor, state: Optional[torch.Tensor] = None, *, mode: str = "sigmoid",
                    inplace: bool = False) -> Tuple[torch.Tensor, torch.Tensor]:
    """One step of `gated_scan` for x, gate [B][N]: returns (h [B][N], new state fp32 [B][N]).  inplace: the new state
    replaces the old one in `state`'s memory."""
    _need_values(x, "x", 2)
    _need_values(gate, "gate", 2)
    _need_like(gate, "gate", x, x.shape, x.dtype, dense=False)
    _need(mode in _MODES, f"mode: {mode!r} is not one of {sorted(_MODES)}")
    _need(state is not None or not inplace, "inplace: needs a state")
    if state is not None:
        _need_like(state, "state", x, x.shape, torch.float32)
    B, N = x.shape
    with _on(x.device):
        h = torch.empty((B, N), dtype=x.dtype, device=x.device)
        last = state if inplace else torch.empty((B, N), dtype=torch.float32, device=x.device)
        a = _scan_args((1, B, N), x.dtype, mode, None)
        a.x, a.gate, a.h, a.state, a.last = x.data_ptr(), gate.data_ptr(), h.data_ptr(), _ptr(state), last.data_ptr()
        a.x_stride[1], a.gate_stride[1], a.h_stride[1] = x.stride(0), gate.stride(0), N
        sb.snn_scan_forward(a, _stream(x.device))
    return h, last


def gated_scan_backward(kept: ScanKept, dh: torch.Tensor, dlast: Optional[torch.Tensor] = None):
    """Gradients of a loss by x, gate and the state of a `gated_scan(..., keep=...)`, from those by h (dh, of x's type,
    [T][B][N]) and by the last state (dlast, fp32 [B][N], zero if None).  Where the inputs were kept in 8 bits, they are
    the gradients at the values those stand for, with the states of each chunk of 64 steps recomputed from its kept
    state.  Returns (dx, dgate of x's type, dstate fp32)."""
    _need(isinstance(kept, ScanKept), "kept: what gated_scan(..., keep=...) returned is required")
    T, B, N = kept.shape
    like = kept.states
    _need_like(dh, "dh", like, (T, B, N), kept.dtype, dense=False)
    if dlast is not None:
        _need_like(dlast, "dlast", like, (B, N), torch.float32)
    with _on(like.device):
        dx = torch.empty((T, B, N), dtype=kept.dtype, device=like.device)
        dgate = torch.empty_like(dx)
        dstate = torch.empty((B, N), dtype=torch.float32, device=like.device)
        a = _scan_args((T, B, N), kept.dtype, kept.mode, kept.lengths)
        for name in ("x", "gate"):
            t = getattr(kept, name)
            if isinstance(t, PackedActivation):
                setattr(a, name + "_format", _FORMATS[t.format])
                setattr(a, name + "_codes", t.codes.data_ptr())
                setattr(a, name + "_scales", t.scales.data_ptr())
            else:
                _set_strided(a, name, t)
        _set_strided(a, "dh", dh)
        _set_strided(a, "dx", dx)
        _set_strided(a, "dgate", dgate)
        a.states, a.dlast, a.dstate = kept.states.data_ptr(), _ptr(dlast), dstate.data_ptr()
        ws = _scan_workspace(a, True, like.device)  # noqa: F841
        sb.snn_scan_backward(a, _stream(like.device))
    return dx, dgate, dstate


# ---- soft-max cross entropy over a vocabulary ------------------------------------------------------------------
def _vocab_args(x, w_out, targets, scale: float, ignore_index: int):
    _need_values(x, "x", 2)
    _need(isinstance(w_out, torch.Tensor) and w_out.device == x.device, f"w_out: a tensor on {x.device} is required")
    _need(w_out.dtype == x.dtype, f"w_out: dtype {w_out.dtype} instead of {x.dtype}")
    rows, dim = x.shape
    _need(w_out.dim() == 2 and w_out.shape[0] == dim, f"w_out: shape {tuple(w_out.shape)} instead of ({dim}, classes)")
    classes = w_out.shape[1]
    _need(dim >= 1 and classes >= 1, "w_out: at least one feature and one class are required")
    _need(max(rows, dim, classes) < 2 ** 30, "x, w_out: too large")
    _need(rows <= 1 or x.stride(0) >= dim, "x: rows overlap")
    by_feature = (classes == 1 or w_out.stride(1) == 1) and (dim == 1 or w_out.stride(0) >= classes)
    by_class = (dim == 1 or w_out.stride(0) == 1) and (classes == 1 or w_out.stride(1) >= dim)
    _need(by_feature or by_class, "w_out: its features or its classes have to be contiguous, without overlap")
    _need(isinstance(targets, torch.Tensor) and targets.device == x.device, f"targets: a tensor on {x.device} is required")
    _need(targets.dtype in (torch.int32, torch.int64), f"targets: dtype {targets.dtype} is not int32 or int64")
    _need(tuple(targets.shape) == (rows,), f"targets: shape {tuple(targets.shape)} instead of ({rows},)")
    _need(targets.is_contiguous(), "targets: has to be contiguous")
    _need(-2 ** 63 <= ignore_index < 2 ** 63, "ignore_index: does not fit 64 bits")
    _need(abs(scale) <= 3.4e38, "scale: has to be finite")
    a = sb.snn_vocab_loss_args()
    a.rows, a.dim, a.classes, a.dtype = rows, dim, classes, _DTYPES[x.dtype]
    a.x, a.x_stride, a.w = x.data_ptr(), x.stride(0), w_out.data_ptr()
    a.w_layout, a.w_stride = (sb.SNN_W_BY_FEATURE, w_out.stride(0)) if by_feature else (sb.SNN_W_BY_CLASS, w_out.stride(1))
    a.targets, a.target_bits, a.ignore_index, a.scale = targets.data_ptr(), targets.element_size() * 8, ignore_index, scale
    return a


def vocab_loss(x: torch.Tensor, w_out: torch.Tensor, targets: torch.Tensor, *, scale: float = 1.0, ignore_index: int = -100):
    """Mean soft-max cross entropy of the logits scale * x w_out, which are never stored.

    x: [rows][dim], w_out: [dim][classes] of the same type (fp32, bf16 or fp16), stored by feature (contiguous) or by class
    (`table.t()` of a [classes][dim] table).  targets: int32 or int64 [rows]; rows with ignore_index do not count, any other
    target outside [0, classes) makes its row's loss and the mean NaN.
    Returns (loss, a 0-d tensor; row_loss [rows]; lse [rows], the log-sum-exp that `vocab_loss_backward` needs), all fp32,
    with zeros for rows that do not count."""
    a = _vocab_args(x, w_out, targets, scale, ignore_index)
    with _on(x.device):
        out = torch.empty((2, a.rows), dtype=torch.float32, device=x.device)
        loss = torch.empty((), dtype=torch.float32, device=x.device)
        a.row_loss, a.lse, a.loss = out[0].data_ptr(), out[1].data_ptr(), loss.data_ptr()
        ws = torch.empty(sb.snn_vocab_loss_workspace(a, False), dtype=torch.uint8, device=x.device)
        a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel()
        sb.snn_vocab_loss_forward(a, _stream(x.device))
    return loss, out[0], out[1]


def vocab_loss_backward(x: torch.Tensor, w_out: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor, *, scale: float = 1.0,
                        ignore_index: int = -100, dloss=1.0):
    """Gradients of `vocab_loss` by x and w_out: (dx [rows][dim], dw [dim][classes], stored as w_out is), in their type.
    dloss: the gradient of the loss, a number or an fp32 0-d tensor on the device."""
    a = _vocab_args(x, w_out, targets, scale, ignore_index)
    _need_like(lse, "lse", x, (a.rows,), torch.float32)
    if isinstance(dloss, torch.Tensor):
        _need_like(dloss, "dloss", x, (), torch.float32)
        a.dloss, a.dloss_device = 1.0, dloss.data_ptr()
    else:
        a.dloss = dloss
    with _on(x.device):
        dx = torch.empty((a.rows, a.dim), dtype=x.dtype, device=x.device)
        if a.w_layout == sb.SNN_W_BY_FEATURE:
            dw = torch.empty((a.dim, a.classes), dtype=x.dtype, device=x.device)
            a.dw_stride = a.classes
        else:
            dw = torch.empty((a.classes, a.dim), dtype=x.dtype, device=x.device).t()
            a.dw_stride = a.dim
        a.lse, a.dx, a.dx_stride, a.dw = lse.data_ptr(), dx.data_ptr(), a.dim, dw.data_ptr()
        ws = torch.empty(sb.snn_vocab_loss_workspace(a, True), dtype=torch.uint8, device=x.device)
        a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel()
        sb.snn_vocab_loss_backward(a, _stream(x.device))
    return dx, dw
