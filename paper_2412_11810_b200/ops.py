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
_KEEPS = {"raw": sb.SNN_KEEP_RAW, **_FORMATS}
_INT32_MAX = 2 ** 31 - 1
_WIDEST = 2 ** 31 - 64           # channels: the last group of 64 ends within 32 bits


# The checks below run before every launch, and small calls take microseconds: conditions are tested in place, and messages
# are put together only when one does not hold.
def _values(t: torch.Tensor, name: str, dim: int) -> None:
    if not (isinstance(t, torch.Tensor) and t.is_cuda):
        raise ValueError(f"{name}: a CUDA tensor is required")
    if t.dtype not in _DTYPES:
        raise ValueError(f"{name}: dtype {t.dtype} is not fp32, bf16 or fp16")
    if t.dim() != dim:
        raise ValueError(f"{name}: {dim} dimensions are required, got {t.dim()}")
    if not t.is_contiguous() and t.shape[-1] > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: the last dimension has to be contiguous")


def _like(t: torch.Tensor, name: str, like: torch.Tensor, shape, dtype, dense: bool = True) -> None:
    if not isinstance(t, torch.Tensor) or t.get_device() != like.get_device():
        raise ValueError(f"{name}: a tensor on {like.device} is required")
    if t.dtype is not dtype:
        raise ValueError(f"{name}: dtype {t.dtype} instead of {dtype}")
    if t.shape != shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)} instead of {tuple(shape)}")
    if not t.is_contiguous():
        if dense:
            raise ValueError(f"{name}: has to be contiguous")
        if t.shape[-1] > 1 and t.stride(-1) != 1:
            raise ValueError(f"{name}: the last dimension has to be contiguous")


def _choice(value, name: str, choices) -> None:
    if value not in choices:
        raise ValueError(f"{name}: {value!r} is not one of {sorted(choices)}")


def _on(t: torch.Tensor):
    """The library launches on the current device."""
    return _HERE if t.get_device() == torch.cuda.current_device() else torch.cuda.device(t.device)


_HERE = contextlib.nullcontext()
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(t: torch.Tensor) -> int:
    """The handle of the current stream of a tensor's device."""
    return _raw_stream(t.get_device()) if _raw_stream else torch.cuda.current_stream(t.device).cuda_stream


def _dense(t: torch.Tensor) -> torch.Tensor:
    """A new contiguous tensor of the same shape and type (empty_like is the cheaper call where it can be used)."""
    return torch.empty_like(t) if t.is_contiguous() else t.new_empty(t.shape)


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


def _empty_codes(like: torch.Tensor, shape) -> Tuple[torch.Tensor, torch.Tensor]:
    return (like.new_empty(shape, dtype=torch.uint8),
            like.new_empty((*shape[:-1], -(-shape[-1] // KEEP_GROUP)), dtype=torch.uint8))


def pack_activation(x: torch.Tensor, format: str = "int8") -> PackedActivation:
    """Encodes a tensor [..., N] to 8 bits ("int8" or "e4m3").  The leading dimensions have to collapse into one without a
    copy, the last one has to be contiguous."""
    if not (isinstance(x, torch.Tensor) and x.is_cuda):
        raise ValueError("x: a CUDA tensor is required")
    if x.dtype not in _DTYPES:
        raise ValueError(f"x: dtype {x.dtype} is not fp32, bf16 or fp16")
    if x.dim() < 1 or x.shape[-1] > _WIDEST:
        raise ValueError("x: at least one dimension is required, the last one at most 2^31 - 64")
    _choice(format, "format", _FORMATS)
    n, count = x.shape[-1], x.numel()
    stride = n
    if not x.is_contiguous():
        try:
            rows = x.view(-1, n) if count else x
        except RuntimeError:
            raise ValueError("x: the leading dimensions have to collapse into one without a copy") from None
        if count and n > 1 and rows.stride(-1) != 1:
            raise ValueError("x: the last dimension has to be contiguous")
        stride = rows.stride(0)
    with _on(x):
        codes, scales = _empty_codes(x, x.shape)
        if count:
            sb.snn_activation_pack(x.data_ptr(), _DTYPES[x.dtype], count // n, n, stride, _FORMATS[format], codes.data_ptr(),
                                   scales.data_ptr(), _stream(x))
    return PackedActivation(codes, scales, format, x.dtype)


def unpack_activation(packed: PackedActivation, dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """The values that `packed` stands for, in `dtype` (that of the packed tensor by default)."""
    dtype = packed.dtype if dtype is None else dtype
    if dtype not in _DTYPES:
        raise ValueError(f"dtype: {dtype} is not fp32, bf16 or fp16")
    _choice(packed.format, "format", _FORMATS)
    codes = packed.codes
    if not (isinstance(codes, torch.Tensor) and codes.is_cuda):
        raise ValueError("codes: a CUDA tensor is required")
    if codes.dim() < 1 or codes.shape[-1] > _WIDEST:
        raise ValueError("codes: at least one dimension is required, the last one at most 2^31 - 64")
    n, count = codes.shape[-1], codes.numel()
    _like(codes, "codes", codes, codes.shape, torch.uint8)
    _like(packed.scales, "scales", codes, (*codes.shape[:-1], -(-n // KEEP_GROUP)), torch.uint8)
    with _on(codes):
        out = torch.empty_like(codes, dtype=dtype)
        if count:
            sb.snn_activation_unpack(codes.data_ptr(), packed.scales.data_ptr(), _FORMATS[packed.format], count // n, n,
                                     out.data_ptr(), _DTYPES[dtype], n, _stream(codes))
    return out


# ---- gated linear recurrence ---------------------------------------------------------------------------------
@dataclass(frozen=True)
class ScanKept:
    """What a forward pass of `gated_scan` kept for the backward pass: the state before every 64th step and the inputs,
    each as the caller's own tensor (do not change it before the backward pass, nor `lengths`) or in 8 bits.  What lies
    behind a sequence's end is not kept."""
    shape: Tuple[int, int, int]
    dtype: torch.dtype
    mode: str
    states: torch.Tensor
    lengths: Optional[torch.Tensor]
    x: object                      # torch.Tensor or PackedActivation
    gate: object


def _scan_workspace(a: sb.snn_scan_args, backward: bool, like: torch.Tensor) -> Optional[torch.Tensor]:
    if a.B * a.N >= 149 * 64 or a.T < 512:   # only few channels and many steps need one
        return None
    n = sb.snn_scan_workspace(a, backward)
    if n == 0:
        return None
    ws = like.new_empty(n, dtype=torch.uint8)
    a.workspace, a.workspace_bytes = ws.data_ptr(), n
    return ws


def gated_scan(x: torch.Tensor, gate: torch.Tensor, state: Optional[torch.Tensor] = None, *,
               lengths: Optional[torch.Tensor] = None, mode: str = "sigmoid", keep: Optional[str] = None,
               keep_gate: Optional[str] = None):
    """The gated linear recurrence over x, gate [T][B][N] (fp32, bf16 or fp16; any strides with contiguous channels):

        mode "sigmoid":  h_t = a_t h_{t-1} + (1 - a_t) x_t,  a_t = sigmoid(gate_t)
        mode "direct":   h_t = gate_t h_{t-1} + x_t; the gate is a decay, at most one in magnitude: steps are combined
                         before the state they start from is known, and where a product of consecutive gates leaves
                         the range of fp32 the result may not be finite, even if that of step after step is

    state: fp32 [B][N], the state before the first step (zero if None).  lengths: int32 [B], sample b ends after
    lengths[b] steps (clamped to [0, T]); h is zero behind that and nothing there is read.
    keep: None keeps nothing; "raw" keeps references to x and gate, "int8" and "e4m3" an 8-bit copy of each, made in the
    same pass; keep_gate overrides the format of the gate.  In mode "direct" the gate, a decay close to one, is kept raw.
    What 8 bits cost the gradients, as norms of their distance to those from raw inputs over 2048 steps of normal x and
    gates with a standard deviation of 1.5 (states held for about ten steps, gates of mean 2, and a hundred, mean 5):
    int8 dx 1.1 and 2.7 %, dgate 1.4 and 2.7 %, dstate 0.5 %; e4m3 dx 1.8 and 4.8 %, dgate 3.6 and 5.9 %, dstate 1.1 %.
    dx owes it to the gate alone (keep_gate="raw": none).  Groups of 64 channels share a scale: a few large ones cost the
    others bits in int8 (every 50th value of x 20 times the others: dgate 2.6 instead of 1.4 %).
    Returns (h [T][B][N], last state fp32 [B][N], what was kept for `gated_scan_backward` or None)."""
    _values(x, "x", 3)
    shape, dtype = x.shape, x.dtype
    _like(gate, "gate", x, shape, dtype, dense=False)
    _choice(mode, "mode", _MODES)
    T, B, N = shape
    if T >= 2 ** 30 or B > _INT32_MAX or N > _WIDEST:
        raise ValueError("x: too large")
    if keep is None:
        if keep_gate is not None:
            raise ValueError("keep_gate: needs keep")
    else:
        _choice(keep, "keep", _KEEPS)
        if keep_gate is None:
            keep_gate = "raw" if mode == "direct" else keep
        _choice(keep_gate, "keep_gate", _KEEPS)
        if mode == "direct" and keep_gate != "raw":
            raise ValueError("keep_gate: the gate of mode 'direct' can only be kept raw")
    if state is not None:
        _like(state, "state", x, (B, N), torch.float32)
    if lengths is not None:
        _like(lengths, "lengths", x, (B,), torch.int32)
    with _on(x):
        h = _dense(x)
        last = x.new_empty((B, N), dtype=torch.float32) if state is None else torch.empty_like(state)
        a = sb.snn_scan_args(T, B, N, _DTYPES[dtype], _MODES[mode], x.data_ptr(), gate.data_ptr(), x.stride()[:2], gate.stride()[:2],
                             _ptr(lengths), _ptr(state), h.data_ptr(), (B * N, N), last.data_ptr())
        kept = None
        if keep is not None:
            states = x.new_empty((-(-T // SCAN_CHUNK), B, N), dtype=torch.float32)
            a.states = states.data_ptr()
            held = {}
            for name, t, f in (("x", x, keep), ("gate", gate, keep_gate)):
                if f == "raw":
                    held[name] = t
                    continue
                codes, scales = _empty_codes(x, shape)
                held[name] = PackedActivation(codes, scales, f, dtype)
                setattr(a, name + "_format", _FORMATS[f])
                setattr(a, name + "_codes", codes.data_ptr())
                setattr(a, name + "_scales", scales.data_ptr())
            kept = ScanKept((T, B, N), dtype, mode, states, lengths, held["x"], held["gate"])
        ws = _scan_workspace(a, False, x)  # noqa: F841  (held until the launch)
        sb.snn_scan_forward(a, _stream(x))
    return h, last, kept


def gated_scan_step(x: torch.Tensor, gate: torch.Tensor, state: Optional[torch.Tensor] = None, *, mode: str = "sigmoid",
                    inplace: bool = False) -> Tuple[torch.Tensor, torch.Tensor]:
    """One step of `gated_scan` for x, gate [B][N]: returns (h [B][N], new state fp32 [B][N]).  inplace: the new state
    replaces the old one in `state`'s memory."""
    _values(x, "x", 2)
    shape, dtype = x.shape, x.dtype
    _like(gate, "gate", x, shape, dtype, dense=False)
    _choice(mode, "mode", _MODES)
    if state is not None:
        _like(state, "state", x, shape, torch.float32)
    elif inplace:
        raise ValueError("inplace: needs a state")
    B, N = shape
    if B > _INT32_MAX or N > _WIDEST:
        raise ValueError("x: too large")
    with _on(x):
        h = _dense(x)
        last = state if inplace else x.new_empty(shape, dtype=torch.float32) if state is None else torch.empty_like(state)
        sb.snn_scan_forward(sb.snn_scan_args(1, B, N, _DTYPES[dtype], _MODES[mode], x.data_ptr(), gate.data_ptr(), (0, x.stride(0)),
                                             (0, gate.stride(0)), None, _ptr(state), h.data_ptr(), (0, N), last.data_ptr()), _stream(x))
    return h, last


def gated_scan_backward(kept: ScanKept, dh: torch.Tensor, dlast: Optional[torch.Tensor] = None):
    """Gradients of a loss by x, gate and the state of a `gated_scan(..., keep=...)`, from those by h (dh, of x's type,
    [T][B][N]) and by the last state (dlast, fp32 [B][N], zero if None).  Where the inputs were kept in 8 bits, they are
    the gradients at the values those stand for, with the states of each chunk of 64 steps recomputed from its kept
    state.  Returns (dx, dgate of x's type, dstate fp32)."""
    if not isinstance(kept, ScanKept):
        raise ValueError("kept: what gated_scan(..., keep=...) returned is required")
    T, B, N = shape = kept.shape
    like = kept.states
    _like(dh, "dh", like, shape, kept.dtype, dense=False)
    if dlast is not None:
        _like(dlast, "dlast", like, (B, N), torch.float32)
    with _on(like):
        dx, dgate = _dense(dh), _dense(dh)
        dstate = like.new_empty((B, N))
        a = sb.snn_scan_args(T, B, N, _DTYPES[kept.dtype], _MODES[kept.mode])
        a.lengths, a.states, a.dlast, a.dstate = _ptr(kept.lengths), like.data_ptr(), _ptr(dlast), dstate.data_ptr()
        for name in ("x", "gate"):
            t = getattr(kept, name)
            if isinstance(t, PackedActivation):
                setattr(a, name + "_format", _FORMATS[t.format])
                setattr(a, name + "_codes", t.codes.data_ptr())
                setattr(a, name + "_scales", t.scales.data_ptr())
            else:
                setattr(a, name, t.data_ptr())
                setattr(a, name + "_stride", t.stride()[:2])
        a.dh, a.dx, a.dgate = dh.data_ptr(), dx.data_ptr(), dgate.data_ptr()
        a.dh_stride, a.dx_stride, a.dgate_stride = dh.stride()[:2], (B * N, N), (B * N, N)
        ws = _scan_workspace(a, True, like)  # noqa: F841
        sb.snn_scan_backward(a, _stream(like))
    return dx, dgate, dstate


# ---- soft-max cross entropy over a vocabulary ------------------------------------------------------------------
def _vocab_args(x, w_out, targets, scale: float, ignore_index: int):
    _values(x, "x", 2)
    rows, dim = x.shape
    if not isinstance(w_out, torch.Tensor) or w_out.get_device() != x.get_device():
        raise ValueError(f"w_out: a tensor on {x.device} is required")
    if w_out.dtype is not x.dtype:
        raise ValueError(f"w_out: dtype {w_out.dtype} instead of {x.dtype}")
    if w_out.dim() != 2 or w_out.shape[0] != dim:
        raise ValueError(f"w_out: shape {tuple(w_out.shape)} instead of ({dim}, classes)")
    classes = w_out.shape[1]
    if dim < 1 or classes < 1:
        raise ValueError("w_out: at least one feature and one class are required")
    if max(rows, dim, classes) >= 2 ** 30:
        raise ValueError("x, w_out: too large")
    if rows > 1 and x.stride(0) < dim:
        raise ValueError("x: rows overlap")
    s0, s1 = w_out.stride()
    by_feature = (classes == 1 or s1 == 1) and (dim == 1 or s0 >= classes)
    if not by_feature and not ((dim == 1 or s0 == 1) and (classes == 1 or s1 >= dim)):
        raise ValueError("w_out: its features or its classes have to be contiguous, without overlap")
    if not isinstance(targets, torch.Tensor) or targets.dtype not in (torch.int32, torch.int64):
        raise ValueError("targets: an int32 or int64 tensor is required")
    _like(targets, "targets", x, (rows,), targets.dtype)
    if not -2 ** 63 <= ignore_index < 2 ** 63:
        raise ValueError("ignore_index: does not fit 64 bits")
    if not abs(scale) <= 2.35e38:
        raise ValueError("scale: has to be at most 2.35e38 in magnitude")
    return sb.snn_vocab_loss_args(rows, dim, classes, _DTYPES[x.dtype], x.data_ptr(), x.stride(0), w_out.data_ptr(), s0 if by_feature else s1,
                                  sb.SNN_W_BY_FEATURE if by_feature else sb.SNN_W_BY_CLASS, targets.element_size() * 8, targets.data_ptr(),
                                  ignore_index, scale)


def _loss_workspace(a: sb.snn_vocab_loss_args, backward: bool, like: torch.Tensor) -> torch.Tensor:
    ws = like.new_empty(sb.snn_vocab_loss_workspace(a, backward), dtype=torch.uint8)
    a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel()
    return ws


def vocab_loss(x: torch.Tensor, w_out: torch.Tensor, targets: torch.Tensor, *, scale: float = 1.0, ignore_index: int = -100):
    """Mean soft-max cross entropy of the logits scale * x w_out, which are never stored.

    x: [rows][dim], w_out: [dim][classes] of the same type (fp32, bf16 or fp16), stored by feature (contiguous) or by class
    (`table.t()` of a [classes][dim] table); 16-bit operands whose rows are not multiples of 16 bytes are copied first.
    targets: int32 or int64 [rows]; rows with ignore_index do not count, any other target outside [0, classes) makes its
    row's loss and the mean NaN.
    Returns (loss, a 0-d tensor; row_loss [rows]; lse [rows], the log-sum-exp that `vocab_loss_backward` needs), all fp32,
    with zeros for rows that do not count.

    Products of fp32 operands are those of fp32 arithmetic (three 16-bit parts of every value, on the tensor cores), of 16-bit
    ones exact; sums are fp32 (of 16-bit products: in the tensor cores' accumulators, which cut what does not fit).
    Workspace: 8 bytes per row and 128 classes (up to four rows: per block), and in fp32 6 bytes per value of x and w."""
    a = _vocab_args(x, w_out, targets, scale, ignore_index)
    with _on(x):
        row_loss = x.new_empty(a.rows, dtype=torch.float32)
        lse, loss = torch.empty_like(row_loss), row_loss.new_empty(())
        a.row_loss, a.lse, a.loss = row_loss.data_ptr(), lse.data_ptr(), loss.data_ptr()
        ws = _loss_workspace(a, False, x)  # noqa: F841  (held until the launch)
        sb.snn_vocab_loss_forward(a, _stream(x))
    return loss, row_loss, lse


def vocab_loss_backward(x: torch.Tensor, w_out: torch.Tensor, targets: torch.Tensor, lse: torch.Tensor, *, scale: float = 1.0,
                        ignore_index: int = -100, dloss=1.0):
    """Gradients of `vocab_loss` by x and w_out: (dx [rows][dim], dw [dim][classes], stored as w_out is), in their type.
    dloss: the gradient of the loss, a number or an fp32 0-d tensor on the device.

    The logits are computed again; their derivatives are rounded to the operands' type before they are multiplied by w and x
    (bf16: to 8 bits, which adds 4e-4 to 6e-4 of their norm to gradients that are themselves rounded to 1.7e-3; fp16: to 11
    bits; fp32: not at all).  Workspace: 512 MB of them at a time at most (less if rows x classes are fewer; at least 256
    classes), a copy of x, in fp32 also one of w of 6 bytes per value, and fp32 sums for dx, several of them where rows x
    dim are few."""
    a = _vocab_args(x, w_out, targets, scale, ignore_index)
    _like(lse, "lse", x, (a.rows,), torch.float32)
    if isinstance(dloss, torch.Tensor):
        _like(dloss, "dloss", x, (), torch.float32)
        a.dloss, a.dloss_device = 1.0, dloss.data_ptr()
    else:
        a.dloss = dloss
    with _on(x):
        dx = _dense(x)
        if a.w_layout == sb.SNN_W_BY_FEATURE:
            dw = x.new_empty((a.dim, a.classes))
            a.dw_stride = a.classes
        else:
            dw = x.new_empty((a.classes, a.dim)).t()
            a.dw_stride = a.dim
        a.lse, a.dx, a.dx_stride, a.dw = lse.data_ptr(), dx.data_ptr(), a.dim, dw.data_ptr()
        ws = _loss_workspace(a, True, x)  # noqa: F841
        sb.snn_vocab_loss_backward(a, _stream(x))
    return dx, dw
