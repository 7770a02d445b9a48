"""Sequence-model operators on torch tensors: argument checks, buffers and streams around the C ABI of include/snn.h.

    h, last, kept = gated_scan(x, gate, state, keep="int8")     # recurrence with learned gates, [T][B][N]
    dx, dgate, dstate = gated_scan_backward(kept, dh, dlast)
    h, state = gated_scan_step(x, gate, state)                  # one token
    packed = pack_activation(x, "int8"); x = unpack_activation(packed)
    loss, row_loss, lse = vocab_loss(x, w_out, targets)         # soft-max cross entropy of x w_out, logits never stored
    dx, dw = vocab_loss_backward(x, w_out, targets, lse)
    y, h, rstd, kept = rms_norm(x, weight, residual, keep="int8")   # the norm in front of a layer, with the residual's addition
    dx, dweight = rms_norm_backward(h, rstd, dy, weight, dh)
    state = adamw_state(params, bits=8); norm = adamw_step(params, grads, state, lr=1e-3, max_norm=1.0)
    tokens, parents, scores, ended, states = beam_step(logits, scores, states=states)   # beam search, [B][K][V]
    states = reorder_states(states, parents)

Gradients are explicit, as in the training step: nothing is recorded for autograd.  Work is launched on the current torch
stream of the tensors' device and the calls return without waiting; they can be captured into a CUDA graph.  Arguments
that do not fit raise ValueError before anything is launched; a status of the library raises `binding.SnnError`.
"""
from __future__ import annotations

import contextlib
from dataclasses import dataclass
from typing import List, Optional, Sequence, Tuple

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


def _launch(call, args, like: torch.Tensor) -> None:
    """A call of the library on the current stream of a tensor's device, which is made the current one where it is another."""
    device = like.get_device()
    if device == torch.cuda.current_device():
        call(args, _stream(like))
    else:
        with torch.cuda.device(device):
            call(args, _stream(like))


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


def _row_stride(t: torch.Tensor, name: str) -> int:
    """The distance of the rows of a tensor [..., N] whose leading dimensions are taken as one."""
    n = t.shape[-1]
    if t.is_contiguous():
        return n
    count = t.numel()
    try:
        rows = t.view(-1, n) if count else t
    except RuntimeError:
        raise ValueError(f"{name}: the leading dimensions have to collapse into one without a copy") from None
    if count and n > 1 and rows.stride(-1) != 1:
        raise ValueError(f"{name}: the last dimension has to be contiguous")
    return rows.stride(0)


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
    stride = _row_stride(x, "x")
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


# ---- root-mean-square norm with the residual's addition --------------------------------------------------------
def _rows(t: torch.Tensor, name: str) -> None:
    if not (isinstance(t, torch.Tensor) and t.is_cuda):
        raise ValueError(f"{name}: a CUDA tensor is required")
    if t.dtype not in _DTYPES:
        raise ValueError(f"{name}: dtype {t.dtype} is not fp32, bf16 or fp16")
    if t.dim() < 1 or not 1 <= t.shape[-1] <= _WIDEST:
        raise ValueError(f"{name}: at least one dimension is required, the last one from 1 to 2^31 - 64")


def _rows_like(t: torch.Tensor, name: str, like: torch.Tensor) -> int:
    """Checks a tensor of the shape and type of another, and returns the distance of its rows."""
    if not isinstance(t, torch.Tensor) or t.get_device() != like.get_device():
        raise ValueError(f"{name}: a tensor on {like.device} is required")
    if t.dtype is not like.dtype:
        raise ValueError(f"{name}: dtype {t.dtype} instead of {like.dtype}")
    if t.shape != like.shape:
        raise ValueError(f"{name}: shape {tuple(t.shape)} instead of {tuple(like.shape)}")
    return _row_stride(t, name)


def _overlap(a: int, a_stride: int, b: int, b_stride: int, rows: int, n: int, size: int) -> bool:
    """Whether two arrays of rows have bytes in common (strides of at least n values; of different strides: whether they could)."""
    if rows == 0 or a >= b + ((rows - 1) * b_stride + n) * size or b >= a + ((rows - 1) * a_stride + n) * size:
        return False
    if a_stride != b_stride or rows == 1:
        return True
    apart = (b - a) % (a_stride * size)     # columns of the same rows, beside one another?
    return apart < n * size or a_stride * size - apart < n * size


def _norm_weight(weight: Optional[torch.Tensor], like: torch.Tensor) -> int:
    """Checks a norm's weight and returns its type's number."""
    if weight is None:
        return _DTYPES[like.dtype]
    if not isinstance(weight, torch.Tensor) or weight.get_device() != like.get_device():
        raise ValueError(f"weight: a tensor on {like.device} is required")
    if weight.dtype is not like.dtype and weight.dtype is not torch.float32:
        raise ValueError(f"weight: dtype {weight.dtype} is neither {like.dtype} nor fp32")
    if weight.shape != like.shape[-1:]:
        raise ValueError(f"weight: shape {tuple(weight.shape)} instead of {tuple(like.shape[-1:])}")
    if not weight.is_contiguous():
        raise ValueError("weight: has to be contiguous")
    return _DTYPES[weight.dtype]


def rms_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None, residual: Optional[torch.Tensor] = None, *, eps: float = 1e-6,
             keep: Optional[str] = None, values: bool = True, inplace: bool = False):
    """Root-mean-square norm of the rows of a tensor [..., N], after the residual has been added to it:

        h = x + residual (in their type),  rstd = 1 / sqrt(mean(h^2) + eps),  y = h rstd weight

    x, residual: fp32, bf16 or fp16, leading dimensions that collapse into one without a copy; weight: [N], of their type or
    fp32 (ones if None).  keep: "int8" or "e4m3" for a copy of y in 8 bits, made in the same pass from the values before they
    are rounded to the type; values=False leaves y itself out.  inplace: h replaces the residual in its memory.
    eps: from 1e-30 to 1.  Rows of any finite values are normed, also where their squares leave fp32.
    Returns (y or None, h, rstd fp32 [...], PackedActivation or None); h is x itself where there is no residual."""
    _rows(x, "x")
    shape, n = x.shape, x.shape[-1]
    weight_dtype = _norm_weight(weight, x)
    if keep is not None:
        _choice(keep, "keep", _FORMATS)
    elif not values:
        raise ValueError("values: without them, keep is required")
    if not 1e-30 <= eps <= 1.0:
        raise ValueError("eps: has to be from 1e-30 to 1")
    count = x.numel()
    a = sb.snn_rms_norm_args(count // n, n, _DTYPES[x.dtype], weight_dtype, eps, x.data_ptr(), _row_stride(x, "x"))
    if residual is not None:
        a.residual, a.residual_stride = residual.data_ptr() if isinstance(residual, torch.Tensor) else None, _rows_like(residual, "residual", x)
    elif inplace:
        raise ValueError("inplace: needs a residual")
    a.weight = _ptr(weight)
    h = x
    if residual is not None:
        if inplace:
            h, a.h_stride = residual, a.residual_stride
            if a.rows > 1 and a.h_stride < n:
                raise ValueError("residual: rows overlap")
            same = a.x == a.residual and a.x_stride == a.residual_stride
            if not same and _overlap(a.x, a.x_stride, a.residual, a.residual_stride, a.rows, n, x.element_size()):
                raise ValueError("residual: overlaps x in memory")
        else:
            h, a.h_stride = _dense(x), n
        a.h = h.data_ptr()
    rstd = x.new_empty(shape[:-1], dtype=torch.float32)
    a.rstd = rstd.data_ptr()
    y = kept = None
    if values:
        y = _dense(x)
        a.y, a.y_stride = y.data_ptr(), n
    if keep is not None:
        codes, scales = _empty_codes(x, shape)
        kept = PackedActivation(codes, scales, keep, x.dtype)
        a.keep_format, a.codes, a.scales = _FORMATS[keep], codes.data_ptr(), scales.data_ptr()
    if count:
        _launch(sb.snn_rms_norm_forward, a, x)
    return y, h, rstd, kept


def rms_norm_backward(h: torch.Tensor, rstd: torch.Tensor, dy: torch.Tensor, weight: Optional[torch.Tensor] = None,
                      dh: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Gradients of a loss from those by y (dy) and by h (dh, what the residual stream hands back; zero if None), with h and
    rstd as `rms_norm` returned them.  Where y was kept in 8 bits, they are those of the values before.
    Returns (dx, the gradient by x and by the residual alike, of their type; dweight, of weight's type, None without one).
    Workspace: 4 N bytes per thread block, of which there are at most 1184, and no more than rows."""
    _rows(h, "h")
    n = h.shape[-1]
    weight_dtype = _norm_weight(weight, h)
    _like(rstd, "rstd", h, h.shape[:-1], torch.float32)
    a = sb.snn_rms_norm_args(h.numel() // n, n, _DTYPES[h.dtype], weight_dtype)
    a.h, a.h_stride, a.weight, a.rstd = h.data_ptr(), _row_stride(h, "h"), _ptr(weight), rstd.data_ptr()
    a.dy_stride, a.dy = _rows_like(dy, "dy", h), dy.data_ptr()
    if dh is not None:
        a.dh_stride, a.dh = _rows_like(dh, "dh", h), dh.data_ptr()
    dx = _dense(h)
    a.dx, a.dx_stride = dx.data_ptr(), n
    dweight = None
    if weight is not None:
        dweight = torch.empty_like(weight)
        a.dweight = dweight.data_ptr()
        ws = h.new_empty(sb.snn_rms_norm_workspace(a), dtype=torch.uint8)
        a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel()
    _launch(sb.snn_rms_norm_backward, a, h)
    return dx, dweight


# ---- AdamW over many tensors -----------------------------------------------------------------------------------
@dataclass(frozen=True)
class AdamWState:
    """The moments of a list of tensors, one behind the other, each tensor's from a multiple of 64 values on, and the number of
    steps done: m and v fp32, or in 8 bits (e4m3), where v holds square roots."""
    m: object                      # torch.Tensor or PackedActivation
    v: object
    step: torch.Tensor             # int64, 0-d, on the device


def _moments(sizes) -> int:
    return sum(-(-n // KEEP_GROUP) * KEEP_GROUP for n in sizes)


def adamw_state(params: Sequence[torch.Tensor], bits: int = 32) -> AdamWState:
    """The state that `adamw_step` starts from: moments of zero in 32 or 8 bits (8 or 2 1/32 bytes per parameter)."""
    if bits not in (32, 8):
        raise ValueError(f"bits: {bits!r} is neither 32 nor 8")
    if len(params) == 0:
        raise ValueError("params: at least one tensor is required")
    for k, p in enumerate(params):
        if not (isinstance(p, torch.Tensor) and p.is_cuda):
            raise ValueError(f"params[{k}]: a CUDA tensor is required")
    n, like = _moments(p.numel() for p in params), params[0]
    step = like.new_zeros((), dtype=torch.int64)
    if bits == 32:
        return AdamWState(like.new_zeros(n, dtype=torch.float32), like.new_zeros(n, dtype=torch.float32), step)
    m, v = (PackedActivation(like.new_zeros(n, dtype=torch.uint8), like.new_zeros(n // KEEP_GROUP, dtype=torch.uint8), "e4m3", torch.float32)
            for _ in range(2))
    return AdamWState(m, v, step)


def _scalar_on(t: torch.Tensor, name: str, like: torch.Tensor, dtype) -> None:
    _like(t, name, like, (), dtype)


def adamw_step(params: Sequence[torch.Tensor], grads: Sequence[torch.Tensor], state: AdamWState, *, lr, betas: Tuple[float, float] = (0.9, 0.999),
               eps: float = 1e-8, weight_decay: float = 0.01, max_norm: Optional[float] = None, scale=1.0, seed: int = 0,
               copies: Optional[Sequence[Optional[torch.Tensor]]] = None) -> Optional[torch.Tensor]:
    """One AdamW step over all tensors in `params`, in place, with the step's number t counted in `state`:

        g = scale grad, times max_norm / norm where the norm of all gradients together is above max_norm
        m = b1 m + (1 - b1) g,  v = b2 v + (1 - b2) g^2
        p = p (1 - lr weight_decay) - lr m / (1 - b1^t) / (sqrt(v / (1 - b2^t)) + eps)

    params, grads: contiguous tensors of fp32, bf16 or fp16, in any mixture; no two of them may overlap.  copies: tensors of
    the parameters' shapes (or None) that receive the new parameters in their own type, as 16-bit copies of fp32 ones; a 16-bit
    parameter whose change is less than half a step stays as it is.
    lr and scale: numbers, or fp32 0-d tensors on the device, so that a captured step follows a schedule.
    max_norm: None computes no norm; otherwise a step whose norm is not finite is left out and not counted.
    A finite gradient beyond 1.8e19 in magnitude, whose square is infinite, stops its parameter (but for the decay).
    Moments in 8 bits are rounded at random, by a hash of seed, t and place: give every list of tensors a seed of its own.
    eps: from 1e-30 to 1.  Returns the norm before the clip (fp32, 0-d), or None without max_norm."""
    if not isinstance(state, AdamWState):
        raise ValueError("state: what adamw_state returned is required")
    count = len(params)
    if len(grads) != count or (copies is not None and len(copies) != count):
        raise ValueError("grads, copies: as many as params are required")
    like = state.step
    device = like.get_device() if isinstance(like, torch.Tensor) else -1
    if device < 0:
        raise ValueError("state.step: a CUDA tensor is required")
    table, dtypes, room = (sb.snn_adamw_tensor * count)(), _DTYPES, 0
    written = []          # (begin, end, of which list, which one)
    for k in range(count):
        p, g = params[k], grads[k]
        n = p.numel() if isinstance(p, torch.Tensor) else 0
        if not isinstance(p, torch.Tensor) or p.get_device() != device or p.dtype not in dtypes or not p.is_contiguous():
            raise ValueError(f"params[{k}]: a contiguous tensor of fp32, bf16 or fp16 on {like.device} is required")
        if not isinstance(g, torch.Tensor) or g.get_device() != device or g.dtype not in dtypes or not g.is_contiguous():
            raise ValueError(f"grads[{k}]: a contiguous tensor of fp32, bf16 or fp16 on {like.device} is required")
        if g.shape != p.shape:
            raise ValueError(f"grads[{k}]: shape {tuple(g.shape)} instead of {tuple(p.shape)}")
        room += n + -n % KEEP_GROUP
        if n == 0:
            continue
        e = table[k]
        at = p.data_ptr()
        e.param, e.grad, e.n, e.param_dtype, e.grad_dtype = at, g.data_ptr(), n, dtypes[p.dtype], dtypes[g.dtype]
        written.append((at, at + n * p.element_size(), "params", k))
        c = None if copies is None else copies[k]
        if c is not None:
            if not isinstance(c, torch.Tensor) or c.get_device() != device or c.dtype not in dtypes or not c.is_contiguous() or c.shape != p.shape:
                raise ValueError(f"copies[{k}]: a contiguous tensor of fp32, bf16 or fp16 and of the parameter's shape is required")
            at = c.data_ptr()
            written.append((at, at + n * c.element_size(), "copies", k))
            e.copy, e.copy_dtype = at, dtypes[c.dtype]
    written.sort()
    for a, b in zip(written, written[1:]):
        if b[0] < a[1]:
            raise ValueError(f"{b[2]}[{b[3]}]: shares memory with {a[2]}[{a[3]}], which is written as well")
    if like.dtype is not torch.int64 or like.dim() != 0:
        raise ValueError("state.step: an int64 0-d tensor is required")
    a = sb.snn_adamw_args()
    a.count, a.tensors, a.step = count, table, like.data_ptr()
    if isinstance(state.m, PackedActivation):
        a.moment_format = sb.SNN_KEEP_E4M3
        for name in ("m", "v"):
            t = getattr(state, name)
            if not isinstance(t, PackedActivation) or t.format != "e4m3":
                raise ValueError(f"state.{name}: not in e4m3, as the other moment is")
            _like(t.codes, f"state.{name}", like, (room,), torch.uint8)
            _like(t.scales, f"state.{name}", like, (room // KEEP_GROUP,), torch.uint8)
            setattr(a, name + "_codes", t.codes.data_ptr())
            setattr(a, name + "_scales", t.scales.data_ptr())
    else:
        for name in ("m", "v"):
            t = getattr(state, name)
            _like(t, f"state.{name}", like, (room,), torch.float32)
            setattr(a, name, t.data_ptr())
    for name, value in (("lr", lr), ("scale", scale)):
        if isinstance(value, torch.Tensor):
            _scalar_on(value, name, like, torch.float32)
            setattr(a, name + "_device", value.data_ptr())
            value = 1.0
        elif not abs(value) <= 3e38 or (name == "lr" and value < 0):
            raise ValueError(f"{name}: has to be finite" + (" and at least zero" if name == "lr" else ""))
        setattr(a, name, value)
    if not (0 <= betas[0] < 1 and 0 <= betas[1] < 1):
        raise ValueError("betas: have to be from 0 to less than 1")
    if not 1e-30 <= eps <= 1.0:
        raise ValueError("eps: has to be from 1e-30 to 1")
    if not 0 <= weight_decay <= 3e38:
        raise ValueError("weight_decay: has to be finite and at least zero")
    if max_norm is not None and not max_norm > 0:
        raise ValueError("max_norm: has to be above zero")
    if not 0 <= seed < 2 ** 64:
        raise ValueError("seed: has to fit 64 bits")
    a.beta1, a.beta2, a.eps, a.weight_decay, a.max_norm, a.seed = *betas, eps, weight_decay, max_norm or 0.0, seed
    norm = None
    if max_norm is not None:
        norm = like.new_empty((), dtype=torch.float32)
        a.norm = norm.data_ptr()
    ws = like.new_empty(sb.SNN_ADAMW_WORKSPACE, dtype=torch.uint8)
    a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel()
    _launch(sb.snn_adamw_step, a, like)
    return norm


# ---- beam search -----------------------------------------------------------------------------------------------
MOST_BEAMS = 32


def _state_table(states, rows: int, out_rows: int, inplace: bool, device: int, read: Optional[torch.Tensor] = None):
    """(table for the library, tensors that receive the rows); read: what the call reads while it writes them."""
    if isinstance(states, torch.Tensor):
        raise ValueError("states: a sequence of tensors is required")
    table, out, held = (sb.snn_state_rows * len(states))(), [], []
    for k, t in enumerate(states):
        if not isinstance(t, torch.Tensor) or t.get_device() != device or not t.is_contiguous():
            raise ValueError(f"states[{k}]: a contiguous tensor on the device of the beams is required")
        if t.dim() < 1 or t.shape[0] != rows:
            raise ValueError(f"states[{k}]: {rows} rows are required, one for each beam")
        at, size = t.data_ptr(), t.numel() * t.element_size()
        if inplace:
            if size:
                held.append((at, at + size, k))
            new = t
        else:
            new = torch.empty_like(t) if rows == out_rows else t.new_empty((out_rows, *t.shape[1:]))
        out.append(new)
        e = table[k]
        e.source, e.to, e.row_bytes = at, new.data_ptr(), size // rows if rows else 0
    held.sort()
    for (_, end, j), (begin, _, k) in zip(held, held[1:]):
        if begin < end:
            raise ValueError(f"states[{max(j, k)}]: shares memory with states[{min(j, k)}], which does not go in place")
    if read is not None and read.numel():
        first, last = read.data_ptr(), read.data_ptr() + read.numel() * read.element_size()
        for begin, end, k in held:
            if begin < last and first < end:
                raise ValueError(f"states[{k}]: shares memory with the parents, which does not go in place")
    return table, out


def beam_step(logits: torch.Tensor, scores: torch.Tensor, *, width: Optional[int] = None, ended: Optional[torch.Tensor] = None,
              end: Optional[int] = None, states: Sequence[torch.Tensor] = (), inplace: bool = False):
    """One step of beam search: the best `width` (K if None) continuations of the K beams of each sample, by

        score(k, c) = scores[b, k] + log_softmax(logits[b, k])[c]

    logits: [B][K][V], fp32, bf16 or fp16, with contiguous classes; scores: fp32 [B][K] (a first step from one beam has K = 1).
    Classes of one beam are ranked by their logits, exactly.  Beams are ranked by scores that are compared in 64 bits, with exponentials
    summed in fp32: good to 1e-6 as a rule and 1e-5 at worst, and what is closer than that may come in either order.  Equal beams have
    equal scores; ties go to the lower beam, then to the lower class.
    end: the class that ends a beam; ended: bool [B][K], the beams that have: they go on with `end` alone, at their score.
    Continuations at -infinity come last, in the order of k V + c: classes masked by logits of -infinity, and all of a
    beam whose score is not finite, or whose logits are all masked or hold a NaN or +infinity.
    states: tensors whose rows [B K, ...] belong to the beams (what gated_scan_step carries, tokens so far): they come back
    as rows [B width, ...] of the beams' parents, with inplace in their own memory (width = K), of which no two may share any.
    K and width are at most 32, V at most 2^22.  Returns (tokens int64 [B][width], parents int64 [B][width], the beam of each,
    scores fp32 [B][width], ended bool [B][width] or None without end, list of states)."""
    _values(logits, "logits", 3)
    B, K, V = logits.shape
    width = K if width is None else width
    if not (1 <= K <= MOST_BEAMS and 1 <= width <= MOST_BEAMS):
        raise ValueError(f"logits, width: from 1 to {MOST_BEAMS} beams are required")
    if not 1 <= V <= 1 << 22 or B * K > 1 << 24:
        raise ValueError("logits: from 1 to 2^22 classes and at most 2^24 beams are required")
    if width > K * V:
        raise ValueError("width: more than there are continuations")
    _like(scores, "scores", logits, (B, K), torch.float32)
    if end is None:
        if ended is not None:
            raise ValueError("ended: needs end")
    elif not 0 <= end < V:
        raise ValueError("end: is not a class")
    if ended is not None:
        _like(ended, "ended", logits, (B, K), torch.bool)
    if inplace and width != K:
        raise ValueError("inplace: needs as many survivors as beams")
    table, out = _state_table(states, B * K, B * width, inplace, logits.get_device())
    tokens = logits.new_empty((B, width), dtype=torch.int64)
    parents = torch.empty_like(tokens)
    new_scores = torch.empty_like(scores) if width == K else scores.new_empty((B, width))
    new_ended = None if end is None else logits.new_empty((B, width), dtype=torch.bool)
    a = sb.snn_beam_args(B, K, width, V, _DTYPES[logits.dtype], logits.data_ptr(), logits.stride(0), logits.stride(1), scores.data_ptr(),
                         _ptr(ended), -1 if end is None else end, tokens.data_ptr(), parents.data_ptr(), new_scores.data_ptr(),
                         _ptr(new_ended), table, len(out))
    if B:
        ws = logits.new_empty(sb.snn_beam_workspace(a), dtype=torch.uint8)
        a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel()
        _launch(sb.snn_beam_step, a, logits)
    return tokens, parents, new_scores, new_ended, out


def reorder_states(states: Sequence[torch.Tensor], parents: torch.Tensor, *, beams: Optional[int] = None, inplace: bool = False) -> List[torch.Tensor]:
    """Rows [B K, ...] of tensors of any type in the order of their parents, int64 [B][W]: row b W + w of a result is row
    b K + parents[b, w]; a parent outside [0, K) leaves zeros.  beams: K, where it is not W.  inplace: in the tensors' own
    memory (K = W), which they may share neither with one another nor with the parents; rows that stay where they are are not
    written.  K and W are at most 32."""
    if not (isinstance(parents, torch.Tensor) and parents.is_cuda and parents.dtype is torch.int64 and parents.dim() == 2 and parents.is_contiguous()):
        raise ValueError("parents: a contiguous int64 CUDA tensor of two dimensions is required")
    B, W = parents.shape
    K = W if beams is None else beams
    if not (1 <= K <= MOST_BEAMS and 1 <= W <= MOST_BEAMS):
        raise ValueError(f"parents, beams: from 1 to {MOST_BEAMS} beams are required")
    if B > 1 << 24:
        raise ValueError("parents: too many samples")
    if inplace and K != W:
        raise ValueError("inplace: needs as many survivors as beams")
    with _on(parents):
        table, out = _state_table(states, B * K, B * W, inplace, parents.get_device(), parents)
        if B and out:
            sb.snn_reorder_rows(table, len(out), parents.data_ptr(), B, K, W, _stream(parents))
    return out
