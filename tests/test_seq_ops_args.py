"""Refusals of the sequence-model operators: before anything is launched, so without a GPU."""
import ctypes as C

import numpy as np
import pytest

import seq_reference as ref
from paper_2412_11810_b200 import binding as sb

torch = pytest.importorskip("torch")
from paper_2412_11810_b200 import ops  # noqa: E402


def _scan_args(**kw):
    a = sb.snn_scan_args()
    a.T, a.B, a.N = 4, 2, 8
    for name in ("x", "gate", "h", "last", "states", "dh", "dx", "dgate", "dstate"):
        setattr(a, name, 1 << 20)   # never read: every call below is refused first
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("change", [{"T": -1}, {"B": -1}, {"N": -1}, {"T": 1 << 30}, {"dtype": 3}, {"dtype": -1}, {"mode": 2},
                                    {"x_format": 3}, {"gate_format": -1}, {"x_format": sb.SNN_KEEP_INT8}, {"gate": None}, {"x": None}])
def test_scan_refuses_invalid_arguments(change):
    for call in (sb.lib.snn_scan_forward, sb.lib.snn_scan_backward):
        assert call(C.byref(_scan_args(**change)), None) == sb.SNN_ERR_INVALID_ARG


def test_scan_refuses_missing_buffers():
    assert sb.lib.snn_scan_forward(None, None) == sb.SNN_ERR_INVALID_ARG
    assert sb.lib.snn_scan_backward(None, None) == sb.SNN_ERR_INVALID_ARG
    assert sb.lib.snn_scan_forward(C.byref(_scan_args(h=None)), None) == sb.SNN_ERR_INVALID_ARG
    # 8-bit copies are made only where states are kept
    assert sb.lib.snn_scan_forward(C.byref(_scan_args(states=None, x_format=1, x_codes=256, x_scales=256)), None) == sb.SNN_ERR_INVALID_ARG
    for name in ("dh", "dx", "dgate", "states"):
        assert sb.lib.snn_scan_backward(C.byref(_scan_args(**{name: None})), None) == sb.SNN_ERR_INVALID_ARG
    direct = _scan_args(mode=sb.SNN_SCAN_DIRECT, gate_format=sb.SNN_KEEP_INT8, gate_codes=256, gate_scales=256)
    assert sb.lib.snn_scan_forward(C.byref(direct), None) == sb.SNN_ERR_UNSUPPORTED
    assert sb.lib.snn_scan_backward(C.byref(direct), None) == sb.SNN_ERR_UNSUPPORTED


def test_scan_workspace():
    """Needed where there are few channels and many steps; small, and refused when it is missing."""
    for backward in (False, True):
        assert sb.snn_scan_workspace(_scan_args(T=64), backward) == 0
        assert sb.snn_scan_workspace(_scan_args(T=4096, B=64, N=1024), backward) == 0
        a = _scan_args(T=65536, B=1, N=1024, dtype=sb.SNN_DTYPE_BF16)
        n = sb.snn_scan_workspace(a, backward)
        assert 0 < n < 65536 * 1024 * 2 // 50
        a.workspace, a.workspace_bytes = 1 << 20, n - 1
        call = sb.lib.snn_scan_backward if backward else sb.lib.snn_scan_forward
        assert call(C.byref(a), None) == sb.SNN_ERR_WORKSPACE_TOO_SMALL
        a.workspace, a.workspace_bytes = (1 << 20) + 16, n
        assert call(C.byref(a), None) == sb.SNN_ERR_INVALID_ARG
    assert sb.lib.snn_scan_workspace(C.byref(_scan_args()), 0, None) == sb.SNN_ERR_INVALID_ARG


@pytest.mark.parametrize("rows,cols,dtype,fmt", [(-1, 4, 0, 1), (4, -1, 0, 1), (4, 4, 3, 1), (4, 4, 0, 0), (4, 4, 0, 3), (4, 4, 0, 1)])
def test_pack_refuses_invalid_arguments(rows, cols, dtype, fmt):
    assert sb.lib.snn_activation_pack(None, dtype, rows, cols, 4, fmt, None, None, None) == sb.SNN_ERR_INVALID_ARG
    assert sb.lib.snn_activation_unpack(None, None, fmt, rows, cols, None, dtype, 4, None) == sb.SNN_ERR_INVALID_ARG


def _loss_args(**kw):
    a = sb.snn_vocab_loss_args()
    a.rows, a.dim, a.classes, a.x_stride, a.w_stride, a.target_bits, a.scale = 4, 8, 16, 8, 16, 64, 1.0
    a.dx_stride, a.dw_stride = 8, 16
    for name in ("x", "w", "targets", "lse", "loss", "dx", "dw"):
        setattr(a, name, 1 << 20)   # never read: every call below is refused first
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("change", [{"rows": -1}, {"dim": 0}, {"classes": 0}, {"rows": 1 << 30}, {"dtype": 3}, {"w_layout": 2},
                                    {"target_bits": 16}, {"scale": float("nan")}, {"scale": float("inf")}, {"x_stride": 7},
                                    {"w_stride": 15}, {"x": None}, {"w": None}, {"targets": None}])
def test_loss_refuses_invalid_arguments(change):
    n = C.c_size_t()
    for call in (lambda a: sb.lib.snn_vocab_loss_forward(C.byref(a), None), lambda a: sb.lib.snn_vocab_loss_backward(C.byref(a), None),
                 lambda a: sb.lib.snn_vocab_loss_workspace(C.byref(a), 0, C.byref(n))):
        assert call(_loss_args(**change)) == sb.SNN_ERR_INVALID_ARG


def test_loss_refuses_missing_buffers():
    for name in ("lse", "loss"):
        assert sb.lib.snn_vocab_loss_forward(C.byref(_loss_args(**{name: None})), None) == sb.SNN_ERR_INVALID_ARG
    for change in ({"dx": None}, {"dw": None}, {"lse": None}, {"dx_stride": 7}, {"dw_stride": 15}):
        assert sb.lib.snn_vocab_loss_backward(C.byref(_loss_args(**change)), None) == sb.SNN_ERR_INVALID_ARG
    assert sb.lib.snn_vocab_loss_forward(None, None) == sb.SNN_ERR_INVALID_ARG
    assert sb.lib.snn_vocab_loss_workspace(C.byref(_loss_args()), 0, None) == sb.SNN_ERR_INVALID_ARG


def test_loss_workspace_does_not_grow_with_the_logits():
    """The forward pass holds a pair of numbers per row and 128 classes, the backward pass a bounded piece of dz."""
    a = _loss_args(rows=8192, dim=1024, classes=131072, x_stride=1024, w_stride=131072, dtype=sb.SNN_DTYPE_BF16)
    logits = 4 * 8192 * 131072
    assert 0 < sb.snn_vocab_loss_workspace(a, False) < logits / 32
    assert 0 < sb.snn_vocab_loss_workspace(a, True) < logits / 4


def test_sequence_operators_need_cuda_tensors():
    x = torch.zeros(4, 2, 8)
    for call in (lambda: ops.gated_scan(x, x), lambda: ops.gated_scan_step(x[0], x[0]), lambda: ops.pack_activation(x),
                 lambda: ops.gated_scan_backward(None, x),
                 lambda: ops.vocab_loss(x[0], x[0].t(), torch.zeros(2, dtype=torch.int64)),
                 lambda: ops.vocab_loss_backward(x[0], x[0].t(), torch.zeros(2, dtype=torch.int64), x[0, :, 0]),
                 lambda: ops.unpack_activation(ops.PackedActivation(x, x, "int8", torch.float32))):
        with pytest.raises(ValueError):
            call()


def test_enumerators_match_the_header():
    import os
    import re
    header = open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "snn.h")).read()
    found = re.findall(r"\b(SNN_(?:DTYPE|KEEP|SCAN|W)_[A-Z0-9_]+)\s*=\s*(\d+)", header)
    found += re.findall(r"#define\s+(SNN_(?:KEEP|SCAN)_[A-Z]+)\s+(\d+)", header)
    assert len(found) == 12
    for name, value in found:
        assert getattr(sb, name) == int(value), name


def test_struct_sizes_match_the_header(tmp_path):
    """The argument structs are spelled twice (include/snn.h and binding.py): same sizes and last offsets."""
    import os
    import subprocess
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "%s/include/snn.h"\nint main(void) {\n'
                   'printf("%%zu %%zu\\n", sizeof(snn_scan_args), offsetof(snn_scan_args, workspace_bytes));\n'
                   'printf("%%zu %%zu\\n", sizeof(snn_vocab_loss_args), offsetof(snn_vocab_loss_args, workspace_bytes));\n'
                   'printf("%%d %%d\\n", SNN_KEEP_GROUP, SNN_SCAN_CHUNK); return 0; }\n' % root)
    subprocess.run(["gcc", str(src), "-o", str(tmp_path / "s")], check=True)
    out = subprocess.run([str(tmp_path / "s")], check=True, capture_output=True, text=True).stdout.split()
    assert [int(v) for v in out] == [C.sizeof(sb.snn_scan_args), sb.snn_scan_args.workspace_bytes.offset, C.sizeof(sb.snn_vocab_loss_args),
                                     sb.snn_vocab_loss_args.workspace_bytes.offset, ops.KEEP_GROUP, ops.SCAN_CHUNK]


# ---- the 64-bit reference itself ---------------------------------------------------------------------------------
@pytest.mark.parametrize("mode", ["sigmoid", "direct"])
def test_reference_gradients_against_differences(mode):
    rng = np.random.default_rng(1)
    T, B, N = 70, 2, 3
    lengths = np.array([70, 41])
    x, gate = rng.standard_normal((T, B, N)), rng.standard_normal((T, B, N))
    gate = gate if mode == "sigmoid" else 0.9 * np.tanh(gate)
    state, dh, dlast = rng.standard_normal((B, N)), rng.standard_normal((T, B, N)), rng.standard_normal((B, N))
    r = ref.scan_backward(x, gate, state, lengths, mode, dh, dlast)

    def loss(p):
        f = ref.scan_forward(p[0], p[1], p[2], lengths, mode)
        return (f["h"] * dh).sum() + (f["last"] * dlast).sum()

    point = [x, gate, state]
    for k, name in enumerate(("dx", "dgate", "dstate")):
        v = rng.standard_normal(point[k].shape)
        at = lambda s: [p + s * v if j == k else p for j, p in enumerate(point)]  # noqa: E731
        slope = (loss(at(1e-6)) - loss(at(-1e-6))) / 2e-6
        assert abs((r[name] * v).sum() - slope) <= 1e-7 * np.abs(r[name] * v).sum() + 1e-6


def test_reference_eight_bits():
    v = np.array([[127.0, 2.5, -0.49, 63.5], [448.0, 450.0, 17.0, 2.0 ** -10]])
    q, s = ref.eight_bits(v, "int8")
    assert np.array_equal(q[0], [127, 2, 0, 64]) and s[0, 0] == 127 and s[1, 0] == 129
    q, s = ref.eight_bits(v, "e4m3")
    assert np.array_equal(q, [[128, 2.5, -0.5, 64], [448, 448, 16, 0]]) and s[0, 0] == 126 and s[1, 0] == 128


def test_loss_wait_selftest_refuses_invalid_arguments():
    call = lambda a, *v: sb.lib.snn_selftest_vocab_loss_wait(C.byref(a), *v, None)  # noqa: E731
    for v in ((0, 1, 0, 0, 10), (1, 3, 0, 0, 10), (1, -1, 0, 0, 10), (1, 0, -1, 0, 10), (1, 0, 0, 0, 0), (1, 0, 0, 0, 1 << 23)):
        assert call(_loss_args(), *v) == sb.SNN_ERR_INVALID_ARG
    assert call(_loss_args(rows=-1), 1, 0, 0, 0, 10) in (sb.SNN_ERR_INVALID_ARG, sb.SNN_ERR_UNSUPPORTED)
    if not sb.lib.snn_debug_checks_enabled():   # the limits of waits are constants there
        assert call(_loss_args(), 1, 0, 0, 0, 10) == sb.SNN_ERR_UNSUPPORTED


@pytest.mark.parametrize("dtype", [sb.SNN_DTYPE_FP32, sb.SNN_DTYPE_BF16])
def test_scan_workspace_has_room_for_the_first_state(dtype):
    """Where the time axis is cut, the blocks of the last part write `last` while others still start: they take `state`, which
    may be the same buffer, from a copy beside the summaries (16 bytes per pair of channels and part)."""
    for T, B, N in ((4096, 1, 64), (65536, 1, 1024), (5000, 3, 100)):
        tiles = B * -(-N // 64)
        n = sb.snn_scan_workspace(_scan_args(T=T, B=B, N=N, dtype=dtype), False)
        assert n > 0 and n % (tiles * 32 * 16) == tiles * 32 * 8


def test_scan_wait_selftest_refuses_invalid_arguments():
    for v in ((0, -1, 0, 10), (1, -1, 0, 10), (0, 0, 0, 0), (1, 0, 0, 1 << 23)):
        assert sb.lib.snn_selftest_scan_wait(C.byref(_scan_args()), *v, None) == sb.SNN_ERR_INVALID_ARG
    assert sb.lib.snn_selftest_scan_wait(C.byref(_scan_args(N=-1)), 1, 0, 0, 10, None) in (sb.SNN_ERR_INVALID_ARG, sb.SNN_ERR_UNSUPPORTED)
    if not sb.lib.snn_debug_checks_enabled():
        assert sb.lib.snn_selftest_scan_wait(C.byref(_scan_args()), 1, 0, 0, 10, None) == sb.SNN_ERR_UNSUPPORTED


@pytest.mark.parametrize("width", [2 ** 31 - 1, 2 ** 31 - 63])
def test_widths_whose_last_group_passes_32_bits_are_refused(width):
    p = 1 << 20   # never read
    assert sb.lib.snn_activation_pack(p, 0, 1, width, width, 1, p, p, None) == sb.SNN_ERR_UNSUPPORTED
    assert sb.lib.snn_activation_unpack(p, p, 1, 1, width, p, 0, width, None) == sb.SNN_ERR_UNSUPPORTED
    for T in (1, 100):
        a = _scan_args(T=T, B=1, N=width)
        assert sb.lib.snn_scan_forward(C.byref(a), None) == sb.SNN_ERR_UNSUPPORTED
        assert sb.lib.snn_scan_backward(C.byref(a), None) == sb.SNN_ERR_UNSUPPORTED
        n = C.c_size_t()
        assert sb.lib.snn_scan_workspace(C.byref(a), 0, C.byref(n)) == sb.SNN_ERR_UNSUPPORTED


@pytest.mark.parametrize("scale", [2.4e38, -3.4e38])
def test_loss_refuses_a_scale_that_leaves_fp32_times_log2_e(scale):
    n = C.c_size_t()
    for call in (lambda a: sb.lib.snn_vocab_loss_forward(C.byref(a), None), lambda a: sb.lib.snn_vocab_loss_backward(C.byref(a), None),
                 lambda a: sb.lib.snn_vocab_loss_workspace(C.byref(a), 0, C.byref(n))):
        assert call(_loss_args(scale=scale)) == sb.SNN_ERR_INVALID_ARG


def test_scan_calls_without_a_workspace_need_none():
    """`ops` asks the library for the size of a workspace only where the time axis may be cut: wherever it does not ask, the
    library wants none."""
    like = torch.zeros(0)
    asked = 0
    for dtype in (sb.SNN_DTYPE_FP32, sb.SNN_DTYPE_BF16):
        for T in (1, 100, 511, 512, 513, 640, 4096, 70000):
            for B, N in ((1, 1), (1, 9472), (1, 9473), (1, 9535), (1, 9536), (1, 9537), (148, 1), (148, 64), (149, 1), (149, 63), (149, 64),
                         (149, 65), (37, 256), (2, 4736), (2, 4800), (600, 16), (3, 3200)):
                for backward in (False, True):
                    a = _scan_args(T=T, B=B, N=N, dtype=dtype)
                    ws = ops._scan_workspace(a, backward, like)
                    assert (0 if ws is None else ws.numel()) == sb.snn_scan_workspace(a, backward)
                    asked += ws is not None
    assert asked > 0
