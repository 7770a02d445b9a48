"""Refusals of the norm, the AdamW step and beam search: before anything is launched, so without a GPU; and their 64-bit references."""
import ctypes as C
import os
import re
import subprocess

import numpy as np
import pytest

import model_reference as ref
from paper_2412_11810_b200 import binding as sb

torch = pytest.importorskip("torch")
from paper_2412_11810_b200 import ops  # noqa: E402

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20   # a pointer that is never read: every call below is refused first


def _norm(**kw):
    a = sb.snn_rms_norm_args(4, 64, 0, 0, 1e-6, P, 64)
    for name in ("h", "y", "rstd", "dy", "dx"):
        setattr(a, name, P)
    for name in ("h_stride", "y_stride", "dy_stride", "dx_stride"):
        setattr(a, name, 64)
    for k, v in kw.items():
        setattr(a, k, v)
    return a


def _norm_calls():
    n = C.c_size_t()
    return (lambda a: sb.lib.snn_rms_norm_forward(C.byref(a), None), lambda a: sb.lib.snn_rms_norm_backward(C.byref(a), None),
            lambda a: sb.lib.snn_rms_norm_workspace(C.byref(a), C.byref(n)))


@pytest.mark.parametrize("change", [{"rows": -1}, {"n": 0}, {"n": -1}, {"dtype": 3}, {"dtype": -1}, {"weight_dtype": 1}, {"weight_dtype": 3},
                                    {"dtype": 1, "weight_dtype": 2}])
def test_norm_refuses_invalid_arguments(change):
    for call in _norm_calls():
        assert call(_norm(**change)) == sb.SNN_ERR_INVALID_ARG


@pytest.mark.parametrize("width", [2 ** 31 - 1, 2 ** 31 - 63])
def test_norm_refuses_widths_whose_last_group_passes_32_bits(width):
    for call in _norm_calls():
        assert call(_norm(n=width)) == sb.SNN_ERR_UNSUPPORTED


def test_norm_refuses_what_does_not_fit():
    forward, backward, _ = _norm_calls()
    for change in ({"eps": 0.0}, {"eps": 1e-31}, {"eps": 1.5}, {"eps": float("nan")}, {"x": None}, {"y": None}, {"keep_format": 3}, {"keep_format": 1},
                   {"keep_format": 1, "codes": P}, {"residual": P, "h": None}, {"residual": P, "h_stride": 63}, {"y_stride": 63}, {"y_stride": 0}):
        assert forward(_norm(**change)) == sb.SNN_ERR_INVALID_ARG, change
    for change in ({"h": None}, {"rstd": None}, {"dy": None}, {"dx": None}, {"dx_stride": 63}, {"dweight": P}, {"dweight": P, "workspace": P + 16}):
        assert backward(_norm(**change)) == sb.SNN_ERR_INVALID_ARG, change
    n = sb.snn_rms_norm_workspace(_norm(rows=100))
    assert n >= 64 * 4
    assert backward(_norm(rows=100, dweight=P, workspace=P, workspace_bytes=64)) == sb.SNN_ERR_WORKSPACE_TOO_SMALL
    assert sb.lib.snn_rms_norm_forward(None, None) == sb.SNN_ERR_INVALID_ARG and sb.lib.snn_rms_norm_backward(None, None) == sb.SNN_ERR_INVALID_ARG
    assert sb.lib.snn_rms_norm_workspace(C.byref(_norm()), None) == sb.SNN_ERR_INVALID_ARG


def test_norm_workspace_is_small():
    """Four bytes a column and thread block, of which there are no more than 148 times 16, nor than rows."""
    for rows in (1, 7, 1000, 1 << 20, 1 << 40):
        for n in (1, 64, 1000, 8192, 20000, 2 ** 31 - 64):
            for dtype in (0, 1):
                size = sb.snn_rms_norm_workspace(_norm(rows=rows, n=n, dtype=dtype, weight_dtype=dtype))
                assert 4 * n <= size <= 4 * n * min(rows, 148 * 16) + 256
    assert sb.snn_rms_norm_workspace(_norm(rows=0)) == 0


def _adamw(listed=((P, P, 64),), **kw):
    a = sb.snn_adamw_args()
    a.count = len(listed)
    a.table = (sb.snn_adamw_tensor * max(1, len(listed)))(*[sb.snn_adamw_tensor(p, g, None, n, 0, 0, 0) for p, g, n in listed])   # (kept alive)
    a.tensors, a.m, a.v, a.step, a.workspace, a.workspace_bytes = a.table, P, P, P, P, sb.SNN_ADAMW_WORKSPACE
    a.lr, a.beta1, a.beta2, a.eps, a.weight_decay, a.scale = 1e-3, 0.9, 0.999, 1e-8, 0.01, 1.0
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("change", [{"count": -1}, {"tensors": None}, {"moment_format": 1}, {"moment_format": 3}, {"lr": -1.0}, {"lr": float("nan")},
                                    {"lr": float("inf")}, {"beta1": 1.0}, {"beta1": -0.1}, {"beta2": 1.0}, {"beta2": float("nan")}, {"eps": 0.0}, {"eps": 1e-31},
                                    {"eps": 2.0}, {"weight_decay": -0.1}, {"scale": float("inf")}, {"scale": float("nan")}, {"max_norm": -1.0},
                                    {"max_norm": float("nan")}])
def test_adamw_refuses_invalid_arguments(change):
    n = C.c_size_t()
    assert sb.lib.snn_adamw_step(C.byref(_adamw(**change)), None) == sb.SNN_ERR_INVALID_ARG
    assert sb.lib.snn_adamw_workspace(C.byref(_adamw(**change)), C.byref(n)) == sb.SNN_ERR_INVALID_ARG


def test_adamw_refuses_what_does_not_fit():
    step = lambda a: sb.lib.snn_adamw_step(C.byref(a), None)  # noqa: E731
    for tensors in (((None, P, 4),), ((P, None, 4),), ((P, P, -1),), ((P, P, 1 << 50),)):
        assert step(_adamw(tensors)) == sb.SNN_ERR_INVALID_ARG
    for field in ("param_dtype", "grad_dtype"):
        a = _adamw()
        setattr(a.table[0], field, 3)
        assert step(a) == sb.SNN_ERR_INVALID_ARG
    a = _adamw()
    a.table[0].copy, a.table[0].copy_dtype = P, 7
    assert step(a) == sb.SNN_ERR_INVALID_ARG
    for change in ({"step": None}, {"workspace": None}, {"workspace": P + 16}, {"m": None}, {"v": None}, {"m": P + 16}, {"v": P + 4}, {"moment_format": 2},
                   {"moment_format": 2, "m_codes": P, "v_codes": P, "m_scales": P}, {"moment_format": 2, "m_codes": P + 4, "v_codes": P, "m_scales": P, "v_scales": P}):
        assert step(_adamw(**change)) == sb.SNN_ERR_INVALID_ARG, change
    assert step(_adamw(workspace_bytes=sb.SNN_ADAMW_WORKSPACE - 1)) == sb.SNN_ERR_WORKSPACE_TOO_SMALL
    assert sb.lib.snn_adamw_step(None, None) == sb.SNN_ERR_INVALID_ARG and sb.lib.snn_adamw_workspace(C.byref(_adamw()), None) == sb.SNN_ERR_INVALID_ARG
    assert sb.snn_adamw_workspace(_adamw()) == sb.SNN_ADAMW_WORKSPACE


def _beam(moved=(), **kw):
    a = sb.snn_beam_args(2, 3, 3, 100, 0, P, 300, 100, P, None, -1, P, P, P)
    a.table = (sb.snn_state_rows * max(1, len(moved)))(*[sb.snn_state_rows(*s) for s in moved])
    a.states, a.n_states, a.workspace, a.workspace_bytes = a.table, len(moved), P, 1 << 30
    for k, v in kw.items():
        setattr(a, k, v)
    return a


@pytest.mark.parametrize("change", [{"B": -1}, {"K": 0}, {"W": 0}, {"V": 0}, {"dtype": 3}, {"W": 31, "K": 1, "V": 30}, {"end": 100}, {"end": -2}, {"ended": P},
                                    {"new_ended": P}])
def test_beam_refuses_invalid_arguments(change):
    n = C.c_size_t()
    assert sb.lib.snn_beam_step(C.byref(_beam(**change)), None) == sb.SNN_ERR_INVALID_ARG
    assert sb.lib.snn_beam_workspace(C.byref(_beam(**change)), C.byref(n)) == sb.SNN_ERR_INVALID_ARG


def test_beam_refuses_what_does_not_fit():
    step = lambda a: sb.lib.snn_beam_step(C.byref(a), None)  # noqa: E731
    for change in ({"K": 33}, {"W": 33}, {"V": (1 << 22) + 1}, {"B": 2 ** 31 - 1, "K": 32, "V": 1 << 22}):
        assert step(_beam(**change)) == sb.SNN_ERR_UNSUPPORTED, change
    for change in ({"logits": None}, {"logits": P + 2}, {"scores": None}, {"tokens": None}, {"parents": None}, {"new_scores": None}, {"workspace": None},
                   {"workspace": P + 8}, {"n_states": -1}, {"n_states": 1, "states": None}):
        assert step(_beam(**change)) == sb.SNN_ERR_INVALID_ARG, change
    for states in (((None, P, 8),), ((P, None, 8),), ((P, P + 64, -1),), ((P, P, 8),)):   # (the last one: in place, with another number of beams)
        assert step(_beam(states, W=2)) == sb.SNN_ERR_INVALID_ARG
    need = sb.snn_beam_workspace(_beam())
    assert need > 0 and step(_beam(workspace_bytes=need - 1)) == sb.SNN_ERR_WORKSPACE_TOO_SMALL
    assert sb.lib.snn_beam_step(None, None) == sb.SNN_ERR_INVALID_ARG and sb.lib.snn_beam_workspace(C.byref(_beam()), None) == sb.SNN_ERR_INVALID_ARG
    table = (sb.snn_state_rows * 1)(sb.snn_state_rows(P, P + 64, 8))
    reorder = lambda *v: sb.lib.snn_reorder_rows(*v, None)  # noqa: E731
    for v in ((table, -1, P, 1, 2, 2), (None, 1, P, 1, 2, 2), (table, 1, None, 1, 2, 2), (table, 1, P, -1, 2, 2), (table, 1, P, 1, 0, 2), (table, 1, P, 1, 2, 0)):
        assert reorder(*v) == sb.SNN_ERR_INVALID_ARG
    assert reorder(table, 1, P, 1, 33, 2) == sb.SNN_ERR_UNSUPPORTED and reorder(table, 1, P, 1, 2, 33) == sb.SNN_ERR_UNSUPPORTED


def test_beam_workspace_does_not_grow_with_the_logits():
    """A list of `W` and two numbers for a warp's part of a row: less than a fiftieth of the logits of wide rows, and never
    more than 1024 parts."""
    for B, K, V in ((1, 4, 32000), (64, 8, 131072), (1, 1, 1 << 22), (1000, 32, 50257)):
        size = sb.snn_beam_workspace(_beam(B=B, K=K, W=4, V=V, dtype=1))
        assert 0 < size <= B * K * 1024 * 40 + 512
        if B * K * V >= 1 << 20:
            assert size <= B * K * V * 2 / 50 + 512


def test_model_operators_need_cuda_tensors():
    x = torch.zeros(4, 8)
    for call in (lambda: ops.rms_norm(x), lambda: ops.rms_norm(x, x[0]), lambda: ops.rms_norm_backward(x, x[:, 0], x), lambda: ops.adamw_state([x]), lambda: ops.adamw_state([]),
                 lambda: ops.adamw_state([x], 16), lambda: ops.adamw_step([x], [x], None, lr=1.0), lambda: ops.adamw_step([x], [x], ops.AdamWState(x, x, x), lr=1.0),
                 lambda: ops.beam_step(x[None], x), lambda: ops.reorder_states([x], torch.zeros(1, 4, dtype=torch.int64))):
        with pytest.raises(ValueError):
            call()


def test_structs_and_constants_match_the_header(tmp_path):
    """The argument structs are spelled twice (include/snn.h and binding.py): same sizes and last offsets."""
    header = os.path.join(ROOT, "include", "snn.h")
    last = {"snn_rms_norm_args": "workspace_bytes", "snn_adamw_tensor": "copy_dtype", "snn_adamw_args": "workspace_bytes", "snn_state_rows": "row_bytes",
            "snn_beam_args": "workspace_bytes"}
    src = tmp_path / "s.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "%s"\nint main(void) {\n' % header
                   + "".join('printf("%%zu %%zu\\n", sizeof(%s), offsetof(%s, %s));\n' % (s, s, f) for s, f in last.items()) + "return 0; }\n")
    subprocess.run(["gcc", str(src), "-o", str(tmp_path / "s")], check=True)
    out = subprocess.run([str(tmp_path / "s")], check=True, capture_output=True, text=True).stdout.split()
    want = [v for s, f in last.items() for v in (C.sizeof(getattr(sb, s)), getattr(getattr(sb, s), f).offset)]
    assert [int(v) for v in out] == want
    assert int(re.search(r"#define\s+SNN_ADAMW_WORKSPACE\s+(\d+)", open(header).read()).group(1)) == sb.SNN_ADAMW_WORKSPACE


# ---- the 64-bit references themselves ------------------------------------------------------------------------------
def test_reference_norm_against_differences():
    rng = np.random.default_rng(1)
    h, w, dy, dh = rng.standard_normal((5, 7)), rng.standard_normal(7), rng.standard_normal((5, 7)), rng.standard_normal((5, 7))
    b = ref.norm_backward(h, ref.norm_forward(h, w, 0.1)["rstd"], w, dy, dh)
    loss = lambda h, w: (ref.norm_forward(h, w, 0.1)["y"] * dy).sum() + (h * dh).sum()  # noqa: E731
    v, u = rng.standard_normal(h.shape), rng.standard_normal(7)
    assert abs((b["dx"] * v).sum() - (loss(h + 1e-6 * v, w) - loss(h - 1e-6 * v, w)) / 2e-6) <= 1e-7
    assert abs((b["dw"] * u).sum() - (loss(h, w + 1e-6 * u) - loss(h, w - 1e-6 * u)) / 2e-6) <= 1e-7


def test_reference_adamw_agrees_with_torch():
    p = torch.randn(50, dtype=torch.float64, generator=torch.Generator().manual_seed(1)).requires_grad_()
    opt = torch.optim.AdamW([p], lr=1e-2, betas=(0.8, 0.95), eps=1e-6, weight_decay=0.1)
    q, m, v = p.detach().numpy().copy(), np.zeros(50), np.zeros(50)
    for t in range(1, 6):
        p.grad = torch.randn(50, dtype=torch.float64, generator=torch.Generator().manual_seed(10 + t))
        f = ref.adamw(q, p.grad.numpy(), m, v, t, 1e-2, (0.8, 0.95), 1e-6, 0.1)
        q, m, v = f["p"], f["m"], f["v"]
        opt.step()
    assert np.abs(q - p.detach().numpy()).max() <= 1e-14


def test_reference_rounding_at_random():
    """All 2^16 random numbers: the mean is the value, neighbours are the two codes around it, exact values stay."""
    r = np.arange(1 << 16, dtype=np.float64).reshape(-1, 64)
    for value, low, high in ((0.3, 0.28125, 0.3125), (-100.0, -96, -104), (0.001, 0, 2.0 ** -9), (448.0, 448, 448), (3.0, 3, 3)):
        v = np.full(r.shape, value)
        v[:, 0] = 448.0
        one, _ = ref.encode_at_random(v, r, False, np.zeros(r.shape))
        one = one.reshape(r.shape)[:, 1:]
        assert set(np.unique(one)) <= {low, high}
        assert abs(one.mean() - value) <= abs(high - low) * 2.0 ** -5
    one, _ = ref.encode_at_random(np.where(np.arange(64) == 0, 448.0, 1e-5), np.zeros((1, 64)), True, np.zeros((1, 64)))
    assert (one[1:] == 2.0 ** -9).all()


def test_reference_beam():
    z = np.array([[1.0, 2.0, 2.0], [0.0, -np.inf, 5.0]])
    flat, scores = ref.beam(z, np.array([0.0, -10.0]), 5)
    assert flat.tolist() == [1, 2, 0, 5, 3]
    p = np.exp(scores)
    assert abs(p[:3].sum() - 1) <= 1e-12 and abs(p[3:].sum() - np.exp(-10)) <= 1e-15
    flat, scores = ref.beam(z, np.array([0.0, -10.0]), 6, np.array([True, False]), 2)
    assert flat.tolist() == [2, 5, 3, 0, 1, 4] and scores[2] == 0
