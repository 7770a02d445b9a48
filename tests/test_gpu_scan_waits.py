"""The bounded waits of the recurrence: a pass in which one of them runs out ends, and its results say so."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.fixture(autouse=True)
def checked_build(monkeypatch):
    """The self-tests of waits are in the bounds-checked build of the same sources."""
    import os
    from paper_2412_11810_b200 import binding as sb
    monkeypatch.setattr(sb, "LIB_PATH", os.path.join(sb.HERE, "libsnnckpt_debug.so"))
    monkeypatch.setattr(sb, "lib", sb._load())
    assert sb.lib.snn_debug_checks_enabled() == 1


POLLS = 1 << 14   # a tile takes microseconds, so many polls some milliseconds
MODES = {"sigmoid": 0, "direct": 1}


def problem(T, B, N, dtype, mode):
    g = torch.Generator(device="cuda").manual_seed(31)
    x, gate, dh = (torch.randn(T, B, N, generator=g, device="cuda").to(dtype) for _ in range(3))
    return x, torch.sigmoid(gate) if mode == "direct" else gate, dh, torch.randn(B, N, generator=g, device="cuda")


def lossy(x, gate, mode, step, quits, **buffers):
    """The forward pass (or with dh the backward pass) with the self-test's limits."""
    from paper_2412_11810_b200 import binding as sb
    T, B, N = x.shape
    a = sb.snn_scan_args(T, B, N, sb.SNN_DTYPE_FP32 if x.dtype == torch.float32 else sb.SNN_DTYPE_BF16, MODES[mode], x.data_ptr(), gate.data_ptr(),
                         (B * N, N), (B * N, N))
    for name, v in buffers.items():
        setattr(a, name, v if isinstance(v, int) else v.data_ptr())
    a.h_stride = a.dh_stride = a.dx_stride = a.dgate_stride = (B * N, N)
    backward = "dh" in buffers
    ws = torch.empty(max(1, sb.snn_scan_workspace(a, backward)), dtype=torch.uint8, device="cuda")
    a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel()
    sb.snn_selftest_scan_wait(a, backward, step, quits, POLLS, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()


@pytest.mark.parametrize("quits", [False, True])
@pytest.mark.parametrize("mode", ["sigmoid", "direct"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_forward(dtype, mode, quits):
    from paper_2412_11810_b200 import ops
    T, B, N, lost = 448, 3, 192, 256   # one segment of the time axis
    x, gate, _, state = problem(T, B, N, dtype, mode)
    want, _, _ = ops.gated_scan(x, gate, state, mode=mode, keep="raw")
    h, last, states = torch.zeros_like(x), torch.zeros_like(state), torch.zeros(T // 64, B, N, device="cuda")
    codes, scales = torch.zeros(T, B, N, dtype=torch.uint8, device="cuda"), torch.zeros(T, B, N // 64, dtype=torch.uint8, device="cuda")
    lossy(x, gate, mode, lost, quits, state=state, h=h, last=last, states=states, x_format=1, x_codes=codes, x_scales=scales)
    first = lost + (40 if quits else 0)      # the warp that does not wait has steps 40 to 47 of a turn
    assert torch.equal(h[:first], want[:first]) and torch.isnan(h[first:]).all() and torch.isnan(last).all()
    assert torch.isnan(states[lost // 64 + 1:]).all() and torch.isfinite(states[:lost // 64]).all()
    assert (scales[first:first + 8] == 255).all()   # what is kept of those steps is no number


@pytest.mark.parametrize("quits", [False, True])
@pytest.mark.parametrize("mode", ["sigmoid", "direct"])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_backward(dtype, mode, quits):
    from paper_2412_11810_b200 import ops
    T, B, N, lost = 448, 3, 192, 256   # one segment of the time axis
    x, gate, dh, state = problem(T, B, N, dtype, mode)
    _, _, kept = ops.gated_scan(x, gate, state, mode=mode, keep="raw")
    want = ops.gated_scan_backward(kept, dh, state)
    dx, dgate, dstate = torch.zeros_like(x), torch.zeros_like(x), torch.zeros_like(state)
    lossy(x, gate, mode, lost, quits, states=kept.states, dh=dh, dlast=state, dx=dx, dgate=dgate, dstate=dstate)
    # from the last step to the first: those of later turns are whole, the turn's own steps from the one that was lost on are not
    assert torch.equal(dx[lost + 64:], want[0][lost + 64:]) and torch.equal(dgate[lost + 64:], want[1][lost + 64:])
    end = lost + (48 if quits else 64)
    assert torch.isnan(dx[:end]).all() and torch.isnan(dgate[:end]).all() and torch.isnan(dstate).all()
    assert all(torch.equal(a, b) for a, b in zip(ops.gated_scan_backward(kept, dh, state), want))
