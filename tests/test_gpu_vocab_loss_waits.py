"""The bounded waits of the vocabulary loss: a pass in which one of them runs out ends, and its results say so."""
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


DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
POLLS = 1 << 14   # a tile takes microseconds, so many polls some milliseconds
GRAD, DX, DW = 0, 1, 2


def problem(n, D, V, dtype):
    g = torch.Generator(device="cuda").manual_seed(21)
    x = torch.randn(n, D, generator=g, device="cuda").to(DT[dtype])
    w = (torch.randn(V, D, generator=g, device="cuda") / D ** 0.5).to(DT[dtype]).t()
    t = torch.randint(0, V, (n,), generator=g, device="cuda")
    t[::9] = -100
    return x, w, t


def backward_with_a_lost_wait(x, w, t, lse, kernel, unit, quits):
    """`vocab_loss_backward` with the self-test's limits."""
    from paper_2412_11810_b200 import binding as sb, ops
    a = ops._vocab_args(x, w, t, 1.0, -100)
    dx, dw = torch.zeros_like(x), x.new_zeros((w.shape[1], w.shape[0])).t()
    a.dloss, a.lse, a.dx, a.dx_stride, a.dw, a.dw_stride = 1.0, lse.data_ptr(), dx.data_ptr(), a.dim, dw.data_ptr(), a.dim
    ws = ops._loss_workspace(a, True, x)  # noqa: F841
    sb.snn_selftest_vocab_loss_wait(a, True, kernel, unit, quits, POLLS, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    return dx, dw


# four warps at 16 k-blocks and more, eight below, sums in registers in fp32
CASES = [("bf16", 1024), ("bf16", 64), ("fp32", 64)]


@pytest.mark.parametrize("quits", [False, True])
@pytest.mark.parametrize("dtype,D", CASES)
def test_pass_ends_when_warps_disagree_about_a_wait(dtype, D, quits):
    """One warp of the derivatives' epilogue gives up (quits) while the others find their tile: all of them have to leave, or
    those that stay would wait for it at their common barrier without end."""
    from paper_2412_11810_b200 import ops
    x, w, t = problem(2600, D, 5000, dtype)
    _, _, lse = ops.vocab_loss(x, w, t)
    want = ops.vocab_loss_backward(x, w, t, lse)
    dx, _ = backward_with_a_lost_wait(x, w, t, lse, GRAD, 100, quits)
    assert torch.isnan(dx[t >= 0]).all() and (dx[t < 0] == 0).all()
    # the device is none the worse for it
    assert all(torch.equal(a, b) for a, b in zip(ops.vocab_loss_backward(x, w, t, lse), want))


@pytest.mark.parametrize("quits", [False, True])
@pytest.mark.parametrize("dtype,D", CASES)
def test_losses_are_nan_when_a_wait_runs_out(dtype, D, quits):
    from paper_2412_11810_b200 import binding as sb, ops
    x, w, t = problem(2600, D, 5000, dtype)
    a = ops._vocab_args(x, w, t, 1.0, -100)
    row, lse, loss = (torch.zeros(s, device="cuda") for s in (2600, 2600, ()))
    a.row_loss, a.lse, a.loss = row.data_ptr(), lse.data_ptr(), loss.data_ptr()
    ws = ops._loss_workspace(a, False, x)  # noqa: F841
    sb.snn_selftest_vocab_loss_wait(a, False, 0, 100, quits, POLLS, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert torch.isnan(loss)
    # the 220 tiles are taken in the order of the rows: those from the 100th on belong to every row (with `quits`, to the
    # rows of the warp that left)
    on = t >= 0
    lost = on if not quits else on & (torch.arange(2600, device="cuda") % 128 // 32 == 2)
    assert torch.isnan(row[lost]).all() and torch.isnan(lse[lost]).all() and (row[~on] == 0).all()


@pytest.mark.parametrize("quits", [False, True])
@pytest.mark.parametrize("kernel", [GRAD, DX, DW])
@pytest.mark.parametrize("dtype,D", CASES + [("fp16", 72), ("bf16", 1001)])
def test_gradients_are_nan_when_a_wait_runs_out(dtype, D, kernel, quits):
    """No gradient is finite that rests on a tile that never came: all of dx, and of dw all if its derivatives are in doubt,
    the tiles left out if it is its own product."""
    from paper_2412_11810_b200 import ops
    x, w, t = problem(2600, D, 5000, dtype)
    _, _, lse = ops.vocab_loss(x, w, t)
    dx, dw = backward_with_a_lost_wait(x, w, t, lse, kernel, 0, quits)
    assert torch.isnan(dx[t >= 0]).all()
    if kernel != DW or not quits:
        assert torch.isnan(dw).all()
    else:   # the warp that left had 32 of every 128 classes
        assert torch.isnan(dw[:, torch.arange(5000, device="cuda") % 128 // 32 == 2][: 128 if dtype == "fp32" else 256]).all()
    if kernel == DW and not quits and D == 1024:   # 20 x 4 tiles, classes by features; those before the 7th are whole
        want = ops.vocab_loss_backward(x, w, t, lse)[1]
        _, dw = backward_with_a_lost_wait(x, w, t, lse, kernel, 7, quits)
        rows = torch.arange(5000, device="cuda") // 256
        cols = torch.arange(D, device="cuda") // 256
        unit = cols[:, None] + 4 * rows[None, :]
        assert torch.isnan(dw[unit >= 7]).all() and torch.equal(dw[unit < 7], want[unit < 7])
