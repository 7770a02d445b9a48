"""Refusals of the sequence-model operators that need tensors on a device."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


@pytest.mark.parametrize("width", [2 ** 31 - 1, 2 ** 31 - 63])
def test_widths_whose_last_group_passes_32_bits(width):
    """Tensors without elements: the widths alone are refused, as an argument."""
    from paper_2412_11810_b200 import ops
    x = torch.empty(0, width, device="cuda")
    y = torch.empty(0, 1, width, device="cuda")
    codes = torch.empty(0, width, dtype=torch.uint8, device="cuda")
    scales = torch.empty(0, -(-width // 64), dtype=torch.uint8, device="cuda")
    for call in (lambda: ops.pack_activation(x), lambda: ops.gated_scan(y, y), lambda: ops.gated_scan_step(x, x),
                 lambda: ops.unpack_activation(ops.PackedActivation(codes, scales, "int8", torch.float32)),
                 lambda: ops.unpack_activation(ops.PackedActivation(codes.sum(), scales, "int8", torch.float32))):
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("rows", [0, 3])
@pytest.mark.parametrize("by_class", [False, True])
def test_stride_of_a_single_row_of_dw_is_not_used(rows, by_class):
    """Through the C ABI: one feature by feature, or one class by class, with no stride given."""
    from paper_2412_11810_b200 import binding as sb
    D, V = (5, 1) if by_class else (1, 7)
    x, w = torch.randn(rows, D, device="cuda"), torch.randn(D * V, device="cuda")
    t, lse = torch.zeros(rows, dtype=torch.int64, device="cuda"), torch.zeros(rows, device="cuda")
    dx, dw, want = torch.empty_like(x), torch.full((D * V,), 9.0, device="cuda"), torch.empty(D * V, device="cuda")
    for stride, out in ((0, dw), (D * V, want)):
        a = sb.snn_vocab_loss_args(rows, D, V, sb.SNN_DTYPE_FP32, x.data_ptr(), D, w.data_ptr(), stride,
                                   sb.SNN_W_BY_CLASS if by_class else sb.SNN_W_BY_FEATURE, 64, t.data_ptr(), -100, 1.0)
        a.dloss, a.lse, a.dx, a.dx_stride, a.dw, a.dw_stride = 1.0, lse.data_ptr(), dx.data_ptr(), D, out.data_ptr(), stride
        ws = torch.empty(sb.snn_vocab_loss_workspace(a, True), dtype=torch.uint8, device="cuda")
        a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel()
        sb.snn_vocab_loss_backward(a, torch.cuda.current_stream().cuda_stream)
    torch.cuda.synchronize()
    assert torch.equal(dw, want) and (rows > 0 or (dw == 0).all())
