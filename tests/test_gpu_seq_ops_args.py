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
