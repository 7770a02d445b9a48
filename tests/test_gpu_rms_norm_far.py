"""8-bit copies of the norm of rows whose squares leave fp32: codes are those of the formula in 64 bits there as well."""
import pytest

import model_reference as ref
from seq_reference import eight_bits

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"fp32": torch.float32, "bf16": torch.bfloat16}


def ops():
    from paper_2412_11810_b200 import ops as o
    return o


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


@pytest.mark.parametrize("keep", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,weight", [("fp32", None), ("bf16", None), ("bf16", "bf16"), ("fp32", "fp32"), ("bf16", "fp32")])
@pytest.mark.parametrize("n", [512, 4096, 1030, 20480])
@pytest.mark.parametrize("size", [1e30, 2.5e38])
def test_rows_whose_squares_leave_fp32(size, n, dtype, weight, keep):
    """As `test_codes_are_those_of_the_formula`, of rows that are summed again scaled (at 2.5e38 rstd is subnormal, too): a scale that is good
    to 2^-28 leaves 0.3 codes of 1.2 million beside their place; one rounded to fp32 a dozen, one that is subnormal thousands."""
    rows = 1200000 // n
    g = torch.Generator().manual_seed(n)
    x = ((torch.rand(rows, n, generator=g, dtype=torch.float64) * 2 - 1) * size).to(DT[dtype]).cuda()
    w = None if weight is None else (1 + 0.3 * torch.randn(n, generator=g)).to(DT[weight]).cuda()
    kept = ops().rms_norm(x, w, keep=keep, values=False)[3]
    want, scales = eight_bits(ref.norm_forward(f64(x), None if w is None else f64(w), 1e-6)["y"], keep)
    assert int((kept.scales.cpu().numpy() != scales).sum()) <= 1
    assert int((f64(ops().unpack_activation(kept, torch.float32)) != want).sum()) <= 3
