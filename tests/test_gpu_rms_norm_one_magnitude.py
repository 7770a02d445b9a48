"""8-bit copies of rows whose values are all of one magnitude, of any size: |y| is below one by eps / (2 h^2), so int8 scales are those of
[1/2, 1), however close to one that is."""
import numpy as np
import pytest

import model_reference as ref
from seq_reference import eight_bits

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


@pytest.mark.parametrize("keep", ["int8", "e4m3"])
@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("n", [1, 3, 16, 64, 100, 513, 1024, 4096, 20480])
def test_scales_and_codes(n, dtype, residual, keep):
    """Sizes up to 100: |y| is below one by 5e-11 or more, and y is computed to 2^-36 (1.5e-11; a 16-bit h times the scale's upper 12 bits
    and a rest of 24) or better, the sums of squares of one magnitude exactly."""
    from paper_2412_11810_b200 import ops
    rows = 4000 if n < 1000 else 300
    g = torch.Generator().manual_seed(n)
    c = torch.exp(torch.rand(rows, 1, generator=g, dtype=torch.float64) * (np.log(100) - np.log(0.01)) + np.log(0.01))
    sign = torch.randint(0, 2, (rows, n), generator=g) * 2 - 1
    x = (c * sign).to(DT[dtype]).cuda()
    half = x / 2 if residual else None     # (exact, and so is their sum)
    kept = ops.rms_norm(half if residual else x, None, half, keep=keep, values=False)[3]
    y = ref.norm_forward(f64(x), None, 1e-6)["y"]
    values, scales = eight_bits(y, keep)
    assert np.array_equal(kept.scales.cpu().numpy(), scales)
    assert np.array_equal(f64(ops.unpack_activation(kept, torch.float32)), values)
