"""The norm's values, h and scales have the same bits whatever else the call returns."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def ops():
    from paper_2412_11810_b200 import ops as o
    return o


@pytest.mark.parametrize("residual", [False, True])
@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("rows,n", [(1, 1), (300, 24), (1000, 64), (2000, 130), (700, 1024), (40, 1030), (3000, 2048), (200, 8192), (64, 16384), (20, 20480), (20, 20001)])
def test_an_8_bit_copy_changes_nothing_else(rows, n, dtype, residual):
    g = torch.Generator().manual_seed(n)
    x = torch.randn(rows, n, generator=g).to(DT[dtype]).cuda()
    r = (3 * torch.randn(rows, n, generator=g)).to(DT[dtype]).cuda() if residual else None
    if dtype != "fp16" and rows > 1:
        x[1] *= 1e30    # squares that leave fp32
    w = (1 + 0.3 * torch.randn(n, generator=g)).to(DT[dtype]).cuda()
    y, h, rstd, _ = ops().rms_norm(x, w, r)
    kept = []
    for keep in ("int8", "e4m3"):
        y2, h2, rstd2, k = ops().rms_norm(x, w, r, keep=keep)
        assert torch.equal(y, y2) and torch.equal(h, h2) and torch.equal(rstd, rstd2), keep
        _, _, rstd3, k2 = ops().rms_norm(x, w, r, keep=keep, values=False)
        assert torch.equal(rstd, rstd3) and torch.equal(k.codes, k2.codes) and torch.equal(k.scales, k2.scales)
        kept.append(k)
    assert kept[0].format != kept[1].format
