"""A norm's residual in place beside x in one buffer: taken where they have no byte in common, refused where they do."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def ops():
    from paper_2412_11810_b200 import ops as o
    return o


def refused(*calls):
    for call in calls:
        with pytest.raises(ValueError):
            call()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows,n,first,second", [(7, 64, 0, 64), (7, 64, 64, 0), (9, 40, 3, 50), (1, 64, 0, 64), (300, 33, 40, 1)])
def test_a_residual_in_other_columns_of_the_same_rows(rows, n, first, second, dtype):
    """x and the residual side by side in one buffer: the sum goes into the residual's columns."""
    wide = torch.randn(rows, 130, device="cuda").to(dtype)
    before = wide.clone()
    x, residual = wide[:, first:first + n], wide[:, second:second + n]
    want = ops().rms_norm(before[:, first:first + n], None, before[:, second:second + n])   # (at the same distance, so with sums in the same order)
    y, h, rstd, _ = ops().rms_norm(x, None, residual, inplace=True)
    assert h is residual and torch.equal(h, want[1]) and torch.equal(y, want[0]) and torch.equal(rstd, want[2])
    wide[:, second:second + n] = before[:, second:second + n]
    assert torch.equal(wide, before)


def test_a_residual_in_place_that_shares_columns():
    r = ops().rms_norm
    wide = torch.randn(6, 130, device="cuda")
    before = wide.clone()
    refused(lambda: r(wide[:, :64], None, wide[:, 63:127], inplace=True), lambda: r(wide[:, 63:127], None, wide[:, :64], inplace=True),
            lambda: r(wide[1:, :64], None, wide[:-1, :64], inplace=True), lambda: r(wide[1:, :64], None, wide[:-1, 60:124], inplace=True),
            # rows that go on into the next row of the other
            lambda: r(wide.view(-1)[70:70 + 5 * 130].view(5, 130)[:, :64], None, wide[:5, :64], inplace=True),
            # rows of another distance
            lambda: r(wide.view(-1)[:320].view(5, 64), None, wide[:5, 64:128], inplace=True))
    assert torch.equal(wide, before)
