"""The vocabulary loss of fp32 operands whose values lie far apart, against its definition in 64 bits: what fp32 arithmetic
keeps has to be kept, whatever else a tensor holds."""
import pytest

import seq_reference as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

UNIT = 2.0 ** -23


def ops():
    from paper_2412_11810_b200 import ops as o
    return o


def steps(K):
    """What a sum of K products is off by, relative to the sum of their magnitudes: six tensor-core instructions per 16
    products (three parts of 8 bits per operand), each cutting two units at most, and the products left out (2^-24)."""
    return (12 * -(-K // 16) + 4) * UNIT


def definition(x, w, t):
    """Results in 64 bits and bounds that scale with every single term: no floor but fp32's own range.  Errors of the
    logits (ez) pass into the probabilities as factors; exp2 and its argument are off by 4 units of 1 + |z| + |lse|, as in
    seq_reference.vocab_loss; derivatives have 24 bits.  Below 2^-109 a value's last part is below 2^-126, where bf16 has steps
    of 2^-133: such a value is off by half a step, 2^-134."""
    x, w = x.double(), w.double()
    n, V = x.shape[0], w.shape[1]
    on = t >= 0
    at = torch.where(on, t, 0)[:, None]
    x = torch.where(on[:, None], x, 0.0)
    count = int(on.sum())
    off_x, off_w = (torch.where((v != 0) & (v.abs() < 2.0 ** -109), 2.0 ** -134, 0.0).double() for v in (x, w))
    z, ez = x @ w, steps(x.shape[1]) * (x.abs() @ w.abs()) + off_x @ w.abs() + x.abs() @ off_w
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    lse_tol = (p * ez).sum(1) + (64 + V / 2048 + 4 * lse.abs() + 2 * z.abs().amax(1)) * UNIT
    zt = z.gather(1, at).squeeze(1)
    row, row_tol = lse - zt, lse_tol + ez.gather(1, at).squeeze(1) + 4 * UNIT * (zt.abs() + (lse - zt).abs())
    ep = p * (ez + lse_tol[:, None] + 4 * UNIT * (1 + z.abs() + lse.abs()[:, None])) + 2.0 ** -126
    dz = p.clone().scatter_add_(1, at, torch.full_like(at, -1.0, dtype=p.dtype))
    ep = ep.scatter_add_(1, at, torch.full_like(at, UNIT, dtype=p.dtype)) + UNIT / 2 * dz.abs()
    dz, ep = torch.where(on[:, None], dz, 0.0), torch.where(on[:, None], ep, 0.0)
    zero = torch.zeros_like(lse)
    return {"row": torch.where(on, row, zero), "row_tol": torch.where(on, row_tol, zero), "lse": torch.where(on, lse, zero),
            "lse_tol": torch.where(on, lse_tol, zero), "dx": dz @ w.t() / count,
            "dx_tol": ((ep + (steps(V) + 8 * UNIT) * dz.abs()) @ w.abs().t() + dz.abs() @ off_w.t()) / count, "dw": x.t() @ dz / count,
            "dw_tol": (x.abs().t() @ (ep + (steps(n) + 8 * UNIT) * dz.abs()) + off_x.t() @ dz.abs()) / count}


def close(got, want, tol, what):
    err = (got.double() - want).abs() - (tol + ref.HALF_STEP["fp32"] * (want.abs() + tol) + ref.TINY["fp32"])
    assert (err <= 0).all(), f"{what}: off by {float(err.max()):.3e} more than allowed"


def inputs(n, D, V, layout, seed=1):
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(n, D, generator=g, device="cuda")
    w = torch.randn(D, V, generator=g, device="cuda") * (2 / D ** 0.5)
    t = torch.randint(0, V, (n,), generator=g, device="cuda")
    t[::11] = -100
    return x, w if layout == "feature" else w.t().contiguous().t(), t


def check(x, w, t):
    r = definition(x, w, t)
    loss, row, lse = ops().vocab_loss(x, w, t)
    dx, dw = ops().vocab_loss_backward(x, w, t, lse)
    for name, got in (("row", row), ("lse", lse), ("dx", dx), ("dw", dw)):
        close(got, r[name], r[name + "_tol"], name)


LAYOUT = pytest.mark.parametrize("layout", ["feature", "class"])
SIZE = pytest.mark.parametrize("n,D,V", [(70, 40, 300), (300, 200, 1003)])


@LAYOUT
@SIZE
@pytest.mark.parametrize("apart", [1e6, 1e9, 1e20])
def test_features_of_different_magnitudes(n, D, V, layout, apart):
    """One feature of x much larger than the others, its weights as much smaller, and the other way round."""
    x, w, t = inputs(n, D, V, layout)
    x[:, 3] *= apart
    w[3] /= apart
    check(x, w, t)
    x[:, 5] /= apart
    w[5] *= apart
    check(x, w, t)


@LAYOUT
@SIZE
def test_a_row_of_large_values_beside_ordinary_ones(n, D, V, layout):
    x, w, t = inputs(n, D, V, layout, 2)
    x[4] *= 1e8
    assert int(t[4]) >= 0
    check(x, w, t)


@LAYOUT
def test_a_class_of_large_weights_beside_ordinary_ones(layout):
    x, w, t = inputs(70, 40, 300, layout, 3)
    w[:, 7] *= 1e7
    check(x, w, t)


@LAYOUT
@SIZE
@pytest.mark.parametrize("size", [1e-2, 1e-6, 1e4])
def test_rows_that_are_not_finite_leave_the_others_alone(n, D, V, layout, size):
    """An infinity or a NaN in a row that counts makes that row's loss no number, and the mean and dw with it; the other rows
    keep theirs."""
    x, w, t = inputs(n, D, V, layout, 4)
    x, w = x * size, w / size
    r = definition(x, w, t)
    bad = torch.zeros(n, dtype=torch.bool, device="cuda")
    for i, v in ((1, float("inf")), (9, float("nan")), (40, float("-inf"))):
        assert int(t[i]) >= 0
        x[i, i % D] = v
        bad[i] = True
    loss, row, lse = ops().vocab_loss(x, w, t)
    dx, dw = ops().vocab_loss_backward(x, w, t, lse)
    assert not torch.isfinite(loss) and not torch.isfinite(row[bad]).any() and torch.isnan(dx[bad]).all()
    for name, got in (("row", row), ("lse", lse), ("dx", dx)):
        close(got[~bad], r[name][~bad], r[name + "_tol"][~bad], name)


@LAYOUT
@SIZE
@pytest.mark.parametrize("size", [1e-30, 1e-32, 1e30])
def test_operands_near_the_ends_of_the_range(n, D, V, layout, size):
    x, w, t = inputs(n, D, V, layout, 5)
    check(x * size, w / size, t)


def test_the_largest_values_of_the_type():
    """Those that round to infinity in 8 bits."""
    x, w, t = inputs(70, 40, 300, "feature", 6)
    top = torch.finfo(torch.float32).max
    x[:, 2], w[2] = top, w[2] / top
    x[5:20, 2] *= -1
    check(x, w, t)


@LAYOUT
def test_classes_of_small_probability(layout):
    """Logits from 0 down to -60: the gradients of rare classes keep their bits too."""
    x, w, t = inputs(300, 64, 500, layout, 7)
    x[:, 0], w[0] = 1.0, torch.linspace(0, -60, 500, device="cuda")
    w[1:] *= 0.1
    t = torch.where(t >= 0, t % 20, t)
    check(x, w, t)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_sums_over_many_rows_stay_within_the_range_of_their_mean(dtype):
    """The gradient by w is a mean over the rows: finite for values whose sum over the rows is not."""
    n, D, V = 3000, 8, 4
    x = torch.full((n, D), 2.0 ** 127, dtype=dtype, device="cuda")
    w = torch.zeros(D, V, dtype=dtype, device="cuda")
    t = torch.zeros(n, dtype=torch.int64, device="cuda")
    _, _, lse = ops().vocab_loss(x, w, t)
    dx, dw = ops().vocab_loss_backward(x, w, t, lse)
    # four classes of the same logit: the derivatives are -3/4 and 1/4, exact but for the roundings of lse and exp2 (below 2^-20)
    want = torch.tensor([-0.75, 0.25, 0.25, 0.25], dtype=torch.float64, device="cuda").expand(D, V) * 2.0 ** 127
    assert ((dw.double() - want).abs() <= want.abs() * (2.0 ** -20 + torch.finfo(dtype).eps / 2)).all() and (dx == 0).all()
