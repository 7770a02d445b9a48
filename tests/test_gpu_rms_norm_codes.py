"""8-bit copies of the norm where y stands on a border: ties between two codes, and a group's largest value at its scale's limit.  Codes and
scales are those of the formula in 64 bits."""
import numpy as np
import pytest

import model_reference as ref
from seq_reference import eight_bits

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def ops():
    from paper_2412_11810_b200 import ops as o
    return o


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def check(x, w, eps, keep, what=""):
    kept = ops().rms_norm(x, w, eps=eps, keep=keep, values=False)[3]
    y = ref.norm_forward(f64(x), None if w is None else f64(w), eps)["y"]
    values, scales = eight_bits(y, keep)
    assert np.array_equal(kept.scales.cpu().numpy(), scales), what
    got = f64(ops().unpack_activation(kept, torch.float32))
    assert np.array_equal(got, values), f"{what}: {int((got != values).sum())} of {got.size}"


# rows by vectors, by pairs, by single values, and rows beyond registers
WIDTHS = [64, 512, 4096, 1024 + 4, 2052, 20480, 20004]


@pytest.mark.parametrize("keep", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,weight", [("fp32", "fp32"), ("bf16", "bf16"), ("bf16", "fp32"), ("fp16", "fp16")])
@pytest.mark.parametrize("n", WIDTHS)
def test_ties_go_to_the_even_code(n, dtype, weight, keep):
    """A quarter of h is +-2^(k+1), the rest zero: the scale is 2^-k exactly, and y = +-2 w where h is not zero.  The weights are all
    multiples of an eighth from a group's largest on down, so that a good part of y lies in the middle between two codes."""
    x = torch.zeros(4, n)
    x[:, ::4] = 2.0
    x[1] *= -1
    x[2, ::8] *= -1
    x[3] *= 2.0 ** -5
    top = 64 if keep == "int8" else 224
    w = torch.arange(n) * 4099 % (8 * top) / 8     # (up to 11 significant bits: bf16 rounds them to 8)
    w[::64] = top
    # mean(h^2) is 1 to the bit, beside which eps vanishes in 64 bits as well; of the last row it is 2^-10
    check(x.to(DT[dtype]).cuda(), w.to(DT[weight]).cuda(), 1e-30, keep)
    # with eps as usual the scale is below one by 5e-7, and no y on a border
    check(x[:3].to(DT[dtype]).cuda(), w.to(DT[weight]).cuda(), 1e-6, keep)
    if n <= 4096:   # rows that begin at an odd element: value by value
        wide = torch.full((4, n + 6), float("nan"), dtype=DT[dtype], device="cuda")
        wide[:, 3:3 + n] = x.to(DT[dtype])
        check(wide[:, 3:3 + n], w.to(DT[weight]).cuda(), 1e-30, keep)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("n", [64, 1028, 20480])
def test_largest_values_at_the_limit_of_a_scale(n, dtype):
    """448 x 2^k is the largest e4m3 value of its scale, 128 x 2^k of int8 belongs to the next one; and the numbers beside them."""
    x = torch.zeros(2, n)
    x[:, ::4] = 2.0
    for half in (224.0, 112.0, 1.75 * 2.0 ** -20, 64.0, 2.0 ** -9, 1.0):
        for beside in (-1, 0, 1):
            w = torch.full((n,), half / 3).to(DT[dtype])
            at = torch.tensor(half, dtype=DT[dtype])
            if beside:
                at = at * (1 + beside * torch.finfo(DT[dtype]).eps)   # (rounded: the neighbour on that side, or the one behind it)
            w[::64] = at
            for keep in ("int8", "e4m3"):
                check(x.to(DT[dtype]).cuda(), w.cuda(), 1e-30, keep, (half, beside))


@pytest.mark.parametrize("keep", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("n", [8, 64, 96, 130, 4096, 20480, 333])
@pytest.mark.parametrize("size", [0.5, 1.0, 4.0, 8.0, 64.0, 512.0])
def test_rows_of_one_magnitude(size, n, dtype, keep):
    """|y| is below one by eps / (2 size^2): the largest values of its scale in int8, 127.99.. or so, and not those of the next one.
    (Squares are powers of four, so that their sum is exact.)"""
    x = torch.full((6, n), size)
    x[1] *= -1
    x[2, ::3] *= -1
    # all but one value of every group are small: the mean is not one, and y of the large ones is somewhere
    x[3, torch.arange(n) % 64 != 5] = size / 1024
    x[4, n // 2:] = 0
    x[5] = torch.where(torch.arange(n) % 4 == 1, 2 * size, 0.0)
    check(x.to(DT[dtype]).cuda(), None, 1e-6, keep)
    if n % 4 == 0:   # here |y| is 1 (and 2) to the bit
        check(x[[0, 1, 2, 5]].to(DT[dtype]).cuda(), None, 1e-30, keep)


@pytest.mark.parametrize("keep", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_rows_of_one_value(dtype, keep):
    """y = +-1 less eps / (2 h^2), or h / sqrt(eps) where h is small.  Powers of two: their squares are exact."""
    x = 2.0 ** torch.arange(-12, 12).float()[:, None] * torch.tensor([1.0, -1.0])
    check(x.reshape(-1, 1).to(DT[dtype]).cuda(), None, 1e-6, keep)
    # (3 less 1e-14 and the like)
    check(x.reshape(-1, 1).to(DT[dtype]).cuda(), torch.tensor([3.0], dtype=DT[dtype]).cuda(), 2.0 ** -24, keep)


@pytest.mark.parametrize("keep", ["int8", "e4m3"])
def test_rows_at_both_ends_beside_one_another(keep):
    """Rows that share a warp: squares beyond fp32, ordinary ones, exact ones, zeros, infinities and NaN; each as it is alone."""
    for dtype in DT:
        n, g = 32, torch.Generator().manual_seed(3)
        x = torch.randn(40, n, generator=g, dtype=torch.float64)
        big = 3e4 if dtype == "fp16" else 2e38
        x[::8] = (torch.rand(5, n, generator=g, dtype=torch.float64) * 2 - 1) * big
        x[1::8] = 4.0
        x[2::8] = 0.0
        x[3, 4], x[11, 5] = float("inf"), float("nan")
        x = x.to(DT[dtype]).cuda()
        y, _, rstd, kept = ops().rms_norm(x, keep=keep)
        for k in range(40):
            a, _, b, c = ops().rms_norm(x[k:k + 1], keep=keep)
            same = lambda p, q: torch.equal(torch.nan_to_num(p.float(), nan=7e30), torch.nan_to_num(q.float(), nan=7e30))  # noqa: E731
            assert same(a[0], y[k]) and same(b[0], rstd[k]) and torch.equal(c.scales[0], kept.scales[k]), k
            assert torch.equal(c.codes[0], kept.codes[k]), k
        keep_rows = [k for k in range(40) if k not in (3, 11)]
        check(x[[k for k in keep_rows if k % 8 in (1, 2)]], None, 1e-6, keep)
