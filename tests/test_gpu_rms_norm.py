"""The norm with the residual's addition on the GPU against its definition in 64 bits."""
import numpy as np
import pytest

import model_reference as ref
from seq_reference import eight_bits, rounding

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def ops():
    from paper_2412_11810_b200 import ops as o
    return o


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def close(got, want, tol, dtype, what):
    got = f64(got)
    assert got.shape == want.shape, what
    err = np.abs(got - want) - (tol + rounding(np.abs(want) + tol, dtype))
    assert not np.isnan(got).any() and (err <= 0).all(), f"{what}: off by {np.nanmax(err):.3e} more than allowed"


def place(v, layout):
    """The same values in rows of a wider buffer, from an odd element on, or two rows apart."""
    if layout == "offset":
        wide = torch.full((v.shape[0], v.shape[1] + 6), float("nan"), dtype=v.dtype, device=v.device)
        wide[:, 3:3 + v.shape[1]] = v
        return wide[:, 3:3 + v.shape[1]]
    if layout == "apart":
        wide = torch.full((v.shape[0], 2, v.shape[1]), float("nan"), dtype=v.dtype, device=v.device)
        wide[:, 0] = v
        return wide[:, 0]
    return v


def inputs(rows, n, dtype, seed, layout="dense", weight="same", residual=True):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    x, res, dy, dh = ((s * r(rows, n)).to(DT[dtype]) for s in (1.0, 3.0, 0.5, 0.5))
    x[:, ::50] *= 20
    w = None if weight is None else (1 + 0.3 * r(n)).to(torch.float32 if weight == "fp32" else DT[dtype]).cuda()
    x, res, dy, dh = (place(v.cuda(), layout) for v in (x, res, dy, dh))
    return x, res if residual else None, w, dy, dh if residual else None


def total(x, res):
    return x if res is None else (x.float() + res.float()).to(x.dtype)


def check(x, res, w, dy, dh, dtype, eps=1e-6, **kw):
    h_want = total(x, res)
    f = ref.norm_forward(f64(h_want), None if w is None else f64(w), eps)
    y, h, rstd, kept = ops().rms_norm(x, w, res, eps=eps, **kw)
    assert kept is None and torch.equal(h, h_want) and (res is not None or h is x)
    close(rstd, f["rstd"], f["rstd_tol"], "fp32", "rstd")
    close(y, f["y"], f["y_tol"], dtype, "y")
    dx, dw = ops().rms_norm_backward(h, rstd, dy, w, dh)
    b = ref.norm_backward(f64(h), f64(rstd), None if w is None else f64(w), f64(dy), None if dh is None else f64(dh))
    close(dx, b["dx"], b["dx_tol"], dtype, "dx")
    if w is None:
        assert dw is None
    else:
        assert dw.dtype is w.dtype
        close(dw, b["dw"], b["dw_tol"], "fp32" if w.dtype is torch.float32 else dtype, "dw")


@pytest.mark.parametrize("keep", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype,weight,n", [("fp32", "same", 512), ("bf16", "same", 512), ("bf16", "fp32", 4096), ("fp16", "same", 1030), ("fp32", None, 321),
                                            ("bf16", "same", 20000)])
def test_codes_are_those_of_the_formula(dtype, weight, n, keep):
    """Codes are rounded once.  The scale is good to 2^-28 or so, and a code of int8 lies 64 steps from zero on average: of 1.2 million
    64 x 2^-28 x 1.2 million = 0.3 are the ones beside it; products rounded to fp32 before leave a dozen."""
    rows = 1200000 // n
    x, res, w, _, _ = inputs(rows, n, dtype, n, weight=weight)
    _, h, _, kept = ops().rms_norm(x, w, res, keep=keep, values=False)
    want, _ = eight_bits(ref.norm_forward(f64(h), None if w is None else f64(w), 1e-6)["y"], keep)
    differ = int((f64(ops().unpack_activation(kept, torch.float32)) != want).sum())
    assert differ <= 3


WIDTHS = [1, 7, 8, 63, 64, 65, 130, 256, 264, 520, 1030, 2048, 2056, 4096, 8192, 8200, 16384, 16392, 20001]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("n", WIDTHS)
def test_norm_and_gradients(n, dtype):
    for rows, weight, residual in ((1, "same", True), (3, "fp32", False), (37, "same", True), (5, None, True)):
        check(*inputs(rows, n, dtype, n + rows, weight=weight, residual=residual), dtype)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("n", [16, 24, 32, 48, 80, 112, 160, 192, 320, 512, 576])
def test_several_rows_of_a_warp(n, dtype):
    for rows in (1, 2, 5, 33, 500):
        x, res, w, dy, dh = inputs(rows, n, dtype, n + rows)
        check(x, res, w, dy, dh, dtype)
        want = ops().rms_norm(x, w, res, keep="int8")
        alone = [ops().rms_norm(x[k:k + 1].clone(), w, res[k:k + 1].clone(), keep="int8")[3] for k in range(0, rows, 7)]
        assert all(torch.equal(a.codes[0], want[3].codes[k * 7]) and torch.equal(a.scales[0], want[3].scales[k * 7]) for k, a in enumerate(alone))


@pytest.mark.parametrize("dtype,weight", [("fp32", "same"), ("bf16", "same"), ("bf16", "fp32"), ("fp16", None)])
@pytest.mark.parametrize("layout", ["dense", "offset", "apart"])
@pytest.mark.parametrize("rows,n", [(700, 96), (3000, 40), (2500, 256), (1500, 1032), (300, 8192), (200, 9000)])
def test_norm_of_many_rows_and_layouts(rows, n, layout, dtype, weight):
    check(*inputs(rows, n, dtype, 7, layout, weight), dtype)


@pytest.mark.parametrize("keep", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("rows,n,layout", [(5, 1, "dense"), (9, 64, "dense"), (33, 130, "offset"), (40, 1030, "dense"), (3, 4096, "apart"), (2, 20008, "dense"),
                                           (70, 200, "dense")])
def test_norm_kept_in_8_bits(rows, n, layout, dtype, keep):
    x, res, w, _, _ = inputs(rows, n, dtype, 3, layout)
    y, h, rstd, kept = ops().rms_norm(x, w, res, keep=keep)
    only, h2, rstd2, kept2 = ops().rms_norm(x, w, res, keep=keep, values=False)
    assert only is None and torch.equal(h, h2) and torch.equal(rstd, rstd2)
    assert torch.equal(kept.codes, kept2.codes) and torch.equal(kept.scales, kept2.scales)
    assert kept.format == keep and kept.dtype is x.dtype and kept.codes.shape == x.shape
    f = ref.norm_forward(f64(h), f64(w), 1e-6)
    close(y, f["y"], f["y_tol"], dtype, "y")
    _, scales = eight_bits(f["y"], keep)
    # a group's scale is that of its largest value, where that is not within its error of a border
    low, high = (eight_bits(np.abs(f["y"]) + s * f["y_tol"], keep)[1] for s in (-1, 1))
    got = kept.scales.cpu().numpy()
    assert ((got == scales) | ((got >= low) & (got <= high))).all()
    step = np.repeat(2.0 ** (got.astype(np.float64) - 127), 64, axis=1)[:, :n]
    values = f64(ops().unpack_activation(kept, torch.float32))
    u = np.abs(f["y"]) / step
    if keep == "int8":   # to nearest, ending at 127
        off = np.maximum(u - 127, 0.5) * step
    else:
        off = 0.5 * 2.0 ** (np.floor(np.log2(np.maximum(u, 2.0 ** -6))) - 3) * step
    assert (np.abs(values - f["y"]) <= off * (1 + 1e-12) + 2 * f["y_tol"]).all()


@pytest.mark.parametrize("n", [24, 1000, 16400])
@pytest.mark.parametrize("dtype,size", [("fp32", 3e38), ("bf16", 3e38), ("fp32", 1e20), ("fp32", 1e-30), ("bf16", 1e-36), ("fp16", 6e4), ("fp16", 6e-8)])
def test_values_at_the_ends_of_the_range(dtype, size, n):
    g = torch.Generator().manual_seed(1)
    x = (torch.rand(6, n, generator=g, dtype=torch.float64) * 2 - 1) * size
    x[3] = size
    x[4] = 0
    x = x.to(DT[dtype]).cuda()
    for eps in (1e-6, 1e-30):
        f = ref.norm_forward(f64(x), None, eps)
        y, _, rstd, _ = ops().rms_norm(x, eps=eps)
        close(rstd, f["rstd"], f["rstd_tol"] + 2.0 ** -126 * 2.0 ** -20, "fp32", "rstd")   # (of the largest values it is subnormal)
        close(y, f["y"], f["y_tol"] + 2.0 ** -126 * 2.0 ** -20 * np.abs(f64(x)), dtype, "y")


@pytest.mark.parametrize("n", [40, 512, 16392])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_rows_that_are_not_finite_stay_by_themselves(dtype, n):
    x, res, w, _, _ = inputs(40, n, dtype, 5)
    want, _, _, want_kept = ops().rms_norm(x, w, res, keep="int8")
    x[7, n // 2], x[20, 3], x[33, n - 1] = float("nan"), float("inf"), -float("inf")
    y, _, rstd, kept = ops().rms_norm(x, w, res, keep="int8")
    other = [k for k in range(40) if k not in (7, 20, 33)]
    assert torch.equal(y[other], want[other]) and torch.equal(kept.codes[other], want_kept.codes[other])
    assert torch.isnan(rstd[7]) and torch.isnan(y[7]).all()
    for k, at in ((20, 3), (33, n - 1)):   # 1 / inf: zero, but for the infinity itself
        assert float(rstd[k]) == 0 and torch.isnan(y[k, at]) and (y[k, [c for c in range(n) if c != at]] == 0).all()
        assert int(kept.scales[k, at // 64]) == 255


def test_residual_in_place_and_three_dimensions():
    x, res, w, dy, dh = inputs(6 * 5, 72, "bf16", 9)
    want = ops().rms_norm(x, w, res)
    held = res.clone().view(6, 5, 72)
    y, h, rstd, _ = ops().rms_norm(x.view(6, 5, 72), w, held, inplace=True)
    assert h is held and torch.equal(h.view(30, 72), want[1]) and torch.equal(y.view(30, 72), want[0]) and rstd.shape == (6, 5)
    a = ops().rms_norm_backward(want[1], want[2], dy, w, dh)
    b = ops().rms_norm_backward(h, rstd, dy.view(6, 5, 72), w, dh.view(6, 5, 72))
    assert torch.equal(a[0], b[0].view(30, 72)) and torch.equal(a[1], b[1])
    # in rows of a wider buffer, whose other columns stay as they are
    wide = torch.full((30, 80), 5.0, dtype=torch.bfloat16, device="cuda")
    wide[:, :72] = res
    y, h, _, _ = ops().rms_norm(x, w, wide[:, :72], inplace=True)
    assert torch.equal(h, want[1]) and torch.equal(y, want[0]) and (wide[:, 72:] == 5).all()
    # one row
    y, h, rstd, _ = ops().rms_norm(x[0], w, res[0])
    assert torch.equal(y, want[0][0]) and rstd.shape == ()


def test_without_rows():
    x = torch.empty(0, 40, device="cuda")
    w = torch.ones(40, device="cuda")
    y, h, rstd, kept = ops().rms_norm(x, w, x, keep="int8")
    assert y.shape == (0, 40) and rstd.shape == (0,) and kept.codes.shape == (0, 40)
    dx, dw = ops().rms_norm_backward(h, rstd, x, w, x)
    assert dx.shape == (0, 40) and (dw == 0).all()


def test_a_gradient_for_all_rows_alike():
    """dy and dh with a row stride of zero."""
    x, _, w, dy, _ = inputs(50, 136, "fp32", 4, residual=False)
    _, h, rstd, _ = ops().rms_norm(x, w)
    want = ops().rms_norm_backward(h, rstd, dy[:1].repeat(50, 1), w, dy[1:2].repeat(50, 1))
    got = ops().rms_norm_backward(h, rstd, dy[:1].expand(50, 136), w, dy[1:2].expand(50, 136))
    assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("rows,n", [(4, 9), (60, 40)])
def test_gradients_against_differences(rows, n):
    x, res, w, dy, dh = inputs(rows, n, "fp32", 6)
    _, h, rstd, _ = ops().rms_norm(x, w, res)
    dx, dw = ops().rms_norm_backward(h, rstd, dy, w, dh)
    point = [f64(x) + f64(res), f64(w)]
    g = np.random.default_rng(2)
    for k, grad in enumerate((f64(dx), f64(dw))):
        v = g.standard_normal(grad.shape)

        def loss(s):
            p = [q + s * v if j == k else q for j, q in enumerate(point)]
            return (ref.norm_forward(p[0], p[1], 1e-6)["y"] * f64(dy)).sum() + (p[0] * f64(dh)).sum()

        slope = (loss(1e-6) - loss(-1e-6)) / 2e-6
        # 64 units and the rounding of h, relative to the magnitudes summed
        assert abs((grad * v).sum() - slope) <= 200 * ref.U * np.abs(grad * v).sum() + 1e-7


def test_streams_and_capture():
    x, res, w, dy, dh = inputs(300, 520, "bf16", 8)

    def both():
        y, h, rstd, kept = ops().rms_norm(x, w, res, keep="e4m3")
        return y, h, rstd, kept.codes, kept.scales, *ops().rms_norm_backward(h, rstd, dy, w, dh)

    want = both()
    assert all(torch.equal(a, b) for a, b in zip(want, both()))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = both()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = both()
    for _ in range(2):
        for t in held:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_offsets_beyond_32_bits():
    rows, n = (1 << 19) + 3, 4104     # 2.15e9 values
    x = torch.empty(rows, n, dtype=torch.bfloat16, device="cuda")
    x[:5], x[-5:] = 1.5, -2.5
    x[5:-5] = 1.0
    x[-5:, ::2] = 0.5
    y, h, rstd, kept = ops().rms_norm(x, keep="int8")
    f = ref.norm_forward(f64(x[-5:]), None, 1e-6)
    close(y[-5:], f["y"], f["y_tol"], "bf16", "y")
    assert torch.equal(kept.codes[-1], kept.codes[-5]) and int(kept.codes[-1].view(torch.int8).min()) < 0 and (y[1000:1100] == 1).all()
    dy = x
    dx, _ = ops().rms_norm_backward(h, rstd, dy)
    b = ref.norm_backward(f64(x[-5:]), f64(rstd[-5:]), None, f64(dy[-5:]), None)
    close(dx[-5:], b["dx"], b["dx_tol"], "bf16", "dx")
