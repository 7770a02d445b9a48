"""Soft-max cross entropy over a vocabulary on the GPU against its definition in 64 bits."""
import pytest

import seq_reference as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def ops():
    from paper_2412_11810_b200 import ops as o
    return o


def inputs(n, D, V, dtype, seed, layout="feature", ignored=0.1, bits=64, spread=2.0):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, D, generator=g).to(DT[dtype]).cuda()
    w = (torch.randn(D, V, generator=g) * (spread / D ** 0.5)).to(DT[dtype]).cuda()
    t = torch.randint(0, V, (n,), generator=g)
    t[torch.rand(n, generator=g) < ignored] = -100
    t = t.to(torch.int32 if bits == 32 else torch.int64).cuda()
    if layout == "class":
        w = w.t().contiguous().t()
    elif layout == "wide":     # rows of wider buffers, from an odd element on
        a = torch.full((n, D + 5), float("nan"), dtype=x.dtype, device="cuda")
        b = torch.full((D, V + 7), float("nan"), dtype=x.dtype, device="cuda")
        a[:, 1:1 + D], b[:, 3:3 + V] = x, w
        x, w = a[:, 1:1 + D], b[:, 3:3 + V]
    elif layout == "wide_class":
        b = torch.full((V, D + 8), float("nan"), dtype=x.dtype, device="cuda")
        b[:, :D] = w.t()
        w = b[:, :D].t()
    return x, w, t


def close(got, want, tol, dtype, what):
    got = got.double()
    bad = torch.isnan(want)
    assert got.shape == want.shape and torch.equal(torch.isnan(got), bad), what
    err = (got - want).abs() - (tol + ref.HALF_STEP[dtype] * (want.abs() + tol) + ref.TINY[dtype])
    err = torch.where(bad, torch.zeros_like(err), err)
    assert (err <= 0).all(), f"{what}: off by {float(err.max()):.3e} more than allowed"


def check(x, w, t, dtype, scale=1.0, ignore=-100, dloss=1.0, backward=True):
    o = ops()
    r = ref.vocab_loss(x.double(), w.double(), t, scale, ignore, dtype, dloss if isinstance(dloss, float) else float(dloss))
    loss, row, lse = o.vocab_loss(x, w, t, scale=scale, ignore_index=ignore)
    close(loss, r["loss"], r["loss_tol"], "fp32", "loss")
    close(row, r["row"], r["row_tol"], "fp32", "row_loss")
    close(lse, r["lse"], r["lse_tol"], "fp32", "lse")
    if backward:
        dx, dw = o.vocab_loss_backward(x, w, t, lse, scale=scale, ignore_index=ignore, dloss=dloss)
        assert dx.dtype == x.dtype and dw.dtype == w.dtype
        close(dx, r["dx"], r["dx_tol"], dtype, "dx")
        close(dw, r["dw"], r["dw_tol"], dtype, "dw")
        return loss, dx, dw


SIZES = [(1, 8, 2), (1, 1, 1), (3, 5, 1), (2, 64, 256), (5, 64, 300), (130, 72, 257), (257, 128, 1000), (300, 1, 513), (64, 200, 5003),
         (256, 256, 256), (513, 640, 777)]


@pytest.mark.parametrize("layout", ["feature", "class"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("n,D,V", SIZES)
def test_loss_and_gradients(n, D, V, dtype, layout):
    check(*inputs(n, D, V, dtype, 1, layout), dtype)


@pytest.mark.parametrize("layout", ["feature", "class", "wide", "wide_class"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("n,D,V", [(1, 1024, 5000), (2, 72, 20001), (3, 2048, 127), (4, 33, 129), (1, 8192, 40), (4, 2056, 50), (1, 4, 70000), (5, 64, 300)])
def test_loss_of_a_few_rows(n, D, V, dtype, layout):
    check(*inputs(n, D, V, dtype, 13, layout), dtype, scale=0.7, backward=False)


@pytest.mark.parametrize("layout", ["wide", "wide_class"])
@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("bits", [32, 64])
def test_loss_layouts_and_target_types(bits, dtype, layout):
    check(*inputs(70, 48, 333, dtype, 2, layout, bits=bits), dtype)
    check(*inputs(70, 51, 330, dtype, 3, layout, bits=bits), dtype)


@pytest.mark.parametrize("dtype", ["bf16", "fp16", "fp32"])
def test_loss_scale_and_upstream_gradient(dtype):
    x, w, t = inputs(90, 100, 400, dtype, 4)
    check(x, w, t, dtype, scale=0.25, dloss=3.0)
    check(x, w, t, dtype, scale=-2.0, dloss=torch.tensor(0.5, device="cuda"))


@pytest.mark.parametrize("layout", ["feature", "class"])
def test_loss_more_than_one_piece_of_the_vocabulary(layout):
    """dz of 5000 rows x 60001 classes is three pieces; also more rows than one wave of tiles, and a split contraction."""
    check(*inputs(5000, 40, 60001, "bf16", 5, layout), "bf16")


def test_loss_of_more_than_32_bits_of_logits():
    """70000 x 40000 logits, never stored: the last rows and the last classes against the definition."""
    o = ops()
    n, D, V = 70000, 16, 40000
    x, w, t = inputs(n, D, V, "bf16", 15, "class")
    _, row, lse = o.vocab_loss(x, w, t)
    dx, dw = o.vocab_loss_backward(x, w, t, lse)
    rows = slice(n - 64, n)
    r = ref.vocab_loss(x[rows].double(), w.double(), t[rows], 1.0, -100, "bf16")
    close(row[rows], r["row"], r["row_tol"], "fp32", "row_loss")
    part, count = int((t[rows] >= 0).sum()), int((t >= 0).sum())
    close(dx[rows], r["dx"] * part / count, r["dx_tol"] * part / count, "bf16", "dx")
    # the gradient of the last 32 classes, from all rows
    z = torch.empty(n, 32, dtype=torch.float64, device="cuda")
    for a in range(0, n, 10000):
        b = slice(a, a + 10000)
        full = x[b].double() @ w.double()
        z[b] = torch.softmax(full, 1)[:, -32:]
    at = t - (V - 32)
    on = (t >= 0).double()[:, None]
    z = (z - torch.nn.functional.one_hot(at.clamp(min=-1) + 1, 33)[:, 1:].double()) * on
    want = x.double().t() @ z / count
    # dz is rounded to bf16 (2^-8 of each) and computed to 2^-16; the sum over the rows is cut 2 n / 16 times by 2^-23
    tol = x.double().abs().t() @ z.abs() / count * (2.0 ** -8 + 2.0 ** -16 + 2 * n / 16 * 2.0 ** -23)
    close(dw[:, -32:], want, tol, "bf16", "dw")


def test_loss_long_contraction_in_fp32():
    check(*inputs(40, 2000, 3001, "fp32", 6), "fp32")


def test_loss_fp32_of_any_magnitude():
    """fp32 operands are scaled as a whole: large ones, small ones, zeros, and padding that is no number."""
    x, w, t = inputs(40, 64, 300, "fp32", 12)
    check(x * 1e12, w * 1e-12, t, "fp32")
    check(x * 1e-30, w * 1e30, t, "fp32")
    check(torch.zeros_like(x), w, t, "fp32")
    check(x, torch.zeros_like(w), t, "fp32")
    x[t < 0] = float("inf")
    check(x, w, t, "fp32")


def test_loss_rows_that_do_not_count():
    o = ops()
    x, w, t = inputs(50, 64, 300, "bf16", 7, ignored=0.0)
    t[::7] = -100
    x[::7] = float("nan")     # padding may hold anything
    x[7] = float("inf")
    _, dx, dw = check(x, w, t, "bf16")
    assert (dx[::7] == 0).all() and torch.isfinite(dw).all()
    # another index to ignore: the class itself
    t = torch.where(t < 0, 5, t)
    x = torch.nan_to_num(x, 0.0, 0.0, 0.0)
    check(x, w, t, "bf16", ignore=5)
    # none counts
    t[:] = -100
    loss, row, lse = o.vocab_loss(x, w, t)
    dx, dw = o.vocab_loss_backward(x, w, t, lse)
    assert float(loss) == 0 and all((v == 0).all() for v in (row, lse, dx, dw))


def test_loss_targets_that_are_no_class():
    o = ops()
    x, w, t = inputs(9, 64, 300, "bf16", 8, ignored=0.0)
    t[3], t[4], t[5], t[6] = 300, -1, 2 ** 32 + 5, -2 ** 40
    loss, row, lse = o.vocab_loss(x, w, t)
    assert torch.isnan(loss) and torch.isnan(row[3:7]).all() and torch.isfinite(row[:3]).all() and torch.isfinite(row[7:]).all()
    dx, dw = o.vocab_loss_backward(x, w, t, lse)
    good = t.clone()
    good[3:7] = -100
    _, _, lse2 = o.vocab_loss(x, w, good)
    dx2, dw2 = o.vocab_loss_backward(x, w, good, lse2)
    assert torch.equal(dx, dx2) and torch.equal(dw, dw2)


def test_loss_nothing_to_do():
    o = ops()
    x, w = torch.zeros(0, 8, device="cuda"), torch.ones(8, 30, device="cuda")
    t = torch.zeros(0, dtype=torch.int64, device="cuda")
    loss, row, lse = o.vocab_loss(x, w, t)
    dx, dw = o.vocab_loss_backward(x, w, t, lse)
    assert float(loss) == 0 and row.shape == (0,) and dx.shape == (0, 8) and (dw == 0).all()


def test_loss_extreme_logits():
    """Logits of hundreds, both signs: the maximum is taken out before anything is exponentiated."""
    x, w, t = inputs(40, 64, 700, "bf16", 9, spread=120.0)
    check(x, w, t, "bf16")


def test_loss_gradient_against_differences():
    x, w, t = inputs(30, 24, 100, "fp32", 10)
    _, dx, dw = check(x, w, t, "fp32")
    g = torch.Generator(device="cuda").manual_seed(0)
    for which, grad in ((0, dx), (1, dw)):
        v = torch.randn(grad.shape, generator=g, device="cuda", dtype=torch.float64)
        eps = 1e-5

        def loss(s):
            a, b = (x.double() + s * v, w.double()) if which == 0 else (x.double(), w.double() + s * v)
            return float(torch.nn.functional.cross_entropy(a @ b, t, ignore_index=-100))

        slope = (loss(eps) - loss(-eps)) / (2 * eps)
        # eps^2 times a third derivative, 1e-16 / eps, and 32-bit gradients
        assert abs(float((grad.double() * v).sum()) - slope) <= 1e-5 * float((grad.double() * v).abs().sum()) + 1e-8


def test_loss_results_do_not_depend_on_the_call():
    o = ops()
    x, w, t = inputs(700, 96, 3001, "bf16", 11, "class")

    def step():
        loss, row, lse = o.vocab_loss(x, w, t)
        return (loss, row, lse, *o.vocab_loss_backward(x, w, t, lse))

    want = [v.clone() for v in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a = step()
    b = step()
    torch.cuda.synchronize()
    for got in (a, b):
        assert all(torch.equal(v, u) for v, u in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for v in held:
        v.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(v, u) for v, u in zip(held, want))
    x.mul_(0.5)
    graph.replay()
    again = step()
    torch.cuda.synchronize()
    assert all(torch.equal(v, u) for v, u in zip(held, again)) and not torch.equal(held[0], want[0])
