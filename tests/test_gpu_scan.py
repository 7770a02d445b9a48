"""The gated linear recurrence and 8-bit activations on the GPU against their definitions in 64 bits."""
import numpy as np
import pytest

import seq_reference as ref

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
    err = np.abs(got - want) - (tol + ref.rounding(np.abs(want) + tol, dtype))
    assert got.shape == want.shape, what
    assert not np.isnan(got).any() and (err <= 0).all(), f"{what}: off by {np.nanmax(err):.3e} more than allowed"


def place(v, layout):
    """The values [T][B][N] in memory of another layout."""
    T, B, N = v.shape
    if layout == "batch_major":
        return v.transpose(0, 1).contiguous().transpose(0, 1)
    if layout == "offset":      # rows of a wider buffer, from an odd element on
        wide = torch.full((T, B, N + 6), float("nan"), dtype=v.dtype, device=v.device)
        wide[..., 3:3 + N] = v
        return wide[..., 3:3 + N]
    return v


def inputs(T, B, N, dtype, mode, seed, lengths=None, layout="dense"):
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(T, B, N, generator=g)
    gate = torch.randn(T, B, N, generator=g) * 2 + 1
    if mode == "direct":
        gate = torch.sigmoid(gate) * torch.where(torch.rand(T, B, N, generator=g) < 0.1, -1.0, 1.0)
    dh = torch.randn(T, B, N, generator=g)
    x, gate, dh = x.to(DT[dtype]), gate.to(DT[dtype]), dh.to(DT[dtype])
    if lengths is not None:   # what lies behind a sequence's end is poison
        dead = torch.from_numpy(~ref._on(T, B, np.asarray(lengths))).expand(T, B, N)
        for v in (x, gate, dh):
            v[dead] = float("nan")
    state, dlast = torch.randn(B, N, generator=g), torch.randn(B, N, generator=g)
    x, gate, dh = (place(v.cuda(), layout) for v in (x, gate, dh))
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    return x, gate, dh, state.cuda(), dlast.cuda(), n


SIZES = [(1, 1, 1), (2, 3, 64), (16, 2, 65), (17, 2, 65), (64, 2, 130), (65, 1, 2), (130, 3, 7), (513, 2, 66), (1100, 1, 100),
         (1100, 3, 1), (130, 600, 3), (200, 300, 2)]


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("mode", ["sigmoid", "direct"])
@pytest.mark.parametrize("T,B,N", SIZES)
def test_scan_with_gradients(T, B, N, mode, dtype):
    x, gate, dh, state, dlast, _ = inputs(T, B, N, dtype, mode, 1)
    f = ref.scan_forward(f64(x), f64(gate), f64(state), None, mode)
    h, last, kept = ops().gated_scan(x, gate, state, mode=mode)
    assert kept is None
    close(h, f["h"], f["h_tol"], dtype, "h")
    close(last, f["last"], f["last_tol"], "fp32", "last")
    h2, last2, kept = ops().gated_scan(x, gate, state, mode=mode, keep="raw")
    close(h2, f["h"], f["h_tol"], dtype, "h with states kept")
    close(last2, f["last"], f["last_tol"], "fp32", "last with states kept")
    r = ref.scan_backward(f64(x), f64(gate), f64(state), None, mode, f64(dh), f64(dlast))
    close(kept.states, r["states"], r["states_tol"], "fp32", "kept states")
    for name, got in zip(("dx", "dgate", "dstate"), ops().gated_scan_backward(kept, dh, dlast)):
        close(got, r[name], r[name + "_tol"], "fp32" if name == "dstate" else dtype, name)


@pytest.mark.parametrize("layout", ["dense", "batch_major", "offset"])
@pytest.mark.parametrize("dtype,keep", [("fp32", "raw"), ("bf16", "raw"), ("fp32", "int8"), ("bf16", "int8"), ("fp16", "e4m3")])
@pytest.mark.parametrize("T,B,N,lengths", [(70, 4, 130, (0, 70, 33, 1)), (600, 3, 67, (64, 599, 777)), (150, 2, 64, (-3, 128)),
                                           (5, 3, 9, (5, 0, 2)), (9, 2, 128, (0, 0)), (700, 3, 80, (700, 65, 129)),
                                           (2000, 1, 16, (1999,)), (2000, 2, 16, (700, 3)), (3000, 1, 33, (2561,)), (300, 200, 48, tuple((i * 37) % 301 for i in range(200)))])
def test_scan_layouts_lengths_and_kept_formats(T, B, N, lengths, dtype, keep, layout):
    x, gate, dh, state, dlast, n = inputs(T, B, N, dtype, "sigmoid", 2, lengths, layout)
    eight = None if keep == "raw" else keep
    f = ref.scan_forward(f64(x), f64(gate), f64(state), np.asarray(lengths), "sigmoid")
    r = ref.scan_backward(f64(x), f64(gate), f64(state), np.asarray(lengths), "sigmoid", f64(dh), f64(dlast), eight, eight)
    h, last, kept = ops().gated_scan(x, gate, state, lengths=n, keep=keep)
    close(h, f["h"], f["h_tol"], dtype, "h")
    close(last, f["last"], f["last_tol"], "fp32", "last")
    h, last, _ = ops().gated_scan(x, gate, state, lengths=n)
    close(h, f["h"], f["h_tol"], dtype, "h, nothing kept")
    close(last, f["last"], f["last_tol"], "fp32", "last, nothing kept")
    dx, dgate, dstate = ops().gated_scan_backward(kept, dh, dlast)
    close(dx, r["dx"], r["dx_tol"], dtype, "dx")
    close(dgate, r["dgate"], r["dgate_tol"], dtype, "dgate")
    close(dstate, r["dstate"], r["dstate_tol"], "fp32", "dstate")
    dead = torch.from_numpy(np.broadcast_to(~f["on"], (T, B, N)).copy()).cuda()
    assert (h[dead] == 0).all() and (dx[dead] == 0).all() and (dgate[dead] == 0).all()


@pytest.mark.parametrize("mode,keep,keep_gate", [("direct", "int8", None), ("direct", "e4m3", "raw"), ("sigmoid", "raw", "int8"),
                                                 ("sigmoid", "int8", "raw"), ("sigmoid", "e4m3", "int8")])
def test_scan_formats_of_the_two_inputs(mode, keep, keep_gate):
    T, B, N = 140, 2, 96
    x, gate, dh, state, dlast, _ = inputs(T, B, N, "fp32", mode, 3)
    _, _, kept = ops().gated_scan(x, gate, state, mode=mode, keep=keep, keep_gate=keep_gate)
    if keep != "raw":   # the copy made on the way is the one that packing makes
        want = ops().pack_activation(x, keep)
        assert torch.equal(kept.x.codes, want.codes) and torch.equal(kept.x.scales, want.scales)
    r = ref.scan_backward(f64(x), f64(gate), f64(state), None, mode, f64(dh), f64(dlast), None if keep == "raw" else keep,
                          None if keep_gate in (None, "raw") else keep_gate)
    for name, got in zip(("dx", "dgate", "dstate"), ops().gated_scan_backward(kept, dh, dlast)):
        close(got, r[name], r[name + "_tol"], "fp32", name)


@pytest.mark.parametrize("mode", ["sigmoid", "direct"])
def test_scan_gradient_against_differences(mode):
    """<gradient, v> is the slope of the loss along v, taken from the 64-bit forward pass."""
    T, B, N = 150, 2, 33
    x, gate, dh, state, dlast, _ = inputs(T, B, N, "fp32", mode, 4)
    _, _, kept = ops().gated_scan(x, gate, state, mode=mode, keep="raw")
    grads = [f64(g) for g in ops().gated_scan_backward(kept, dh, dlast)]
    point = [f64(x), f64(gate), f64(state)]
    rng = np.random.default_rng(0)

    def loss(p):
        f = ref.scan_forward(p[0], p[1], p[2], None, mode)
        return (f["h"] * f64(dh)).sum() + (f["last"] * f64(dlast)).sum()

    for k in range(3):
        v = rng.standard_normal(point[k].shape)
        at = lambda s: [p + s * v if j == k else p for j, p in enumerate(point)]  # noqa: E731
        eps = 1e-6
        slope = (loss(at(eps)) - loss(at(-eps))) / (2 * eps)
        # the difference quotient is off by eps^2 times a third derivative and by the losses' rounding over eps (about
        # 1e-16 x 1e3 / 1e-6); the gradient by its 32-bit arithmetic, 32 x 2^-23 of the magnitudes that are summed
        room = 1e-5 * np.abs(grads[k] * v).sum() + 1e-5
        assert abs((grads[k] * v).sum() - slope) <= room


def test_scan_extreme_gates():
    """Gates of either infinity pass the input resp. the state on untouched."""
    T, B, N = 70, 1, 64
    x, gate, dh, state, dlast, _ = inputs(T, B, N, "fp32", "sigmoid", 5)
    gate[:] = float("inf")
    gate[40] = float("-inf")
    h, last, kept = ops().gated_scan(x, gate, state, keep="raw")
    assert torch.equal(h[:40], state.expand(40, B, N)) and torch.equal(h[40:], x[40].expand(30, B, N))
    assert torch.equal(last, x[40])
    dx, dgate, dstate = ops().gated_scan_backward(kept, dh, dlast)
    assert (dgate == 0).all() and (dx[:40] == 0).all() and (dx[41:] == 0).all()
    # the sums of the gradients that flow into the one open input and into the first state: <= 71 additions of values
    # below 8 in magnitude
    assert (dx[40] - (dh[40:].double().sum(0) + dlast)).abs().max() <= 71 * 8 * 71 * 2.0 ** -24
    assert (dstate - dh[:40].double().sum(0)).abs().max() <= 71 * 8 * 71 * 2.0 ** -24


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("mode", ["sigmoid", "direct"])
@pytest.mark.parametrize("B,N", [(1, 1), (5, 33), (64, 256)])
def test_scan_step(B, N, mode, dtype):
    x, gate, _, state, _, _ = inputs(1, B, N, dtype, mode, 6)
    f = ref.scan_forward(f64(x), f64(gate), f64(state), None, mode)
    h, new = ops().gated_scan_step(x[0], gate[0], state, mode=mode)
    close(h, f["h"][0], f["h_tol"][0], dtype, "h")
    close(new, f["last"], f["last_tol"], "fp32", "state")
    held = state.clone()
    h2, same = ops().gated_scan_step(x[0], gate[0], held, mode=mode, inplace=True)
    assert same is held and torch.equal(held, new) and torch.equal(h, h2)


def test_scan_steps_follow_the_scan():
    """A prompt by gated_scan and tokens by gated_scan_step give what one longer scan gives."""
    T, B, N = 40, 2, 70
    x, gate, _, state, _, _ = inputs(T, B, N, "fp32", "sigmoid", 7)
    f = ref.scan_forward(f64(x), f64(gate), f64(state), None, "sigmoid")
    h, s, _ = ops().gated_scan(x[:33], gate[:33], state)
    close(h, f["h"][:33], f["h_tol"][:33], "fp32", "prompt")
    for t in range(33, T):
        h, s = ops().gated_scan_step(x[t], gate[t], s)
        close(h, f["h"][t], f["h_tol"][t], "fp32", f"token {t}")


def test_scan_offsets_beyond_32_bits():
    """2.4e9 values per tensor: the last group of channels against the reference."""
    T, N = 40000, 60000
    g = torch.Generator(device="cuda").manual_seed(14)
    x, dh = (torch.empty(T, 1, N, dtype=torch.bfloat16, device="cuda").normal_(generator=g) for _ in range(2))
    gate = torch.empty(T, 1, N, dtype=torch.bfloat16, device="cuda").normal_(1.0, 2.0, generator=g)
    h, last, kept = ops().gated_scan(x, gate, keep="int8")
    part = slice(N - N % 64, N)
    small = [f64(v[:, :, part]) for v in (x, gate, dh)]
    r = ref.scan_backward(small[0], small[1], None, None, "sigmoid", small[2], None, "int8", "int8")
    f = ref.scan_forward(small[0], small[1], None, None, "sigmoid")
    close(h[:, :, part], f["h"], f["h_tol"], "bf16", "h")
    close(last[:, part], f["last"], f["last_tol"], "fp32", "last")
    dx, dgate, _ = ops().gated_scan_backward(kept, dh)
    close(dx[:, :, part], r["dx"], r["dx_tol"], "bf16", "dx")
    close(dgate[:, :, part], r["dgate"], r["dgate_tol"], "bf16", "dgate")
    back = ops().unpack_activation(kept.x)
    assert np.array_equal(f64(back[-5:, :, part]), ref.eight_bits(small[0][-5:], "int8")[0])


def test_scan_nothing_to_do():
    o = ops()
    for T, B, N in ((0, 2, 5), (3, 0, 5), (3, 2, 0)):
        x = torch.zeros(T, B, N, device="cuda")
        s = torch.ones(B, N, device="cuda")
        h, last, kept = o.gated_scan(x, x, s, keep="int8")
        assert h.shape == (T, B, N)
        dx, dgate, dstate = o.gated_scan_backward(kept, x, s * 3)
        if T == 0:
            assert torch.equal(last, s) and torch.equal(dstate, s * 3)
    h, last, kept = o.gated_scan(torch.zeros(4, 1, 3, device="cuda"), torch.zeros(4, 1, 3, device="cuda"))
    assert (h == 0).all() and (last == 0).all()


def test_scan_results_do_not_depend_on_the_call():
    """The same bits on another stream, out of a replayed graph, and beside another call in flight."""
    o = ops()
    x, gate, dh, state, dlast, _ = inputs(900, 2, 130, "bf16", "sigmoid", 8)

    def step():
        h, last, kept = o.gated_scan(x, gate, state, keep="int8")
        return (h, last, *o.gated_scan_backward(kept, dh, dlast))

    want = [v.clone() for v in step()]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        a = step()
    b = step()
    torch.cuda.synchronize()
    for got in (a, b):
        assert all(torch.equal(v, w) for v, w in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for v in held:
        v.zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(v, w) for v, w in zip(held, want))
    x.mul_(0.5)
    graph.replay()
    again = step()
    torch.cuda.synchronize()
    assert all(torch.equal(v, w) for v, w in zip(held, again)) and not torch.equal(held[0], want[0])


# ---- 8-bit activations -----------------------------------------------------------------------------------------
@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("shape", [(1, 1), (3, 63), (2, 5, 64), (7, 65), (1, 1000), (33, 130), (130,), (5, 72), (700, 136), (3, 4096)])
def test_pack_and_unpack(shape, dtype, fmt):
    g = torch.Generator().manual_seed(9)
    x = (torch.randn(*shape, generator=g) * torch.exp(3 * torch.randn(*shape, generator=g))).to(DT[dtype]).cuda()
    p = ops().pack_activation(x, fmt)
    want, scales = ref.eight_bits(f64(x), fmt)
    assert np.array_equal(p.scales.cpu().numpy(), scales)
    # (a group with a value that fp16 turned into an infinity is all NaN)
    assert np.array_equal(f64(ops().unpack_activation(p, torch.float32)), want, equal_nan=True)
    # an 8-bit value has at most 7 significant bits: exact in all three types, but for fp16's subnormal values
    want, _ = ref.eight_bits(f64(x), fmt, dtype)
    back = ops().unpack_activation(p)
    assert back.dtype == x.dtype and np.array_equal(f64(back), f64(torch.from_numpy(want).to(x.dtype)), equal_nan=True)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_pack_borders(fmt):
    """Largest values next to the ones at which the scale changes, ties, zeros, the ends of fp32."""
    rows = []
    for top in (1.0, 1.75, np.nextafter(np.float32(1.75), np.float32(2)), 1.9921875, np.nextafter(np.float32(1.9921875), np.float32(1)),
                2.0, 2.0 ** -126, 2.0 ** -149, 2.0 ** -121, 2.0 ** -119 * 1.9999, 3.4e38, 0.0):
        r = np.zeros(64, np.float32)
        r[:] = np.float32(top) * np.linspace(-1, 1, 64, dtype=np.float32)
        r[5] = top
        r[6] = np.float32(top) * np.float32(2.5 / 127)
        rows.append(r)
    x = torch.from_numpy(np.stack(rows)).cuda()
    p = ops().pack_activation(x, fmt)
    want, scales = ref.eight_bits(f64(x), fmt)
    assert np.array_equal(p.scales.cpu().numpy(), scales)
    assert np.array_equal(f64(ops().unpack_activation(p)), want)


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_pack_keeps_the_largest_values_finite(dtype, fmt):
    x = torch.full((1, 64), torch.finfo(DT[dtype]).max, dtype=DT[dtype], device="cuda")
    x[0, 1::2] *= -1
    back = ops().unpack_activation(ops().pack_activation(x, fmt))
    assert torch.isfinite(back).all() and np.array_equal(f64(back), ref.eight_bits(f64(x), fmt, dtype)[0])


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_unpack_to_a_narrower_type(fmt):
    x = torch.tensor([[1e6, -3e5, 100.0, 7.0]], device="cuda")
    p = ops().pack_activation(x, fmt)
    want = np.clip(ref.eight_bits(f64(x), fmt)[0], -65504, 65504)
    assert np.array_equal(f64(ops().unpack_activation(p, torch.float16)), want.astype(np.float16).astype(np.float64))


@pytest.mark.parametrize("fmt", ["int8", "e4m3"])
def test_pack_not_finite(fmt):
    x = torch.ones(4, 200, device="cuda")
    x[1, 70], x[2, 199], x[3, 0] = float("nan"), float("inf"), float("-inf")
    p = ops().pack_activation(x, fmt)
    want, scales = ref.eight_bits(f64(x), fmt)
    assert np.array_equal(p.scales.cpu().numpy(), scales)
    got = f64(ops().unpack_activation(p))
    assert np.array_equal(got, want, equal_nan=True) and np.isnan(got).sum() == 64 + 8 + 64


def test_pack_strided_rows_and_long_tensors():
    wide = torch.randn(50, 201, device="cuda")
    view = wide[:, 1:132]
    p = ops().pack_activation(view)
    assert np.array_equal(f64(ops().unpack_activation(p)), ref.eight_bits(f64(view), "int8")[0])
    assert ops().unpack_activation(ops().pack_activation(torch.zeros(0, 5, device="cuda"))).shape == (0, 5)
    assert ops().unpack_activation(ops().pack_activation(torch.zeros(5, 0, device="cuda"))).shape == (5, 0)


@pytest.mark.parametrize("T,B,N,length", [(40007, 1, 2048, None), (40007, 1, 2048, 37003), (3001, 2, 70, 1500), (70001, 3, 33, None)])
def test_segments_of_the_time_axis_lose_nothing(T, B, N, length):
    """With gates of one and small whole numbers the states are running sums that fp32 holds exactly, in any order: every
    part of a segment has to arrive, whether or not the pass keeps states (which cuts the time axis differently)."""
    g = torch.Generator(device="cuda").manual_seed(T + N)
    whole = lambda *shape: torch.randint(-1, 2, shape, generator=g, device="cuda").float()  # noqa: E731
    x, dh, state, dlast, gate = whole(T, B, N), whole(T, B, N), whole(B, N), whole(B, N), torch.ones(T, B, N, device="cuda")
    lengths, end = None, T
    if length is not None:
        lengths, end = torch.full((B,), length, dtype=torch.int32, device="cuda"), length
    want = torch.zeros(T, B, N, device="cuda")
    want[:end] = state + x[:end].cumsum(0)
    d = torch.zeros_like(want)
    d[:end] = dlast + dh[:end].flip(0).cumsum(0).flip(0)
    before = torch.cat([state[None], want[:-1]])
    for keep in (None, "raw"):
        h, last, kept = ops().gated_scan(x, gate, state, lengths=lengths, mode="direct", keep=keep)
        assert torch.equal(h, want) and torch.equal(last, want[end - 1])
    dx, dgate, dstate = ops().gated_scan_backward(kept, dh, dlast)
    assert torch.equal(dx, d) and torch.equal(dstate, d[0])
    assert float((d * before).abs().max()) < 2 ** 24   # so the products are exact too
    assert torch.equal(dgate, d * before)
