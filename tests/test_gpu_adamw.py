"""The AdamW step over many tensors on the GPU against its definition in 64 bits."""
import numpy as np
import pytest

import model_reference as ref
from seq_reference import rounding

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
HYPER = dict(lr=3e-3, betas=(0.9, 0.99), eps=1e-6, weight_decay=0.1)


def ops():
    from paper_2412_11810_b200 import ops as o
    return o


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy().reshape(-1)


def room(n):
    return -(-n // 64) * 64


def tensors(shapes, dtypes, seed, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return [(std * torch.randn(*s, generator=g)).to(DT[d]).cuda() for s, d in zip(shapes, dtypes)]


def within(got, want, tol, what):
    err = np.abs(got - want) - tol
    assert not np.isnan(got).any() and (err <= 0).all(), f"{what}: off by {err.max():.3e} more than allowed"


def check_step(params, grads, state, hyper=HYPER, factor=1.0, copies=None, seed=0, **kw):
    """One step and its comparison; factor: what the gradients are multiplied by."""
    before = [f64(p) for p in params]
    t = int(state.step) + 1
    eight = not isinstance(state.m, torch.Tensor)
    if eight:
        old = [ref.e4m3(s.codes.cpu().numpy(), s.scales.cpu().numpy()) for s in (state.m, state.v)]
        old[1] = old[1] ** 2
    else:
        old = [f64(state.m), f64(state.v)]
    norm = ops().adamw_step(params, grads, state, copies=copies, seed=seed, **hyper, **kw)
    assert int(state.step) == t
    at = 0
    new = [ops().unpack_activation(s, torch.float32) if eight else s for s in (state.m, state.v)]
    new = [f64(s) for s in new]
    for k, (p, g) in enumerate(zip(params, grads)):
        n = p.numel()
        b1, b2 = hyper["betas"]
        r = ref.adamw(before[k], f64(g) * factor, old[0][at:at + n], old[1][at:at + n], t, hyper["lr"], hyper["betas"], hyper["eps"], hyper["weight_decay"])
        # a factor of the gradients is rounded once more, and so is the product
        more = 0.0 if factor == 1.0 else 4 * ref.U
        dtype = {v: key for key, v in DT.items()}[p.dtype]
        update = np.abs(r["p"] - before[k] * (1 - hyper["lr"] * hyper["weight_decay"]))
        # through the root a relative error of g counts at most once, through m as its own term
        tol = r["p_tol"] + 2 * more * (update + hyper["lr"] / (1 - b1 ** t) * np.abs((1 - b1) * f64(g) * factor) / (np.sqrt(r["v"] / (1 - b2 ** t)) + hyper["eps"]))
        within(f64(p), r["p"], tol + rounding(np.abs(r["p"]) + tol, dtype), f"p[{k}]")
        if copies is not None and copies[k] is not None:
            name = {v: key for key, v in DT.items()}[copies[k].dtype]
            within(f64(copies[k]), r["p"], tol + rounding(np.abs(r["p"]) + tol, name), f"copies[{k}]")
        m_tol = r["m_tol"] + more * np.abs((1 - b1) * f64(g) * factor)
        if not eight:
            within(new[0][at:at + n], r["m"], m_tol + rounding(r["m"], "fp32"), f"m[{k}]")
            within(new[1][at:at + n], r["v"], r["v_tol"] + 2 * more * r["v"] + rounding(r["v"], "fp32"), f"v[{k}]")
        else:
            bits = ref.random_bits(at + np.arange(room(n)), seed, t)
            pad = lambda a: np.concatenate([a, np.zeros(room(n) - n)])  # noqa: E731
            for s, v, tol, r16, root in ((0, r["m"], m_tol, bits & np.uint64(0xFFFF), False),
                                         (1, np.sqrt(r["v"]), (4 * ref.U + more) * np.sqrt(r["v"]) + 2.0 ** -100, bits >> np.uint64(16), True)):
                v, tol = pad(v), pad(tol)
                with np.errstate(all="ignore"):
                    unsure = np.where(v != 0, tol / np.abs(v), 0.0).reshape(-1, 64)
                one, other = ref.encode_at_random(v, r16.astype(np.float64), root, unsure)
                got = new[s][at:at + room(n)]
                bad = (got != one) & (got != other)
                if root:
                    # v is a sum of two fp32 products: where they are subnormal, each of the four roundings leaves up to 2^-150, so that
                    # the root is that of something within 2^-148 of v, and its code (which rises with it) between those of the ends
                    ends = [ref.encode_at_random(np.sqrt(np.maximum(v ** 2 + d, 0.0)), r16.astype(np.float64), True, np.zeros_like(unsure))[0]
                            for d in (-2.0 ** -148, 2.0 ** -148)]
                    bad &= (got < ends[0]) | (got > ends[1])
                # the largest value of a group is as unsure as its values: within that of 448 scales, its scale is either of the two
                # (0.0034179687500000013 here may be 448 x 2^-17 there), and right codes are those of the scale that was taken
                if bad.any():
                    for shift in (-(4 * ref.U + more), 4 * ref.U + more):
                        a, b = ref.encode_at_random(v, r16.astype(np.float64), root, unsure, shift)
                        same = np.repeat(((got == a) | (got == b)).reshape(-1, 64).all(1), 64)
                        bad &= ~same
                assert not bad.any(), f"{'mv'[s]}[{k}]: {int(bad.sum())} of {n}, first at {np.argmax(bad)}: {got[bad][:4]} instead of {one[bad][:4]}"
                # close decisions are few: what is unsure is a few units in 2^24 of at most 16 steps (where squares are not subnormal)
                if factor == 1.0 and n > 1000:
                    assert ((got != one) & (v ** 2 >= 2.0 ** -110)).mean() <= 2e-3
        at += room(n)
    return norm


SHAPES = [(1,), (7, 9), (64,), (65, 3), (0, 5), (2048,), (2049,), (33, 130), (5000,)]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("p_dtype,g_dtype", [("fp32", "fp32"), ("bf16", "bf16"), ("fp16", "fp32"), ("fp32", "bf16"), ("bf16", "fp16")])
def test_steps_from_the_start(p_dtype, g_dtype, bits):
    params = tensors(SHAPES, [p_dtype] * len(SHAPES), 1)
    state = ops().adamw_state(params, bits)
    for step in range(4):
        grads = tensors(SHAPES, [g_dtype] * len(SHAPES), 10 + step, std=10.0 ** -(step % 3))
        grads[3][::2] = 0
        assert check_step(params, grads, state, seed=3) is None


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("p_dtype,g_dtype", [("bf16", "bf16"), ("fp32", "fp32"), ("fp32", "bf16"), ("fp16", "fp16"), ("bf16", "fp32")])
def test_enough_for_tiles_of_several_turns(p_dtype, g_dtype, bits):
    """Ten million parameters: whole parts of tiles, tensors' ends inside them, and small tensors in between."""
    shapes = [(3000, 2001), (77,), (1500, 2100), (2048,), (1111, 1003), (16384,)]
    params = tensors(shapes, [p_dtype] * len(shapes), 30)
    grads = tensors(shapes, [g_dtype] * len(shapes), 31, std=0.01)
    grads[0][::7] = 0
    copies = [None if k % 2 else torch.zeros(s, dtype=torch.bfloat16, device="cuda") for k, s in enumerate(shapes)]
    state = ops().adamw_state(params, bits)
    total = np.sqrt(sum((f64(g) ** 2).sum() for g in grads))
    check_step(params, grads, state, copies=copies, seed=5)
    norm = check_step(params, grads, state, copies=copies, seed=5, factor=1 / total, max_norm=1.0)
    assert abs(float(norm) - total) <= 4 * ref.U * total


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("size", [1e17, 1e9, 1e4, 1e-4, 1e-10, 1e-17])
def test_gradients_of_all_magnitudes(size, bits):
    """Groups whose scales lie far from one on both sides, and some that hold both ends at once."""
    shapes = [(700,), (33, 64), (20000,)]
    params = tensors(shapes, ["fp32"] * 3, 15)
    state = ops().adamw_state(params, bits)
    for step in range(3):
        grads = tensors(shapes, ["fp32"] * 3, 20 + step, std=size)
        grads[1][:, ::3] *= 1e-5
        grads[2][::7] = 0
        check_step(params, grads, state, seed=11)


def test_roots_of_subnormal_squares_do_not_blow_up():
    """8-bit moments, no eps to speak of, one large gradient beside some whose squares are subnormal: every update stays at
    the size of a step (the sign of the gradient times lr, up to rounding)."""
    g = torch.full((64,), 1e-19, device="cuda")
    g[5], g[9] = 1.0, 0.0
    p = torch.zeros(64, device="cuda")
    ops().adamw_step([p], [g], ops().adamw_state([p], 8), lr=1e-3, betas=(0.9, 0.999), eps=1e-30, weight_decay=0.0)
    assert float(p[9]) == 0 and (p.abs() <= 1.01e-3).all() and abs(float(p[5]) + 1e-3) <= 1e-8


@pytest.mark.parametrize("bits", [32, 8])
def test_mixed_types_copies_and_places_in_memory(bits):
    """Every combination of types in one list, some of them at odd places of a larger buffer."""
    names = list(DT)
    combos = [(a, b, c) for a in names for b in names for c in (*names, None)]
    shapes = [(31 + 40 * k,) for k in range(len(combos))]
    params = tensors(shapes, [c[0] for c in combos], 2)
    grads = tensors(shapes, [c[1] for c in combos], 3)
    copies = [None if c[2] is None else torch.zeros(s, dtype=DT[c[2]], device="cuda") for s, c in zip(shapes, combos)]
    for k in range(0, len(params), 2):   # contiguous, but from an odd element on
        for held in (params, grads, copies):
            if held[k] is not None:
                buffer = torch.full((held[k].numel() + 9,), 7.0, dtype=held[k].dtype, device="cuda")
                at = 1 + k % 3
                buffer[at:at + held[k].numel()] = held[k]
                held[k] = buffer[at:at + held[k].numel()]
    state = ops().adamw_state(params, bits)
    for _ in range(2):
        check_step(params, grads, state, copies=copies)
    for held in (params, grads, copies):   # nothing beside them was written
        for k in range(0, len(params), 2):
            if held[k] is not None:
                base = held[k]._base
                assert (base[:1 + k % 3] == 7).all() and (base[1 + k % 3 + held[k].numel():] == 7).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("count", [64, 65, 600, 1030])
def test_more_tensors_than_a_table_holds(count, bits):
    shapes = [(1 + (7 * k) % 90,) for k in range(count)]
    params, grads = tensors(shapes, ["fp32"] * count, 4), tensors(shapes, ["fp32"] * count, 5)
    state = ops().adamw_state(params, bits)
    total = np.sqrt(sum((f64(g) ** 2).sum() for g in grads))
    check_step(params, grads, state)
    norm = check_step(params, grads, state, factor=0.5 / total, max_norm=0.5)
    assert abs(float(norm) - total) <= 4 * ref.U * total


@pytest.mark.parametrize("bits", [32, 8])
def test_clip_scale_and_schedule_on_the_device(bits):
    shapes = [(300, 70), (4001,), (1,)]
    params, grads = tensors(shapes, ["fp32"] * 3, 6), tensors(shapes, ["bf16", "fp32", "fp16"], 7)
    state = ops().adamw_state(params, bits)
    total = np.sqrt(sum((f64(g) ** 2).sum() for g in grads))
    norm = check_step(params, grads, state, max_norm=2 * total)   # below it: nothing is clipped
    assert abs(float(norm) - total) <= 4 * ref.U * total
    norm = check_step(params, grads, state, factor=0.25 * 0.1 / (0.25 * total), max_norm=0.1, scale=0.25)
    assert abs(float(norm) - 0.25 * total) <= 4 * ref.U * total
    on_device = torch.tensor(0.5, device="cuda")
    check_step(params, grads, state, factor=0.5, scale=on_device)
    lr = torch.tensor(HYPER["lr"], device="cuda")
    hyper = dict(HYPER, lr=float(lr.double()))
    before, held = [p.clone() for p in params], (state.step.clone(), state.m, state.v)
    if bits == 32:
        held = (held[0], state.m.clone(), state.v.clone())
        check_step(params, grads, state, hyper=hyper)
        again = ops().AdamWState(held[1], held[2], held[0])
        ops().adamw_step(before, grads, again, **dict(HYPER, lr=lr))
        assert all(torch.equal(a, b) for a, b in zip(before, params)) and torch.equal(again.v, state.v)


@pytest.mark.parametrize("value", [float("inf"), -float("inf"), float("nan")])
@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_without_a_finite_norm_is_left_out(bits, value):
    shapes = [(100, 30), (77,)]
    params, grads = tensors(shapes, ["fp32", "bf16"], 8), tensors(shapes, ["fp32"] * 2, 9)
    copies = [torch.zeros(s, device="cuda", dtype=torch.bfloat16) for s in shapes]
    state = ops().adamw_state(params, bits)
    check_step(params, grads, state, copies=copies)
    parts = lambda: [*params, *copies, state.step, *((state.m, state.v) if bits == 32 else (state.m.codes, state.m.scales, state.v.codes, state.v.scales))]  # noqa: E731
    before = [t.clone() for t in parts()]
    grads[1][40] = value
    norm = ops().adamw_step(params, grads, state, copies=copies, max_norm=1.0, **HYPER)
    assert not torch.isfinite(norm) and all(torch.equal(a, b) for a, b in zip(before, parts()))
    # without a clip nothing looks: the parameter alone is lost, in 8 bits its group
    ops().adamw_step(params, grads, state, copies=copies, **HYPER)
    lost = torch.isnan(params[1])
    assert lost[40] or value != value and lost[40]
    assert int(lost.sum()) == 1 and not torch.isnan(params[0]).any()
    if bits == 8:
        m = ops().unpack_activation(state.m)
        assert torch.isnan(m[47 * 64:48 * 64]).all() and not torch.isnan(m[:47 * 64]).any() and int(state.m.scales[-1]) != 255


def test_norms_of_very_large_and_small_gradients():
    p = torch.zeros(5000, device="cuda")
    for size in (1e30, 1e19, 1e-25, 1e-38):
        state = ops().adamw_state([p])
        g = torch.full_like(p, size)
        norm = ops().adamw_step([p], [g], state, max_norm=1e38, **HYPER)
        want = float(g[0].double()) * np.sqrt(5000)
        assert abs(float(norm) - want) <= 4 * ref.U * want
        # clipped, the squares fit
        norm = ops().adamw_step([p], [g], ops().adamw_state([p]), max_norm=1e-3, **HYPER)
        assert torch.isfinite(p).all()


def test_moments_in_8_bits_keep_their_mean():
    """Decay alone (gradients of zero): a moment of one million places that moves by a thousandth a step, less than a hundredth
    of a step of its codes, still falls as it should on average; rounded to nearest it would not move."""
    n, steps = 1 << 20, 40
    p, g = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda")
    state = ops().adamw_state([p], 8)
    # e4m3 codes of magnitudes 8 .. 15 in steps, of both signs in m
    codes = (torch.arange(n, device="cuda") % 8 + 0x40).to(torch.uint8)
    state.m.codes.copy_(codes)
    state.v.codes.copy_(codes)
    state.m.scales.fill_(127)
    state.v.scales.fill_(127)
    start = [float(ops().unpack_activation(s, torch.float32).double().mean()) for s in (state.m, state.v)]
    for k in range(steps):
        ops().adamw_step([p], [g], state, lr=0.0, betas=(0.999, 0.999), eps=1e-8, seed=5)
    got = [float(ops().unpack_activation(s, torch.float32).double().mean()) for s in (state.m, state.v)]
    # a rounding has a standard deviation of at most half a step (2^-2 of values from 2 to 4): over n places and all steps the mean
    # is off by 5 standard deviations, 5 * 0.125 * sqrt(steps / n), at most; r takes 2^16 values, which moves the mean by at
    # most 2^-17 of a step each time
    bound = 5 * 0.125 * np.sqrt(steps / n) + steps * 0.25 * 2.0 ** -16
    for s, decay in ((0, 0.999), (1, 0.999 ** 0.5)):
        assert abs(got[s] - start[s] * decay ** steps) <= bound, (s, got, start)


def test_random_bits_are_even():
    """The reference's own hash: every bit is set half of the time, and two bits agree half of the time."""
    r = ref.random_bits(np.arange(1 << 16), 12345678901, 77)
    bits = (r[:, None] >> np.arange(32, dtype=np.uint64)) & np.uint64(1)
    bits = bits.astype(np.float64)
    # 5 standard deviations of a mean of 2^16 fair bits
    assert np.abs(bits.mean(0) - 0.5).max() <= 5 * 0.5 / 256
    agree = bits.T @ bits + (1 - bits).T @ (1 - bits)
    assert np.abs(agree / (1 << 16) - np.eye(32) - 0.5 * (1 - np.eye(32))).max() <= 5 * 0.5 / 256


@pytest.mark.parametrize("bits", [32, 8])
def test_streams_and_captured_steps(bits):
    shapes = [(129, 65), (3000,)]

    def fresh():
        params = tensors(shapes, ["fp32", "bf16"], 11)
        return params, tensors(shapes, ["fp32"] * 2, 12), ops().adamw_state(params, bits)

    def parts(params, state):
        return [*params, state.step, *((state.m, state.v) if bits == 32 else (state.m.codes, state.m.scales, state.v.codes, state.v.scales))]

    kw = dict(HYPER, max_norm=1.0, seed=9)
    params, grads, state = fresh()
    for _ in range(3):
        ops().adamw_step(params, grads, state, **kw)
    want = [t.clone() for t in parts(params, state)]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        params, grads, state = fresh()
        for _ in range(3):
            ops().adamw_step(params, grads, state, **kw)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(parts(params, state), want))
    # a captured step counts itself
    params, grads, state = fresh()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norm = ops().adamw_step(params, grads, state, **kw)
    assert int(state.step) == 0
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert int(state.step) == 3 and all(torch.equal(a, b) for a, b in zip(parts(params, state), want)) and float(norm) > 1


def test_a_long_run_follows_the_definition():
    """Fifty steps in fp32 against float64, and the same in 8 bits within what their rounding costs."""
    n = 4096
    p0 = tensors([(n,)], ["fp32"], 13)[0]
    target = tensors([(n,)], ["fp32"], 14)[0]
    p, state = p0.clone(), ops().adamw_state([p0])
    q, eight = p0.clone(), ops().adamw_state([p0], 8)
    r, m, v = f64(p0), np.zeros(n), np.zeros(n)
    for t in range(1, 51):
        ops().adamw_step([p], [p - target], state, **HYPER)
        ops().adamw_step([q], [q - target], eight, seed=1, **HYPER)
        f = ref.adamw(r, r - f64(target), m, v, t, HYPER["lr"], HYPER["betas"], HYPER["eps"], HYPER["weight_decay"])
        r, m, v = f["p"], f["m"], f["v"]
    # 50 updates of at most 3e-3 each, all off by 24 units and by what p itself is off (a rounding of it a step)
    assert np.abs(f64(p) - r).max() <= 50 * (24 * ref.U * 3e-3 + 4 * ref.U * np.abs(r).max()) * 4
    # in 8 bits m and sqrt(v) are off by up to an eighth each: every update by less than 0.3 of its size of at most 4e-3
    assert np.abs(f64(q) - r).max() <= 50 * 0.3 * 4e-3


@pytest.mark.parametrize("bits", [32, 8])
def test_step_of_a_spiking_network(bits):
    """Session.adamw_step updates the weights that its own training step made gradients for."""
    import snn_workloads as wl
    from gpu_helpers import make_session
    w = wl.small(sizes=(40, 260, 132, 6), T=21, B=5, p_in=0.1, g_ff=(2.5, 1.6), seed=13)
    s, bits_in, targets = make_session(w, wl.make(w))
    losses = []
    for step in range(3):
        losses.append(s.train_step(bits_in, targets, max_activity=1.0))
        weights, grads = s.parameters(), s.parameter_gradients()
        before = [f64(t) for t in weights]
        old = None if step == 0 else [f64(s.adamw.m), f64(s.adamw.v)] if bits == 32 else None
        norm = s.adamw_step(lr=1e-3, weight_decay=0.0, bits=bits, max_norm=1e9)
        total = np.sqrt(sum((f64(g) ** 2).sum() for g in grads))
        assert abs(float(norm) - total) <= 4 * ref.U * total and int(s.adamw.step) == step + 1
        if bits == 32:
            at = 0
            for b, t, g in zip(before, weights, grads):
                n = t.numel()
                m, v = (np.zeros(n), np.zeros(n)) if old is None else (old[0][at:at + n], old[1][at:at + n])
                r = ref.adamw(b, f64(g), m, v, step + 1, 1e-3, (0.9, 0.999), 1e-8, 0.0)
                within(f64(t), r["p"], r["p_tol"] + rounding(r["p"], "fp32"), "weights")
                at += room(n)
    assert all(np.isfinite(losses)) and s.parameters()[0].data_ptr() == s.W_ff[0].data_ptr()
    s.close()


def test_long_offsets():
    """A tensor of more than 2^31 values, whose last tile is checked."""
    n = (1 << 31) + 131
    p = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g = torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    g[-200:] = 0.5
    p[-200:] = 1.0
    state = ops().adamw_state([p], 8)
    ops().adamw_step([p], [g], state, seed=2, **HYPER)
    r = ref.adamw(np.ones(200), np.full(200, 0.5), np.zeros(200), np.zeros(200), 1, HYPER["lr"], HYPER["betas"], HYPER["eps"], HYPER["weight_decay"])
    tol = r["p_tol"]
    within(f64(p[-200:]), r["p"], tol + rounding(r["p"], "bf16"), "p")
    first = n - 200
    codes, scales = state.m.codes[first // 64 * 64:].cpu().numpy(), state.m.scales[first // 64:].cpu().numpy()
    got = ref.e4m3(codes, scales)[first % 64:first % 64 + 200]
    assert (np.abs(got - 0.05) <= 0.05 / 8).all() and not state.m.codes[:first // 64 * 64].any()
    places = first + np.arange(200)
    want = np.concatenate([np.zeros(first % 64), r["m"], np.zeros(-n % 64)])
    bits = np.concatenate([np.zeros(first % 64), (ref.random_bits(places, 2, 1) & np.uint64(0xFFFF)).astype(np.float64), np.zeros(-n % 64)])
    one, other = ref.encode_at_random(want, bits, False, np.full((want.size // 64, 64), 8 * ref.U))
    one, other = one[first % 64:first % 64 + 200], other[first % 64:first % 64 + 200]
    assert ((got == one) | (got == other)).all()
