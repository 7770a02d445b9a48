"""AdamW on the GPU where the square of a finite gradient leaves fp32: the parameter stops, and nothing else is lost."""
import numpy as np
import pytest

import model_reference as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

LR, DECAY = 1e-3, 0.01


def ops():
    from paper_2412_11810_b200 import ops as o
    return o


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def moments(state):
    return [f64(s if isinstance(s, torch.Tensor) else ops().unpack_activation(s, torch.float32)) for s in (state.m, state.v)]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,at,size", [(64, 5, 1e30), (200, 130, 6e20), (5000, 4999, 1e25), (5000, 64, -1e30), (200, 199, 3e38), (10_000_000, 7_654_321, 1e30)])
def test_a_gradient_whose_square_is_infinite_stops_its_parameter(n, at, size, dtype, bits):
    """Its v is infinite: p (1 - lr weight_decay) is what is left of the formula.  (At 6e20 the product with 1 - beta2 is beyond
    fp32 as well.)  The last size takes parts of tiles of several turns."""
    g = torch.Generator(device="cuda").manual_seed(n)
    p = torch.randn(n, generator=g, device="cuda").to(dtype)
    grads = [torch.randn(n, generator=g, device="cuda").to(dtype) for _ in range(3)]
    grads[0][at] = size
    state = ops().adamw_state([p], bits)
    group = slice(at // 64 * 64, min(at // 64 * 64 + 64, n))
    for step in range(3):
        before = f64(p)
        old = moments(state)
        ops().adamw_step([p], [grads[step]], state, lr=LR, weight_decay=DECAY, seed=3)
        got = f64(p)
        assert np.isfinite(got).all(), step
        # kept but for the decay and two roundings (of half a step and of the decay), then one of the type
        kept = before[at] * (1 - LR * DECAY)
        half = 2.0 ** -24 if dtype is torch.float32 else 2.0 ** -8
        assert abs(got[at] - kept) <= (2 * ref.U + half) * abs(kept), step
        m, v = moments(state)
        assert np.isfinite(m).all()
        if bits == 8:   # (in 32 bits v says infinity, which is what keeps the parameter where it is)
            assert np.isfinite(v).all()
            assert 384 * 2.0 ** 55 <= v[at] <= 448 * 2.0 ** 55   # the largest root that is kept, and two codes less
        else:
            assert np.isinf(v[at]) and np.isfinite(np.delete(v, at)).all()
        # everything outside its group, and in the first step everything but itself, is as if it were not there
        r = ref.adamw(before, f64(grads[step]), np.zeros(n) if step == 0 else old[0][:n], np.zeros(n) if step == 0 else old[1][:n] ** (2 if bits == 8 else 1), step + 1, LR, (0.9, 0.999), 1e-8,
                      DECAY)
        others = np.ones(n, bool)
        others[at if step == 0 else group] = False
        tol = r["p_tol"] + half * (np.abs(r["p"]) + r["p_tol"])
        assert (np.abs(got - r["p"]) <= tol)[others].all(), step


@pytest.mark.parametrize("bits", [32, 8])
def test_the_largest_gradients_whose_squares_are_finite(bits):
    """Just below the border: an ordinary update, and again one in the next step (in 8 bits roots end at 448 x 2^55, a code's value,
    so that their squares are finite when they are read back)."""
    p = torch.zeros(192, device="cuda")
    g = torch.full((192,), 1.8e19, device="cuda")
    g[64:128] = 1.7e19
    g[128:] = -1.6e19
    state = ops().adamw_state([p], bits)
    for step in range(3):
        before = f64(p)
        ops().adamw_step([p], [g], state, lr=LR, betas=(0.5, 0.0), weight_decay=0.0, seed=3)   # (v is the square itself)
        # m / (1 - b1^t) and v are those of a constant gradient: sign(g) lr, off by an eighth in 8 bits where a code is rounded or cut
        assert (np.abs(f64(p) - before + LR * np.sign(f64(g))) <= LR * (1e-5 if bits == 32 else 0.15)).all(), step
        assert all(np.isfinite(s).all() for s in moments(state))


@pytest.mark.parametrize("bits", [32, 8])
def test_an_infinite_gradient_is_still_lost(bits):
    """An infinity or a NaN is not a large value: its parameter is NaN, in 8 bits its group's moments are, and others stay."""
    p, g = torch.ones(256, device="cuda"), torch.ones(256, device="cuda")
    g[70], g[140] = float("inf"), float("nan")
    state = ops().adamw_state([p], bits)
    ops().adamw_step([p], [g], state, lr=LR, weight_decay=DECAY)
    lost = torch.isnan(p).cpu().numpy()
    assert lost[70] and lost[140] and lost.sum() == 2
    m, v = moments(state)
    if bits == 8:
        assert np.isnan(m[64:192]).all() and np.isnan(v[64:192]).all()
        m, v = np.delete(m, slice(64, 192)), np.delete(v, slice(64, 192))
        assert np.isfinite(m).all() and np.isfinite(v).all()
