"""Weight decay of the AdamW step: small factors count in full."""
import numpy as np
import pytest

import model_reference as ref
from seq_reference import rounding

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def ops():
    from paper_2412_11810_b200 import ops as o
    return o


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("lr,decay", [(2e-5, 0.01), (3e-6, 0.01), (1e-6, 0.02), (1e-3, 0.1), (0.5, 1.5), (1.0, 3.0), (1.0, 1.0), (1e-3, 0.0)])
def test_a_step_without_gradients_is_the_decay_rounded_once(lr, decay, bits):
    """Without gradients p' = p (1 - lr wd).  It is rounded once to fp32 (half a step), from a factor that is good to 2^-46 or better."""
    n = 40_000
    p = torch.randn(n, generator=torch.Generator().manual_seed(1)).cuda()
    before = f64(p)
    ops().adamw_step([p], [torch.zeros_like(p)], ops().adamw_state([p], bits), lr=lr, weight_decay=decay)
    want = before * (1 - lr * decay)
    err = np.abs(f64(p) - want)
    assert (err <= rounding(want, "fp32") + 2.0 ** -46 * np.abs(before)).all()


@pytest.mark.parametrize("bits", [32, 8])
def test_a_step_is_rounded_once(bits):
    """With gradients: half a step of p', and the roundings of the update's own terms."""
    n, lr, decay = 40_000, 2e-5, 0.01
    g = torch.Generator().manual_seed(2)
    p, grad = torch.randn(n, generator=g).cuda(), torch.randn(n, generator=g).cuda()
    before = f64(p)
    ops().adamw_step([p], [grad], ops().adamw_state([p], bits), lr=lr, weight_decay=decay)
    r = ref.adamw(before, f64(grad), np.zeros(n), np.zeros(n), 1, lr, (0.9, 0.999), 1e-8, decay)
    # the bound of `adamw` with half a step of p instead of four
    tol = r["p_tol"] - 4 * ref.U * np.abs(before) + 2.0 ** -46 * np.abs(before)
    assert (np.abs(f64(p) - r["p"]) <= tol + rounding(np.abs(r["p"]) + tol, "fp32")).all()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("decay", [0.0, 0.01, 1e-6, 500.0, 1500.0])
def test_infinite_parameters_and_small_ones_stay(decay, bits):
    """A parameter of -infinity (a mask that is kept among the weights) stays one, as in the formula; zeros of both signs, the
    smallest values and the largest are not moved by a decay of nothing."""
    lr = 1e-3
    p = torch.tensor([float("-inf"), float("inf"), 0.0, -0.0, 1e-45, -1e-40, 1.2e-38, 3.4e38, -3.4e38, 1.0], device="cuda")
    before = f64(p)
    ops().adamw_step([p], [torch.zeros_like(p)], ops().adamw_state([p], bits), lr=lr, weight_decay=decay)
    got, keep = f64(p), 1 - lr * decay
    assert (got[:2] == before[:2] * np.sign(keep)).all()
    err = np.abs(got[2:] - before[2:] * keep)
    assert (err <= rounding(before[2:] * keep, "fp32") + 2.0 ** -46 * np.abs(before[2:])).all()
    if decay == 0:
        assert np.array_equal(got, before)
