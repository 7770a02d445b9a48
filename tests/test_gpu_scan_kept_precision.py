"""What keeping the inputs of the recurrence in 8 bits costs its gradients: as much as the formats say, and no more."""
import numpy as np
import pytest

import seq_reference as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def f64(t):
    return t.to(torch.float64).cpu().numpy()


# the figures that gated_scan states, of dx, dgate and dstate
@pytest.mark.parametrize("keep,mean,stated", [("int8", 2.0, (0.011, 0.014, 0.0055)), ("int8", 5.0, (0.027, 0.027, 0.0055)),
                                              ("e4m3", 2.0, (0.018, 0.036, 0.011)), ("e4m3", 5.0, (0.048, 0.059, 0.011))])
def test_distance_to_the_gradients_from_raw_inputs(keep, mean, stated):
    """The distance between the kernels' gradients from 8-bit and from raw inputs is that of the definitions, to within what
    either is off by (triangle inequality over their bounds)."""
    from paper_2412_11810_b200 import ops
    T, B, N = 2048, 2, 128
    g = torch.Generator().manual_seed(41)
    x, gate = torch.randn(T, B, N, generator=g).cuda(), (mean + 1.5 * torch.randn(T, B, N, generator=g)).cuda()
    state, dlast, dh = torch.randn(B, N, generator=g).cuda(), 0.1 * torch.randn(B, N, generator=g).cuda(), 0.1 * torch.randn(T, B, N, generator=g).cuda()
    got, want = [], []
    for k in (keep, "raw"):
        _, _, kept = ops.gated_scan(x, gate, state, keep=k)
        got.append([f64(v) for v in ops.gated_scan_backward(kept, dh, dlast)])
        eight = None if k == "raw" else k
        want.append(ref.scan_backward(f64(x), f64(gate), f64(state), None, "sigmoid", f64(dh), f64(dlast), eight, eight))
    for i, name in enumerate(("dx", "dgate", "dstate")):
        size = np.linalg.norm(want[1][name])
        far = np.linalg.norm(got[0][i] - got[1][i]) / size
        defined = np.linalg.norm(want[0][name] - want[1][name]) / size
        room = sum(np.linalg.norm(w[name + "_tol"] + ref.rounding(np.abs(w[name]) + w[name + "_tol"], "fp32")) for w in want) / size
        assert abs(far - defined) <= room
        # the figures are means over other inputs: of half a million values, or for the state of 256 channels, each of which
        # is dominated by the first few steps (the norm of 256 such values scatters by a quarter)
        assert abs(defined - stated[i]) <= (0.25 if name == "dstate" else 0.1) * stated[i]
