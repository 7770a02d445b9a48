"""The AdamW step with moments in 8 bits where it is called by others: in a network's training loop, and with a schedule on the device."""
import numpy as np
import pytest

import model_reference as ref
from seq_reference import rounding

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def ops():
    from paper_2412_11810_b200 import ops as o
    return o


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy().reshape(-1)


def moments(state):
    m, v = (ref.e4m3(s.codes.cpu().numpy(), s.scales.cpu().numpy()) for s in (state.m, state.v))
    return m, v ** 2


def test_weights_of_a_spiking_network_follow_the_definition():
    import snn_workloads as wl
    from gpu_helpers import make_session
    w = wl.small(sizes=(40, 260, 132, 6), T=21, B=5, p_in=0.1, g_ff=(2.5, 1.6), seed=13)
    s, bits_in, targets = make_session(w, wl.make(w))
    for step in range(4):
        s.train_step(bits_in, targets, max_activity=1.0)
        weights, grads = s.parameters(), s.parameter_gradients()
        before = [f64(t) for t in weights]
        total = sum(-(-t.numel() // 64) * 64 for t in weights)
        old = (np.zeros(total), np.zeros(total)) if step == 0 else moments(s.adamw)
        s.adamw_step(lr=1e-3, weight_decay=0.1, bits=8, seed=4)
        assert int(s.adamw.step) == step + 1
        at = 0
        for b, t, g in zip(before, weights, grads):
            n = t.numel()
            r = ref.adamw(b, f64(g), old[0][at:at + n], old[1][at:at + n], step + 1, 1e-3, (0.9, 0.999), 1e-8, 0.1)
            assert (np.abs(f64(t) - r["p"]) <= r["p_tol"] + rounding(r["p"], "fp32")).all(), step
            assert (np.abs(r["p"] - b) > 1e-4).any()   # (there is something to compare)
            at += -(-n // 64) * 64
    s.close()


@pytest.mark.parametrize("p_dtype", list(DT))
@pytest.mark.parametrize("bits", [8, 32])
def test_rates_and_scales_on_the_device_are_those_of_the_host(bits, p_dtype):
    shapes = [(300, 70), (4001,), (1,)]
    g = torch.Generator().manual_seed(6)
    start = [torch.randn(*k, generator=g).to(DT[p_dtype]).cuda() for k in shapes]
    grads = [torch.randn(*k, generator=g).cuda() for k in shapes]
    rates = [3e-3, 1e-3, 0.0, 2e-4]

    def run(on_device):
        params, state = [p.clone() for p in start], ops().adamw_state(start, bits)
        norms = []
        for k, lr in enumerate(rates):
            lr, scale = torch.tensor(lr, device="cuda"), torch.tensor(0.25 * (k + 1), device="cuda")
            if not on_device:
                lr, scale = float(lr.double()), float(scale)
            norms.append(float(ops().adamw_step(params, grads, state, lr=lr, scale=scale, max_norm=1.0, seed=8, weight_decay=0.1)))
        parts = (state.m, state.v) if bits == 32 else (state.m.codes, state.m.scales, state.v.codes, state.v.scales)
        return norms, [*params, *parts, state.step]

    norms, host = run(False)
    again, device = run(True)
    assert norms == again and all(torch.equal(a, b) for a, b in zip(host, device))
    assert int(host[-1]) == 4 and not torch.equal(host[0], start[0])
