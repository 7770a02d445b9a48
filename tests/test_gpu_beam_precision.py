"""How good the scores of beam search are: what its documentation says of sums in fp32, on rows that are made for their errors."""
import numpy as np
import pytest

import model_reference as ref
from seq_reference import rounding

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def log_sum_bound(z):
    """Of log sum exp(z - max), in fp32: a difference, its product with log2 e (which is off by 1.4e-8 itself) and a rounding each, so
    |d| (2 x 2^-24 + 1.4e-8) of every exponential; ex2.approx, 2^-22; and sums of a lane, 16 terms and then up to 128 segments one after
    the other.  Parts are joined in 64 bits."""
    d = z - z.max()
    p = np.exp(d)
    p /= p.sum()
    return (p * np.abs(np.where(p > 0, d, 0))).sum() * (2 * ref.U + 1.4e-8) + 2.0 ** -22 + (16 + 128) * ref.U


@pytest.mark.parametrize("dtype", list(DT))
@pytest.mark.parametrize("B,V", [(1, 1 << 22), (6, 131072), (400, 50257)])
def test_scores_are_as_good_as_sums_in_fp32(B, V, dtype):
    """A tail of one value below the largest, whose every term is rounded alike; values that rise, so that sums are scaled again and
    again; random ones.  The documented 1e-5 is above the bound of each."""
    from paper_2412_11810_b200 import ops
    rise = torch.arange(V, device="cuda", dtype=torch.float64) / V
    rows = [torch.where(rise == 0, 0.0, -14.9), torch.where(rise < 0.999, -3.3, 2.2), rise * 20, -rise * 20 + 3e-3,
            torch.randn(V, device="cuda", dtype=torch.float64, generator=torch.Generator(device="cuda").manual_seed(1)) * 2.5]
    K = len(rows)
    logits = torch.stack([r.to(DT[dtype]) for r in rows])[None].repeat(B, 1, 1)
    scores = torch.zeros(B, K, device="cuda")
    tokens, parents, new, _, _ = ops.beam_step(logits, scores, width=32)
    tokens, parents, new = tokens.cpu().numpy(), parents.cpu().numpy(), f64(new)
    z = f64(logits[0])
    bound = np.array([log_sum_bound(v) for v in z])
    assert (bound < 1e-5).all()
    _, exact = ref.beam(z, np.zeros(K), 1)
    for b in {0, B - 1}:
        want = exact[parents[b] * V + tokens[b]]
        assert (np.abs(new[b] - want) <= bound[parents[b]] + rounding(want, "fp32")).all()
        # the order is that of scores which are off by no more than that
        least = np.sort(exact)[::-1][31]
        assert (want >= least - 2 * bound.max()).all()
        # and within a beam that of the logits, to the bit
        for k in range(K):
            mine = z[k][tokens[b][parents[b] == k]]
            assert (np.diff(mine) <= 0).all()
            assert np.array_equal(mine, np.sort(z[k])[::-1][:len(mine)])
