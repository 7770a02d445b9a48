"""Refusals of the norm, the AdamW step and beam search that need tensors on a device."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def ops():
    from paper_2412_11810_b200 import ops as o
    return o


def refused(*calls):
    for call in calls:
        with pytest.raises(ValueError):
            call()


def test_norm():
    o, x, w = ops(), torch.randn(6, 40, device="cuda"), torch.ones(40, device="cuda")
    y, h, rstd, _ = o.rms_norm(x, w, x)
    r, b = o.rms_norm, o.rms_norm_backward
    refused(lambda: r(x.double()), lambda: r(x[0, 0]), lambda: r(x[:, :0]), lambda: r(x.t()), lambda: r(x.view(2, 3, 40).transpose(0, 1)), lambda: r(x, w[:39]),
            lambda: r(x, w.bfloat16()), lambda: r(x, w.cpu()), lambda: r(x, w[:, None]), lambda: r(x, torch.ones(80, device="cuda")[::2]), lambda: r(x, w, x[:5]),
            lambda: r(x, w, x.bfloat16()), lambda: r(x, w, x.cpu()), lambda: r(x, w, 3.0), lambda: r(x, w, inplace=True), lambda: r(x, eps=0.0), lambda: r(x, eps=2.0),
            lambda: r(x, keep="raw"), lambda: r(x, keep="e5m2"), lambda: r(x, values=False), lambda: r(x, w, x[:1].expand(6, 40), inplace=True),
            lambda: r(x[1:], w, x[:-1], inplace=True),
            lambda: b(h, rstd[:5], x), lambda: b(h, rstd.double(), x), lambda: b(h, rstd, x[:5]), lambda: b(h, rstd, x.bfloat16()), lambda: b(h, rstd, x.t()),
            lambda: b(h, rstd, x, w[:3]), lambda: b(h, rstd, x, w, x[:1]), lambda: b(h, rstd, None), lambda: b(h, None, x))
    y, h, _, _ = r(x, w, x)
    held = x.clone()
    y2, h2, _, _ = r(held, w, held, inplace=True)   # twice itself
    assert torch.equal(y, y2) and torch.equal(h, held) and h2 is held


def test_adamw():
    o = ops()
    p, g = [torch.randn(8, 9, device="cuda"), torch.randn(5, device="cuda")], [torch.randn(8, 9, device="cuda"), torch.randn(5, device="cuda")]
    s, e = o.adamw_state(p), o.adamw_state(p, 8)
    assert s.m.shape == (192,) and e.m.codes.shape == (192,) and e.v.scales.shape == (3,)
    before = [t.clone() for t in p]
    step = lambda **k: o.adamw_step(**{**dict(params=p, grads=g, state=s, lr=1e-3), **k})  # noqa: E731
    refused(lambda: step(grads=g[:1]), lambda: step(copies=[None]), lambda: step(params=[p[0], p[0]], grads=[g[0], g[0]], state=o.adamw_state([p[0], p[0]])),
            lambda: step(copies=[p[0], None]), lambda: step(params=[p[0].t(), p[1]]), lambda: step(grads=[g[0].t(), g[1]]), lambda: step(params=[p[0].double(), p[1]]),
            lambda: step(grads=[g[0].long(), g[1]]), lambda: step(grads=[g[0].view(-1), g[1]]), lambda: step(grads=[g[0].cpu(), g[1]]), lambda: step(grads=[None, g[1]]),
            lambda: step(copies=[torch.zeros(8, device="cuda"), None]), lambda: step(copies=[p[0].double(), None]), lambda: step(state=o.adamw_state(p[:1])),
            lambda: step(state=o.AdamWState(s.m, e.v, s.step)), lambda: step(state=o.AdamWState(e.m, s.v, s.step)), lambda: step(state=o.AdamWState(s.m, s.v, s.step.int())),
            lambda: step(state=o.AdamWState(s.m, s.v, s.step.cpu())), lambda: step(state=o.AdamWState(s.m.double(), s.v, s.step)),
            lambda: step(state=o.AdamWState(o.PackedActivation(e.m.codes, e.m.scales, "int8", torch.float32), e.v, s.step)), lambda: step(state=(s.m, s.v)),
            lambda: step(lr=-1.0), lambda: step(lr=float("nan")), lambda: step(lr=torch.tensor(1.0)), lambda: step(lr=torch.ones(1, device="cuda")),
            lambda: step(scale=float("inf")), lambda: step(scale=torch.ones((), device="cuda", dtype=torch.float64)), lambda: step(betas=(1.0, 0.9)),
            lambda: step(betas=(0.9, -0.1)), lambda: step(eps=0.0), lambda: step(eps=3.0), lambda: step(weight_decay=-1.0), lambda: step(max_norm=0.0),
            lambda: step(max_norm=float("nan")), lambda: step(seed=-1), lambda: step(seed=1 << 64), lambda: o.adamw_state(p, 4))
    assert all(torch.equal(a, b) for a, b in zip(before, p)) and int(s.step) == 0


def test_an_empty_list_of_values_counts_its_step():
    o = ops()
    p = torch.empty(0, 4, device="cuda")
    s = o.adamw_state([p])
    assert o.adamw_step([p], [p], s, lr=1e-3) is None
    assert float(o.adamw_step([p], [p], s, lr=1e-3, max_norm=1.0)) == 0 and int(s.step) == 2


def test_beam():
    o = ops()
    z, s, e = torch.randn(2, 3, 50, device="cuda"), torch.zeros(2, 3, device="cuda"), torch.zeros(2, 3, device="cuda", dtype=torch.bool)
    t = torch.randn(6, 4, device="cuda")
    b, r = o.beam_step, o.reorder_states
    parents = torch.zeros(2, 3, device="cuda", dtype=torch.int64)
    refused(lambda: b(z[0], s), lambda: b(z.double(), s), lambda: b(z.transpose(1, 2), s), lambda: b(z, s[:1]), lambda: b(z, s.double()), lambda: b(z, s.cpu()),
            lambda: b(z, s, width=0), lambda: b(z, s, width=33), lambda: b(z[:, :1, :2], s[:, :1].contiguous(), width=3), lambda: b(z, s, ended=e),
            lambda: b(z, s, ended=e.int(), end=1), lambda: b(z, s, ended=e[:1], end=1), lambda: b(z, s, end=50), lambda: b(z, s, end=-1),
            lambda: b(z[:, :, :0], s), lambda: b(z[:, :0], s[:, :0]), lambda: b(torch.zeros(1, 33, 4, device="cuda"), torch.zeros(1, 33, device="cuda")),
            lambda: b(torch.empty(0, 1, (1 << 22) + 1, device="cuda"), torch.empty(0, 1, device="cuda")),
            lambda: b(z, s, states=t), lambda: b(z, s, states=[t[:5]]), lambda: b(z, s, states=[t.t()]), lambda: b(z, s, states=[t.cpu()]), lambda: b(z, s, states=[None]),
            lambda: b(z, s, states=[t, t], inplace=True), lambda: b(z, s, width=2, states=[t], inplace=True),
            lambda: r([t], parents.int()), lambda: r([t], parents[0]), lambda: r([t], parents.t()), lambda: r([t], parents.cpu()), lambda: r([t[:5]], parents),
            lambda: r([t], parents, beams=4), lambda: r([t], parents, beams=0), lambda: r([t], parents, beams=33), lambda: r([t, t], parents, inplace=True),
            lambda: r(t, parents), lambda: r([torch.randn(4, 2, device="cuda")], parents, beams=2, inplace=True))
