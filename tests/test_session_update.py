"""Session.adamw_step without gradients to apply, or with other moments than it has: refused before anything is launched, so without a GPU."""
import pytest

torch = pytest.importorskip("torch")
from paper_2412_11810_b200 import binding as sb  # noqa: E402
from paper_2412_11810_b200 import ops, session  # noqa: E402


@pytest.fixture
def net(monkeypatch):
    """A Session whose tensors are on the CPU and whose library calls are recorded; (session, calls)."""
    calls = []
    s = object.__new__(session.Session)
    s.net, s.sizes, s.L, s.cell, s.device = None, [4, 3, 2], 1, sb.SNN_CELL_LIF, torch.device("cpu")
    s.device_ws, s.pinned_ws, s.adamw, s.debug_V, s._last = torch.empty(64, dtype=torch.uint8), None, None, None, None

    class Stream:
        cuda_stream = 0

        def synchronize(self):
            pass

    s.main = s.side = Stream()
    monkeypatch.setattr(session.Session, "ensure_workspace", lambda self, *a: (0, 0))
    monkeypatch.setattr(torch.cuda, "current_stream", lambda *a: Stream())
    monkeypatch.setattr(sb, "snn_train_step", lambda net, a: calls.append("train") or 1.0)
    monkeypatch.setattr(ops, "adamw_step", lambda params, grads, state, **kw: calls.append(("adamw", state)))
    monkeypatch.setattr(ops, "adamw_state", lambda params, bits=32: calls.append(("state", bits)) or ops.AdamWState(
        *([ops.PackedActivation(None, None, "e4m3", torch.float32)] * 2 if bits == 8 else [torch.zeros(1)] * 2), torch.zeros((), dtype=torch.int64)))
    weights(s)
    return s, calls


def weights(s):
    s.set_weights([torch.ones(4, 3).numpy()], [torch.ones(3, 3).numpy()], torch.ones(3, 2).numpy())


class OnDevice(torch.Tensor):
    is_cuda = True


def train(s, **kw):
    bits = torch.zeros(5, 2, 1, dtype=torch.int32).as_subclass(OnDevice)
    return s.train_step(bits, torch.zeros(2, dtype=torch.int32), **kw)


def refused(s, calls, *errors, **kw):
    before = list(calls)
    with pytest.raises(errors or RuntimeError):
        s.adamw_step(lr=1e-3, **kw)
    assert calls == before


def test_before_the_first_training_step(net):
    s, calls = net
    refused(s, calls)
    train(s)
    s.adamw_step(lr=1e-3)
    assert [c[0] for c in calls] == ["t", "state", "adamw"]


def test_after_a_forward_pass_alone(net):
    s, calls = net
    train(s, forward_only=True)
    refused(s, calls)
    train(s)
    s.adamw_step(lr=1e-3)
    train(s, extra_flags=sb.SNN_FLAG_FORWARD_ONLY)
    refused(s, calls)
    train(s)
    s.adamw_step(lr=1e-3)


def test_after_new_weights(net):
    s, calls = net
    train(s)
    weights(s)
    refused(s, calls)


def test_after_a_step_that_failed(net, monkeypatch):
    s, calls = net
    train(s)

    def fails(net, a):
        raise RuntimeError("event pool overflow")

    with monkeypatch.context() as m:
        m.setattr(sb, "snn_train_step", fails)
        with pytest.raises(RuntimeError, match="overflow"):
            train(s)
    refused(s, calls)
    train(s)
    s.adamw_step(lr=1e-3)


def test_moments_of_other_bits_than_the_first_step_chose(net):
    s, calls = net
    train(s)
    s.adamw_step(lr=1e-3, bits=8)
    assert ("state", 8) in calls
    refused(s, calls, ValueError, bits=32)
    s.adamw_step(lr=1e-3)           # those that it has
    s.adamw_step(lr=1e-3, bits=8)
    weights(s)
    train(s)
    s.adamw_step(lr=1e-3)           # anew: 32
    assert ("state", 32) in calls
    refused(s, calls, ValueError, bits=8)
    s.adamw_step(lr=1e-3, bits=32)
