"""Parameters and copies that share memory are refused by AdamW's check on the host, before anything is launched."""
import itertools

import pytest

torch = pytest.importorskip("torch")
from paper_2412_11810_b200 import binding as sb  # noqa: E402
from paper_2412_11810_b200 import ops  # noqa: E402


@pytest.fixture
def step(monkeypatch):
    """adamw_step with tensors that say they are on device 0, whose library call is recorded instead."""
    calls = []

    class OnDevice(torch.Tensor):
        is_cuda = True

        def get_device(self):
            return 0

    def on(t):
        return t.as_subclass(OnDevice)

    monkeypatch.setattr(ops, "_launch", lambda call, a, like: calls.append(a.count))
    monkeypatch.setattr(ops, "_like", lambda *a, **k: None)

    def call(params, copies=None):
        room = sum(-(-p.numel() // 64) * 64 for p in params)
        state = ops.AdamWState(on(torch.zeros(room)), on(torch.zeros(room)), on(torch.zeros((), dtype=torch.int64)))
        grads = [on(torch.zeros(p.shape)) for p in params]
        ops.adamw_step([on(p) for p in params], grads, state, lr=1e-3, copies=None if copies is None else [None if c is None else on(c) for c in copies])
        return calls

    return call, calls


def test_parameters_and_copies_that_share_memory(step):
    call, calls = step
    buffer, other = torch.zeros(100), torch.zeros(100, dtype=torch.bfloat16)
    a, b, c, empty = buffer[:24].view(4, 6), buffer[24:50], buffer[60:61], buffer[5:5]
    for some in itertools.permutations((a, b, c, empty, empty)):
        call(list(some))
    call([a, b, c], [other[:24].view(4, 6), other[24:50], None])
    done = len(calls)
    for one in (a, buffer[23:30], buffer[:1], buffer[:70], buffer[2:4].view(2, 1), buffer.view(torch.bfloat16)[100:103], buffer.view(torch.float16)[99:100]):
        if one.dtype is torch.bfloat16:
            one = buffer.view(torch.bfloat16)[97:103]    # from the middle of a value on
        for some in itertools.permutations((a, b, c, one)):
            with pytest.raises(ValueError, match="params|copies"):
                call(list(some))
    for copies in ([a, None, None], [None, None, buffer[49:50]], [other[:24].view(4, 6), other[23:49], None], [buffer.view(torch.bfloat16)[:24].view(4, 6), None, None],
                   [None, buffer[40:66], None]):
        with pytest.raises(ValueError, match="params|copies"):
            call([a, b, c], copies)
    assert len(calls) == done
