"""Beams' states in place that share memory are refused by the host's check, before anything is launched."""
import itertools

import pytest

torch = pytest.importorskip("torch")
from paper_2412_11810_b200 import ops  # noqa: E402


def table(states, *read):
    return ops._state_table(states, 6, 6, True, -1, *read)   # (-1: tensors on the CPU)


def test_states_that_share_memory():
    buffer = torch.arange(100.0)
    a, b, c, d = buffer[:24].view(6, 4), buffer[24:48].view(6, 4), buffer[48:54].view(6), buffer[54:66].view(6, 2)
    nothing = buffer[30:30].view(6, 0)
    for some in itertools.permutations((a, b, c, d, nothing, nothing)):
        assert table(list(some))[1] == list(some)
    for other in (a, buffer[:24].view(6, 2, 2), buffer[23:29].view(6), buffer[23:47].view(6, 4), buffer[6:12].view(6), buffer[:60].view(6, 10), buffer[65:71].view(6)):
        for some in itertools.permutations((a, b, d, other)):
            with pytest.raises(ValueError, match="states"):
                table(list(some))
        # copies may come from anywhere
        ops._state_table([a, b, d, other], 6, 6, False, -1)


def test_states_that_share_memory_with_the_parents():
    buffer = torch.arange(30)
    parents, state = buffer[6:12].view(2, 3), torch.zeros(6, 5)
    assert len(table([buffer[:6], state, buffer[12:18]], parents)[1]) == 3
    for other in (parents.view(6), buffer[1:7], buffer[11:17], buffer[:30].view(6, 5), parents.view(6).view(torch.uint8).view(6, 8)):
        for states in ([other], [state, other], [other, state]):
            with pytest.raises(ValueError, match="parents"):
                table(states, parents)
