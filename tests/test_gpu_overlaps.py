"""Beams' states in place that share memory, with one another or with the parents: refused, since the result would depend on the order of writes."""
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


def test_states_in_place():
    o = ops()
    logits, scores = torch.randn(2, 3, 50, device="cuda"), torch.zeros(2, 3, device="cuda")
    parents = torch.tensor([[2, 0, 1], [1, 1, 0]], device="cuda")
    rows = torch.tensor([2, 0, 1, 4, 4, 3], device="cuda")
    buffer = torch.randn(100, device="cuda")
    before = buffer.clone()
    a, b, c = buffer[:24].view(6, 4), buffer[20:44].view(6, 4), buffer[44:56].view(6, 2)
    again, inside = buffer[:24].view(6, 2, 2), buffer[6:18].view(6, 2)
    for pair in ([a, b], [b, a], [c, a, b], [a, again], [a, inside], [inside, a], [a, c, buffer[55:61].view(6, 1)]):
        refused(lambda: o.beam_step(logits, scores, states=pair, inplace=True), lambda: o.reorder_states(pair, parents, inplace=True))
    assert torch.equal(buffer, before)
    # one behind the other: no byte in common; states without values are nowhere
    out = o.reorder_states([b, buffer[44:50].view(6, 1), buffer[:0].view(6, 0), buffer[:0].view(6, 0), buffer[8:20].view(6, 2)], parents, inplace=True)
    assert torch.equal(out[0], before[20:44].view(6, 4)[rows]) and torch.equal(out[1], before[44:50].view(6, 1)[rows])
    assert torch.equal(out[4], before[8:20].view(6, 2)[rows]) and torch.equal(buffer[:8], before[:8]) and torch.equal(buffer[50:], before[50:])
    # copies may come from anywhere
    out = o.reorder_states([a, b, a, inside], parents)
    assert all(torch.equal(p, q[rows]) for p, q in zip(out, (a, b, a, inside)))


def test_parents_are_not_moved_while_they_are_read():
    o = ops()
    parents = torch.tensor([[2, 0, 1], [1, 1, 0]], device="cuda")
    rows = torch.tensor([2, 0, 1, 4, 4, 3], device="cuda")
    held, state = parents.clone(), torch.randn(6, 5, device="cuda")
    refused(lambda: o.reorder_states([parents.view(6)], parents, inplace=True), lambda: o.reorder_states([state, parents.view(6, 1)], parents, inplace=True))
    assert torch.equal(parents, held)
    assert torch.equal(o.reorder_states([parents.view(6)], parents)[0], held.view(6)[rows])
