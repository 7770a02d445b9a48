"""The sequence-model operators together, as a recurrent language model uses them: a gated recurrence over its inputs, kept
for the backward pass, and the vocabulary loss of what it puts out."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def model(T, B, N, V, dtype, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g, device="cuda")  # noqa: E731
    x, gate = r(T, B, N).to(dtype), (r(T, B, N) + 1).to(dtype)
    table = (r(V, N) * 3 / N ** 0.5).to(dtype)     # one row per class: w_out is its transpose
    targets = torch.randint(0, V, (T, B), generator=g, device="cuda")
    targets[T // 2:, 0] = -100                      # the first sequence is shorter
    lengths = torch.full((B,), T, dtype=torch.int32, device="cuda")
    lengths[0] = T // 2
    return x, gate, r(B, N), table, targets, lengths


def step(x, gate, state, table, targets, lengths, keep):
    from paper_2412_11810_b200 import ops
    T, B, N = x.shape
    h, last, kept = ops.gated_scan(x, gate, state, lengths=lengths, keep=keep)
    loss, _, lse = ops.vocab_loss(h.view(T * B, N), table.t(), targets.view(-1))
    dh, dw = ops.vocab_loss_backward(h.view(T * B, N), table.t(), targets.view(-1), lse)
    return (loss, last, *ops.gated_scan_backward(kept, dh.view(T, B, N)), dw.t())


def exact_loss(x, gate, state, table, targets, lengths):
    """The same loss in 64 bits, differentiable."""
    T, B, N = x.shape
    on = (torch.arange(T, device=x.device)[:, None] < lengths[None, :])[:, :, None]
    a = torch.sigmoid(gate)
    h, out = state, []
    for t in range(T):
        h = torch.where(on[t], a[t] * h + (1 - a[t]) * x[t], h)
        out.append(torch.where(on[t], h, torch.zeros_like(h)))
    z = torch.stack(out).reshape(T * B, N) @ table.t()
    return torch.nn.functional.cross_entropy(z, targets.view(-1), ignore_index=-100), h


@pytest.mark.parametrize("T,B,N,V", [(70, 3, 64, 500), (130, 2, 33, 1003)])
def test_training_step_in_fp32(T, B, N, V):
    m = model(T, B, N, V, torch.float32, 1)
    leaves = [t.double().requires_grad_() for t in m[:4]]
    want_loss, want_last = exact_loss(*leaves, *m[4:])
    want_loss.backward()
    got = step(*m, "raw")
    # every stage is off by less than 64 units of 2^-23 of the magnitudes it sums (the bounds of its own tests); over the
    # four stages of a gradient, with sums whose magnitudes are up to ten times the result, 4 * 64 * 2^-23 * 10 < 4e-4
    want_loss = float(want_loss.detach())
    assert abs(float(got[0]) - want_loss) <= 4e-4 * want_loss
    for name, g, w in zip(("last", "dx", "dgate", "dstate", "dtable"), got[1:], (want_last.detach(), *(v.grad for v in leaves))):
        assert float((g.double() - w).norm()) <= 4e-4 * float(w.norm()), name


def test_training_step_against_differences():
    T, B, N, V = 40, 2, 16, 60
    m = model(T, B, N, V, torch.float32, 2)
    grads = step(*m, "raw")[2:]
    point = [t.double() for t in m[:4]]
    g = torch.Generator(device="cuda").manual_seed(3)
    for k, grad in enumerate(grads):
        v = torch.randn(grad.shape, generator=g, device="cuda", dtype=torch.float64)

        def loss(s):
            return float(exact_loss(*[p + s * v if j == k else p for j, p in enumerate(point)], *m[4:])[0])

        slope = (loss(1e-5) - loss(-1e-5)) / 2e-5
        assert abs(float((grad.double() * v).sum()) - slope) <= 4e-4 * float((grad.double() * v).abs().sum()) + 1e-8


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
@pytest.mark.parametrize("keep", ["raw", "int8", "e4m3"])
def test_training_step_in_16_bits_and_captured(dtype, keep):
    """Runs in every type and format, gives the same bits again, and out of a graph."""
    m = model(200, 2, 96, 700, dtype, 4)
    want = step(*m, keep)
    assert all(torch.isfinite(t).all() for t in want) and all(float(t.abs().max()) > 0 for t in want)
    assert all(torch.equal(a, b) for a, b in zip(want, step(*m, keep)))
    want = [t.clone() for t in want]
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step(*m, keep)
    graph.replay()
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(held, want))
    # padding of the shorter sequence takes no part
    assert (want[2][100:, 0] == 0).all() and (want[3][100:, 0] == 0).all()


def test_scoring_token_by_token():
    """A serving loop (one step of the recurrence, the loss of one row) agrees with the whole sequence at once."""
    from paper_2412_11810_b200 import ops
    T, N, V = 12, 40, 300
    x, gate, state, table, targets, _ = model(T, 1, N, V, torch.float32, 5)
    targets = targets.clamp(min=0)
    h, last, _ = ops.gated_scan(x, gate, state)
    _, rows, _ = ops.vocab_loss(h.view(T, N), table.t(), targets.view(-1))
    s = state
    for t in range(T):
        out, s = ops.gated_scan_step(x[t], gate[t], s)
        _, row, _ = ops.vocab_loss(out, table.t(), targets[t])
        # two orders of the same arithmetic: 64 units of 2^-23 each of magnitudes below 40
        assert abs(float(row) - float(rows[t])) <= 2 * 64 * 2.0 ** -23 * 40
    assert float((s - last).abs().max()) <= 2 * 64 * 2.0 ** -23 * 8
