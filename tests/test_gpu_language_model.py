"""The sequence-model operators together, as a small recurrent language model trains and answers with them: norms around a gated
recurrence, the vocabulary loss, the AdamW step, and beam search whose beams carry the recurrent state."""
import numpy as np
import pytest


pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

T, B, N, V = 20, 3, 48, 61


def ops():
    from paper_2412_11810_b200 import ops as o
    return o


def parameters(dtype, seed=1):
    g = torch.Generator().manual_seed(seed)
    r = lambda *s: torch.randn(*s, generator=g)  # noqa: E731
    return [t.to(dtype).cuda() for t in (r(V, N) * 0.5, 1 + 0.1 * r(N), r(N, N) / N ** 0.5, r(N, N) / N ** 0.5, 1 + 0.1 * r(N))]


def batch(seed=2):
    g = torch.Generator().manual_seed(seed)
    tokens = torch.randint(0, V, (T + 1, B), generator=g).cuda()
    return tokens[:-1], tokens[1:].contiguous()


def training_step(params, tokens, targets, keep="raw"):
    """Loss and gradients."""
    table, w1, wx, wg, w2 = params
    o = ops()
    x = table[tokens]
    y1, _, s1, _ = o.rms_norm(x, w1)
    h, last, kept = o.gated_scan(y1 @ wx, y1 @ wg, keep=keep)
    y2, h2, s2, _ = o.rms_norm(h, w2, x)
    flat = lambda t: t.view(T * B, N)  # noqa: E731
    loss, _, lse = o.vocab_loss(flat(y2), table.t(), targets.view(-1))
    dy2, dtable = o.vocab_loss_backward(flat(y2), table.t(), targets.view(-1), lse)
    dh, dw2 = o.rms_norm_backward(h2, s2, dy2.view(T, B, N), w2)
    dz, dgate, _ = o.gated_scan_backward(kept, dh)
    dy1 = dz @ wx.t() + dgate @ wg.t()
    dx, dw1 = o.rms_norm_backward(x, s1, dy1, w1, dh)
    # (the embedding's rows of equal tokens are added by a product, in the same order every time)
    chosen = (torch.arange(V, device=x.device)[:, None] == tokens.reshape(1, -1)).to(x.dtype)
    dtable = dtable.t() + chosen @ flat(dx)
    return loss, [dtable, dw1, flat(y1).t() @ flat(dz), flat(y1).t() @ flat(dgate), dw2]


def exact_loss(params, tokens, targets):
    table, w1, wx, wg, w2 = params
    norm = lambda v, w: v / torch.sqrt((v * v).mean(-1, keepdim=True) + 1e-6) * w  # noqa: E731
    x = table[tokens]
    y1 = norm(x, w1)
    z, a = y1 @ wx, torch.sigmoid(y1 @ wg)
    h, out = torch.zeros(B, N, dtype=x.dtype, device=x.device), []
    for t in range(T):
        h = a[t] * h + (1 - a[t]) * z[t]
        out.append(h)
    return torch.nn.functional.cross_entropy((norm(torch.stack(out) + x, w2) @ table.t()).view(T * B, V), targets.view(-1))


def test_gradients_of_the_whole_model():
    params, (tokens, targets) = parameters(torch.float32), batch()
    leaves = [p.double().requires_grad_() for p in params]
    want = exact_loss(leaves, tokens, targets)
    want.backward()
    loss, grads = training_step(params, tokens, targets)
    # ten stages, each off by less than 64 units of 2^-23 of the magnitudes it sums, which are up to ten times the result:
    # 10 * 64 * 2^-23 * 10 < 8e-4
    assert abs(float(loss) - float(want.detach())) <= 8e-4 * float(want.detach())
    for k, (g, w) in enumerate(zip(grads, leaves)):
        assert float((g.double() - w.grad).norm()) <= 8e-4 * float(w.grad.norm()), k


def test_gradients_of_the_whole_model_against_differences():
    params, (tokens, targets) = parameters(torch.float32), batch()
    _, grads = training_step(params, tokens, targets)
    g = torch.Generator(device="cuda").manual_seed(3)
    for k, grad in enumerate(grads):
        v = torch.randn(grad.shape, generator=g, device="cuda", dtype=torch.float64)
        loss = lambda s: float(exact_loss([p.double() + s * v if j == k else p.double() for j, p in enumerate(params)], tokens, targets))  # noqa: E731
        slope = (loss(1e-5) - loss(-1e-5)) / 2e-5
        assert abs(float((grad.double() * v).sum()) - slope) <= 8e-4 * float((grad.double() * v).abs().sum()) + 1e-8


@pytest.mark.parametrize("dtype,bits,keep", [(torch.float32, 32, "raw"), (torch.bfloat16, 8, "int8"), (torch.float16, 8, "e4m3")])
def test_training_steps_eager_and_captured(dtype, bits, keep):
    """Steps of the whole model with the update in them give the same bits out of a graph, which counts its own steps."""
    tokens, targets = batch()
    kw = dict(lr=1e-2, max_norm=1.0, seed=7)

    def run(captured):
        params = parameters(dtype)
        state = ops().adamw_state(params, bits)

        def step():
            loss, grads = training_step(params, tokens, targets, keep)
            ops().adamw_step(params, grads, state, **kw)
            return loss

        if not captured:
            return [step().clone() for _ in range(4)], params, state
        loss = step().clone()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            held = step()
        losses = [loss]
        for _ in range(3):
            graph.replay()
            losses.append(held.clone())
        torch.cuda.synchronize()
        return losses, params, state

    losses, params, state = run(False)
    again, params2, state2 = run(True)
    assert int(state.step) == int(state2.step) == 4
    assert all(torch.isfinite(v) for v in losses) and [float(v) for v in losses] == [float(v) for v in again]
    for a, b in zip(params, params2):
        assert torch.isfinite(a).all() and torch.equal(a, b)


def test_answers_by_beam_search():
    """Beams that carry the recurrent state, token by token, against the score of each answer over the whole sequence at once."""
    o = ops()
    table, w1, wx, wg, w2 = parameters(torch.float32, 4)
    steps, K, end = 6, 5, 7
    first = torch.tensor([3, 11], device="cuda")
    rows = first.numel()
    state, scores, ended = torch.zeros(rows, N, device="cuda"), torch.zeros(rows, 1, device="cuda"), None
    history = first[:, None].clone()
    for t in range(steps):
        x = table[history[:, -1]]
        y, _, _, _ = o.rms_norm(x, w1)
        h, state = o.gated_scan_step(y @ wx, y @ wg, state)
        y, _, _, _ = o.rms_norm(h, w2, x)
        logits = (y @ table.t()).view(rows, -1, V)
        tokens, parents, scores, ended, (state, history) = o.beam_step(logits, scores, width=K, ended=ended, end=end, states=[state, history])
        history = torch.cat([history, tokens.view(-1, 1)], 1)
    answers = history.view(rows, K, steps + 1)
    assert (scores[:, :-1] >= scores[:, 1:]).all()
    for b in range(rows):
        seen = set()
        for k in range(K):
            a = answers[b, k].tolist()
            seen.add(tuple(a))
            stop = a.index(end, 1) + 1 if end in a[1:] else len(a)
            assert all(v == end for v in a[stop:]) and bool(ended[b, k]) == (end in a[1:])
            # the same tokens at once, in 64 bits
            p = [v.double() for v in (table, w1, wx, wg, w2)]
            seq = torch.tensor(a[:stop], device="cuda")
            x = p[0][seq[:-1]]
            norm = lambda v, w: v / torch.sqrt((v * v).mean(-1, keepdim=True) + 1e-6) * w  # noqa: E731
            y = norm(x, p[1])
            z, g = y @ p[2], torch.sigmoid(y @ p[3])
            h, total = torch.zeros(N, dtype=torch.float64, device="cuda"), 0.0
            for t in range(stop - 1):
                h = g[t] * h + (1 - g[t]) * z[t]
                total += float(torch.log_softmax(norm(h + x[t], p[4]) @ p[0].t(), -1)[seq[t + 1]])
            # six steps of logits below 30, each the end of four stages off by 64 units of 2^-23 of what they sum
            assert abs(total - float(scores[b, k])) <= steps * 4 * 64 * 2.0 ** -23 * 30
        assert len(seen) == K
    assert np.isfinite(scores.cpu().numpy()).all()
