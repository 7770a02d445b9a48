"""Beam search over a vocabulary on the GPU against its definition in 64 bits."""
import numpy as np
import pytest

import model_reference as ref

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")

DT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
INF = float("inf")


def ops():
    from paper_2412_11810_b200 import ops as o
    return o


def f64(t):
    return t.detach().to(torch.float64).cpu().numpy()


def check(logits, scores, width=None, ended=None, end=None, states=(), **kw):
    B, K, V = logits.shape
    W = K if width is None else width
    before = [t.clone() for t in states]
    tokens, parents, new, gone, out = ops().beam_step(logits, scores, width=width, ended=ended, end=end, states=states, **kw)
    assert tokens.shape == parents.shape == new.shape == (B, W) and tokens.dtype is torch.int64 and parents.dtype is torch.int64
    z, s = f64(logits), f64(scores)
    t, p = tokens.cpu().numpy(), parents.cpu().numpy()
    e = None if ended is None else ended.cpu().numpy()
    assert ((t >= 0) & (t < V) & (p >= 0) & (p < K)).all()
    for b in range(B):
        ref.check_beam(p[b] * V + t[b], f64(new)[b], z[b], s[b], W, None if e is None else e[b], end, f"sample {b}")
    if end is None:
        assert gone is None
    else:
        want = t == end
        if e is not None:
            want = want | np.take_along_axis(e, p, 1)
        assert np.array_equal(gone.cpu().numpy(), want)
    rows = (parents + K * torch.arange(B, device=parents.device)[:, None]).reshape(-1)
    assert len(out) == len(before) and all(torch.equal(o, f[rows]) for o, f in zip(out, before))
    return tokens, parents, new, gone, out


def inputs(B, K, V, dtype, seed, std=2.5):
    g = torch.Generator().manual_seed(seed)
    logits = (std * torch.randn(B, K, V, generator=g)).to(DT[dtype]).cuda()
    return logits, (-5 * torch.rand(B, K, generator=g)).cuda(), g


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("B,K,W,V", [(1, 1, 1, 1), (2, 1, 3, 3), (3, 4, 4, 5), (1, 4, 4, 2047), (2, 3, 3, 2048), (2, 3, 5, 2049), (5, 1, 32, 4096), (1, 32, 32, 8191),
                                     (3, 8, 8, 8193), (2, 5, 5, 16385), (1, 2, 2, 50257), (40, 4, 4, 32000), (30, 20, 20, 8200), (1, 1, 32, 32), (4, 32, 1, 33)])
def test_sizes(B, K, W, V, dtype):
    logits, scores, _ = inputs(B, K, V, dtype, B + K + V)
    check(logits, scores, W)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("W", [4, 32])
def test_parts_of_many_segments(W, dtype):
    """Enough rows for a warp to walk through a dozen of segments: ordinary rows, equal values, rising and falling ones, steps of
    a few values, the best at the end, and masks."""
    B, K, V = 300, 4, 20001
    logits, scores, g = inputs(B, K, V, dtype, 13)
    rise = torch.arange(V, device="cuda") / V
    logits[1] = 0.5
    logits[2, 0], logits[2, 1] = rise.to(logits), (-rise).to(logits)
    logits[3] = (rise * 40).floor().to(logits)
    logits[4] = (-rise * 40).floor().to(logits)
    logits[5, :, -3:] = 30
    logits[6, :, :-2] = -INF
    logits[7, 1] = torch.where(torch.rand(V, generator=g) < 0.5, -INF, 1.0).to(logits)
    logits[8] = torch.randint(0, 3, (K, V), generator=g).to(logits)
    logits[9, 2], logits[10, 3, 15000] = -INF, float("nan")
    check(logits, scores, W)


@pytest.mark.parametrize("V", [(1 << 22) - 3, 1 << 22])
def test_the_largest_vocabulary(V):
    logits, scores, _ = inputs(1, 2, V, "bf16", 3)
    check(logits, scores, 7)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("layout", ["offset", "beams_first", "last_position"])
def test_layouts(layout, dtype):
    B, K, V = 3, 4, 3001
    logits, scores, _ = inputs(B, K, V, dtype, 4)
    if layout == "offset":
        wide = torch.full((B, K, V + 9), INF, dtype=logits.dtype, device="cuda")
        wide[..., 5:5 + V] = logits
        view = wide[..., 5:5 + V]
    elif layout == "beams_first":
        view = logits.transpose(0, 1).contiguous().transpose(0, 1)
    else:   # of several positions of each beam
        wide = torch.full((B, K, 3, V), INF, dtype=logits.dtype, device="cuda")
        wide[:, :, 2] = logits
        view = wide[:, :, 2]
    want = check(logits, scores)
    got = check(view, scores)
    assert all(torch.equal(a, b) for a, b in zip(want[:2], got[:2]))
    assert torch.equal(want[2], got[2])   # sums go by the classes, not by the address of a row


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_equal_logits_go_by_their_class(dtype):
    """Rows of equal values, of few different ones, and of both zeros."""
    B, K, V = 2, 3, 9000
    logits, scores, g = inputs(B, K, V, dtype, 5)
    logits[0, 0] = 1.25
    logits[0, 1] = torch.randint(0, 3, (V,), generator=g).to(logits)
    logits[0, 2] = torch.where(torch.rand(V, generator=g) < 0.5, 0.0, -0.0).to(logits)
    logits[1] = 0
    scores[1] = -1.5   # beams that are the same as well: the lower one first
    tokens, parents, *_ = check(logits, scores, 32)
    assert tokens[1].tolist() == list(range(32)) and (parents[1] == 0).all()
    # all of a beam's best behind the others' in a rising and a falling row
    logits[0, 0] = torch.arange(V).to(logits) / V
    logits[0, 1] = -torch.arange(V).to(logits) / V
    check(logits, scores, 32)


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("V", [4999, 50257])
def test_equal_beams_tie(V, dtype):
    """Copies of a beam, at odd addresses of all kinds: the lower one first, with the same scores to the bit."""
    logits, scores, _ = inputs(5, 1, V, dtype, 12)
    logits, scores = logits.repeat(1, 8, 1), scores.repeat(1, 8)
    tokens, parents, new, _, _ = check(logits, scores, 32)
    for b in range(5):
        for t in tokens[b].unique():
            at = tokens[b] == t
            assert len(set(new[b][at].tolist())) == 1 and parents[b][at].tolist() == list(range(int(at.sum())))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_masked_classes(dtype):
    """Masks of -infinity and of the type's lowest value, rows with few classes left, with one, and with none."""
    B, K, V = 6, 3, 5000
    logits, scores, g = inputs(B, K, V, dtype, 6)
    low = torch.finfo(DT[dtype]).min
    logits[0, :, 10:] = -INF
    logits[1, :, 10:] = low
    logits[2] = -INF
    logits[2, 1, 4321] = 3.0       # one continuation for the whole sample
    logits[3] = low
    logits[4] = -INF               # none at all
    logits[5, 0] = -INF
    logits[5, 1, ::2] = -INF
    for width in (3, 32):
        tokens, parents, new, _, _ = check(logits, scores, width)
        assert (int(parents[2, 0]), int(tokens[2, 0])) == (1, 4321) and tokens[2, 1:].tolist() == list(range(width - 1)) and torch.isneginf(new[2, 1:]).all()
        assert tokens[4].tolist() == list(range(width)) and (parents[4] == 0).all() and torch.isneginf(new[4]).all()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V", [40, 20000])
def test_dead_beams(dtype, V):
    """NaN and +infinity in the logits or the score: no continuation, and no trace in the others."""
    B, K = 4, 4
    logits, scores, _ = inputs(B, K, V, dtype, 7)
    logits[0, 0, V // 2] = float("nan")
    logits[0, 2, V - 1] = INF
    logits[1] = float("nan")
    logits[2, 3] = -INF
    logits[2, 3, 5] = float("nan")     # NaN beside masked classes alone
    scores[2, 0], scores[2, 1], scores[3, 1] = float("nan"), -INF, INF
    tokens, parents, new, _, _ = check(logits, scores, 6)
    assert set(parents[0].tolist()) <= {1, 3} and set(parents[2].tolist()) == {2} and torch.isneginf(new[1]).all()


@pytest.mark.parametrize("K,W,V,end", [(4, 4, 7000, 2), (5, 5, 33, 0), (3, 8, 4, 3), (1, 4, 100, 50), (32, 32, 2100, 2099)])
def test_ended_beams(K, W, V, end):
    B = 6
    logits, scores, g = inputs(B, K, V, "bf16", 8)
    ended = torch.rand(B, K, generator=g) < 0.4
    ended[0], ended[1] = True, False
    ended = ended.cuda()
    logits[ended] = float("nan")       # never looked at
    logits[1, 0, end] = 30.0           # ends in this step
    scores[2, 0] = -INF
    tokens, parents, _, gone, _ = check(logits, scores, W, ended, end)
    # (where that is among the survivors, which the scores of the other beams decide)
    assert gone[1][(tokens[1] == end) & (parents[1] == 0)].all()
    check(logits[1:2], scores[1:2], W, None, end)


def test_states_of_all_kinds():
    B, K, W, V = 5, 3, 4, 300
    logits, scores, g = inputs(B, K, V, "fp32", 9)
    r = lambda *s: torch.randn(B * K, *s, generator=g).cuda()  # noqa: E731
    states = [r(64), r(7).to(torch.bfloat16), r(3, 5).to(torch.float16), torch.randint(0, 99, (B * K, 11), generator=g).cuda(),
              torch.randint(0, 99, (B * K, 13), generator=g).to(torch.uint8).cuda(), r(), r(0), r(20000), r(2, 1000).double()]
    check(logits, scores, W, states=states)
    check(logits, scores, K, states=states)
    check(logits, scores, K, states=[t.clone() for t in states], inplace=True)
    check(logits, scores, W, states=[r(k) for k in range(1, 151)])


def test_reorder_states():
    g = torch.Generator().manual_seed(10)
    B, K, W = 3, 5, 4
    parents = torch.randint(0, K, (B, W), generator=g).cuda()
    t = torch.randn(B * K, 37, generator=g).cuda()
    rows = (parents + K * torch.arange(B, device="cuda")[:, None]).reshape(-1)
    assert torch.equal(ops().reorder_states([t], parents, beams=K)[0], t[rows])
    # parents that are none are never an index
    parents = torch.tensor([[0, -1, 5, 2 ** 62, -2 ** 62], [4, 3, 2, 1, 0]], device="cuda")
    t = torch.randn(10, 6, generator=g).cuda()
    want = torch.cat([t[:1], torch.zeros(4, 6, device="cuda"), t[5:].flip(0)])
    assert torch.equal(ops().reorder_states([t], parents)[0], want)
    held = t.clone()
    out = ops().reorder_states([held], parents, inplace=True)
    assert out[0] is held and torch.equal(held, want)
    assert ops().reorder_states([], parents) == []
    empty = ops().reorder_states([torch.empty(0, 3, device="cuda")], torch.empty(0, 2, dtype=torch.int64, device="cuda"))
    assert empty[0].shape == (0, 3)


def test_without_samples():
    tokens, parents, new, gone, out = ops().beam_step(torch.empty(0, 4, 50, device="cuda"), torch.empty(0, 4, device="cuda"), end=1,
                                                      states=[torch.empty(0, 8, device="cuda")])
    assert tokens.shape == parents.shape == new.shape == gone.shape == (0, 4) and out[0].shape == (0, 8)


def test_streams_and_capture():
    B, K, V = 4, 4, 9001
    logits, scores, g = inputs(B, K, V, "bf16", 11)
    ended = (torch.rand(B, K, generator=g) < 0.3).cuda()
    states = [torch.randn(B * K, 100, generator=g).cuda()]

    def step():
        t, p, s, e, out = ops().beam_step(logits, scores, ended=ended, end=3, states=states)
        return t, p, s, e, *out

    want = step()
    assert all(torch.equal(a, b) for a, b in zip(want, step()))
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        got = step()
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(want, got))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        held = step()
    for _ in range(2):
        for t in held:
            t.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(held, want))


def test_offsets_beyond_32_bits():
    B, K, V = 17, 32, (1 << 22) - 1     # 2.28e9 logits
    logits = torch.zeros(B, K, V, dtype=torch.bfloat16, device="cuda")
    logits[:, :, 7] = 1.0
    logits[-1, -1, V - 2] = 9.0
    logits[-1, 30, V - 1] = 8.0
    scores = torch.zeros(B, K, device="cuda")
    tokens, parents, new, _, _ = ops().beam_step(logits, scores, width=3)
    assert parents[-1].tolist()[:2] == [31, 30] and tokens[-1].tolist()[:2] == [V - 2, V - 1]
    assert (tokens[:-1] == 7).all() and (parents[:-1] == torch.arange(3, device="cuda")).all()
    want = 9 - np.log(np.exp(9.0) + np.exp(1.0) + V - 2)
    assert abs(float(new[-1, 0]) - want) <= 1e-6
