"""The recurrence with its first state and its last one in the same buffer, which the C ABI allows."""
import pytest

pytestmark = pytest.mark.gpu
torch = pytest.importorskip("torch")


def forward(x, gate, state, last, lengths, h, states):
    from paper_2412_11810_b200 import binding as sb
    T, B, N = x.shape
    a = sb.snn_scan_args(T, B, N, {torch.float32: sb.SNN_DTYPE_FP32, torch.bfloat16: sb.SNN_DTYPE_BF16}[x.dtype], sb.SNN_SCAN_SIGMOID,
                         x.data_ptr(), gate.data_ptr(), x.stride()[:2], gate.stride()[:2], None if lengths is None else lengths.data_ptr(),
                         None if state is None else state.data_ptr(), h.data_ptr(), (B * N, N), last.data_ptr())
    a.states = None if states is None else states.data_ptr()
    ws = torch.empty(max(1, sb.snn_scan_workspace(a, False)), dtype=torch.uint8, device="cuda")
    a.workspace, a.workspace_bytes = ws.data_ptr(), ws.numel()
    sb.snn_scan_forward(a, torch.cuda.current_stream().cuda_stream)


# a step, few steps, one segment of the time axis, several, with sequences that end in any of them
@pytest.mark.parametrize("T,B,N,lengths", [(1, 3, 70, None), (9, 3, 70, (9, 0, 4)), (200, 2, 33, (200, 7)), (2000, 1, 16, None),
                                           (5000, 2, 64, (5000, 1)), (5000, 3, 100, (2500, 0, 4990)), (20011, 1, 640, (64,))])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("keep", [False, True])
def test_state_and_last_in_one_buffer(T, B, N, lengths, dtype, keep):
    g = torch.Generator(device="cuda").manual_seed(T)
    x, gate = (torch.randn(T, B, N, generator=g, device="cuda").to(dtype) for _ in range(2))
    state = torch.randn(B, N, generator=g, device="cuda")
    n = None if lengths is None else torch.tensor(lengths, dtype=torch.int32, device="cuda")
    states = torch.zeros(-(-T // 64), B, N, device="cuda") if keep else None
    h, last = torch.empty_like(x), torch.empty_like(state)
    forward(x, gate, state, last, n, h, states)
    want_states = None if states is None else states.clone()
    for _ in range(5):
        both, h2 = state.clone(), torch.empty_like(x)
        if keep:
            states.zero_()
        forward(x, gate, both, both, n, h2, states)
        assert torch.equal(h2, h) and torch.equal(both, last)
        assert states is None or torch.equal(states, want_states)
    # no first state at all is a state of zeros
    none, zero, h3 = torch.empty_like(state), torch.empty_like(state), torch.empty_like(x)
    forward(x, gate, None, none, n, h2, states)
    forward(x, gate, torch.zeros_like(state), zero, n, h3, states)
    assert torch.equal(h2, h3) and torch.equal(none, zero)
