"""Cases and plain forms of the sequence-model operators in `paper_2412_11810_b200.ops`.

Three operators that a recurrent sequence model trains and answers with, next to the spiking training step:

  scan  the gated linear recurrence h_t = a_t h_{t-1} + (1 - a_t) x_t with a_t = sigmoid(gate_t), or
        h_t = gate_t h_{t-1} + x_t ("direct"), over [T][B][N]: forward, one token, and forward with backward, where the
        inputs kept for the backward pass are held raw or in 8 bits beside one fp32 state every 64 steps
  pack  activations to 8 bits (groups of 64 values of a row share a power-of-two scale) and back
  loss  mean soft-max cross entropy of scale * x w_out over a large vocabulary, without keeping the logits: forward, and
        forward with the gradients of x and w_out

`own` selects who computes: False the plain form (elementary torch operations in 32 bits), True the CUDA library.
`exact` is the definition in 64 bits, written apart from the plain form.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
CHUNK = 64     # steps between kept states
GROUP = 64     # values that share a scale
IGNORE = -100  # target of a row that does not count

# bounds of the drawn cases: no more work than the largest listed case of the kind
MOST_SCAN = 65536 * 2048
MOST_PACK = 16384 * 4096
MOST_LOSS = 8192 * 2048 * 131072


def listed():
    return [
        # one new token for each of 64 sequences in flight: the state update of a serving loop
        {"name": "scan_token", "op": "scan", "dtype": "bf16", "T": 1, "B": 64, "N": 1024, "mode": "sigmoid", "ragged": False, "train": False, "keep": "raw"},
        # evaluation of a small batch in the library's own type, padded sequences of different lengths
        {"name": "scan_eval_ragged", "op": "scan", "dtype": "fp32", "T": 1000, "B": 8, "N": 1030, "mode": "sigmoid", "ragged": True, "train": False, "keep": "raw"},
        # a prompt of one long document: few channels, a long time axis
        {"name": "scan_prompt_long", "op": "scan", "dtype": "bf16", "T": 65536, "B": 1, "N": 1024, "mode": "sigmoid", "ragged": False, "train": False, "keep": "raw"},
        # training with decays that the caller computes, odd sizes, raw inputs kept
        {"name": "scan_train_direct", "op": "scan", "dtype": "fp16", "T": 777, "B": 5, "N": 1001, "mode": "direct", "ragged": True, "train": True, "keep": "raw"},
        # training of an ordinary batch, kept inputs in 8 bits
        {"name": "scan_train_int8", "op": "scan", "dtype": "bf16", "T": 2048, "B": 16, "N": 2048, "mode": "sigmoid", "ragged": False, "train": True, "keep": "int8"},
        # training on one very long sequence, kept inputs in 8 bits: what checkpoints are for
        {"name": "scan_train_long_e4m3", "op": "scan", "dtype": "bf16", "T": 65536, "B": 1, "N": 2048, "mode": "sigmoid", "ragged": False, "train": True, "keep": "e4m3"},
        # the activations of a short odd batch
        {"name": "pack_small", "op": "pack", "dtype": "fp32", "rows": 33, "N": 1001, "format": "int8"},
        # the activations of one layer of a large batch
        {"name": "pack_large", "op": "pack", "dtype": "bf16", "rows": 16384, "N": 4096, "format": "e4m3"},
        # scoring the last position of one sequence
        {"name": "loss_one_row", "op": "loss", "dtype": "bf16", "rows": 1, "D": 1024, "V": 32000, "tied": True, "train": False},
        # the library's own readout: fp32, features by row, few hundred samples
        {"name": "loss_train_fp32", "op": "loss", "dtype": "fp32", "rows": 500, "D": 1000, "V": 5003, "tied": False, "train": True},
        # one training micro-batch, an odd vocabulary
        {"name": "loss_train_mid", "op": "loss", "dtype": "bf16", "rows": 4096, "D": 1024, "V": 50257, "tied": True, "train": True},
        # the largest: a long training batch over a large vocabulary
        {"name": "loss_train_large", "op": "loss", "dtype": "bf16", "rows": 8192, "D": 2048, "V": 131072, "tied": True, "train": True},
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    kind = rng.choice(["scan", "scan", "pack", "loss", "loss"])
    dtype = rng.choice(["fp32", "bf16", "fp16"])
    if kind == "scan":
        train = rng.random() < 0.6
        mode = rng.choice(["sigmoid", "sigmoid", "direct"])
        while True:
            T, B, N = _log_int(rng, 1, 65536), _log_int(rng, 1, 64), _log_int(rng, 1, 4096)
            if T * B * N * SIZE[dtype] <= 2 * MOST_SCAN:
                break
        return {"op": "scan", "dtype": dtype, "T": T, "B": B, "N": N, "mode": mode, "ragged": rng.random() < 0.5, "train": train,
                "keep": rng.choice(["raw", "int8", "e4m3"])}
    if kind == "pack":
        while True:
            rows, N = _log_int(rng, 1, 65536), _log_int(rng, 1, 8192)
            if rows * N * SIZE[dtype] <= 2 * MOST_PACK:
                break
        return {"op": "pack", "dtype": dtype, "rows": rows, "N": N, "format": rng.choice(["int8", "e4m3"])}
    while True:
        rows, D, V = _log_int(rng, 1, 8192), _log_int(rng, 8, 2048), _log_int(rng, 2, 131072)
        if rows * D * V * (6 if dtype == "fp32" else 1) <= MOST_LOSS:
            break
    return {"op": "loss", "dtype": dtype, "rows": rows, "D": D, "V": V, "tied": rng.random() < 0.5, "train": rng.random() < 0.6}


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    dt = DTYPES[case["dtype"]]

    def normal(*shape, mean=0.0, std=1.0, dtype=dt):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(mean, std, generator=g).to(dtype)

    s = {"case": case}
    if case["op"] == "scan":
        T, B, N = case["T"], case["B"], case["N"]
        s["x"] = normal(T, B, N)
        # a gate of mean 2 holds on to a state for about ten steps; decays given directly lie in (0, 1)
        s["gate"] = normal(T, B, N, mean=2.0, std=1.5)
        if case["mode"] == "direct":
            s["gate"] = torch.sigmoid(s["gate"].float()).to(dt)
        s["state"] = normal(B, N, dtype=torch.float32)
        s["lengths"] = None
        if case["ragged"]:
            s["lengths"] = torch.randint(0, T + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
            s["lengths"][0] = T
        if case["train"]:
            s["dh"] = normal(T, B, N, std=0.1)
            s["dlast"] = normal(B, N, std=0.1, dtype=torch.float32)
    elif case["op"] == "pack":
        # activations: every 50th feature is an outlier
        s["x"] = normal(case["rows"], case["N"])
        s["x"][:, ::50] *= 20
    else:
        n, D, V = case["rows"], case["D"], case["V"]
        s["x"] = normal(n, D)
        # logits of a trained model spread over a few units; a tied table is stored with one row per class
        w = normal(V, D, std=2.0 / math.sqrt(D)) if case["tied"] else normal(D, V, std=2.0 / math.sqrt(D))
        s["w"] = w.t() if case["tied"] else w
        s["targets"] = torch.randint(0, V, (n,), generator=g, device="cuda", dtype=torch.int64)
        if n > 4:   # padding rows
            s["targets"][torch.rand(n, generator=g, device="cuda") < 0.05] = IGNORE
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------

def _quantised(v, fmt):
    """The values that fp32 `v` [..., N] has in 8 bits: groups of 64 along the last axis, a power of two as scale."""
    n = v.shape[-1]
    u = torch.nn.functional.pad(v, (0, -n % GROUP)).unflatten(-1, (-1, GROUP))
    m, k = torch.frexp(u.abs().amax(-1, keepdim=True))
    if fmt == "int8":      # the smallest scale at which the largest value is below 128; codes end at 127
        e = k - 7
    else:                  # ... is no more than 448, the largest e4m3 value
        e = k - 9 + (m > 0.875)
    e = e.clamp(min=-127)
    q = torch.ldexp(u, -e)
    q = torch.round(q).clamp(-127, 127) if fmt == "int8" else q.to(torch.float8_e4m3fn).float()
    q = torch.ldexp(q, e)
    return q.flatten(-2)[..., :n]


def _scanned(a, b):
    """(A, H) with A_t = a_t .. a_1 and H_t = a_t H_{t-1} + b_t, by doubling the distance."""
    a, h, d = a.clone(), b.clone(), 1
    while d < a.shape[0]:
        h[d:] = h[d:] + a[d:] * h[:-d]
        a[d:] = a[d:] * a[:-d]
        d *= 2
    return a, h


def _coefficients(x, gate, mode):
    """a, the factor of x, and their derivatives by the gate's share: a' and whether x is scaled."""
    if mode == "direct":
        return gate, torch.ones_like(gate)
    return torch.sigmoid(gate), torch.sigmoid(-gate)


def _plain_scan(s):
    c = s["case"]
    T, B, N = s["x"].shape
    dt = s["x"].dtype
    x, gate, h0 = s["x"].float(), s["gate"].float(), s["state"]
    on = None
    if s["lengths"] is not None:
        on = (torch.arange(T, device=x.device)[:, None] < s["lengths"][None, :])[:, :, None]

    def masked(a, b):   # steps behind a sequence's end hand the state on
        return (a, b) if on is None else (torch.where(on, a, 1.0), torch.where(on, b, 0.0))

    a, i = _coefficients(x, gate, c["mode"])
    a, b = masked(a, i * x)
    A, H = _scanned(a, b)
    h = H + A * h0
    last = h[-1].clone()
    shown = h if on is None else torch.where(on, h, 0.0)
    if not c["train"]:
        return shown.to(dt), last
    # the backward pass on what was kept: the inputs, raw or in 8 bits, and the state before every 64th step
    if c["keep"] != "raw":
        x = _quantised(x, c["keep"])
        if c["mode"] == "sigmoid":
            gate = _quantised(gate, c["keep"])
        a, i = _coefficients(x, gate, c["mode"])
        a, b = masked(a, i * x)
        kept = torch.cat([h0[None], h[CHUNK - 1:-1:CHUNK]])
        n, pad = kept.shape[0], -T % CHUNK
        ca = torch.nn.functional.pad(a, (0, 0, 0, 0, 0, pad)).reshape(n, CHUNK, B, N).transpose(0, 1)
        cb = torch.nn.functional.pad(b, (0, 0, 0, 0, 0, pad)).reshape(n, CHUNK, B, N).transpose(0, 1)
        A, H = _scanned(ca, cb)
        h = (H + A * kept[None]).transpose(0, 1).reshape(n * CHUNK, B, N)[:T]
        before = torch.cat([h0[None], h[:-1]])
        before[::CHUNK] = kept
    else:
        before = torch.cat([h0[None], h[:-1]])
    dh = s["dh"].float()
    if on is not None:
        dh = torch.where(on, dh, 0.0)
    dh[-1] += s["dlast"]
    # D_t = dh_t + a_{t+1} D_{t+1}, from the last step to the first
    back = torch.cat([torch.ones_like(a[:1]), a[1:].flip(0)])
    D = _scanned(back, dh.flip(0))[1].flip(0)
    dstate = a[0] * D[0]
    if c["mode"] == "direct":
        dx, dgate = D, D * before
    else:
        dx, dgate = D * i, D * (before - x) * a * i
    if on is not None:
        dx, dgate = torch.where(on, dx, 0.0), torch.where(on, dgate, 0.0)
    return shown.to(dt), last, dx.to(dt), dgate.to(dt), dstate


def _plain_loss(s):
    x, w = s["x"].float(), s["w"].float()
    on = s["targets"] != IGNORE
    count = on.sum().clamp(min=1)
    x = torch.where(on[:, None], x, 0.0)
    z = x @ w
    m = z.amax(1, keepdim=True)
    lse = (torch.exp(z - m).sum(1, keepdim=True).log() + m).squeeze(1)
    at = torch.where(on, s["targets"], 0)[:, None]
    row = torch.where(on, lse - z.gather(1, at).squeeze(1), 0.0)
    loss = (row.double().sum() / count).float()
    shown = torch.where(on, lse, 0.0)
    if not s["case"]["train"]:
        return loss, row, shown
    z = torch.exp(z - lse[:, None])
    z.scatter_add_(1, at, torch.full_like(at, -1.0, dtype=torch.float32))
    z *= (on.float() / count)[:, None]
    dx, dw = z @ w.t(), x.t() @ z
    return loss, row, shown, dx.to(s["x"].dtype), dw.to(s["w"].dtype)


# ---- the library's operators -------------------------------------------------------------------------------

def _own(s):
    from paper_2412_11810_b200 import ops
    c = s["case"]
    if c["op"] == "scan":
        if not c["train"]:
            if c["T"] == 1 and s["lengths"] is None:
                h, last = ops.gated_scan_step(s["x"][0], s["gate"][0], s["state"], mode=c["mode"])
                return h[None], last
            h, last, _ = ops.gated_scan(s["x"], s["gate"], s["state"], lengths=s["lengths"], mode=c["mode"])
            return h, last
        h, last, kept = ops.gated_scan(s["x"], s["gate"], s["state"], lengths=s["lengths"], mode=c["mode"], keep=c["keep"])
        return (h, last, *ops.gated_scan_backward(kept, s["dh"], s["dlast"]))
    if c["op"] == "pack":
        return ops.unpack_activation(ops.pack_activation(s["x"], c["format"]))
    loss, row, lse = ops.vocab_loss(s["x"], s["w"], s["targets"], ignore_index=IGNORE)
    if not c["train"]:
        return loss, row, lse
    return (loss, row, lse, *ops.vocab_loss_backward(s["x"], s["w"], s["targets"], lse, ignore_index=IGNORE))


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    if op == "scan":
        return _plain_scan(state)
    if op == "pack":
        return _quantised(state["x"].float(), state["case"]["format"]).to(state["x"].dtype)
    return _plain_loss(state)


def work(case):
    e = SIZE[case["dtype"]]
    if case["op"] == "scan":
        n, states = case["T"] * case["B"] * case["N"], 4 * case["B"] * case["N"]
        if case["train"]:   # x, gate, dh in; h, dx, dgate out; state, dlast in; last, dstate out
            return {"bytes": 6 * n * e + 4 * states, "flops": 25 * n}
        return {"bytes": 3 * n * e + 2 * states, "flops": 8 * n}
    if case["op"] == "pack":   # to 8 bits and back: the values in, the bytes out; the bytes in, the values out
        n = case["rows"] * case["N"]
        scales = case["rows"] * -(-case["N"] // GROUP)
        return {"bytes": 2 * n * e + 2 * n + 2 * scales, "flops": 6 * n}
    n, D, V = case["rows"], case["D"], case["V"]
    operands, rows = (n * D + D * V) * e, n * 12 + 4
    if case["train"]:
        return {"bytes": 2 * operands + rows, "flops": 6 * n * D * V}
    return {"bytes": operands + rows, "flops": 2 * n * D * V}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------

def _exact_eight_bits(v, fmt):
    """The 8-bit values of the rows of `v` (float64), group by group from the definition."""
    n = v.shape[-1]
    out = torch.empty_like(v)
    for c0 in range(0, n, GROUP):
        u = v[..., c0:c0 + GROUP]
        top = u.abs().amax(-1, keepdim=True)
        # exponent e of the scale: the smallest with top / 2^e below 128 (int8) or up to 448 (e4m3)
        e = torch.floor(torch.log2(top.clamp(min=2.0 ** -140))) - (8 if fmt == "e4m3" else 6)
        e = e.clamp(min=-127) - 1
        over = (lambda t: t > 448) if fmt == "e4m3" else (lambda t: t >= 128)
        for _ in range(3):
            e = torch.where(over(top / torch.exp2(e)), e + 1, e)
        e = e.clamp(min=-127)
        q = u / torch.exp2(e)
        if fmt == "int8":
            q = torch.round(q).clamp(-127, 127)
        else:   # three fraction bits, normal exponents down to -6
            step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
            q = torch.round(q / step) * step
        out[..., c0:c0 + GROUP] = q * torch.exp2(e)
    return out


def _exact_scan(s):
    c = s["case"]
    T, B, N = s["x"].shape
    x, gate, h0 = s["x"].double(), s["gate"].double(), s["state"].double()
    lengths = s["lengths"] if s["lengths"] is not None else torch.full((B,), T, device=x.device)
    dead = torch.arange(T, device=x.device)[:, None] >= lengths[None, :]

    def parts(x, gate):
        a = gate.clone() if c["mode"] == "direct" else 1 / (1 + torch.exp(-gate))
        i = torch.ones_like(gate) if c["mode"] == "direct" else 1 / (1 + torch.exp(gate))
        b = i * x
        a[dead], b[dead] = 1.0, 0.0
        return a, i, b

    a, i, b = parts(x, gate)
    h = torch.empty(T + 1, B, N, dtype=torch.float64, device=x.device)
    h[0] = h0
    for t in range(T):
        torch.addcmul(b[t], a[t], h[t], out=h[t + 1])
    shown = h[1:].clone()
    shown[dead] = 0.0
    if not c["train"]:
        return shown, h[T].clone()
    last, before = h[T].clone(), h[:T]
    if c["keep"] != "raw":
        x = _exact_eight_bits(x, c["keep"])
        if c["mode"] == "sigmoid":
            gate = _exact_eight_bits(gate, c["keep"])
        a, i, b = parts(x, gate)
        before = h[:T].clone()
        for j in range(1, CHUNK):   # the j-th step behind every kept state at once
            at = torch.arange(j, T, CHUNK, device=x.device)
            before[at] = a[at - 1] * before[at - 1] + b[at - 1]
    dh = s["dh"].double()
    dh[dead] = 0.0
    D = torch.empty_like(dh)
    carry = s["dlast"].double()
    for t in range(T - 1, -1, -1):
        torch.add(dh[t], carry, out=D[t])
        carry = a[t] * D[t]
    if c["mode"] == "direct":
        dx, dgate = D.clone(), D * before
    else:
        dx, dgate = D * i, D * (before - x) * a * i
    dx[dead], dgate[dead] = 0.0, 0.0
    return shown, last, dx, dgate, carry


def _exact_loss(s):
    n, D = s["x"].shape
    w = s["w"].double()
    on = s["targets"] != IGNORE
    count = max(1, int(on.sum()))
    row = torch.zeros(n, dtype=torch.float64, device=w.device)
    lse = torch.zeros_like(row)
    dx = torch.zeros(n, D, dtype=torch.float64, device=w.device)
    dw = torch.zeros_like(w) if s["case"]["train"] else None
    for r in range(0, n, 1024):   # rows at a time, those that count
        rows = torch.nonzero(on[r:r + 1024]).squeeze(1) + r
        if rows.numel() == 0:
            continue
        x, y = s["x"][rows].double(), s["targets"][rows]
        z = x @ w
        lse[rows] = torch.logsumexp(z, dim=1)
        logp = torch.log_softmax(z, dim=1)
        row[rows] = -logp[torch.arange(rows.numel(), device=w.device), y]
        if dw is not None:
            p = torch.exp(logp)
            p[torch.arange(rows.numel(), device=w.device), y] -= 1
            dx[rows] = p @ w.t() / count
            dw += x.t() @ p / count
    loss = row.sum() / count
    return (loss, row, lse) if dw is None else (loss, row, lse, dx, dw)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "scan":
        return _exact_scan(s)
    if case["op"] == "pack":
        return _exact_eight_bits(s["x"].double(), case["format"])
    return _exact_loss(s)
