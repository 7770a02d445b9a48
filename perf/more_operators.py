"""Cases and plain forms of the operators in `paper_2412_11810_b200.ops` that stand around the recurrence and the loss.

What a recurrent sequence model needs between its layers, at the end of a training step and when it answers:

  norm   h = x + residual, y = h / sqrt(mean(h^2) + eps) * weight, y in the inputs' type, in 8 bits, or both; with "train"
         also the gradients by x (which is that by the residual) and by the weight
  adamw  one AdamW step over all tensors of a model, moments in 32 bits, or in 8 bits (groups of 64 e4m3 codes under a
         power-of-two scale, the second moment as its root, rounded up or down at random by a hash of seed, step and place)
  beam   beam search: the best `width` continuations of all beams of a sample by score + log soft-max, ties to the lowest
         index, ended beams carried along, and the beams' recurrent states put into the new order

`own` selects who computes: False the plain form (elementary torch operations in 32 bits), True the CUDA library.
`exact` is the definition in 64 bits, written apart from the plain form.
"""
import math

import torch

own = False

DTYPES = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
GROUP = 64          # values that share a scale
EPS_NORM = 1e-6
LR, BETAS, EPS, DECAY = 2e-5, (0.9, 0.999), 1e-8, 0.01
END = 2             # token that ends a beam

# bounds of the drawn cases: no more work than the largest listed case of the kind
MOST_NORM = 32768 * 2048 * 2
MOST_ADAMW = 340_000_000
MOST_BEAM = 64 * 8 * 131072 * 4


def listed():
    return [
        # one new token for each of 64 sequences in flight
        {"name": "norm_token", "op": "norm", "dtype": "bf16", "rows": 64, "N": 1024, "residual": True, "keep": "none", "values": True, "train": False},
        # a prompt's activations for a product in 8 bits: no 16-bit copy is written
        {"name": "norm_prompt_int8", "op": "norm", "dtype": "bf16", "rows": 16384, "N": 4096, "residual": True, "keep": "int8", "values": False, "train": False},
        # training in the library's own type, odd sizes, the output kept in 8 bits beside the values
        {"name": "norm_train_odd", "op": "norm", "dtype": "fp32", "rows": 999, "N": 1030, "residual": False, "keep": "e4m3", "values": True, "train": True},
        # training of a large batch: 32 sequences of 1024 steps
        {"name": "norm_train_large", "op": "norm", "dtype": "bf16", "rows": 32768, "N": 2048, "residual": True, "keep": "none", "values": True, "train": True},
        # a small spiking network's three matrices, gradients clipped to a norm
        {"name": "adamw_small", "op": "adamw", "net": "64,128,10", "layers": 0, "N": 0, "V": 0, "dtype": "fp32", "grads": "fp32", "bits": 32, "clip": True, "copies": "none"},
        # a sequence model of 50 tensors in 16 bits with moments in 8
        {"name": "adamw_model_8bit", "op": "adamw", "net": "", "layers": 12, "N": 1024, "V": 32000, "dtype": "bf16", "grads": "bf16", "bits": 8, "clip": False, "copies": "none"},
        # fp32 parameters with the 16-bit copies that the products read, odd widths, gradients clipped
        {"name": "adamw_copies_odd", "op": "adamw", "net": "", "layers": 5, "N": 1001, "V": 50257, "dtype": "fp32", "grads": "bf16", "bits": 8, "clip": True, "copies": "bf16"},
        # the largest: the seven matrices of a network of 3 x 8192 neurons
        {"name": "adamw_large", "op": "adamw", "net": "1024,8192,8192,8192,100", "layers": 0, "N": 0, "V": 0, "dtype": "fp32", "grads": "fp32", "bits": 32, "clip": False, "copies": "none"},
        # one sequence in flight, four beams
        {"name": "beam_one", "op": "beam", "dtype": "bf16", "B": 1, "K": 4, "W": 4, "V": 32000, "ended": False, "states": 2, "N": 1024},
        # the first step behind the prompts of a batch: one beam becomes eight
        {"name": "beam_first", "op": "beam", "dtype": "fp16", "B": 64, "K": 1, "W": 8, "V": 50257, "ended": False, "states": 2, "N": 1001},
        # odd numbers of samples, beams and classes; some beams have ended
        {"name": "beam_odd", "op": "beam", "dtype": "fp32", "B": 7, "K": 5, "W": 5, "V": 5003, "ended": True, "states": 1, "N": 1030},
        # the largest batch and vocabulary
        {"name": "beam_large", "op": "beam", "dtype": "fp32", "B": 64, "K": 8, "W": 8, "V": 131072, "ended": True, "states": 4, "N": 2048},
    ]


def _log_int(rng, low, high):
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    kind = rng.choice(["norm", "adamw", "beam"])
    dtype = rng.choice(["fp32", "bf16", "fp16"])
    if kind == "norm":
        while True:
            rows, N = _log_int(rng, 1, 65536), _log_int(rng, 16, 16384)
            if rows * N * SIZE[dtype] <= MOST_NORM:
                break
        keep = rng.choice(["none", "int8", "e4m3"])
        return {"op": "norm", "dtype": dtype, "rows": rows, "N": N, "residual": rng.random() < 0.7, "keep": keep,
                "values": keep == "none" or rng.random() < 0.5, "train": rng.random() < 0.5}
    if kind == "adamw":
        bits, clip = rng.choice([8, 32]), rng.random() < 0.5
        if rng.random() < 0.4:
            sizes = [_log_int(rng, 10, 4096) for _ in range(rng.randint(3, 5))]
            return {"op": "adamw", "net": ",".join(str(n) for n in sizes), "layers": 0, "N": 0, "V": 0, "dtype": "fp32", "grads": "fp32", "bits": bits,
                    "clip": clip, "copies": "none"}
        while True:
            layers, N, V = rng.randint(1, 6), _log_int(rng, 16, 4096), _log_int(rng, 16, 65536)
            if sum(r * c for r, c in _model(layers, N, V)) <= MOST_ADAMW // 3:
                break
        grads = rng.choice([dtype, "fp32"])
        copies = rng.choice(["none", "bf16", "fp16"]) if dtype == "fp32" else "none"
        return {"op": "adamw", "net": "", "layers": layers, "N": N, "V": V, "dtype": dtype, "grads": grads, "bits": bits, "clip": clip, "copies": copies}
    while True:
        B, K, V = _log_int(rng, 1, 128), rng.randint(1, 16), _log_int(rng, 16, 200000)
        if B * K * V * SIZE[dtype] <= MOST_BEAM:
            break
    return {"op": "beam", "dtype": dtype, "B": B, "K": K, "W": K if K > 1 else rng.randint(1, 16), "V": V, "ended": rng.random() < 0.5,
            "states": rng.randint(1, 4), "N": _log_int(rng, 1, 2048)}


def _model(layers, N, V):
    """Rows and columns of a sequence model's tensors: a table, and per layer a norm's weight and three matrices."""
    return [(V, N), (1, N)] + [(1, N), (N, N), (N, N), (N, N)] * layers


def _shapes(case):
    if not case["net"]:
        return _model(case["layers"], case["N"], case["V"])
    n = [int(v) for v in case["net"].split(",")]
    hidden = n[1:-1]
    return [*zip(n[:-2], hidden), *((h, h) for h in hidden), (n[-2], n[-1])]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)

    def normal(*shape, std=1.0, dtype=torch.float32):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, std, generator=g).to(dtype)

    s = {"case": case}
    if case["op"] == "norm":
        dt, rows, N = DTYPES[case["dtype"]], case["rows"], case["N"]
        # activations: every 50th feature is an outlier; a residual stream grows over the layers
        s["x"] = normal(rows, N, dtype=dt)
        s["x"][:, ::50] *= 20
        s["residual"] = normal(rows, N, std=3.0, dtype=dt) if case["residual"] else None
        s["weight"] = (1 + normal(N, std=0.2)).to(dt)
        if case["train"]:
            s["dy"] = normal(rows, N, std=0.01, dtype=dt)
            s["dh"] = normal(rows, N, std=0.01, dtype=dt) if case["residual"] else None
    elif case["op"] == "adamw":
        shapes = _shapes(case)
        s["params"] = [normal(r, c, std=1 / math.sqrt(max(r, 16)), dtype=DTYPES[case["dtype"]]) for r, c in shapes]
        # gradients of different magnitudes from tensor to tensor; rows that nothing touched have none
        size = [10 ** (-2 - k % 3) for k in range(len(shapes))]
        s["grads"] = [normal(r, c, std=e, dtype=DTYPES[case["grads"]]) for (r, c), e in zip(shapes, size)]
        for t in s["grads"]:
            t[::7][1:] = 0
        # moments of such gradients, each tensor's from a multiple of 64 on
        first = _flat([normal(r, c, std=0.3 * e) for (r, c), e in zip(shapes, size)])
        second = _flat([(normal(r, c, std=0.2).exp_() * e) ** 2 for (r, c), e in zip(shapes, size)])
        if case["bits"] == 8:
            s["m"], s["v"] = _nearest_codes(first), _nearest_codes(second.sqrt_())
        else:
            s["m"], s["v"] = first, second
        s["step"] = torch.tensor(100 + seed % 900, dtype=torch.int64, device="cuda")
        s["copies"] = None if case["copies"] == "none" else [p.to(DTYPES[case["copies"]]) for p in s["params"]]
        s["max_norm"] = 0.1 if case["clip"] else None
        s["seed"] = seed
    else:
        B, K, V = case["B"], case["K"], case["V"]
        s["logits"] = normal(B, K, V, std=2.5, dtype=DTYPES[case["dtype"]])
        if V > 100:
            s["logits"][:, :, 7::97] = float("-inf")    # classes that are never an answer
        s["scores"] = -5 * torch.rand(B, K, generator=g, device="cuda")
        s["ended"] = (torch.rand(B, K, generator=g, device="cuda") < 0.2) if case["ended"] else None
        s["states"] = [normal(B * K, case["N"]) for _ in range(case["states"])]
    return s


# ---- the plain forms ---------------------------------------------------------------------------------------

def _flat(tensors):
    """All values in fp32 one behind the other, each tensor from a multiple of 64 on."""
    return torch.cat([torch.nn.functional.pad(t.reshape(-1).float(), (0, -t.numel() % GROUP)) for t in tensors])


def _unflat(flat, tensors):
    sizes = [t.numel() + -t.numel() % GROUP for t in tensors]
    return [f[:t.numel()].view_as(t) for f, t in zip(flat.split(sizes), tensors)]


def _exponent(top, most):
    """The exponent of the smallest power of two, not below 2^-127, at which `top` is no more than 448 (below 128)."""
    m, k = torch.frexp(top)
    return (k - 9 + (m > 0.875) if most == 448 else k - 7).clamp(min=-127)


def _quantised(v, fmt):
    """The values that fp32 `v` [..., N] has in 8 bits, rounded to nearest."""
    n = v.shape[-1]
    u = torch.nn.functional.pad(v, (0, -n % GROUP)).unflatten(-1, (-1, GROUP))
    e = _exponent(u.abs().amax(-1, keepdim=True), 128 if fmt == "int8" else 448)
    q = torch.ldexp(u, -e)
    q = torch.round(q).clamp(-127, 127) if fmt == "int8" else q.to(torch.float8_e4m3fn).float()
    return torch.ldexp(q, e).flatten(-2)[..., :n]


def _nearest_codes(flat):
    u = flat.view(-1, GROUP)
    e = _exponent(u.abs().amax(-1, keepdim=True), 448)
    return torch.ldexp(u, -e).to(torch.float8_e4m3fn).view(torch.uint8).flatten(), (e + 127).to(torch.uint8).flatten()


def _values_of(codes, scales):
    return torch.ldexp(codes.view(torch.float8_e4m3fn).float().view(-1, GROUP), scales.int()[:, None] - 127).flatten()


def _mix(x):
    """A hash of 32 bits (whole numbers in int64): multiplications by odd numbers between shifts."""
    x = ((x ^ (x >> 16)) * 0xEE1F5725) & 0xFFFFFFFF
    x = ((x ^ (x >> 15)) * 0x5DE0A3B7) & 0xFFFFFFFF
    return x ^ (x >> 16)


def _random_bits(n, seed, step):
    key = torch.full_like(step, 0x2545F491)
    for word in (seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF, step & 0xFFFFFFFF, step >> 32):
        key = _mix(key ^ word)
    j = torch.arange(n, device=step.device)
    return _mix((j & 0xFFFFFFFF) ^ key ^ _mix(j >> 32))


def _random_codes(v, r, root):
    """(codes, scales) of fp32 `v` with magnitudes rounded up where the fraction of a step and r / 2^16 reach one; in 64 bits,
    since a value lies near a border now and then.  A root above zero stays above zero."""
    u = v.double().view(-1, GROUP)
    e = _exponent(v.view(-1, GROUP).abs().amax(-1, keepdim=True), 448)
    u = torch.ldexp(u, -e)
    a = u.abs()
    step = torch.ldexp(torch.ones_like(a), (torch.frexp(a)[1] - 1).clamp(min=-6) - 3)
    q = ((a / step + r.view(-1, GROUP) / 65536.0).floor() * step).clamp(max=448)
    if root:
        q = torch.where(a > 0, q.clamp(min=2.0 ** -9), q)
    return torch.copysign(q, u).float().to(torch.float8_e4m3fn).view(torch.uint8).flatten(), (e + 127).to(torch.uint8).flatten()


def _plain_norm(s):
    c = s["case"]
    dt = s["x"].dtype
    h = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(dt)
    f, w = h.float(), s["weight"].float()
    rstd = torch.rsqrt((f * f).mean(-1) + EPS_NORM)
    n = f * rstd[:, None]
    y = n * w
    out = [h, rstd]
    if c["values"]:
        out.append(y.to(dt))
    if c["keep"] != "none":
        out.append(_quantised(y, c["keep"]).to(torch.bfloat16))
    if not c["train"]:
        return out
    dy = s["dy"].float()
    g = dy * w
    dx = rstd[:, None] * (g - n * (g * n).mean(-1, keepdim=True))
    if s["dh"] is not None:
        dx = dx + s["dh"].float()
    return [*out, dx.to(dt), (dy * n).sum(0).to(dt)]


def _plain_adamw(s):
    c = s["case"]
    p, g = _flat(s["params"]), _flat(s["grads"])
    norm = None
    if s["max_norm"] is not None:
        norm = g.square().sum(dtype=torch.float64).sqrt()
        g = g * torch.where(norm > s["max_norm"], s["max_norm"] / norm, 1.0).float()
        norm = norm.float()
    s["step"] += 1
    t = s["step"].double()
    first, second = (1 - BETAS[0] ** t).float(), (1 - BETAS[1] ** t).float()
    if c["bits"] == 8:
        m, v = _values_of(*s["m"]), _values_of(*s["v"]).square_()
    else:
        m, v = s["m"], s["v"]
    m = m.mul_(BETAS[0]).add_(g * (1 - BETAS[0]))
    v = v.mul_(BETAS[1]).add_(g.square_().mul_(1 - BETAS[1]))
    del g
    root = v.sqrt()
    p = p.mul_(1 - LR * DECAY).sub_(LR / first * m / (root / second.sqrt() + EPS))
    new = _unflat(p, s["params"])
    torch._foreach_copy_(s["params"], new)
    if s["copies"] is not None:
        torch._foreach_copy_(s["copies"], new)
    if c["bits"] == 32:
        return s["params"], s["m"], s["v"], s["step"], norm, s["copies"]
    r = _random_bits(p.numel(), s["seed"], s["step"])
    s["m"], s["v"] = _random_codes(m, r & 0xFFFF, False), _random_codes(root, r >> 16, True)
    return s["params"], _values_of(*s["m"]).bfloat16(), _values_of(*s["v"]).bfloat16(), s["step"], norm, s["copies"]


def _plain_beam(s):
    c = s["case"]
    B, K, V, W = c["B"], c["K"], c["V"], c["W"]
    z = s["logits"].float()
    # the best of each beam by (logit, lower class): whole numbers that order as the pair does
    b = z.view(torch.int32).long()
    key = (torch.where(b < 0, -2147483648 - b, b) << 32) + (0x7FFFFFFF - torch.arange(V, device=z.device))
    kept = min(W, V)
    token = 0x7FFFFFFF - (key.topk(kept, -1).values & 0xFFFFFFFF)
    del b, key
    z = z.double()
    m = z.amax(-1, keepdim=True)
    total = torch.exp(z - m).sum(-1, keepdim=True).log()
    score = s["scores"].double()[:, :, None] + (z.gather(-1, token) - m - total)
    if s["ended"] is not None:
        # an ended beam goes on with the end token alone; the others of its candidates are at -infinity
        first = torch.arange(kept, device=z.device)
        mine = torch.where(first == 0, END, torch.where(first <= END, first - 1, first))
        token = torch.where(s["ended"][:, :, None], mine, token)
        score = torch.where(s["ended"][:, :, None], torch.where(mine == END, s["scores"].double()[:, :, None], -math.inf), score)
    flat, order = (token + V * torch.arange(K, device=z.device)[:, None]).view(B, -1).sort(-1)
    score = score.view(B, -1).gather(1, order)
    score, order = score.sort(dim=-1, descending=True, stable=True)
    flat, score = flat.gather(1, order[:, :W]), score[:, :W].float()
    parent, token = flat // V, flat % V
    ended = token == END
    if s["ended"] is not None:
        ended = ended | s["ended"].gather(1, parent)
    rows = (parent + K * torch.arange(B, device=z.device)[:, None]).view(-1)
    return token, parent, score, ended, [t[rows] for t in s["states"]]


# ---- the library's operators -------------------------------------------------------------------------------

def _own(s):
    from paper_2412_11810_b200 import ops
    c = s["case"]
    if c["op"] == "norm":
        keep = None if c["keep"] == "none" else c["keep"]
        y, h, rstd, kept = ops.rms_norm(s["x"], s["weight"], s["residual"], eps=EPS_NORM, keep=keep, values=c["values"])
        out = [h, rstd]
        if c["values"]:
            out.append(y)
        if keep is not None:
            out.append(ops.unpack_activation(kept, torch.bfloat16))
        if not c["train"]:
            return out
        return [*out, *ops.rms_norm_backward(h, rstd, s["dy"], s["weight"], s["dh"])]
    if c["op"] == "adamw":
        m, v = s["m"], s["v"]
        if c["bits"] == 8:
            m, v = (ops.PackedActivation(*t, "e4m3", torch.float32) for t in (m, v))
        state = ops.AdamWState(m, v, s["step"])
        norm = ops.adamw_step(s["params"], s["grads"], state, lr=LR, betas=BETAS, eps=EPS, weight_decay=DECAY, max_norm=s["max_norm"], seed=s["seed"],
                              copies=s["copies"])
        if c["bits"] == 8:
            m, v = ops.unpack_activation(m, torch.bfloat16), ops.unpack_activation(v, torch.bfloat16)
        return s["params"], m, v, s["step"], norm, s["copies"]
    return ops.beam_step(s["logits"], s["scores"], width=c["W"], ended=s["ended"], end=END, states=s["states"])


def run(state):
    if own:
        return _own(state)
    op = state["case"]["op"]
    return _plain_norm(state) if op == "norm" else _plain_adamw(state) if op == "adamw" else _plain_beam(state)


def work(case):
    if case["op"] == "norm":
        n, e = case["rows"] * case["N"], SIZE[case["dtype"]]
        rows = 4 * case["rows"] + e * case["N"]
        values = 2 if case["residual"] else 1              # x and residual in
        values += 1 if case["residual"] else 0             # h out, where it is not x itself
        values += 1 if case["values"] else 0               # y out
        codes = 1 + 1 / GROUP if case["keep"] != "none" else 0
        flops = 8 * n
        if case["train"]:                                  # dy (and dh) in, dx out; h and rstd are at hand
            values += 3 if case["residual"] else 2
            flops += 16 * n
        return {"bytes": n * (values * e + codes) + rows, "flops": flops}
    if case["op"] == "adamw":
        n = sum(r * c for r, c in _shapes(case))
        moments = 16 if case["bits"] == 32 else 4 * (1 + 1 / GROUP)
        copies = 0 if case["copies"] == "none" else SIZE[case["copies"]]
        return {"bytes": n * (2 * SIZE[case["dtype"]] + SIZE[case["grads"]] + moments + copies), "flops": 15 * n}
    B, K, W = case["B"], case["K"], case["W"]
    logits = B * K * case["V"]
    return {"bytes": logits * SIZE[case["dtype"]] + B * case["states"] * case["N"] * 4 * (K + W) + B * (5 * K + 21 * W), "flops": 5 * logits}


# ---- the definitions in 64 bits ----------------------------------------------------------------------------

def _exact_eight_bits(v, fmt):
    out = torch.empty_like(v)
    for c0 in range(0, v.shape[-1], GROUP):
        u = v[..., c0:c0 + GROUP]
        e = _exact_scale(u.abs().amax(-1, keepdim=True), fmt)
        q = u / torch.exp2(e)
        if fmt == "int8":
            q = torch.round(q).clamp(-127, 127)
        else:   # three fraction bits, normal exponents down to -6
            step = torch.exp2(torch.floor(torch.log2(q.abs().clamp(min=2.0 ** -6))) - 3)
            q = torch.round(q / step) * step
        out[..., c0:c0 + GROUP] = q * torch.exp2(e)
    return out


def _exact_scale(top, fmt):
    """The smallest exponent e, at least -127, with top / 2^e below 128 (int8) or up to 448 (e4m3)."""
    e = torch.floor(torch.log2(top.clamp(min=2.0 ** -140))) - (8 if fmt == "e4m3" else 6)
    e = e.clamp(min=-127) - 1
    over = (lambda t: t > 448) if fmt == "e4m3" else (lambda t: t >= 128)
    for _ in range(3):
        e = torch.where(over(top / torch.exp2(e)), e + 1, e)
    return e.clamp(min=-127)


def _exact_norm(s):
    c = s["case"]
    h = s["x"].double()
    if s["residual"] is not None:   # what is kept and normed is the sum in the inputs' type
        h = (h + s["residual"].double()).to(s["x"].dtype).double()
    w = s["weight"].double()
    N = h.shape[1]
    rstd = (h.square().sum(1) / N + EPS_NORM) ** -0.5
    y = w * (h * rstd[:, None])
    out = [h, rstd]
    if c["values"]:
        out.append(y)
    if c["keep"] != "none":
        out.append(_exact_eight_bits(y, c["keep"]))
    if not c["train"]:
        return out
    # the Jacobian of h / r with r^2 = mean(h^2) + eps: (dy w) / r - h (dy w . h) / (N r^3)
    g = s["dy"].double() * w
    dx = g * rstd[:, None] - h * ((g * h).sum(1) / N * rstd ** 3)[:, None]
    if s["dh"] is not None:
        dx += s["dh"].double()
    dw = torch.einsum("rn,rn,r->n", s["dy"].double(), h, rstd)
    return [*out, dx, dw]


def _exact_bits(first, count, seed, step):
    """The random bits of `count` places from `first` on, by whole-number arithmetic."""
    def mix(x):
        x = (x ^ x >> 16) * 0xEE1F5725 % 2 ** 32
        x = (x ^ x >> 15) * 0x5DE0A3B7 % 2 ** 32
        return x ^ x >> 16
    key = 0x2545F491
    for word in (seed % 2 ** 32, seed >> 32, step % 2 ** 32, step >> 32):
        key = mix(key ^ word)
    x = torch.arange(first, first + count, device="cuda") ^ key    # (fewer than 2^32 places)
    x = torch.remainder((x ^ x >> 16) * 0xEE1F5725, 2 ** 32)
    x = torch.remainder((x ^ x >> 15) * 0x5DE0A3B7, 2 ** 32)
    return x ^ x >> 16


def _exact_adamw(s):
    c = s["case"]
    norm, factor = None, 1.0
    if s["max_norm"] is not None:
        norm = math.sqrt(sum(float((t.double() ** 2).sum()) for t in s["grads"]))
        factor = min(1.0, s["max_norm"] / norm)
    t = int(s["step"]) + 1
    params, ms, vs, at = [], [], [], 0

    def eight_bits(v, r, root):
        v = torch.nn.functional.pad(v, (0, -v.numel() % GROUP)).view(-1, GROUP)
        e = _exact_scale(v.abs().amax(1, keepdim=True), "e4m3")
        a = v.abs() / torch.exp2(e)
        step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3)
        low = torch.floor(a / step)
        q = torch.where(a / step - low >= 1 - r.view(-1, GROUP) / 65536, low + 1, low) * step
        q = torch.minimum(q, torch.full_like(q, 448.0))
        if root:
            q = torch.where((a > 0) & (q == 0), torch.full_like(q, 2.0 ** -9), q)
        return (torch.sign(v) * q * torch.exp2(e)).view(-1)

    for p, g in zip(s["params"], s["grads"]):
        n = p.numel()
        room = -(-n // GROUP) * GROUP
        if c["bits"] == 8:
            m, r = ((codes[at:at + n].view(torch.float8_e4m3fn).double() * torch.exp2(scales[at // GROUP:(at + room) // GROUP].double() - 127)
                     .repeat_interleave(GROUP)[:n]) for codes, scales in (s["m"], s["v"]))
            v = r ** 2
        else:
            m, v = s["m"][at:at + n].double(), s["v"][at:at + n].double()
        g = g.reshape(-1).double() * factor
        m = BETAS[0] * m + (1 - BETAS[0]) * g
        v = BETAS[1] * v + (1 - BETAS[1]) * g ** 2
        mh, vh = m / (1 - BETAS[0] ** t), v / (1 - BETAS[1] ** t)
        x = p.reshape(-1).double()
        params.append((x - LR * DECAY * x - LR * mh / (vh ** 0.5 + EPS)).view_as(p))
        if c["bits"] == 8:
            r = _exact_bits(at, room, s["seed"], t)
            m, v = eight_bits(m, r % 65536, False), eight_bits(v ** 0.5, r // 65536, True)
        else:
            m, v = (torch.nn.functional.pad(u, (0, room - n)) for u in (m, v))
        ms.append(m)
        vs.append(v)
        at += room
    return params, torch.cat(ms), torch.cat(vs), None, norm, None if s["copies"] is None else params


def _exact_beam(s):
    c = s["case"]
    B, K, V, W = c["B"], c["K"], c["V"], c["W"]
    out = []
    for b in range(B):
        x = torch.log_softmax(s["logits"][b].double(), -1) + s["scores"][b].double()[:, None]
        if s["ended"] is not None:
            for k in torch.nonzero(s["ended"][b]).flatten().tolist():
                x[k] = -math.inf
                x[k, END] = s["scores"][b, k].double()
        out.append(torch.sort(x.view(-1), descending=True, stable=True))
        out[-1] = (out[-1].values[:W], out[-1].indices[:W])
    score, flat = torch.stack([o[0] for o in out]), torch.stack([o[1] for o in out])
    states = [torch.stack([t.view(B, K, -1)[b][flat[b] // V] for b in range(B)]).view(B * W, -1).double() for t in s["states"]]
    return None, None, score, None, states


def exact(case, seed):
    s = prepare(case, seed)
    return _exact_norm(s) if case["op"] == "norm" else _exact_adamw(s) if case["op"] == "adamw" else _exact_beam(s)
