"""The sequence-model operators from their definitions, in 64 bits on the CPU (numpy), with bounds on what 32-bit
arithmetic may be off by.

Bounds are carried by recursions of their own.  For h_t = a_t h_{t-1} + i_t x_t let M_t = |a_t| M_{t-1} + |i_t x_t| be the
sum of the magnitudes of all terms of h_t.  If a step's coefficients and its arithmetic are off by a relative DELTA at
most, h_t is off by E_t with E_t = |a_t| E_{t-1} + DELTA M_t at most (to first order).

DELTA: exp(-|g|) by CUDA's __expf is off by 2 + 1.173 |g| units of 2^-23 (its documented bound), 1 / (1 + e) by 2 + 0.5
units more, one product and one sum add half a unit each; a step is composed with its neighbours once per step and about
24 times more per chunk of 64 steps.  With |g| <= 16 that is below 2 + 19 + 2.5 + 1 + 0.5 (1 + 24 / 64) < 26 units; DELTA
takes 32 units.
"""
import numpy as np

DELTA = 32 * 2.0 ** -23
CHUNK, GROUP = 64, 64
HALF_STEP = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}   # a rounding, relative to the value
TINY = {"fp32": 2.0 ** -150, "bf16": 2.0 ** -134, "fp16": 2.0 ** -25}     # a rounding of a subnormal value


def rounding(v, dtype):
    return HALF_STEP[dtype] * np.abs(v) + TINY[dtype]


# ---- 8-bit values ---------------------------------------------------------------------------------------------
LARGEST = {"fp32": float(np.finfo(np.float32).max), "bf16": 2.0 ** 127 * (2 - 2.0 ** -7), "fp16": 65504.0}


def eight_bits(v, fmt, dtype="fp32"):
    """(values, codes' scale bytes) of float array v [..., N] of a type in the 8-bit format."""
    v = np.asarray(v, np.float64)
    n = v.shape[-1]
    groups = -(-n // GROUP)
    out = np.empty_like(v)
    scales = np.zeros((*v.shape[:-1], groups), np.uint8)
    for j in range(groups):
        u = v[..., j * GROUP:(j + 1) * GROUP]
        bad = ~np.isfinite(u).all(-1)
        u = np.where(bad[..., None], 0.0, u)
        top = np.abs(u).max(-1)
        e = np.full(top.shape, -127)
        for k in range(-127, 128):   # the smallest exponent that fits
            fits = (top / 2.0 ** k < 128) if fmt == "int8" else (top / 2.0 ** k <= 448)
            e = np.where((e == k) & ~fits, k + 1, e)
        q = u / 2.0 ** e[..., None].astype(np.float64)
        if fmt == "e4m3":
            step = 2.0 ** (np.floor(np.log2(np.maximum(np.abs(q), 2.0 ** -6))) - 3)
            q = np.rint(q / step) * step
        else:
            q = np.clip(np.rint(q), -127, 127)
        out[..., j * GROUP:(j + 1) * GROUP] = np.where(bad[..., None], np.nan, q * 2.0 ** e[..., None].astype(np.float64))
        out[..., j * GROUP:(j + 1) * GROUP] = np.clip(out[..., j * GROUP:(j + 1) * GROUP], -LARGEST[dtype], LARGEST[dtype])
        scales[..., j] = np.where(bad, 255, e + 127)
    return out, scales


# ---- gated linear recurrence ----------------------------------------------------------------------------------
def coefficients(gate, mode):
    if mode == "direct":
        return gate.copy(), np.ones_like(gate)
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-gate)), 1 / (1 + np.exp(gate))


def _on(T, B, lengths):
    if lengths is None:
        return np.ones((T, B, 1), bool)
    return (np.arange(T)[:, None] < np.clip(lengths, 0, T)[None, :])[:, :, None]


def scan_forward(x, gate, state, lengths, mode):
    """h, last and the bounds of both; also everything the backward pass needs."""
    T, B, N = x.shape
    on = _on(T, B, lengths)
    x, gate = np.where(on, x, 0.0), np.where(on, gate, 0.0)
    a, i = coefficients(gate, mode)
    a, i = np.where(on, a, 1.0), np.where(on, i, 0.0)
    h = np.zeros((T + 1, B, N)); M = np.zeros_like(h); E = np.zeros_like(h)
    h[0] = 0.0 if state is None else state
    M[0] = np.abs(h[0])
    for t in range(T):
        h[t + 1] = a[t] * h[t] + i[t] * x[t]
        M[t + 1] = np.abs(a[t]) * M[t] + np.abs(i[t] * x[t])
        E[t + 1] = np.abs(a[t]) * E[t] + np.where(on[t], DELTA * M[t + 1], 0.0)
    return {"h": np.where(on, h[1:], 0.0), "h_tol": np.where(on, E[1:], 0.0), "last": h[T], "last_tol": E[T],
            "states": h[0:T:CHUNK], "all": h, "M": M, "E": E, "a": a, "i": i, "x": x, "on": on}


def scan_backward(x, gate, state, lengths, mode, dh, dlast, keep=None, keep_gate=None):
    """dx, dgate, dstate and their bounds.  keep / keep_gate: the inputs were kept in 8 bits."""
    T, B, N = x.shape
    f = scan_forward(x, gate, state, lengths, mode)
    on, xs, a, i = f["on"], f["x"], f["a"], f["i"]
    before, Mb, Eb = f["all"][:T].copy(), f["M"][:T].copy(), f["E"][:T].copy()
    if keep or keep_gate:
        xs = np.where(on, eight_bits(np.where(on, x, 0.0), keep)[0], 0.0) if keep else xs
        g = np.where(on, eight_bits(np.where(on, gate, 0.0), keep_gate)[0], 0.0) if keep_gate else np.where(on, gate, 0.0)
        a, i = coefficients(g, mode)
        a, i = np.where(on, a, 1.0), np.where(on, i, 0.0)
        for t in range(1, T):
            if t % CHUNK:   # recomputed from the chunk's kept state
                before[t] = a[t - 1] * before[t - 1] + i[t - 1] * xs[t - 1]
                Mb[t] = np.abs(a[t - 1]) * Mb[t - 1] + np.abs(i[t - 1] * xs[t - 1])
                Eb[t] = np.abs(a[t - 1]) * Eb[t - 1] + DELTA * Mb[t]
    dh = np.where(on, dh, 0.0)
    D = np.zeros((T, B, N)); MD = np.zeros_like(D); ED = np.zeros_like(D)
    e = np.zeros((B, N)) if dlast is None else np.asarray(dlast, np.float64)
    me, ee = np.abs(e), np.zeros((B, N))
    for t in range(T - 1, -1, -1):
        D[t], MD[t] = dh[t] + e, np.abs(dh[t]) + me
        ED[t] = ee + np.where(on[t], DELTA * MD[t], 0.0)
        e, me, ee = a[t] * D[t], np.abs(a[t]) * MD[t], np.abs(a[t]) * ED[t] + np.where(on[t], DELTA * np.abs(a[t]) * MD[t], 0.0)
    if mode == "direct":
        dx, dx_tol = D, ED
        dg, dg_tol = D * before, ED * Mb + MD * (Eb + DELTA * Mb)
    else:
        s = np.abs(a * i)
        dx, dx_tol = D * i, np.abs(i) * (ED + DELTA * MD)
        dg = D * (before - xs) * a * i
        dg_tol = s * (ED * (Mb + np.abs(xs)) + MD * (Eb + 3 * DELTA * (Mb + np.abs(xs))))
    z = lambda v: np.where(on, v, 0.0)  # noqa: E731
    return {"dx": z(dx), "dx_tol": z(dx_tol), "dgate": z(dg), "dgate_tol": z(dg_tol), "dstate": e, "dstate_tol": ee,
            "states": f["states"], "states_tol": f["E"][0:T:CHUNK]}


# ---- vocabulary loss (torch, float64, on the tensors' device) ----------------------------------------------------
def vocab_loss(x, w, targets, scale, ignore, dtype, dloss=1.0):
    """loss, row_loss, lse, dx, dw and their bounds, for float64 x [n][D], w [D][V].

    Bounds.  A tensor-core instruction adds 16 products to a fp32 accumulator; it cuts or rounds, and two units of 2^-23 of
    the sum of magnitudes cover it.  fp32 operands, in two fp16 parts, take three instructions where 16-bit ones take one;
    each operand is off by 2^-22 of its value (2^-11 of what the first part, off by 2^-11, leaves) and the product left out
    is below 2^-22: six units of 2^-23 in all.  So a sum of K products is off by (2 ceil(K / 16) P + 4) 2^-23 of the sum of
    magnitudes, P = 1, or (2 ceil(K / 16) P + 10) 2^-23, P = 3.  exp2 is off by 2^-22, its argument by a rounding of
    2^-24 of each of its two parts, and what is below 2^-126, the smallest normal number, counts as zero; a row's sum of exponentials has 32 + 8 + V / 2048 + 8 roundings.  dz is rounded to its
    type (fp32: two fp16 parts, 2^-22) before it is multiplied.
    """
    import torch
    P, more = (3, 10) if dtype == "fp32" else (1, 4)
    unit, half = 2.0 ** -23, 2.0 ** -22 if dtype == "fp32" else HALF_STEP[dtype]

    def steps(K):
        return (2 * -(-K // 16) * P + more) * unit

    n, D = x.shape
    V = w.shape[1]
    valid = (targets >= 0) & (targets < V) & (targets != ignore)
    bad = ~valid & (targets != ignore)
    on = valid[:, None]
    x = torch.where(on, x, 0.0)
    count = max(1, int(valid.sum()))
    z = scale * (x @ w)
    ez = steps(D) * abs(scale) * (x.abs() @ w.abs())
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    # the error of lse: that of the logits weighted by p, and of the sum
    lse_tol = (p * ez).sum(1) + (60 + V / 2048) * unit + 4 * unit * lse.abs() + 2 * unit * z.abs().amax(1)
    at = torch.where(valid, targets, 0).long()[:, None]
    zt, ezt = z.gather(1, at).squeeze(1), ez.gather(1, at).squeeze(1)
    row = lse - zt
    row_tol = lse_tol + ezt + 4 * unit * (zt.abs() + row.abs())
    zero = torch.zeros_like(lse)
    out = {"row": torch.where(valid, row, zero), "row_tol": torch.where(valid, row_tol, zero),
           "lse": torch.where(valid, lse, zero), "lse_tol": torch.where(valid, lse_tol, zero)}
    out["row"] = torch.where(bad, torch.full_like(row, float("nan")), out["row"])
    out["loss"], out["loss_tol"] = out["row"].sum() / count, out["row_tol"].sum() / count + unit * out["row"].abs().sum() / count
    dz = p.clone()
    dz.scatter_add_(1, at, torch.full_like(at, -1.0, dtype=dz.dtype))
    ep = p * (ez + lse_tol[:, None] + 4 * unit * (1 + z.abs() + lse.abs()[:, None]))
    ep.scatter_add_(1, at, torch.full_like(at, unit, dtype=dz.dtype))
    ep = ep + 2.0 ** -126 + half * dz.abs() + (0.0 if dtype == "bf16" else 2.0 ** -25 / 16384)
    dz, ep = torch.where(on, dz, 0.0), torch.where(on, ep, 0.0)
    k = abs(scale * dloss) / count
    out["dx"] = scale * dloss / count * (dz @ w.t())
    out["dx_tol"] = k * ((ep + (steps(V) + 8 * unit) * dz.abs()) @ w.abs().t())
    out["dw"] = scale * dloss / count * (x.t() @ dz)
    out["dw_tol"] = k * (x.abs().t() @ (ep + (steps(n) + 8 * unit) * dz.abs()))
    return out
