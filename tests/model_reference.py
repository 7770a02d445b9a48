"""The norm, the AdamW step and beam search from their definitions, in 64 bits on the CPU (numpy), with bounds on what 32-bit
arithmetic may be off by.  U is half a unit in the last place of a value in fp32, relative to it: what one rounding costs.
"""
import numpy as np

from seq_reference import GROUP, rounding

U = 2.0 ** -24


# ---- root-mean-square norm --------------------------------------------------------------------------------------
def norm_units(n):
    """Roundings that a sum over a row goes through: 16 terms at most one after the other (two octets), eight steps of
    joining lanes and warps, in rows that are walked through 4 more for every 8192 columns; and as many again as are left for
    the product with 1/n, eps, the reciprocal root (CUDA's bound: 2 units of 2^-23) and the products that follow."""
    return 32 + 4 * (n // 8192)


def norm_forward(h, weight, eps):
    """h float64 [rows][n] (the sum, as it was rounded): dict of float64 arrays and bounds."""
    n = h.shape[1]
    with np.errstate(all="ignore"):
        rstd = 1 / np.sqrt((h * h).sum(1) / n + eps)
        y = h * rstd[:, None] * (1.0 if weight is None else weight)
    k = norm_units(n) * U
    return {"rstd": rstd, "rstd_tol": k * rstd + 2.0 ** -148, "y": y, "y_tol": k * np.abs(y) + 2.0 ** -140}


def norm_backward(h, rstd, weight, dy, dh):
    n, rows = h.shape[1], h.shape[0]
    g = dy * (1.0 if weight is None else weight)
    x = h * rstd[:, None]
    c = (g * x).sum(1, keepdims=True) / n
    size = np.abs(g * x).sum(1, keepdims=True) / n
    dx = rstd[:, None] * (g - x * c)
    k = 2 * norm_units(n) * U
    tol = k * rstd[:, None] * (np.abs(g) + np.abs(x) * size)
    if dh is not None:
        dx = dx + dh
        tol = tol + 2 * U * (np.abs(dx) + np.abs(dh))
    # a column's sum: rows of a block one after the other, blocks joined 8 at a time; no more roundings than rows and 160
    dw, dw_size = (dy * x).sum(0), np.abs(dy * x).sum(0)
    return {"dx": dx, "dx_tol": tol, "dw": dw, "dw_tol": (rows + 160 + norm_units(n)) * U * dw_size}


# ---- AdamW ------------------------------------------------------------------------------------------------------
def mix(x):
    x = np.asarray(x, np.uint64)
    mask = np.uint64(0xFFFFFFFF)
    x = ((x ^ (x >> np.uint64(16))) * np.uint64(0xEE1F5725)) & mask
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0x5DE0A3B7)) & mask
    return x ^ (x >> np.uint64(16))


def random_bits(place, seed, step):
    key = np.uint64(0x2545F491)
    for word in (seed & 0xFFFFFFFF, seed >> 32, step & 0xFFFFFFFF, step >> 32):
        key = mix(key ^ np.uint64(word))
    place = np.asarray(place, np.uint64)
    return mix((place & np.uint64(0xFFFFFFFF)) ^ key ^ mix(place >> np.uint64(32)))


def e4m3(codes, scales):
    """The values of e4m3 codes in groups of 64 (uint8 arrays of one dimension)."""
    codes = codes.astype(np.int64)
    exponent, fraction = codes >> 3 & 15, codes & 7
    value = np.where(exponent == 0, fraction * 2.0 ** -9, (1 + fraction / 8) * 2.0 ** (exponent - 7.0))
    value = np.where(codes & 127 == 127, np.nan, np.where(codes & 128, -value, value))
    scale = np.where(scales == 255, np.nan, 2.0 ** (scales.astype(np.float64) - 127))
    with np.errstate(all="ignore"):
        return value * np.repeat(scale, GROUP)


def encode_at_random(v, r, root, unsure, shift=0.0):
    """(values after rounding, the other candidate where the decision is closer than `unsure` steps (relative to v), else the same);
    shift: the groups' scales are those of tops larger by that, relatively."""
    v = v.reshape(-1, GROUP)
    top = np.abs(v).max(1, keepdims=True) * (1 + shift)
    e = np.full(top.shape, -127.0)
    for k in range(-127, 128):
        e = np.where((e == k) & (top > 448 * 2.0 ** k), k + 1, e)
    a = np.abs(v) / 2.0 ** e
    step = 2.0 ** (np.floor(np.log2(np.maximum(a, 2.0 ** -6))) - 3)
    at = a / step + r.reshape(-1, GROUP) / 65536.0

    def value(q):
        q = np.minimum(q * step, 448.0)
        if root:
            q = np.where((a > 0) & (q == 0), 2.0 ** -9, q)
        return (np.sign(v) * q * 2.0 ** e).reshape(-1)

    low, off = np.floor(at), unsure * (a / step) + 2.0 ** -20
    other = np.where(at - low < off, low - 1, np.where(low + 1 - at < off, low + 1, low))
    return value(low), value(np.maximum(other, 0))


def adamw(p, g, m, v, t, lr, betas, eps, decay):
    """One step in float64, with bounds: each of m, v is two products and a sum with coefficients that are rounded as well."""
    b1, b2 = betas
    with np.errstate(all="ignore"):
        m1, v1 = b1 * m + (1 - b1) * g, b2 * v + (1 - b2) * g * g
        rate, below = lr / (1 - b1 ** t), np.sqrt(v1 / (1 - b2 ** t)) + eps
        new = p * (1 - lr * decay) - rate * m1 / below
        m_size = np.abs(b1 * m) + np.abs((1 - b1) * g)
        # the update: 4 units of m's terms, 4 of its root (half of v's), 8 of the factors and the quotient (CUDA's bound: 2 x 2^-23)
        tol = 4 * U * np.abs(p) + 24 * U * rate * m_size / below
    return {"p": new, "p_tol": tol, "m": m1, "m_tol": 4 * U * m_size + 2.0 ** -148, "v": v1, "v_tol": 6 * U * v1 + 2.0 ** -148}


# ---- beam search ------------------------------------------------------------------------------------------------
def beam(logits, scores, width, ended=None, end=None):
    """(flat continuation k V + c, score) of the best `width` of one sample: logits [K][V], scores [K] in float64."""
    K, V = logits.shape
    out = np.full((K, V), -np.inf)
    for k in range(K):
        if not np.isfinite(scores[k]):
            continue
        if ended is not None and ended[k]:
            out[k, end] = scores[k]
            continue
        z = logits[k]
        if np.isnan(z).any() or np.isposinf(z).any() or np.isneginf(z).all():
            continue
        d = z - z.max()
        out[k] = scores[k] + (d - np.log(np.exp(d).sum()))
    flat = np.argsort(-out.reshape(-1), kind="stable")
    return flat[:width], out.reshape(-1)


def check_beam(got_flat, got_scores, logits, scores, width, ended=None, end=None, where=""):
    """The result's order is that of the definition, but for neighbours whose scores are closer than 1e-6 (sums of 2^22
    exponentials in fp32 and their logarithm are off by less), and its scores are off by no more than that and a rounding."""
    want, all_scores = beam(logits, scores, width, ended, end)
    mine = all_scores[got_flat]
    with np.errstate(invalid="ignore"):
        same = (got_flat == want) | (np.abs(mine - all_scores[want]) <= 1e-6)
    assert len(set(got_flat.tolist())) == width, where
    assert same.all(), f"{where}: {got_flat} instead of {want}"
    # within a beam equal logits go by their class, exactly
    V = logits.shape[1]
    for i in range(width):
        for j in range(i + 1, width):
            a, b = got_flat[i], got_flat[j]
            if a // V == b // V and all_scores[a] == all_scores[b]:
                assert a < b, where
    dead = np.isneginf(mine)
    assert np.array_equal(np.isneginf(got_scores), dead), where
    assert (np.abs(got_scores[~dead] - mine[~dead]) <= 1e-6 + rounding(mine[~dead], "fp32")).all(), where
    assert np.array_equal(got_flat[dead], want[dead]), where
