"""Plain references in 64 bits for the operators in few bits (microscaled 4-bit products, the 8-bit cache and its attention,
sampling), written from their definitions.  Host only."""
import math

import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
HALF_STEP = 2.0 ** -11                 # of a half, relative: a rounding is off by at most this
HALF_TINY = 2.0 ** -25                 # half of the smallest half


# ---------------------------------------------------------------- microscaled 4-bit floating point

def mx4_quantize(x):
    """x [M, K] halves -> codes [M, K] (0 .. 15), scale bytes [M, K / 32]."""
    x = np.asarray(x, dtype=np.float16)
    b = x.astype(np.float64).reshape(x.shape[0], -1, 32)
    top = np.abs(b).max(-1)
    bad = ~np.isfinite(b).all(-1)
    e = np.zeros(top.shape, dtype=np.int64)
    ok = (top > 0) & ~bad
    e[ok] = np.floor(np.log2(top[ok])).astype(np.int64) - 2
    y = np.abs(np.where(bad[..., None], 0.0, b)) / np.exp2(e.astype(np.float64))[..., None]
    far = np.abs(y[..., None] - LEVELS)
    near = far.min(-1, keepdims=True)
    is_near = far == near
    # of two equally near ones the even code; above 6 the last
    code = np.where(is_near[..., 0::2].any(-1), 2 * is_near[..., 0::2].argmax(-1), 2 * is_near[..., 1::2].argmax(-1) + 1)
    code = np.where(y >= 6.0, 7, code)
    code = np.where(np.signbit(b) & ~bad[..., None], code + 8, code)
    code = np.where(bad[..., None], 0, code)
    return code.reshape(x.shape).astype(np.uint8), np.where(bad, 255, e + 127).astype(np.uint8)


def pack4(code):
    return (code[:, 0::2] | (code[:, 1::2] << 4)).astype(np.uint8)


def unpack4(q):
    return np.stack([q & 15, q >> 4], -1).reshape(q.shape[0], -1)


def mx4_values(code, scale):
    v = np.where(code >= 8, -LEVELS[code & 7], LEVELS[code & 7]).reshape(code.shape[0], -1, 32)
    s = np.where(scale == 255, np.nan, np.exp2(scale.astype(np.float64) - 127.0))
    return (v * s[..., None]).reshape(code.shape)


# ---------------------------------------------------------------- the 8-bit cache and attention over it

BLOCK = 64


def turn(x, pos, base=10000.0):
    """x [rows, heads, d] halves at positions pos [rows]: half-split rotation in binary64, rounded to binary32 and that to half."""
    d = x.shape[-1]
    a = np.asarray(pos, dtype=np.float64)[:, None, None] * base ** (-2.0 * np.arange(d // 2) / d)
    lo, hi = x[..., :d // 2].astype(np.float64), x[..., d // 2:].astype(np.float64)
    return np.concatenate([lo * np.cos(a) - hi * np.sin(a), hi * np.cos(a) + lo * np.sin(a)], -1).astype(np.float32).astype(np.float16)


def block_codes(x):
    """x [64, d] halves -> codes, scale (binary32)."""
    top = np.abs(x.astype(np.float64)).max() if np.isfinite(x).all() else np.nan
    if not np.isfinite(top):
        return np.zeros(x.shape), np.float32(np.nan)
    scale = np.float32(top) / np.float32(127.0)
    return (np.rint(127.0 * x.astype(np.float64) / top) if top > 0 else np.zeros(x.shape)), scale


def held(x):
    """x [n, d] halves of one head, as the cache holds them: values in binary64 (a NaN scale makes a block NaN)."""
    out = x.astype(np.float64)
    for j in range(x.shape[0] // BLOCK):
        codes, scale = block_codes(x[j * BLOCK:(j + 1) * BLOCK])
        out[j * BLOCK:(j + 1) * BLOCK] = codes * np.float64(scale)
    return out


def attend(q, k, v, sees):
    """q [rows, d], k, v [n, d] values, row i sees positions 0 .. sees[i]: outputs, sum of p |v|, and how far the scores may be off in
    binary32 (d products and a few operations, each rounded or truncated), relative to a probability."""
    s = q @ k.T / math.sqrt(q.shape[1])
    hidden = np.arange(k.shape[0])[None] > np.asarray(sees)[:, None]
    s = np.where(hidden, -np.inf, s)
    p = np.exp(s - s.max(-1, keepdims=True))
    p = np.where(hidden, 0.0, p)
    p = p / p.sum(-1, keepdims=True)
    vv = np.where(np.isfinite(v), v, 0.0)
    o = p @ vv
    for i in range(q.shape[0]):                                    # infinities and NaN only where they are seen
        seen = v[:sees[i] + 1]
        odd = ~np.isfinite(seen)
        if odd.any():
            with np.errstate(invalid="ignore"):
                o[i] = o[i] + np.where(odd, seen, 0.0).sum(0)
    size = (np.abs(q) @ np.where(np.isfinite(k), np.abs(k), 0.0).T / math.sqrt(q.shape[1])).max(-1, keepdims=True)
    return o, p @ np.abs(vv), (q.shape[1] + 16) * 2.0 ** -23 * size


def attention_bound(o, mass, score_off, n, v_top, single_half):
    """Largest difference of a half output from `o`.  A probability is off by the scores' error, a few roundings of binary32 and, where it
    enters as one half, half a step of it; numerator and denominator count.  A probability below the normal halves is off by
    up to 2^-25 of the largest one; the output is rounded once."""
    rel = 2.0 * (score_off + (n / 32 + 16) * 2.0 ** -23) + (HALF_STEP if single_half else 2.0 ** -21)
    return HALF_STEP * np.abs(o) * (1 + rel) + HALF_TINY + rel * mass + n * 2.0 ** -25 * v_top


# ---------------------------------------------------------------- sampling

def sample(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, u=0.0):
    """One row of halves -> token, probability, and how near a decision came to its border (relative to the mass it is about)."""
    x = logits.astype(np.float64)
    can = ~np.isnan(x) & (x > -np.inf)
    if not can.any():
        return -1, 0.0, 1.0
    order = np.flatnonzero(can)
    order = order[np.argsort(-x[order], kind="stable")]
    top = x[order[0]]
    if not temperature > 0:
        return int(order[0]), 1.0, 1.0
    w = np.zeros(x.shape)
    w[can] = np.where(x[can] == top, 1.0, 0.0) if np.isinf(top) else np.exp((x[can] - top) / temperature)
    near = 1.0
    if top_k > 0:
        order = order[:top_k]
    if not top_p >= 1.0:
        mass = w[order]
        before = np.cumsum(mass) - mass
        share = (top_p if top_p > 0 else 0.0) * mass.sum()
        near = min(near, (np.abs(before[1:] - share) / mass.sum()).min(initial=1.0)) if top_p > 0 else near
        order = order[:max(1, int((before < share).sum()))]
    if min_p > 0:
        least = min(min_p, 1.0)
        near = min(near, np.abs(w[order[1:]] - least).min(initial=1.0)) if least < 1.0 else near
        order = order[(w[order] >= least)]
    index = np.sort(order)
    cum = np.cumsum(w[index])
    u = min(max(u, 0.0), np.nextafter(1.0, 0.0)) if u == u else 0.0
    hit = int((cum <= u * cum[-1]).sum())
    near = min(near, (np.abs(cum[:-1] - u * cum[-1]) / cum[-1]).min(initial=1.0)) if u > 0 else near
    if (w[w > 0] == 1.0).all():
        near = 1.0                                                 # whole masses: both sides add them exactly
    return int(index[hit]), float(w[index[hit]] / cum[-1]), float(near)
