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
