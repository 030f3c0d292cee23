"""Plain 64-bit forms of the operators on 4-bit values, for the tests: numpy."""

import numpy as np

VALUES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def quantize(x):
    """(codes [.., K], scale bytes [.., blocks], values [.., K]) of float64 x, one code per element."""
    x = np.asarray(x, np.float64)
    K = x.shape[-1]
    n = -(-K // 32)
    full = np.zeros(x.shape[:-1] + (n * 32,))
    full[..., :K] = x
    b = full.reshape(x.shape[:-1] + (n, 32))
    bad = ~np.isfinite(b).all(-1)
    big = np.where(bad, 1.0, np.abs(b).max(-1))
    e = np.zeros(big.shape, np.int64)
    for i in np.ndindex(big.shape):
        m = big[i]
        if m > 0:
            p = -126
            while m > 7 * 2.0 ** p and p < 125:
                p += 1
            e[i] = p
    a = np.where(bad[..., None], 0.0, np.abs(b)) * 2.0 ** -e[..., None].astype(np.float64)
    off = np.abs(a[..., None] - VALUES)
    # the nearest; of two as near, the even one comes first
    order = np.array([0, 2, 4, 6, 1, 3, 5, 7])
    code = order[np.argmin(off[..., order], -1)]
    code = np.where(np.signbit(b), code + 8, code)
    v = values(code.reshape(b.shape[:-2] + (-1,)), np.where(bad, 255, e + 127))
    return code.reshape(b.shape[:-2] + (-1,))[..., :K], np.where(bad, 255, e + 127).astype(np.uint8), v[..., :K]


def values(code, scale):
    """float64 values of one code per element (whole blocks) and scale bytes."""
    v = VALUES[code & 7] * np.where(code & 8, -1.0, 1.0)
    s = np.where(scale == 255, np.nan, 2.0 ** (scale.astype(np.float64) - 127))
    return v * np.repeat(s, 32, -1)[..., :v.shape[-1]]


def pack(code):
    """Two codes to a byte."""
    if code.shape[-1] % 2:
        code = np.concatenate([code, np.zeros(code.shape[:-1] + (1,), code.dtype)], -1)
    return (code[..., 0::2] | code[..., 1::2] << 4).astype(np.uint8)


def attend(q, k, v, pos, scale, window):
    """One row and head: q [D], k and v [L, D] float64, tokens up to pos, of these the last `window` (0: all).
    (out, lse, sum p |v - out| / sum p, sum p |v| / sum p, max |q| |k| scale over the tokens)"""
    lo = max(0, pos - window + 1) if window else 0
    if pos < 0:
        z = np.zeros(q.shape)
        return z, -np.inf, z, z, 0.0
    k, v = k[lo:pos + 1], v[lo:pos + 1]
    with np.errstate(invalid="ignore"):
        s = scale * (k @ q)
        m = s.max()
        p = np.exp(s - m)
        out = (p @ v) / p.sum()
        return (out, m + np.log(p.sum()), p @ np.abs(v - out) / p.sum(), p @ np.abs(v) / p.sum(),
                scale * (np.abs(k) @ np.abs(q)).max())
