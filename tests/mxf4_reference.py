"""The 4-bit format on the host, from its definition: what the tests of the quantiser and the products compare with."""
import numpy as np

LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])


def decode(q, scale, cols):
    """Values, in 64 bits, of codes q [M, >= cols/2] and scale bytes [M, >= cols/32] (NaN where a byte is 255)."""
    n = np.empty(q.shape[:-1] + (2 * q.shape[-1],), np.uint8)
    n[..., 0::2], n[..., 1::2] = q & 15, q >> 4
    n = n[..., :cols]
    v = np.where(n & 8, -1.0, 1.0) * LEVELS[n & 7]
    s = np.repeat(scale.astype(np.int64), 32, axis=-1)[..., :cols]
    return np.where(s == 255, np.nan, v * np.ldexp(1.0, s - 127))


def encode(x):
    """Codes and scale bytes of the rows of x (64 bits): the nearest level, of two the one with the even code."""
    rows, cols = x.shape
    q, scale = np.zeros((rows, (cols + 1) // 2), np.uint8), np.zeros((rows, (cols + 31) // 32), np.uint8)
    for b in range(scale.shape[1]):
        v = x[:, 32 * b:32 * b + 32]
        amax = np.abs(v).max(axis=1)
        fine = np.isfinite(amax)
        e = np.where(fine & (amax > 0), np.frexp(np.where(fine, amax, 1.0))[1] - 1 - 2, -127)
        e = np.clip(e, -127, 127)
        scale[:, b] = np.where(fine, e + 127, 255)
        a = np.where(fine[:, None], np.abs(v), 0.0) * np.ldexp(1.0, -e)[:, None]
        gap = np.abs(a[:, :, None] - LEVELS)
        # even codes first among equals
        order = np.array([0, 2, 4, 6, 1, 3, 5, 7])
        code = order[np.argmin(gap[:, :, order], axis=2)]
        code = code + 8 * (np.signbit(v) & fine[:, None])
        for i in range(v.shape[1]):
            k = 32 * b + i
            q[:, k // 2] |= (code[:, i] << (4 * (k % 2))).astype(np.uint8)
    return q, scale
