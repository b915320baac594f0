"""Philox4x32 with ten rounds on the host, and the mask that entwine_dropout makes of it."""
import numpy as np


def philox(counter, key):
    """counter: four uint64 arrays of 32-bit words; key: two numbers."""
    c, (a, b) = [np.asarray(x, np.uint64) for x in counter], key
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        m, n = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(n >> half) ^ c[1] ^ np.uint64(a), n & low, (m >> half) ^ c[3] ^ np.uint64(b), m & low]
        a, b = (a + 0x9E3779B9) & 0xFFFFFFFF, (b + 0xBB67AE85) & 0xFFFFFFFF
    return c


def numbers(seed, offset, row0, rows, cols):
    """The 16-bit numbers of a matrix's elements."""
    seed, offset = seed % (1 << 64), offset % (1 << 64)
    group, row = np.meshgrid(np.arange(-(-cols // 8), dtype=np.uint64), np.arange(row0, row0 + rows, dtype=np.uint64))
    c = philox([group, row, np.full(group.shape, offset & 0xFFFFFFFF, np.uint64), np.full(group.shape, offset >> 32, np.uint64)],
               (seed & 0xFFFFFFFF, seed >> 32))
    n = np.stack([x for w in c for x in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=-1)
    return n.reshape(rows, -1)[:, :cols].astype(np.int64)


def factors(p, seed, offset, row0, rows, cols):
    """What dropout multiplies each element with (64 bits)."""
    t = int(np.rint(p * 65536))
    return np.where(numbers(seed, offset, row0, rows, cols) >= t, 65536 / (65536 - t), 0.0)
