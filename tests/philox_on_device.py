"""The mask of entwine_dropout on the GPU, in torch's 64-bit integers, for matrices too large for philox_reference.py (with
which a test compares it)."""
import functools

import torch

LOW = 0xFFFFFFFF


def _times(x, c):
    """Halves of the 64-bit product of 32-bit words: it may wrap into the sign, whose bits are masked away."""
    m = x * c
    return (m >> 32) & LOW, m & LOW


@functools.lru_cache(maxsize=4)
def factors(p, seed, offset, row0, rows, cols):
    """What dropout multiplies each element with (64 bits)."""
    seed, offset = seed % (1 << 64), offset % (1 << 64)
    shape = (rows, -(-cols // 8))
    w = [torch.arange(shape[1], device="cuda").expand(shape), torch.arange(row0, row0 + rows, device="cuda")[:, None].expand(shape),
         torch.full(shape, offset & LOW, device="cuda"), torch.full(shape, offset >> 32, device="cuda")]
    a, b = seed & LOW, seed >> 32
    for _ in range(10):
        (mh, ml), (nh, nl) = _times(w[0], 0xD2511F53), _times(w[2], 0xCD9E8D57)
        w = [nh ^ w[1] ^ a, nl, mh ^ w[3] ^ b, ml]
        a, b = (a + 0x9E3779B9) & LOW, (b + 0xBB67AE85) & LOW
    n = torch.stack([h for v in w for h in (v & 0xFFFF, v >> 16)], -1).reshape(rows, -1)[:, :cols]
    t = round(p * 65536)
    return (n >= t).double() * (65536 / (65536 - t))
