"""What the tests of the norm, dropout and 8-bit integers compare with: the generator on the host, and bounds of roundings."""
import numpy as np


def philox(c0, c1, c2, c3, k0, k1):
    """Four 32-bit words of Philox4x32-10; counters and keys broadcast as uint64."""
    low, w = np.uint64(0xFFFFFFFF), np.uint64(32)
    c = [np.asarray(x, dtype=np.uint64) for x in (c0, c1, c2, c3)]
    k0, k1 = int(k0), int(k1)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> w) ^ c[1] ^ np.uint64(k0), b & low, (a >> w) ^ c[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return c


def numbers(rows, cols, seed, offset, call=0):
    """The 32-bit numbers of a matrix [rows, cols] as uint64."""
    o = (offset + call) % 2 ** 64
    quad = np.arange(-(-cols // 4), dtype=np.uint64)[None, :].repeat(rows, 0)
    row = np.arange(rows, dtype=np.uint64)[:, None].repeat(quad.shape[1], 1)
    words = philox(quad, row, np.full_like(row, o & 0xFFFFFFFF), np.full_like(row, o >> 32), seed & 0xFFFFFFFF, seed >> 32 & 0xFFFFFFFF)
    return np.stack(words, axis=2).reshape(rows, -1)[:, :cols]


def keep(rows, cols, p, seed, offset, call=0):
    return numbers(rows, cols, seed, offset, call) >= np.uint64(int(np.floor(p * 2.0 ** 32)))
