"""What dropout drops, in numpy: Philox4x32-10 with 64-bit products."""
import numpy as np


def philox(counter, key):
    """(4, n) words of a counter and (2,) of a key, or numbers that go with them"""
    c = [np.asarray(v, np.uint64) for v in counter]
    k = [int(v) for v in key]
    low, half = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [b >> half ^ c[1] ^ np.uint64(k[0]), b & low, a >> half ^ c[3] ^ np.uint64(k[1]), a & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def kept(rows, cols, p, seed, offset, first=0):
    """(rows, cols) of truth values, and what the kept are multiplied by; rows from `first` on"""
    seed, offset = seed & (1 << 64) - 1, offset & (1 << 64) - 1
    groups = (cols + 7) // 8
    row, group = np.meshgrid(np.arange(first, first + rows, dtype=np.uint64), np.arange(groups, dtype=np.uint64), indexing="ij")
    zero = np.zeros_like(row)
    words = philox([group, row, zero + np.uint64(offset & 0xFFFFFFFF), zero + np.uint64(offset >> 32)], [seed & 0xFFFFFFFF, seed >> 32])
    bits = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], 2).reshape(rows, groups * 8)[:, :cols]
    T = round(p * 65536)
    return bits >= T, 65536 / (65536 - T) if T < 65536 else 0.0
