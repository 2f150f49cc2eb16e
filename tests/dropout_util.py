"""The dropout's mask by its definition, in whole numbers on the CPU."""
import numpy as np


def philox(counter, key, rounds=10):
    """Philox-4x32 (Salmon et al., 2011) on Python's integers."""
    a, b, c, d = counter
    k0, k1 = key
    for _ in range(rounds):
        u, v = 0xD2511F53 * a, 0xCD9E8D57 * c
        a, b, c, d = v >> 32 ^ b ^ k0, v & 0xffffffff, u >> 32 ^ d ^ k1, u & 0xffffffff
        k0, k1 = (k0 + 0x9E3779B9) & 0xffffffff, (k1 + 0xBB67AE85) & 0xffffffff
    return a, b, c, d


def bits(rows, cols, seed, offset):
    """The 16 bits of every element of the given rows (an iterable of row numbers)."""
    out = []
    offset &= 2 ** 64 - 1
    for r in rows:
        half = []
        for g in range(-(-cols // 8)):
            for w in philox((g, r, offset & 0xffffffff, offset >> 32),
                            (seed & 0xffffffff, seed >> 32)):
                half += [w & 0xffff, w >> 16]
        out.append(half[:cols])
    return np.array(out, dtype=np.int64).reshape(len(out), cols)


def mask(rows, cols, seed, offset, p):
    """(kept, factor) for a probability p."""
    t = round(float(np.float32(p)) * 65536)
    factor = float(np.float32(65536 / (65536 - t))) if t < 65536 else 0.0
    return bits(rows, cols, seed, offset) >= t, factor
