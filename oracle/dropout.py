"""Dropout's definition in numpy: Philox4x32-10 (Salmon, Moraes, Dror and Shaw,
"Parallel random numbers: as easy as 1, 2, 3", 2011) in 64-bit integers, the
mask of rows [m][c], and the output in float64."""
import numpy as np

LOW = np.uint64(0xFFFFFFFF)


def philox4x32(counter, key):
    """counter: four arrays (or numbers) below 2^32; key: two numbers below 2^32.  Four uint64 arrays below 2^32."""
    x = [np.asarray(v, dtype=np.uint64) for v in counter]
    k = [int(v) for v in key]
    for _ in range(10):
        a, b = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(b >> np.uint64(32)) ^ x[1] ^ np.uint64(k[0]), b & LOW, (a >> np.uint64(32)) ^ x[3] ^ np.uint64(k[1]), a & LOW]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return x


def limit(p):
    return int(np.floor(p * 65536.0 + 0.5))


def bits(m, c, seed, site=0, step=0):
    """The 16 bits of every element, [m][c]."""
    blocks = -(-c // 8)
    col, row = np.meshgrid(np.arange(blocks), np.arange(m))
    words = philox4x32((col, row, np.full_like(col, site), np.full_like(col, step)), (seed & 0xFFFFFFFF, seed >> 32))
    out = np.empty((m, blocks, 8), dtype=np.int64)
    for j, w in enumerate(words):
        w = np.broadcast_to(w, col.shape).astype(np.int64)
        out[:, :, 2 * j], out[:, :, 2 * j + 1] = w & 0xFFFF, w >> 16
    return out.reshape(m, blocks * 8)[:, :c]


def dropout(x, p, seed, site=0, step=0, add=None):
    """x, add: float64 [m][c]."""
    t = limit(p)
    keep = bits(*x.shape, seed, site, step) >= t
    y = np.where(keep, x * (65536.0 / (65536 - t) if t < 65536 else 0.0), 0.0)
    return y if add is None else y + add
