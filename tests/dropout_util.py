"""Philox4x32-10 in numpy's 64-bit words, and the mask that dapple_dropout_norm makes of it."""
import numpy as np

LOW = np.uint64(0xFFFFFFFF)


def philox(counter, key):
    """counter: four arrays of 32-bit words (as uint64), key: two numbers; the four arrays of output words."""
    c, k = [np.asarray(x, dtype=np.uint64) for x in counter], list(key)
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        hi, lo = (lambda x: x >> np.uint64(32)), (lambda x: x & LOW)
        c = [hi(b) ^ c[1] ^ np.uint64(k[0]), lo(b), hi(a) ^ c[3] ^ np.uint64(k[1]), lo(a)]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def keep_mask(seed, step, site, rows, H, p):
    groups = -(-H // 8)
    g = np.arange(rows * groups, dtype=np.uint64)
    full = lambda v: np.full_like(g, v)  # noqa: E731
    w = philox([g, full(step & 0xFFFFFFFF), full(step >> 32), full(site & 0xFFFFFFFF)], [seed & 0xFFFFFFFF, seed >> 32])
    halves = np.stack([h for x in w for h in (x & np.uint64(0xFFFF), x >> np.uint64(16))], axis=-1).reshape(rows, groups * 8)
    return halves[:, :H] >= round(65536 * float(np.float32(p)))
