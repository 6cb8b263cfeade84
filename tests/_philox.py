"""Philox4x32-10 on the host and what dropout keeps by it (written from the published description, for tests)."""
import numpy as np


def philox4x32(counter, key):
    """counter: four arrays of 32-bit numbers (in 64 bits); key: two numbers."""
    mask = np.uint64(0xFFFFFFFF)
    c = [np.asarray(x, dtype=np.uint64) for x in counter]
    k = [int(key[0]), int(key[1])]
    for _ in range(10):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & mask, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & mask]
        k = [(k[0] + 0x9E3779B9) % 2 ** 32, (k[1] + 0xBB67AE85) % 2 ** 32]
    return c


def threshold(p):
    return int(np.floor(p * 65536.0 + 0.5))


def kept(rows, columns, p, seed, step=0, first_row=0):
    """Truth values [rows, columns]: which elements dropout keeps."""
    row = (np.arange(rows, dtype=np.uint64) + np.uint64(first_row))[:, None]
    block = np.arange(-(-columns // 8), dtype=np.uint64)[None, :]
    zero = np.zeros((rows, block.shape[1]), dtype=np.uint64)
    words = philox4x32([zero + block, zero + (row & np.uint64(0xFFFFFFFF)), zero + (row >> np.uint64(32)), zero + np.uint64(step)],
                       (seed % 2 ** 32, seed // 2 ** 32))
    halves = np.stack([h for w in words for h in (w & np.uint64(0xFFFF), w >> np.uint64(16))], axis=2)
    return halves.reshape(rows, -1)[:, :columns] >= np.uint64(threshold(p))
