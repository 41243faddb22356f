"""Philox4x32-10 and the dropout mask made of it, restated with numpy's unsigned 64-bit arithmetic."""
import numpy as np
import torch

M = np.uint64(0xFFFFFFFF)
S = np.uint64(32)


def philox4x32(counter, key, rounds=10):
    """counter: four arrays of 32-bit words; key: two.  Four arrays."""
    a, b, c, d = (np.asarray(v, np.uint64) & M for v in counter)
    k0, k1 = (np.uint64(v) & M for v in key)
    for _ in range(rounds):
        p, q = a * np.uint64(0xD2511F53), c * np.uint64(0xCD9E8D57)
        a, b, c, d = (q >> S) ^ b ^ k0, q & M, (p >> S) ^ d ^ k1, p & M
        k0, k1 = (k0 + np.uint64(0x9E3779B9)) & M, (k1 + np.uint64(0xBB67AE85)) & M
    return a, b, c, d


def threshold(p):
    return round(p * 65536)


def numbers(first, count, seed, offset):
    """The 16-bit numbers of elements first .. first + count."""
    e = np.arange(first, first + count, dtype=np.uint64)
    g = e >> np.uint64(3)
    seed, offset = seed % 2 ** 64, offset % 2 ** 64
    words = np.stack(philox4x32((g & M, g >> S, np.full_like(g, offset & 0xFFFFFFFF), np.full_like(g, offset >> 32)),
                                (seed & 0xFFFFFFFF, seed >> 32)))
    j = (e & np.uint64(7)).astype(np.int64)
    w = words[j // 2, np.arange(count)]
    return (w >> (np.uint64(16) * (j % 2).astype(np.uint64))) & np.uint64(0xFFFF)


def kept(shape, p, seed, offset, first=0):
    count = int(np.prod(shape))
    return torch.from_numpy(numbers(first, count, seed, offset) >= threshold(p)).view(shape)
