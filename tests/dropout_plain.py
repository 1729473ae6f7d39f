"""The dropout mask in plain numpy: Philox 4x32-10 (Salmon et al., 2011) on unsigned 64-bit integers, and the mask of a call."""
import numpy as np
import torch

LOW = np.uint64(0xffffffff)


def philox(counter, key, rounds=10):
    """counter: four arrays of 32-bit numbers (as uint64), key: two numbers.  Returns four arrays."""
    c, k = [np.asarray(v, np.uint64) for v in counter], [int(v) for v in key]
    for _ in range(rounds):
        a, b = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(b >> np.uint64(32)) ^ c[1] ^ np.uint64(k[0]), b & LOW, (a >> np.uint64(32)) ^ c[3] ^ np.uint64(k[1]), a & LOW]
        k = [(k[0] + 0x9E3779B9) & 0xffffffff, (k[1] + 0xBB67AE85) & 0xffffffff]
    return c


def bits16(n, seed, at, first=0):
    """The 16 bits of elements first .. first + n - 1 of a call; `first` a multiple of eight."""
    i = np.arange(first // 8, first // 8 + -(-n // 8), dtype=np.uint64)
    at %= 2 ** 64
    words = philox((i & LOW, i >> np.uint64(32), np.full_like(i, at & 0xffffffff), np.full_like(i, at >> 32)), (seed & 0xffffffff, seed >> 32))
    return np.stack([v for w in words for v in (w & np.uint64(0xffff), w >> np.uint64(16))], 1).reshape(-1)[:n].astype(np.int64)


def mask(n, p, seed, at, first=0):
    """(which elements are kept, the factor of those)"""
    dropped = int(np.rint(p * 65536))
    return torch.from_numpy(bits16(n, seed, at, first) >= dropped), 0.0 if dropped == 65536 else 65536 / (65536 - dropped)
