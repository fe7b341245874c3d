"""The operators at a layer's end from their definitions in 64 bits, on the host: what the tests of lr_dense_*, lr_dropout and lr_group_norm_* compare with."""
import numpy as np
from scipy.special import erfc

MASK = 0xFFFFFFFF


def philox(counter, key, rounds=10):
    """Philox4x32 of Salmon et al. 2011 in Python's whole numbers: four words from four words and a key of two."""
    c, k = list(counter), list(key)
    for _ in range(rounds):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & MASK, (a >> 32) ^ c[3] ^ k[1], a & MASK]
        k = [(k[0] + 0x9E3779B9) & MASK, (k[1] + 0xBB67AE85) & MASK]
    return c


def mask16(seed, at, first, count):
    """The 16 random bits of elements first .. first + count - 1."""
    blocks = np.arange(first // 8, (first + count + 7) // 8, dtype=np.uint64)
    u, low = np.uint64, np.uint64(MASK)
    at = at % (1 << 64)
    x = [blocks & low, blocks >> u(32), np.full_like(blocks, at & MASK), np.full_like(blocks, at >> 32)]
    for i in range(10):
        k0, k1 = u(((seed & MASK) + i * 0x9E3779B9) & MASK), u((((seed >> 32) & MASK) + i * 0xBB67AE85) & MASK)
        a, b = x[0] * u(0xD2511F53), x[2] * u(0xCD9E8D57)
        x = [(b >> u(32)) ^ x[1] ^ k0, b & low, (a >> u(32)) ^ x[3] ^ k1, a & low]
    words = np.stack(x, 1).astype("<u4").view("<u2").reshape(-1)
    return words[first % 8:first % 8 + count]


def multipliers(p, seed, offset, site, shape):
    """What drop() multiplies with."""
    t = int(np.floor(p * 65536 + 0.5))
    if t == 0:
        return np.ones(shape)
    bits = mask16(seed, offset + site, 0, int(np.prod(shape))).reshape(shape)
    return np.where(bits >= t, 65536 / max(65536 - t, 1), 0.0)


def act(z, name):
    """(value, slope)"""
    if name == "relu":
        return np.maximum(z, 0), (z > 0) * 1.0
    if name == "gelu":
        below = erfc(-z / np.sqrt(2)) / 2
        return z * below, below + z * np.exp(-z * z / 2) / np.sqrt(2 * np.pi)
    if name == "gelu_tanh":
        c = np.sqrt(2 / np.pi)
        t = np.tanh(c * (z + 0.044715 * z ** 3))
        return z * (1 + t) / 2, (1 + t) / 2 + z / 2 * (1 - t * t) * c * (1 + 3 * 0.044715 * z * z)
    if name == "silu":
        s = 1 / (1 + np.exp(-z))
        return z * s, s + z * s * (1 - s)
    return z, np.ones_like(z)
