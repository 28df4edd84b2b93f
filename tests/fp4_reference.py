"""Plain implementations of the operators in 4-bit floating point and of dropout's generator, written from their definitions: quantising in
32 bits (the definition's own), products and layers in 64."""
import math

import numpy as np

BLOCK = {"nvfp4": 16, "mxfp4": 32}
LEVELS = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E4M3 = np.array([(c % 8) / 512 if c < 8 else (1 + (c % 8) / 8) * 2.0 ** (c // 8 - 7) for c in range(127)])  # codes 0 .. 126


def nearest(v, table):
    """Code of the nearest entry, ties to the even code."""
    v = np.asarray(v, dtype=np.float64)
    hi = np.clip(np.searchsorted(table, v), 1, len(table) - 1)
    lo = hi - 1
    below, above = v - table[lo], table[hi] - v
    pick = np.where(below < above, lo, np.where(above < below, hi, np.where(lo % 2 == 0, lo, hi)))
    return np.where(v >= table[-1], len(table) - 1, pick)


def quantise(x, fmt, wide=1.0):
    """codes [M, K] (sign in bit 3), scale bytes [M, blocks] of float32 rows."""
    x = np.asarray(x, dtype=np.float32)
    M, K = x.shape
    B = BLOCK[fmt]
    blocks = -(-K // B)
    padded = np.zeros((M, blocks * B), dtype=np.float32)
    padded[:, :K] = x
    b = padded.reshape(M, blocks, B)
    top = np.abs(b).max(-1) if b.size else np.zeros((M, blocks), dtype=np.float32)
    bad = ~np.isfinite(top)
    t = np.where(bad, np.float32(0), top).astype(np.float32)
    if fmt == "nvfp4":
        with np.errstate(over="ignore"):
            scale = nearest(np.minimum(t / (np.float32(6) * np.float32(wide)), np.float32(448)), E4M3)
        d = (E4M3[scale].astype(np.float32) * np.float32(wide)).astype(np.float32)
    else:
        m, e = np.frexp(t)
        code = np.where(m > 0.75, e - 2, e - 3) + 127
        scale = np.maximum(np.where(t > 0, code, 1), 1)
        d = np.exp2(scale.astype(np.float64) - 127).astype(np.float32)
    with np.errstate(all="ignore"):
        q = np.where((d > 0)[..., None] & ~bad[..., None], np.abs(b) / np.where(d > 0, d, np.float32(1))[..., None], np.float32(0)).astype(np.float32)
    codes = nearest(q, LEVELS) + np.where((np.signbit(b)) & (d > 0)[..., None] & ~bad[..., None], 8, 0)
    scale = np.where(bad, 0x7F if fmt == "nvfp4" else 0xFF, scale)
    return codes.reshape(M, -1)[:, :K].astype(np.uint8), scale.astype(np.uint8)


def pack(codes):
    M, K = codes.shape
    c = np.zeros((M, K + K % 2), dtype=np.uint8)
    c[:, :K] = codes
    return c[:, 0::2] | (c[:, 1::2] << 4)


def unpack(q, K):
    return np.stack((q & 15, q >> 4), -1).reshape(q.shape[:-1] + (-1,))[..., :K]


def steps(scale, fmt, wide=1.0):
    scale = scale.astype(np.int64)
    if fmt == "nvfp4":
        table = np.concatenate([E4M3, [np.nan]])
        return (table[scale & 127].astype(np.float32) * np.float32(wide)).astype(np.float64)
    return np.where(scale == 255, np.nan, np.exp2(scale - 127.0))


def values(codes, scale, fmt, wide=1.0):
    """What rows stand for, in 64 bits."""
    v = np.where(codes >= 8, -1.0, 1.0) * LEVELS[codes & 7]
    return v * np.repeat(steps(scale, fmt, wide), BLOCK[fmt], -1)[..., : codes.shape[-1]]


def rounded(x, fmt, wide=1.0):
    return values(*quantise(x, fmt, wide), fmt, wide)


def weights(rng, shape, fmt, wide=1.0):
    """Random codes and scales: (packed, scale bytes, values in 64 bits) of [.., N, K]."""
    K, B = shape[-1], BLOCK[fmt]
    codes = rng.integers(0, 16, shape).astype(np.uint8)
    lo, hi = (96, 120) if fmt == "nvfp4" else (118, 124)
    scale = rng.integers(lo, hi, shape[:-1] + (-(-K // B),)).astype(np.uint8)
    flat = pack(codes.reshape(-1, K)).reshape(shape[:-1] + (-1,))
    return flat, scale, values(codes, scale, fmt, wide)


def act(name, g):
    """Activation, slope, and the largest magnitude of the slope."""
    if name == "silu":
        s = 1 / (1 + np.exp(-g))
        return g * s, s * (1 + g * (1 - s)), 1.1
    if name == "gelu":
        phi = np.array([0.5 * math.erfc(-v / math.sqrt(2)) for v in np.ravel(g)]).reshape(np.shape(g))
        return g * phi, phi + g * np.exp(-0.5 * g * g) / math.sqrt(2 * math.pi), 1.13
    return np.maximum(g, 0), (g > 0).astype(np.float64), 1.0


def philox(counter, key):
    """Philox-4x32-10: four words for a counter of four words and a key of two."""
    c, k, M = list(counter), list(key), 0xFFFFFFFF
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [(b >> 32) ^ c[1] ^ k[0], b & M, (a >> 32) ^ c[3] ^ k[1], a & M]
        k = [(k[0] + 0x9E3779B9) & M, (k[1] + 0xBB67AE85) & M]
    return c


def keep(M, I, p, seed):
    """Which elements of [M, I] stay."""
    M32 = 0xFFFFFFFF
    s0, s1 = int(seed[0]) & (2 ** 64 - 1), int(seed[1]) & (2 ** 64 - 1)
    words = []
    for n in range(-(-M * I // 4)):
        words += philox((n & M32, n >> 32, s1 & M32, s1 >> 32), (s0 & M32, s0 >> 32))
    return (np.array(words[: M * I], dtype=np.int64).reshape(M, I) >= min(round(p * 2.0 ** 32), 2 ** 32 - 1)) if M * I else np.zeros((M, I), dtype=bool)
