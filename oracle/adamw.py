"""fp64 oracle of the optimiser's step: the formulas of include/pods.h on numpy arrays, with the 8-bit states' grid and the
random bits that decide a rounding.  (The paper names the optimiser only.)"""
import numpy as np

M32 = np.uint64(0xFFFFFFFF)


def mix(x):
    x = np.asarray(x, np.uint64) & M32
    x = x ^ (x >> np.uint64(16))
    x = (x * np.uint64(0x888EC647)) & M32
    x = x ^ (x >> np.uint64(15))
    x = (x * np.uint64(0x246CE511)) & M32
    return x ^ (x >> np.uint64(16))


def random_bits(seed, step, first, n):
    """16 random bits each for the parameter, m and v of elements first .. first + n - 1."""
    key = mix(mix(mix((seed + 0x9E3779B9) & 0xFFFFFFFF) ^ np.uint64(seed >> 32 & 0xFFFFFFFF)) ^ np.uint64(step & 0xFFFFFFFF))
    i = np.uint64(first) + np.arange(n, dtype=np.uint64)
    w = mix((i & M32) ^ mix((key + (i >> np.uint64(32))) & M32))
    return w & np.uint64(0xFFFF), w >> np.uint64(16), ((w * np.uint64(0x9E3779B1)) & M32) >> np.uint64(16)


def e4m3_values():
    """What the codes 0 .. 126 stand for."""
    c = np.arange(127)
    e, m = c >> 3, c & 7
    return np.where(e == 0, m * 2.0 ** -9, (1 + m / 8.0) * 2.0 ** (e - 7.0))


def decode(codes, scales):
    c = np.asarray(codes).astype(np.int64)
    v = np.append(e4m3_values(), np.nan)[c & 127] * np.where(c & 128, -1.0, 1.0)
    k = np.repeat(np.asarray(scales).astype(np.float64), 32)[:c.size]
    return v * np.where(k == 0, 0.0, np.exp2(k - 127.0))


def block_exponents(x):
    """The smallest k >= 1 with |block| / 2^(k - 127) <= 448."""
    n = x.size
    top = np.abs(np.pad(x, (0, -n % 32))).reshape(-1, 32).max(1)
    k = np.ones(top.size, np.int64)
    for i, t in enumerate(top):
        while t * 2.0 ** (127 - k[i]) > 448.0:
            k[i] += 1
    return k


def place_on_grid(x, k):
    """|x| / 2^(k - 127) as a code with a fraction: whole codes below 2^-6 are multiples of 2^-9, above it eighths of a power."""
    y = np.abs(x) * np.exp2(127.0 - np.repeat(k, 32)[:x.size])
    e = np.clip(np.floor(np.log2(np.maximum(y, 2.0 ** -60))), -6, 8)
    return np.where(y < 2.0 ** -6, y * 512.0, (y / np.exp2(e) - 1.0) * 8.0 + (e + 7.0) * 8.0)


def step(p, g, m, v, step, lr, beta1, beta2, eps, decay=0.0, grad_scale=1.0, norm=None, max_norm=0.0):
    """fp64 (p, m, v) after the step; v the second moment itself."""
    p, g, m, v = (np.asarray(a, np.float64) for a in (p, g, m, v))
    g = g * grad_scale
    if max_norm > 0 and norm > max_norm:
        g = g * (max_norm / norm)
    m = beta1 * m + (1.0 - beta1) * g
    v = beta2 * v + (1.0 - beta2) * g * g
    p = p * (1.0 - lr * decay) - lr / (1.0 - beta1 ** step) * m / (np.sqrt(v) / np.sqrt(1.0 - beta2 ** step) + eps)
    return p, m, v
