"""AdamW over many tensors and the norm of their gradients in 64 bits, from the formulas of include/sasgd.h (numpy; test infrastructure)."""
import numpy as np

M32 = np.uint64(0xFFFFFFFF)


def alphas(lr_mode, staleness):
    """(rate / alpha0, shares) of a window."""
    tau = np.asarray(staleness, np.float64)
    if lr_mode == "per_gradient":
        a = 1 / np.maximum(tau, 1)
    elif lr_mode == "mean_staleness":
        a = np.full(len(tau), 1 / max(tau.mean(), 1))
    else:
        a = np.ones(len(tau))
    return a.mean(), a / a.sum()


def step(theta, grads, m, v, t, staleness, lr_mode, alpha0, beta1, beta2, eps, wd, factor=1.0):
    """(theta, m, v) after one step of one tensor; grads: c arrays."""
    mean, share = alphas(lr_mode, staleness)
    rate = alpha0 * mean
    g = factor * sum(s * np.asarray(x, np.float64) for s, x in zip(share, grads))
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    mh, vh = m / (1 - beta1 ** t), v / (1 - beta2 ** t)
    return theta - rate * (mh / (np.sqrt(vh) + eps) + wd * theta), m, v


def mix(x):
    x = np.asarray(x, np.uint64) & M32
    x ^= x >> np.uint64(16)
    x = (x * np.uint64(0x6A09E667)) & M32
    x ^= x >> np.uint64(15)
    x = (x * np.uint64(0xB7E15163)) & M32
    return x ^ (x >> np.uint64(16))


def chance(first, n, seed, t):
    """The 32 bits of the moments' elements first .. first + n - 1."""
    e = np.arange(first, first + n, dtype=np.uint64)
    key = mix((seed + t * 0x9E3779B1) & 0xFFFFFFFF)
    return mix(((e & M32) * np.uint64(0x9E3779B1) & M32) ^ ((e >> np.uint64(32)) * np.uint64(0x243F6A89) & M32) ^ key)


def grid_below(y):
    """Largest e4m3 value not above y (0 <= y <= 448), and the distance to the next."""
    gap = np.exp2(np.floor(np.log2(np.maximum(y, 2.0 ** -6))) - 3)
    return np.floor(y / gap) * gap, gap


def e4m3(byte):
    """The value of an e4m3 byte."""
    byte = np.asarray(byte, np.int64)
    sign, e, f = np.where(byte & 128, -1.0, 1.0), (byte >> 3) & 15, byte & 7
    val = np.where(e == 0, f * 2.0 ** -9, (1 + f / 8) * np.exp2(e - 7.0))
    return sign * np.where((byte & 127) == 127, np.nan, val)


def stored(x, bits, floor):
    """(values / scale on the grid, scale, y) of a padded vector in 8 bits: y is what is rounded, up where its cut-off part in
    1/65536 and the 16 bits carry."""
    x = x.reshape(-1, 256)
    most = np.abs(x).max(1, keepdims=True)
    most[most < 1e-30] = 0
    y = np.abs(x) * np.divide(448.0, most, out=np.zeros_like(most), where=most > 0)
    low, gap = grid_below(np.minimum(y, 448))
    q = np.minimum(low + gap * np.floor((y - low) / gap + bits.reshape(-1, 256) / 65536), 448)
    if floor:
        q = np.where((y > 0) & (q == 0), 2.0 ** -9, q)
    return np.sign(x) * q, most[:, 0] / 448, y
