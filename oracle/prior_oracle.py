"""Double-precision definitions of the prior's operators (layer norm, dropout, residual tail) in numpy, on arrays viewed as
(outer, features, inner).  Test infrastructure; shares no code with the CUDA path."""
import math
import struct

import numpy as np


def philox(counter, key):
    """Philox4x32-10 on one 4-word counter and 2-word key, in Python's whole numbers (Salmon et al. 2011)."""
    c, k = list(counter), list(key)
    for _ in range(10):
        p0, p1 = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(p1 >> 32) ^ c[1] ^ k[0], p1 & 0xFFFFFFFF, (p0 >> 32) ^ c[3] ^ k[1], p0 & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def words(n, seed, offset, step=0):
    """The first n words of the mask, as numpy whole numbers (vectorised; philox() is its own check)."""
    low, wide = np.uint64(0xFFFFFFFF), np.uint64(32)
    with np.errstate(over="ignore"):
        block = np.uint64(offset % 2 ** 64) + np.arange((n + 3) // 4, dtype=np.uint64)
    c = [block & low, block >> wide, np.full_like(block, step & 0xFFFFFFFF), np.full_like(block, (step >> 32) & 0xFFFFFFFF)]
    k = [seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF]
    for _ in range(10):
        p0, p1 = np.uint64(0xD2511F53) * c[0], np.uint64(0xCD9E8D57) * c[2]
        c = [(p1 >> wide) ^ c[1] ^ np.uint64(k[0]), p1 & low, (p0 >> wide) ^ c[3] ^ np.uint64(k[1]), p0 & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return np.stack(c, 1).reshape(-1)[:n]


def kept(shape, p, seed, offset, step=0):
    n = int(np.prod(shape))
    return (words(n, seed, offset, step) >= np.uint64(math.floor(p * 2 ** 32))).reshape(shape)


def scale(p):
    """1 / (1 - p) as a number of 32 bits; 0 where everything is dropped."""
    return struct.unpack("f", struct.pack("f", 1.0 / (1.0 - p)))[0] if p < 1 else 0.0


def dropout(x, p, seed, offset, step=0):
    keep = kept(x.shape, p, seed, offset, step)
    return np.where(keep, np.where(keep, x, 0.0).astype(np.float64) * scale(p), 0.0)


def layer_norm(x, weight, bias, eps):
    x = x.astype(np.float64)
    mean = x.mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt(((x - mean) ** 2).mean(1, keepdims=True) + eps)
    return (x - mean) * rstd * weight[None, :, None] + bias[None, :, None], mean[:, 0], rstd[:, 0]


def layer_norm_vjp(grad, x, weight, mean, rstd):
    grad, x = grad.astype(np.float64), x.astype(np.float64)
    h = (x - mean[:, None]) * rstd[:, None]
    g = grad * weight[None, :, None]
    gx = rstd[:, None] * (g - g.mean(1, keepdims=True) - h * (g * h).mean(1, keepdims=True))
    return gx, (grad * h).sum((0, 2)), grad.sum((0, 2))
