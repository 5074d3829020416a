"""Layer norm and AdamW (oracle; numpy float64; test infrastructure only).

Layer norm of a row x of d numbers:  mean = sum x / d, var = sum (x - mean)^2 / d, rstd = 1 / sqrt(var + eps),
xh = (x - mean) rstd, y = xh w + b;  u = dy w, dx = rstd (u - mean(u) - xh mean(u xh)), dw = sum dy xh, db = sum dy.

AdamW with decoupled weight decay, gradients clipped by the norm over all tensors, and states held as e4m3 codes in units
of a scale per block of 256 elements, rounded stochastically by a counter hash (include/legend.h has the text).
"""

from __future__ import annotations

import numpy as np

from .negatives import fold

BLOCK, TOP, LEAST = 256, 448.0, 2.0**-9


def layer_norm(x, weight, bias, eps):
    x = np.asarray(x, np.float64)
    mean = x.mean(1)
    c = x - mean[:, None]
    rstd = 1.0 / np.sqrt((c * c).mean(1) + eps)
    xh = c * rstd[:, None]
    y = xh if weight is None else xh * np.asarray(weight, np.float64)
    return (y if bias is None else y + np.asarray(bias, np.float64)), mean, rstd


def layer_norm_backward(x, dy, mean, rstd, weight):
    """(dx, dweight, dbias) from the statistics that the forward pass left."""
    x, dy = np.asarray(x, np.float64), np.asarray(dy, np.float64)
    rstd = np.asarray(rstd, np.float64)[:, None]
    xh = (x - np.asarray(mean, np.float64)[:, None]) * rstd
    u = dy if weight is None else dy * np.asarray(weight, np.float64)
    dx = rstd * (u - u.mean(1, keepdims=True) - xh * (u * xh).mean(1, keepdims=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


def gradient_norm(grads, grad_scale=1.0):
    return abs(grad_scale) * np.sqrt(sum(float((np.asarray(g, np.float64) ** 2).sum()) for g in grads))


def clip_factor(norm, max_norm):
    return max_norm / (norm + 1e-6) if max_norm > 0 and norm > max_norm else 1.0


def adamw(p, g, m, v, t, *, lr, beta1, beta2, eps, weight_decay=0.0):
    """Step t (from 1) of one tensor; (p, m, v) after it.  g is scaled and clipped already."""
    p, g, m, v = (np.asarray(a, np.float64) for a in (p, g, m, v))
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    return p * (1 - lr * weight_decay) - lr * (m / (1 - beta1**t)) / (np.sqrt(v / (1 - beta2**t)) + eps), m, v


def e4m3_values():
    """What the 256 codes stand for: sign, 4 exponent bits (bias 7), 3 mantissa bits; exponent 0 is subnormal, 0x7f is NaN."""
    code = np.arange(256)
    e, f = (code >> 3) & 15, code & 7
    mag = np.where(e == 0, f * 2.0**-9, (1 + f / 8) * 2.0 ** (e - 7.0))
    mag[(code & 127) == 127] = np.nan
    return np.where(code & 128, -mag, mag)


def random_words(seed, t, tensor, count, first=0):
    """The 32-bit words of elements first .. first + count - 1 of a tensor at step t."""
    key = np.uint64(fold(fold(np.uint64(seed), t), tensor)) & np.uint64(0xFFFFFFFF)
    i = np.arange(first, first + count, dtype=np.uint64)
    mask = np.uint64(0xFFFFFFFF)
    w = (i & mask) ^ (((i >> np.uint64(32)) * np.uint64(0x9E3779B1)) & mask) ^ key
    w ^= w >> np.uint64(16)
    w = (w * np.uint64(0x9E3779B1)) & mask
    w ^= w >> np.uint64(15)
    w = (w * np.uint64(0x85157AF5)) & mask
    return w ^ (w >> np.uint64(16))


def block_scales(x):
    """One scale per block of 256 values: the largest finite magnitude over 448; 0 below 2^-100."""
    x = np.abs(np.asarray(x, np.float64))
    x = np.where(np.isfinite(x), x, 0.0)
    x = np.pad(x, (0, -len(x) % BLOCK)).reshape(-1, BLOCK).max(1) / TOP
    return np.where(x > 2.0**-100, x, 0.0)


def rounded_up_share(x, scales, least):
    """Values in units of their scales as (code value below, step to the next one, fraction of the step)."""
    s = np.repeat(scales, BLOCK)[: len(x)]
    with np.errstate(divide="ignore", invalid="ignore"):
        a = np.where(s > 0, np.abs(x) / s, 0.0)
    a = np.minimum(a, TOP)
    if least:
        a = np.where(a > 0, np.maximum(a, LEAST), a)
    step = np.exp2(np.maximum(np.frexp(a)[1] - 1, -6) - 3.0)
    low = np.floor(a / step) * step
    return low, step, (a - low) / step
