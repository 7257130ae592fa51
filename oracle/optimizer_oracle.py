"""fp64 oracle of the operators over lists of tensors, written from their definitions (numpy, one tensor at a time): gradient norm, AdamW with
moments in 32 or 8 bits."""
from __future__ import annotations

import math

import numpy as np

BLOCK = 256
#: All magnitudes of the 8-bit type (e4m3: four exponent bits of bias 7, three mantissa bits, no infinity), by their code.
E4M3 = np.array([m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)][:-1])


def grad_norm(grads) -> float:
    return math.sqrt(sum(float(np.square(np.asarray(g, np.float64)).sum()) for g in grads))


def moments(g, m, v, beta1: float, beta2: float):
    return beta1 * m + (1 - beta1) * g, beta2 * v + (1 - beta2) * g * g


def coefficient(grad_scale: float, norm=None, max_norm: float = math.inf) -> float:
    return grad_scale * (1.0 if not norm else min(1.0, max_norm / (grad_scale * norm)))


def param(p, m, v, t: int, lr: float, beta1: float, beta2: float, eps: float, weight_decay: float):
    """The new parameter from the new moments."""
    return (1 - lr * weight_decay) * p - lr / (1 - beta1 ** t) * m / (np.sqrt(v / (1 - beta2 ** t)) + eps)


def thresholds(n: int, t: int):
    """u of elements 0 .. n - 1 at step t, in parts of 2^24."""
    return (12664745 * np.arange(n, dtype=object) + 9560335 * t) % (1 << 24)


def scales(x):
    """Of each block of x [n]: the largest magnitude / 448, or 0 or NaN."""
    top = np.array([np.abs(b).max() if np.isfinite(b).all() else math.nan for b in blocks(x)])
    return np.where(top < 2.0 ** -100, 0.0, top / 448)


def blocks(x):
    return [x[i:i + BLOCK] for i in range(0, len(x), BLOCK)]


def quantise(x, t: int, root: bool):
    """(values of the codes of x [n], scales, how far each magnitude is from the border between its two codes, in parts of their distance)."""
    u = thresholds(len(x), t)
    if root:
        u = (1 << 24) - 1 - u
    s = scales(x)
    y = np.zeros(len(x))
    for i, (b, at) in enumerate(zip(blocks(x), range(0, len(x), BLOCK))):
        y[at:at + BLOCK] = np.minimum(np.abs(b) / s[i], 448.0) if s[i] > 0 else 0.0
    low = np.searchsorted(E4M3, y, side="right") - 1
    high = np.minimum(low + 1, len(E4M3) - 1)
    apart = np.where(high > low, E4M3[high] - E4M3[low], 32.0)
    rest = (y - E4M3[low]) / apart + u.astype(np.float64) / (1 << 24)
    code = np.where(rest >= 1, E4M3[high], E4M3[low])
    if root:
        code = np.where((y > 0) & (code == 0), E4M3[1], code)
    return code * np.where(x < 0, -1.0, 1.0), s, np.abs(rest - 1)
