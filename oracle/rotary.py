"""Oracle of the rotary positions: numpy float64, pair by pair."""
import math

import numpy as np


def frequencies(rot_dim, theta, scaling="none", factor=1.0, original=4096.0, slow=1.0, fast=32.0):
    """(radians of each pair for one position, factor of the result)."""
    n = rot_dim // 2
    if scaling == "base":
        theta = theta * factor ** (rot_dim / (rot_dim - 2))
    f = [math.exp(-2.0 * i / rot_dim * math.log(theta)) for i in range(n)]
    if scaling == "linear":
        f = [x / factor for x in f]
    if scaling == "parts":
        turns = [original * x / (2 * math.pi) for x in f]            # full turns over the original context
        keep = [min(1.0, max(0.0, (t - slow) / (fast - slow))) for t in turns]
        f = [k * x + (1 - k) * x / factor for k, x in zip(keep, f)]
    return f, 0.1 * math.log(factor) + 1.0 if scaling == "parts" else 1.0


def rotate(x, positions, freq, scale=1.0, interleaved=False, inverse=False):
    """Rows x [rows, heads, head_dim] turned by their positions; also the sum of the magnitudes behind each element."""
    y, size = np.array(x, dtype=np.float64), np.abs(np.asarray(x, dtype=np.float64))
    n = len(freq)
    size[..., :2 * n] = 0.0
    for i, f in enumerate(freq):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + n)
        t = np.asarray(positions, dtype=np.float64)[:, None] * f * (-1.0 if inverse else 1.0)
        c, s = scale * np.cos(t), scale * np.sin(t)
        y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
        size[..., a] = size[..., b] = abs(scale) * (np.abs(x[..., a]) + np.abs(x[..., b]))
    return y, size
