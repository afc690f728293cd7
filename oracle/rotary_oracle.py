"""TEST INFRASTRUCTURE ONLY - plain fp64 reference of rotary positions in general form: frequencies (plain, linear, by
parts), half and interleaved pairs, the first `rot` elements of a head.

    pair p of a head's first `rot` elements:  half: (x[p], x[p + rot/2]);  interleaved: (x[2p], x[2p + 1])
    y = magnitude * (a cos - b sin, b cos + a sin),  angle = position * f_p;  inverse: angle negated
    f_p = base^(-2p / rot);  linear: f_p / factor
    by parts: r = original_length f_p / (2 pi);  w = clamp((r - low) / (high - low), 0, 1);  w f_p + (1 - w) f_p / factor

One row and one pair at a time.  Only tests/ may import this module.
"""
import math

import numpy as np


def frequencies(rot, base, scaling="plain", factor=1.0, original_length=0.0, low=1.0, high=32.0):
    out = []
    for p in range(rot // 2):
        f = math.exp(-2.0 * p / rot * math.log(base))
        if scaling == "linear":
            f /= factor
        elif scaling == "parts":
            w = min(max((original_length * f / (2.0 * math.pi) - low) / (high - low), 0.0), 1.0)
            f = w * f + (1.0 - w) * f / factor
        out.append(f)
    return np.array(out)


def positions(cu, total, starts=None):
    """Position of every packed row; None for rows of no sequence."""
    pos = [None] * total
    for s in range(len(cu) - 1):
        for t in range(int(cu[s]), int(cu[s + 1])):
            pos[t] = t - int(cu[s]) + (int(starts[s]) if starts is not None else 0)
    return pos


def rotate(x, pos, freqs, layout="half", magnitude=1.0, inverse=False):
    """x [T, H, d] -> rotated copy (fp64); rows whose position is None are nan."""
    y = np.array(x, dtype=np.float64)
    half = len(freqs)
    for t in range(y.shape[0]):
        if pos[t] is None:
            y[t] = np.nan
            continue
        for p in range(half):
            i, j = (p, p + half) if layout == "half" else (2 * p, 2 * p + 1)
            c, s = math.cos(pos[t] * freqs[p]) * magnitude, math.sin(pos[t] * freqs[p]) * magnitude
            if inverse:
                s = -s
            a, b = y[t, :, i].copy(), y[t, :, j].copy()
            y[t, :, i], y[t, :, j] = a * c - b * s, b * c + a * s
    return y
