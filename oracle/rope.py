"""CPU oracle for rotary positions.  TEST INFRASTRUCTURE ONLY.

fp64 numpy, from the definition: pair p of a token is a complex number that is multiplied by
magnitude * exp(i * coordinate * f_p); the transpose multiplies by the conjugate.  Shares nothing with the CUDA path.
"""
from __future__ import annotations

import math

import numpy as np


def frequencies(axis_pairs, base, scaling="none", factor=1.0, scaled_axes=None, original_length=4096.0, ramp_low=1.0,
                ramp_high=32.0):
    """(radians per position, axis) of every pair."""
    f, axis = [], []
    for a, n in enumerate(axis_pairs):
        on = scaled_axes is None or a in scaled_axes
        for i in range(n):
            b = base
            if on and scaling == "base" and n > 1:
                b = base * factor ** (n / (n - 1))
            x = math.exp(-math.log(b) * i / n)
            if on and scaling == "linear":
                x = x / factor
            if on and scaling == "ramp":
                turns = original_length * x / (2 * math.pi)
                g = min(1.0, max(0.0, (turns - ramp_low) / (ramp_high - ramp_low)))
                x = x * g + x / factor * (1 - g)
            f.append(x)
            axis.append(a)
    return np.array(f), np.array(axis)


def magnitude(scaling, factor):
    return 0.1 * math.log(factor) + 1.0 if scaling == "ramp" else 1.0


def rotate(x, positions, f, axis, layout, size=1.0, inverse=False):
    """x [B, n, H, D] float64, positions [B or 1, n, axes]; rotates the first 2 len(f) elements of every head."""
    pairs = len(f)
    pos = np.broadcast_to(np.asarray(positions, np.float64), (x.shape[0],) + tuple(np.shape(positions))[1:])
    z = size * np.exp(1j * (pos[..., axis] * f))[:, :, None, :]
    if inverse:
        z = z.conj()
    y = np.array(x, np.float64)
    a, b = (slice(0, 2 * pairs, 2), slice(1, 2 * pairs, 2)) if layout == "interleaved" else (slice(0, pairs), slice(pairs, 2 * pairs))
    w = (y[..., a] + 1j * y[..., b]) * z
    y[..., a], y[..., b] = w.real, w.imag
    return y
