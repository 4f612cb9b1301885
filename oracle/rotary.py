"""Rotary positions in numpy and 64 bits, from the definitions in include/flowmm.h."""
import math

import numpy as np

HALVES, PAIRS = 0, 1
PLAIN, LINEAR, BY_PARTS = 0, 1, 2


def frequencies(R, base, scaling=PLAIN, factor=1.0, low=1.0, high=32.0, trained=0):
    f = np.array([base ** (-2.0 * i / R) for i in range(R // 2)])
    if scaling == LINEAR:
        return f / factor
    if scaling == BY_PARTS:
        g = np.clip((trained * f / (2 * math.pi) - low) / (high - low), 0.0, 1.0)
        return g * f + (1 - g) * f / factor
    return f


def rotate(x, positions, freq, layout=HALVES, sections=None, amplitude=1.0, adjoint=False):
    """x [U, H, T, D], positions [U, axes, T]; float64 out."""
    R = 2 * len(freq)
    axis = np.repeat(np.arange(len(sections)), sections) if sections is not None else np.zeros(R // 2, int)
    angle = positions[:, axis].astype(np.longdouble) * freq.astype(np.longdouble)[:, None]
    angle = np.moveaxis(np.fmod(angle, 2 * np.longdouble("3.14159265358979323846264338327950288")).astype(np.float64), 1, 2)[:, None]
    c, s = amplitude * np.cos(angle), amplitude * np.sin(angle)
    if adjoint:
        s = -s
    y = x.astype(np.float64).copy()
    a, b = (slice(0, R // 2), slice(R // 2, R)) if layout == HALVES else (slice(0, R, 2), slice(1, R, 2))
    y[..., a], y[..., b] = x[..., a] * c - x[..., b] * s, x[..., b] * c + x[..., a] * s
    return y
