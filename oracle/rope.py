"""Rotary positions from their definition (TEST INFRASTRUCTURE ONLY, see the package docstring).

Pair i of a row at position p turns by the angle p * f_i: (x, y) -> m (x cos - y sin, x sin + y cos).  The pairs
are elements (i, i + rot / 2), or (2 i, 2 i + 1) in the interleaved layout; elements from rot on stay.  Angles are
formed and reduced in extended precision (64 significant bits: off by 2^-32 at positions up to 2^31).
"""
import numpy as np

_TURN = np.longdouble("6.283185307179586476925286766559005768")


def rotate(x, at, freq, interleaved=False, magnitude=1.0):
    """x [n, d] fp64 rows, at [n, pairs] integer positions of each pair, freq [pairs] -> (rows, length of each
    element's pair, 0 for elements that stay)."""
    freq = np.asarray(freq, dtype=np.float64)
    pairs = freq.shape[0]
    angle = np.asarray(at, dtype=np.longdouble) * freq.astype(np.longdouble)
    angle = (angle - np.floor(angle / _TURN) * _TURN).astype(np.float64)
    one = 2 * np.arange(pairs) if interleaved else np.arange(pairs)
    two = one + 1 if interleaved else one + pairs
    c, s = magnitude * np.cos(angle), magnitude * np.sin(angle)
    out, size = x.copy(), np.zeros_like(x)
    out[:, one] = x[:, one] * c - x[:, two] * s
    out[:, two] = x[:, one] * s + x[:, two] * c
    size[:, one] = size[:, two] = abs(magnitude) * np.hypot(x[:, one], x[:, two])
    return out, size
