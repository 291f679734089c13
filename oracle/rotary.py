"""Rotary positions (oracle; test infrastructure), evaluated in float64."""

import numpy as np

__all__ = ["rotary_ref"]


def rotary_ref(x, positions, inv_freq, interleaved=False, scale=1.0):
    """Rows [T, heads, D] -> float64 [T, heads, D], and the bound |x1| + |x2| of each channel's pair."""
    x = np.asarray(x, np.float64)
    f = np.asarray(inv_freq, np.float64)
    angle = np.asarray(positions, np.float64)[:, None] * f
    turn = np.exp(1j * angle)[:, None] * scale
    n = len(f)
    first = np.arange(n) * 2 if interleaved else np.arange(n)
    second = first + (1 if interleaved else n)
    z = (x[..., first] + 1j * x[..., second]) * turn
    y, size = x.copy(), np.zeros_like(x)
    y[..., first], y[..., second] = z.real, z.imag
    size[..., first] = size[..., second] = abs(scale) * (np.abs(x[..., first]) + np.abs(x[..., second]))
    return y, size
