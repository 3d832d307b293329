"""Per-head RMS norm and rotary position embedding in float64.  Test infrastructure only.

The paper takes a model's queries and keys as given; what produces them from the projections in the models it
evaluates is y = x / sqrt(mean(x^2) + eps) * w per head (models with normed queries and keys) and the rotation of
pairs of elements by the angle position * inv_freq.
"""
import numpy as np


def norm_heads(x, w, eps):
    """x [..., D] -> x / sqrt(mean x^2 + eps) * w; w None leaves x alone."""
    x = np.asarray(x, dtype=np.float64)
    if w is None:
        return x
    return x / np.sqrt((x * x).mean(axis=-1, keepdims=True) + eps) * np.asarray(w, dtype=np.float64)


def rotate(x, positions, inv_freq, interleaved=False):
    """x [heads, T, D], positions [T], inv_freq [rot / 2]: the first rot elements rotated pair by pair."""
    x = np.array(x, dtype=np.float64)
    freq = np.asarray(inv_freq, dtype=np.float64)
    half = len(freq)
    # the turns are reduced in extended precision, so that far positions keep their fraction
    turns = np.asarray(positions, dtype=np.longdouble)[:, None] * freq.astype(np.longdouble) / (2 * np.pi * np.longdouble(1))
    angle = (2 * np.pi * (turns - np.rint(turns))).astype(np.float64)
    c, s = np.cos(angle), np.sin(angle)
    ia, ib = (np.arange(0, 2 * half, 2), np.arange(1, 2 * half, 2)) if interleaved else (np.arange(half), np.arange(half, 2 * half))
    a, b = x[..., ia].copy(), x[..., ib].copy()
    x[..., ia], x[..., ib] = a * c - b * s, b * c + a * s
    return x
