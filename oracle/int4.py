"""4-bit rows for quantised K/V slabs.  Test infrastructure only.

The paper names quantisation as a complement to budget allocation without fixing a scheme; the scheme here: fp32 scales
per channel (the caller's, with their reciprocals) and one fp32 scale per row.  With y = fl32(x * (1 / channel scale)):
row scale s = fl32(max |y| / 7), code u = clamp(rint(fl32(y / s)), -7, 7) + 8, which stands for
(u - 8) * s * channel scale; a row of zeros has s = 0 and u = 8.  A byte holds an even channel in its low half and the
next one in its high half.
"""
import numpy as np


def quantise_rows(rows, inv_chan):
    """rows [..., D] (values a float32 holds exactly) -> (codes uint8 [..., D] in 1 .. 15, row scales float32 [...])."""
    y = np.asarray(rows, dtype=np.float32) * np.asarray(inv_chan, dtype=np.float32)
    s = np.abs(y).max(axis=-1) / np.float32(7.0)
    safe = np.where(s > 0, s, np.float32(1.0))[..., None]
    u = np.clip(np.rint(y / safe), -7, 7) + 8
    return np.where(s[..., None] > 0, u, 8).astype(np.uint8), s


def pack(codes):
    """codes [..., D] -> bytes [..., D / 2]."""
    c = np.asarray(codes, dtype=np.uint8)
    return (c[..., 0::2] | (c[..., 1::2] << 4)).astype(np.uint8)


def unpack(data):
    d = np.asarray(data, dtype=np.uint8)
    return np.stack([d & 15, d >> 4], axis=-1).reshape(d.shape[:-1] + (2 * d.shape[-1],))


def values(codes, scale, chan):
    """codes [..., D], row scales [...], channel scales [D] -> float64 values."""
    return ((np.asarray(codes).astype(np.float64) - 8.0) * np.asarray(scale, dtype=np.float64)[..., None]
            * np.asarray(chan, dtype=np.float64))
