"""Rows of q and k on their way to the attention, in 64 bits: norm of every head, rotation by the position."""
import numpy as np


def qk_rows(x, positions, inv_freq=None, rot_scale=1.0, interleaved=False, norm=False, weight=None, eps=1e-6):
    """x [N,H,D]; returns (rows [N,H,D], length of the pair that each channel belongs to, before the turn)."""
    x = np.array(x, dtype=np.float64)
    if norm:
        x = x / np.sqrt(np.mean(x * x, axis=-1, keepdims=True) + eps)
        if weight is not None:
            x = x * np.asarray(weight, dtype=np.float64)
    size = np.abs(x)
    half = 0 if inv_freq is None else len(inv_freq)
    for i in range(half):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        t = np.asarray(positions, dtype=np.float64)[:, None] * float(inv_freq[i])
        c, s, u, v = np.cos(t) * rot_scale, np.sin(t) * rot_scale, x[..., a].copy(), x[..., b].copy()
        x[..., a], x[..., b] = u * c - v * s, u * s + v * c
        size[..., a] = size[..., b] = np.hypot(u, v) * rot_scale
    return x, size
