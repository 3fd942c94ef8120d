"""Oracle of the RMS norm of a residual stream and its gradients, in fp64 from the rounded h.

Pinned by loops and by differences."""
from __future__ import annotations

import numpy as np

from .ep import bf16_bits_to_f64, f64_to_bf16_bits

__all__ = ["stream", "norm", "backward"]


def stream(x, r=None):
    """h = bf16(x + r): the sum of two bf16 values as fp32 has it, rounded to nearest even."""
    if r is None:
        return np.asarray(x, dtype=np.float64)
    s = (np.asarray(x, dtype=np.float32) + np.asarray(r, dtype=np.float32)).astype(np.float64)
    return bf16_bits_to_f64(f64_to_bf16_bits(s))


def norm(h, w, eps):
    h = np.asarray(h, dtype=np.float64)
    return h / np.sqrt((h * h).mean(1, keepdims=True) + eps) * w


def backward(h, w, dy, eps, dh=None):
    """(dx, dw, magnitudes of the terms of each)."""
    h, w, dy = (np.asarray(t, dtype=np.float64) for t in (h, w, dy))
    i = 1.0 / np.sqrt((h * h).mean(1, keepdims=True) + eps)
    u, g = h * i, dy * w
    dx = i * (g - u * (g * u).mean(1, keepdims=True))
    mag = i * (np.abs(g) + np.abs(u) * np.abs(g * u).mean(1, keepdims=True))
    if dh is not None:
        dx, mag = dx + dh, mag + np.abs(dh)
    return dx, (dy * u).sum(0), mag, np.abs(dy * u).sum(0)
