"""Norms and rotations of queries and keys by their positions in float64 numpy, from the definitions.

TEST INFRASTRUCTURE ONLY, like the rest of this package.  A pair of channels is a
complex number, turned by a product.
"""
from __future__ import annotations

import numpy as np

CAP = 15.5 * 65536.0
TINY = 2.0 ** -90


def turned(x, inv_freq, pos, axes=None, weight=None, eps=None, interleaved=False, scale=1.0):
    """x [..., heads, D]; pos [A, ...] whole numbers; weight [D] or [heads, D].  Returns z and, for
    error bounds, h: the length of each number's pair before it is turned (times scale), or the
    number's own size."""
    x = np.asarray(x, np.float64)
    D, half = x.shape[-1], len(inv_freq)
    if eps is not None:
        norm = np.sqrt((x * x).sum(-1, keepdims=True) / D + eps)
        if weight is not None:
            x = x * np.asarray(weight, np.float64)    # exact: products that are equal stay so
        x = x / norm
    z, h = x.copy(), np.abs(x)
    for j in range(half):
        u, v = (2 * j, 2 * j + 1) if interleaved else (j, j + half)
        a = 0 if axes is None else int(np.clip(axes[j], 0, len(pos) - 1))
        t = np.exp(1j * (np.asarray(pos[a], np.float64) * float(inv_freq[j])))[..., None]
        c = (x[..., u] + 1j * x[..., v]) * t * scale
        z[..., u], z[..., v] = c.real, c.imag
        h[..., u] = h[..., v] = np.hypot(x[..., u], x[..., v]) * scale
    return z, h


def held(x):
    """The numbers that a 4-bit cache holds for rows x [..., D] (oracle/kv4.py's format, many rows at once)."""
    D = x.shape[-1]
    g = np.asarray(x, np.float64).reshape(x.shape[:-1] + (8, D // 8))
    g = np.where(np.isnan(g), 0.0, np.clip(g, -CAP, CAP))
    at = np.abs(g).argmax(-1)[..., None]              # the first of the largest
    a = np.take_along_axis(g, at, -1)
    m, e = np.frexp(a)
    s = np.where(np.abs(a) < TINY, 0.0, -np.ldexp(np.rint(m * 32.0), e - 8))
    with np.errstate(divide="ignore", invalid="ignore"):
        r = np.where(s == 0.0, 0.0, np.clip(np.rint(g / s), -8, 7))
    return (r * s).reshape(x.shape)
