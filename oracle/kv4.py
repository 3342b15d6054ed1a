"""The 4-bit KV cache and attention over it in float64 numpy, from the definitions.

TEST INFRASTRUCTURE ONLY, like the rest of this package.  Nothing here is
blocked, fused or shared with the CUDA library: rows are taken apart byte by
byte, scores and weights are whole matrices.
"""
from __future__ import annotations

import numpy as np

CAP = 15.5 * 65536.0
TINY = 2.0 ** -90


def step_of(group):
    """The step of one group of numbers."""
    x = np.where(np.isnan(group), 0.0, np.clip(group, -CAP, CAP)).astype(np.float64)
    a = x[np.argmax(np.abs(x))]              # numpy's argmax: the first of the largest
    if abs(a) < TINY:
        return 0.0
    m, e = np.frexp(abs(a))                  # a = m * 2^e, 1/2 <= m < 1
    return float(-np.sign(a) * np.ldexp(np.rint(m * 32.0) / 32.0, e) / 8.0)


def row_of(x):
    """Bytes of one row of D numbers."""
    D = len(x)
    G = D // 8
    words, ts = [0] * (D // 8), []
    for g in range(8):
        group = np.asarray(x[g * G:(g + 1) * G], np.float64)
        s = step_of(group)
        ts.append(s / 65536.0)
        for i, v in enumerate(np.where(np.isnan(group), 0.0, np.clip(group, -CAP, CAP))):
            c = 0 if s == 0.0 else int(np.clip(np.rint(v / s), -8, 7))   # a quotient of a 24-bit by a 5-bit number
            d = g * G + i                                                # never rounds onto a half in 53 bits
            words[d // 8] |= (c + 8) << (4 * ((d % 8) // 2) + 16 * (d % 2))
    t32 = np.asarray(ts, np.float32)
    assert np.array_equal(t32.astype(np.float64), ts)
    return np.concatenate([np.asarray(words, np.uint32).view(np.uint8), (t32.view(np.uint32) >> 16).astype(np.uint16).view(np.uint8)])


def rows_of(x):
    """Bytes [..., D / 2 + 16] of rows [..., D]."""
    flat = np.asarray(x, np.float64).reshape(-1, x.shape[-1])
    return np.stack([row_of(r) for r in flat]).reshape(*x.shape[:-1], -1)


def values_of(rows):
    """Numbers [..., D] of rows of bytes (any bytes: an exponent of 2 or more loses its top bit)."""
    half = rows.shape[-1] - 16
    D = 2 * half
    r = rows.astype(np.int64)
    out = np.empty(rows.shape[:-1] + (D,))
    for d in range(D):
        i, j, odd = d // 8, (d % 8) // 2, d % 2
        code = (r[..., 4 * i + 2 * odd + j // 2] >> (4 * (j % 2))) & 15
        w = r[..., half + 2 * (d // (D // 8))] | (r[..., half + 2 * (d // (D // 8)) + 1] << 8)
        w = w & 0xBFFF
        e, m = (w >> 7) & 255, w & 127
        t = np.where(e > 0, np.ldexp(1.0 + m / 128.0, (e - 127).astype(int)), np.ldexp(m / 128.0, -126))
        out[..., d] = (code - 8) * np.where(w >> 15, -t, t) * 65536.0
    return out


def visible(P, cnt, n, S, mask=None, depth=None, window=0, sinks=0):
    """bool [n, S]: which cached positions new token i sees.  mask: bool [n, n]."""
    ok = np.zeros((n, S), bool)
    for i in range(cnt):
        pos = P + (i if depth is None else int(depth[i]))
        for j in range(P + cnt):
            at = j
            if j >= P:
                t = j - P
                if not (t <= i if mask is None else mask[i, t]):
                    continue
                at = P + (t if depth is None else int(depth[t]))
            if window and not (at > pos - window or at < sinks):
                continue
            ok[i, j] = True
    return ok


def attend(q, K, V, ok, scale):
    """One head: q [n, D], K, V [S, D], ok [n, S] -> out [n, D], lse [n], and for
    error bounds: A [n, D] = sum of the weights times |v|, M [n] = the largest
    scale * sum |q| |k| among what is seen."""
    x = np.where(ok, (q @ K.T) * scale, -np.inf)
    top = np.where(ok.any(1), x.max(1, initial=-np.inf), 0.0)
    w = np.where(ok, np.exp(x - top[:, None]), 0.0)
    tot = w.sum(1)
    with np.errstate(divide="ignore"):
        lse = np.where(tot > 0, top + np.log(tot), -np.inf)
    w = w / np.where(tot > 0, tot, 1.0)[:, None]
    M = np.where(ok, (np.abs(q) @ np.abs(K).T) * scale, 0.0).max(1, initial=0.0)
    return w @ V, lse, w @ np.abs(V), M
