"""Plain 64-bit forms of the workers' local-gradient operators: embedding
lookup and gradient, 8-bit activation checkpoints, and the weight gradient of
a linear layer.  numpy only; nothing here is shared with the library.

Section 3 step (1) of the paper ("each worker computes its local gradient on
its own replica"); the paper names no model operators, so these follow the
operators' own definitions.
"""
from __future__ import annotations

import numpy as np

GROUP = 32
MIN_EXP = -117
NAN_CODE = 0x7F


def embed(tokens, table, first, scale):
    """tokens [t] ints, table [v][h] fp64 -> [t][h]; zeros outside the table."""
    v, h = table.shape
    out = np.zeros((len(tokens), h))
    for j, tok in enumerate(tokens):
        row = int(tok) - int(first)
        if 0 <= row < v:
            out[j] = scale * table[row]
    return out


def embed_grad(tokens, dy, v, first, scale):
    """(gradient [v][h], tokens per row [v], sum of |dy| [v][h])."""
    h = dy.shape[1]
    grad, size = np.zeros((v, h)), np.zeros((v, h))
    count = np.zeros(v, np.int64)
    for j, tok in enumerate(tokens):
        row = int(tok) - int(first)
        if 0 <= row < v:
            grad[row] += dy[j]
            size[row] += np.abs(dy[j])
            count[row] += 1
    return scale * grad, count, abs(scale) * size


def e4m3_table() -> np.ndarray:
    """Values of the 256 e4m3 codes: sign, 4 exponent bits of bias 7, 3
    mantissa bits, subnormals, no infinity; 0x7F and 0xFF are NaN."""
    out = np.empty(256)
    for code in range(256):
        e, m = (code >> 3) & 15, code & 7
        x = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        if code & 0x7F == 0x7F:
            x = np.nan
        out[code] = -x if code & 0x80 else x
    return out


def e4m3_nearest(z) -> np.ndarray:
    """Codes of the nearest e4m3 values of z (|z| <= 448), ties to the even
    code."""
    pos = e4m3_table()[:0x7F]
    a = np.abs(z)
    hi = np.searchsorted(pos, a, side="left").clip(0, 0x7E)
    lo = (hi - 1).clip(0)
    dl, dh = a - pos[lo], pos[hi] - a
    code = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    return (code | np.where(np.signbit(z), 0x80, 0)).astype(np.uint8)


def pack(x):
    """x [t][h] fp64 -> (codes [t][h], exponent bytes [t][ceil(h / 32)])."""
    t, h = x.shape
    g = (h + GROUP - 1) // GROUP
    q, s = np.empty((t, h), np.uint8), np.empty((t, g), np.uint8)
    for j in range(g):
        y = x[:, j * GROUP:(j + 1) * GROUP]
        fin = np.isfinite(y)
        top = np.where(fin, np.abs(y), 0.0).max(axis=1)
        k = np.full(t, MIN_EXP)
        while True:  # the smallest k that holds the largest value
            more = top > 448.0 * np.exp2(k.astype(np.float64))
            if not more.any():
                break
            k = k + more
        z = np.where(fin, y, 0.0) * np.exp2(-k.astype(np.float64))[:, None]
        # 256 * 2^120 is beyond fp32: the largest finite value below stands in
        z = np.where((k == 120)[:, None], z.clip(-240.0, 240.0), z)
        q[:, j * GROUP:(j + 1) * GROUP] = np.where(fin, e4m3_nearest(z), NAN_CODE)
        s[:, j] = k + 127
    return q, s


def unpack(q, s):
    """fp64 values of a checkpoint."""
    h = q.shape[1]
    scale = np.exp2(s.astype(np.float64) - 127.0)
    return e4m3_table()[q] * np.repeat(scale, GROUP, axis=1)[:, :h]


def wgrad(dy, x, scale):
    """(scale * dy^T x [o][h], the same of absolute values)."""
    return scale * (dy.T @ x), abs(scale) * (np.abs(dy).T @ np.abs(x))
