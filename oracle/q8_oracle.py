"""Rows in 8 bits, from their definition, in 64-bit numbers.

A row of values is kept as whole numbers q (codes) and a scale s of 16
significant bits; it stands for s q.  ``quantize`` gives codes and scales,
``product`` the product of rows and weights kept so, ``transform_bwd`` the
gradients of a product whose left operand was kept so.
"""
from __future__ import annotations

from fractions import Fraction

import numpy as np

LEVELS = {"signed": 127, "relu": 255}


def cut16(x: Fraction) -> Fraction:
    """x > 0 cut off after 16 significant bits."""
    e = 0
    while x >= 2 ** 16:
        x, e = x / 2, e + 1
    while x < 2 ** 15:
        x, e = x * 2, e - 1
    return Fraction(int(x)) * Fraction(2) ** e


def row_scale(top: float, kind: str) -> float:
    """The scale of a row whose largest value (|h| or h) is top >= 0."""
    least = Fraction(1, 2 ** 126)
    x = Fraction(float(top)) / LEVELS[kind]
    return float(max(cut16(x), least)) if x > least else float(least)


def quantize(h, kind: str):
    """Codes (int64) and scales (float64) of the rows of h; a row that is not
    finite has codes 0 and scale NaN."""
    h = np.asarray(h, np.float64)
    q = np.zeros(h.shape, np.int64)
    s = np.full(h.shape[0], np.nan)
    for i, row in enumerate(h):
        if not np.all(np.isfinite(row)):
            continue
        top = np.max(np.abs(row)) if kind == "signed" else max(np.max(row), 0.0)
        s[i] = row_scale(top, kind)
        # 24-bit over 16-bit numbers: a quotient in 64 bits lies on the right side of every half
        r = np.rint(row / s[i])
        if kind == "relu":
            r = np.where(row > 0, np.maximum(r, 1), 0)
        q[i] = r.astype(np.int64)
    return q, s


def product(q, s, wq, ws):
    """S = s_i ws_j sum_k q_ik wq_jk."""
    return (np.asarray(q, np.int64) @ np.asarray(wq, np.int64).T).astype(np.float64) * s[:, None] * ws[None, :]


def transform_bwd(h, w, g, mask=None, p: float = 0.0):
    """dW = h^T g, dZ = (g w^T) * mask / (1 - p), db = column sums of dZ, for
    the rows h as they are taken back."""
    dw = h.T @ g
    dz = g @ w.T
    if mask is not None:
        dz = np.where(mask, dz / (1.0 - p), 0.0)
    return dw, dz, dz.sum(0)
