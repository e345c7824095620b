"""Definitions, in float64, of the operators around a dense layer: the norm with its gradients, matrices in 4 bits, and
the entry drawn from logits.  Shares nothing with the library.
"""

from __future__ import annotations

import math

import numpy as np

BLOCK = 32
SIZES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
TABLE = np.concatenate([SIZES, -SIZES])


# --------------------------------------------------------------------------- #
# Norm
# --------------------------------------------------------------------------- #
def norm(h, weight=None, eps=1e-6):
    """(y, 1 / root) of rows h."""
    h = np.asarray(h, dtype=np.float64)
    r = 1.0 / np.sqrt(np.mean(h * h, axis=1, keepdims=True) + eps)
    return h * r * (1.0 if weight is None else np.asarray(weight, np.float64)), r


def norm_grad(dy, h, weight=None, dsum=None, eps=1e-6):
    """(dx, dweight)."""
    dy, h = np.asarray(dy, np.float64), np.asarray(h, np.float64)
    r = norm(h, None, eps)[1]
    g = dy if weight is None else dy * np.asarray(weight, np.float64)
    dx = r * g - r ** 3 * h * np.mean(g * h, axis=1, keepdims=True)
    return dx + (0.0 if dsum is None else np.asarray(dsum, np.float64)), np.sum(dy * h * r, axis=0)


# --------------------------------------------------------------------------- #
# 4 bits
# --------------------------------------------------------------------------- #
def scale_exponent(a):
    """The smallest e with a <= 6 * 2^e, in -125..125; 0 for a = 0."""
    if a == 0.0:
        return 0
    e = -200
    while a > 6.0 * 2.0 ** e:
        e += 1
    return min(max(e, -125), 125)


def nearest(v):
    """Codes of the nearest sizes to v, |v| <= 6, ties to the even code; the sign of a zero is kept."""
    size = np.abs(v)
    hi = np.searchsorted(SIZES, size).clip(1, 7)
    lo = hi - 1
    a, b = size - SIZES[lo], SIZES[hi] - size
    code = np.where(a < b, lo, np.where(b < a, hi, np.where(lo % 2 == 0, lo, hi)))
    return (code | np.where(np.signbit(v), 8, 0)).astype(np.uint8)


def quantize(x):
    """(codes [rows][cols], one to a byte, scales [rows][blocks]) of x."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    codes, scales = np.zeros((rows, cols), np.uint8), np.zeros((rows, -(-cols // BLOCK)), np.uint8)
    for i in range(rows):
        for j in range(scales.shape[1]):
            at = slice(j * BLOCK, min(cols, (j + 1) * BLOCK))
            b = x[i, at]
            if not np.all(np.isfinite(b)):
                scales[i, j] = 255
                continue
            e = scale_exponent(np.abs(b).max())
            scales[i, j] = e + 127
            codes[i, at] = nearest(np.clip(b * 2.0 ** -e, -6.0, 6.0))
    return codes, scales


def packed(codes):
    """Two codes to a byte, the even column in the low half; an odd row's last high half is zero."""
    rows, cols = codes.shape
    c = np.concatenate([codes, np.zeros((rows, cols % 2), np.uint8)], axis=1)
    return c[:, 0::2] | c[:, 1::2] << 4


def value(codes, scales):
    s = np.repeat(np.asarray(scales).astype(np.float64), BLOCK, axis=1)[:, :codes.shape[1]]
    return TABLE[codes] * np.where(s == 255, np.nan, 2.0 ** (s - 127))


# --------------------------------------------------------------------------- #
# Drawing
# --------------------------------------------------------------------------- #
def kept(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(entries that stay, by rising index; their weights), both empty where nothing can be drawn; and how near the nearest
    decision was to going the other way, in parts of the whole sum."""
    l = np.asarray(logits, dtype=np.float64)
    if np.any(np.isnan(l)) or np.any(l == np.inf) or not np.any(l > -np.inf):
        return np.zeros(0, int), np.zeros(0), 1.0
    order = np.argsort(-l, kind="stable")
    if not temperature > 0:
        return order[:1], np.ones(1), 1.0
    with np.errstate(over="ignore"):
        w = np.exp((l[order] - l.max()) / temperature)
    w[l[order] == -np.inf] = 0.0
    n, near = len(l), 1.0
    if 0 < top_k < n:
        n = top_k
    w = w[:n]
    if top_p < 1.0:
        total = math.fsum(w)
        before = np.concatenate([[0.0], np.cumsum(w)[:-1]])
        stay = max(1, int(np.sum(before < top_p * total)))
        near = min(near, np.abs(before[1:] / total - top_p).min(initial=1.0))
        w = w[:stay]
    if min_p > 0:
        stay = w >= min(min_p, 1.0)
        near = min(near, np.abs(w - min(min_p, 1.0))[1:].min(initial=1.0))
        w = w[:max(1, int(stay.sum()))]
    at = np.sort(order[:len(w)])
    back = np.argsort(order[:len(w)], kind="stable")
    return at, w[back], near


def draw(logits, u, **kw):
    """(entry, its probability, how near the decision was)."""
    at, w, near = kept(logits, **kw)
    if len(at) == 0:
        return -1, 0.0, near
    sums = np.cumsum(w)
    i = min(int(np.searchsorted(sums, u * sums[-1], side="right")), len(at) - 1)
    near = min(near, np.abs(sums[:-1] / sums[-1] - u).min(initial=1.0))
    return int(at[i]), float(w[i] / sums[-1]), near
