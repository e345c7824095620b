"""Definitions, in float64, of the operators on coded matrices and of the policy from
logits.  Shares nothing with the library.
"""

from __future__ import annotations

import numpy as np

from .az_oracle import e4m3_decode, e4m3_round, softmax_legal

BLOCK = 128
NAN_CODE = 0x7F
TABLE = np.array([e4m3_decode(c) for c in range(256)], dtype=np.float64)
_FINITE = np.array([c for c in range(256) if np.isfinite(TABLE[c])])


def spread(scales, rows, cols, scale_rows):
    """An entry's block's scale byte for each entry."""
    s = np.repeat(np.asarray(scales), BLOCK, axis=1)[:, :cols]
    return np.repeat(s, scale_rows, axis=0)[:rows]


def scale_exponent(a):
    """The smallest e with a <= 448 * 2^e, in -117..119; 0 for a = 0."""
    if a == 0.0:
        return 0
    e = -200
    while a > 448.0 * 2.0 ** e:
        e += 1
    return min(max(e, -117), 119)


def encode(v):
    """Bytes of values on the e4m3 grid; the sign of a zero is kept."""
    order = np.argsort(TABLE[_FINITE], kind="stable")
    codes, values = _FINITE[order], TABLE[_FINITE][order]
    at = codes[np.searchsorted(values, v)]
    assert np.array_equal(TABLE[at], v)
    return np.where(v == 0, np.where(np.signbit(v), 0x80, 0x00), at).astype(np.uint8)


def quantize(x, scale_rows=1):
    """(codes [rows][cols], scales) of x, both uint8."""
    x = np.asarray(x, dtype=np.float64)
    rows, cols = x.shape
    scales = np.zeros((-(-rows // scale_rows), -(-cols // BLOCK)), np.uint8)
    size = np.where(np.isfinite(x), np.abs(x), 0.0)
    for i in range(scales.shape[0]):
        for j in range(scales.shape[1]):
            a = size[i * scale_rows:(i + 1) * scale_rows, j * BLOCK:(j + 1) * BLOCK].max()
            scales[i, j] = scale_exponent(a) + 127
    z = np.where(np.isfinite(x), x, 0.0) * 2.0 ** -(spread(scales, rows, cols, scale_rows).astype(np.float64) - 127)
    codes = encode(np.copysign(e4m3_round(np.clip(z, -448.0, 448.0)), z))
    return np.where(np.isfinite(x), codes, NAN_CODE).astype(np.uint8), scales


def value(codes, scales, scale_rows=1):
    codes = np.asarray(codes)
    s = spread(scales, *codes.shape, scale_rows).astype(np.float64)
    return TABLE[codes] * np.where(s == 255, np.nan, 2.0 ** (s - 127))


def adjusted_logits(logits, allowed=None, bias=None, history=None, lengths=None, penalties=None):
    """history: list of sequences of entries per row."""
    l = np.array(logits, dtype=np.float64)
    rows, vocab = l.shape
    if history is not None:
        for b in range(rows):
            h = np.asarray(history[b])[:max(0, lengths[b])] if lengths is not None else np.asarray(history[b])
            h = h[(h >= 0) & (h < vocab)]
            c = np.bincount(h, minlength=vocab) if h.size else np.zeros(vocab, int)
            r, f, p = (float(v) for v in penalties[b])
            with np.errstate(invalid="ignore"):
                l[b] = np.where(c > 0, np.where(l[b] > 0, l[b] / r, l[b] * r) - (f * c + p), l[b])
    if bias is not None:
        l = l + np.asarray(bias, dtype=np.float64)
    if allowed is not None:
        l = np.where(np.asarray(allowed) != 0, l, -np.inf)
    return l


def policy(logits, allowed=None, **kw):
    """The policy: softmax over the allowed entries, zero elsewhere and in a row without one."""
    l = adjusted_logits(logits, allowed, **kw)
    return softmax_legal(l, l > -np.inf)
