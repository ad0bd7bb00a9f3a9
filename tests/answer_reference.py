"""The operators that answer, from their definitions: rows in 8-bit integers, logits and statistics from them, verification of
drafted tokens.  NumPy in 64 bits (integers in exact arithmetic)."""
import math
from fractions import Fraction

import numpy as np


def quantize_rows(x):
    """x: float64 values of the stored elements.  (q, scales) with the quotient 127 x / max |x| in exact arithmetic."""
    q, scales = np.zeros(x.shape, np.int64), np.zeros(x.shape[0], np.float32)
    for i, row in enumerate(x):
        if not np.isfinite(row).all():
            scales[i] = np.nan
            continue
        a = float(np.abs(row).max()) if row.size else 0.0
        scales[i] = np.float32(np.float32(a) / np.float32(127))
        if a:
            q[i] = [round(Fraction(float(v)) * 127 / Fraction(a)) for v in row]      # (round: ties to even)
    return q, scales


def quantize_rows_fast(x):
    """The same for larger matrices of finite rows: the quotient in 64 bits is the exact one where that is a half integer, and on
    its side of one where it is not (127 x has 31 bits, the divisor 24)."""
    a = np.abs(x).max(1)
    q = np.rint(x * 127 / np.where(a > 0, a, 1)[:, None]).astype(np.int64)
    return q, (a.astype(np.float32) / np.float32(127)).astype(np.float32)


def logits(qH, sH, qW, sW):
    return (qH.astype(np.float64) @ qW.astype(np.float64).T) * sH.astype(np.float64)[:, None] * sW.astype(np.float64)


def probabilities(Y, m, s):
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        return np.exp(Y.astype(np.float64) - np.float64(m)) / np.float64(s)


def verify(Y, gmax, gsum, drafts, starts, uniforms, tokens, order, Z=None, zmax=None, zsum=None):
    """Y, Z [N, V]: the logits of the vocabulary's tokens `order` (shards in the order of the call).  tokens: what the output held
    before.  Returns (accepted, tokens, and for each sequence the distance of the draw from the nearest border between two tokens,
    as a share of the whole)."""
    N, V = Y.shape
    place = {int(t): j for j, t in enumerate(order)}
    tokens, accepted, margins = tokens.copy(), [], []
    for b in range(len(starts) - 1):
        first, last = (min(max(int(v), 0), N) for v in (starts[b], starts[b + 1]))
        last -= 1
        if last < first:
            accepted.append(0)
            margins.append(1.0)
            continue
        i = first
        while i < last:
            j = place.get(int(drafts[i]))
            p = 0.0 if j is None else probabilities(Y[i, j], gmax[i], gsum[i])
            q = 1.0 if Z is None or j is None else probabilities(Z[i, j], zmax[i], zsum[i])
            if not float(uniforms[i]) * q < p:
                break
            i += 1
        p = probabilities(Y[i], gmax[i], gsum[i])
        w = p
        if i < last:
            if Z is None:
                w = p.copy()
                if int(drafts[i]) in place:
                    w[place[int(drafts[i])]] = 0.0
            else:
                w = np.maximum(p - probabilities(Z[i], zmax[i], zsum[i]), 0.0)      # (a NaN stays one)
            if not math.isnan(w.sum()) and w.sum() == 0:
                w = p
        token, margin = -1, 1.0
        total = w.sum()
        if np.isfinite(total) and total > 0:
            total = math.fsum(w)
            c = np.cumsum(w)
            t = float(uniforms[last]) * total
            j = int(np.argmax(c > t)) if (c > t).any() else int(np.flatnonzero(w)[-1])
            token = int(order[j])
            margin = float(min(abs(c[j] - t), abs((c[j - 1] if j else 0.0) - t) if w[:j].any() else 1.0) / total)
        tokens[first:i] = drafts[first:i]
        tokens[i] = token
        tokens[i + 1:last + 1] = -1
        accepted.append(i - first)
        margins.append(margin)
    return np.array(accepted, np.int32), tokens, np.array(margins)
