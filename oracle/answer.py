"""Float64 reference of the answering operators: row quantisation, 8-bit products, log probabilities.

Written from the formulas in include/horizon.h, with NumPy alone.
"""
from __future__ import annotations

from fractions import Fraction
from typing import Dict, Optional

import numpy as np


def quantize_rows(x: np.ndarray, gain: Optional[np.ndarray], eps: float):
    """x [rows, d] (any float type; its values are taken exactly) -> (q int8, scale float64).

    The integers are those of exact arithmetic: a quotient within 2^-40 of a border is decided in
    rational numbers."""
    x = np.asarray(x, np.float64)
    y = x if gain is None else x * np.asarray(gain, np.float64)   # 24 + 8 bits: exact
    q = np.zeros(x.shape, np.int8)
    scale = np.zeros(x.shape[0])
    for r in range(x.shape[0]):
        if not np.all(np.isfinite(y[r])) or not np.all(np.isfinite(x[r])):
            scale[r] = np.nan
            continue
        a = np.max(np.abs(y[r]))
        if a == 0:
            continue
        t = 127.0 * (y[r] / a)
        v = np.rint(t)
        for i in np.flatnonzero(np.abs(np.abs(t - np.floor(t)) - 0.5) < 2.0 ** -40):
            v[i] = round(127 * Fraction(float(y[r, i])) / Fraction(float(a)))   # half to even
        q[r] = v
        scale[r] = a / 127.0
        if gain is not None:
            scale[r] /= np.sqrt(np.mean(x[r] * x[r]) + eps)
    return q, scale


def linear_i8(a, a_scale, w, w_scale, bias, out_dtype=np.float32) -> np.ndarray:
    """The documented roundings, in order, in float32 (bit-exact before the last rounding)."""
    acc = np.asarray(a, np.float64) @ np.asarray(w, np.float64).T   # integers below 2^31: exact
    with np.errstate(over="ignore", invalid="ignore"):
        v = acc.astype(np.float32) * (np.asarray(a_scale, np.float32)[:, None] * np.asarray(w_scale, np.float32))
        if bias is not None:
            v = v + np.asarray(bias, np.float32)
        return v.astype(out_dtype)


def logprobs(z: np.ndarray, tokens: Optional[np.ndarray], top_k: int) -> Dict[str, np.ndarray]:
    """z [rows, vocab].  Also returns what an error bound needs: the sums s = sum over all but one largest
    token of e^(z - m), t1 = sum p |z - m| and t2 = sum p (z - m)^2."""
    z = np.asarray(z, np.float64)
    rows, vocab = z.shape
    n = 0 if tokens is None else tokens.shape[1]
    out = {"token": np.zeros((rows, n)), "entropy": np.zeros(rows), "top": np.full((rows, top_k), -np.inf),
           "top_tokens": np.full((rows, top_k), -1, np.int32), "s": np.zeros(rows), "t1": np.zeros(rows),
           "t2": np.zeros(rows)}
    for r in range(rows):
        bad = bool(np.any(np.isnan(z[r])) or np.any(z[r] == np.inf))
        seen = np.flatnonzero(z[r] > -np.inf) if not bad else np.zeros(0, int)
        lp = np.full(vocab, np.nan if bad else -np.inf)
        if bad:
            out["entropy"][r] = np.nan
            out["top"][r] = np.nan
        elif len(seen):
            at = seen[np.lexsort((seen, -z[r, seen]))]      # by value, then by token
            d = z[r, at] - z[r, at[0]]
            e = np.exp(d)
            s = e[1:].sum()
            lp[at] = d - np.log1p(s)
            p = e / (1 + s)
            out["entropy"][r] = np.log1p(s) - (p * d).sum()
            out["s"][r], out["t1"][r], out["t2"][r] = s, (p * -d).sum(), (p * d * d).sum()
            k = min(top_k, len(at))
            out["top_tokens"][r, :k] = at[:k]
            out["top"][r, :k] = lp[at[:k]]
        for j in range(n):
            t = int(tokens[r, j])
            out["token"][r, j] = 0.0 if t == -1 else lp[t] if 0 <= t < vocab else np.nan
    return out
