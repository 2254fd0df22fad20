"""Float64 reference of decoding on a shared cache: selection over beams, copies of
cache positions, attention of one row a sequence behind a shared prefix.

Each function comes straight from the definition and also returns what a test needs
to bound a kernel's roundings.
"""
from __future__ import annotations

import numpy as np


def beam_values(logits, scores, finished=None, end_token=-1):
    """value(b, t) = score[b] + z[b, t] - log sum e^z of one group: float64 [beams, vocab], -inf for no continuation.

    Also, per beam, the mean distance of its tokens from the largest logit under its distribution."""
    z = np.asarray(logits, np.float64)
    scores = np.asarray(scores, np.float64)
    values = np.full(z.shape, -np.inf)
    distance = np.zeros(len(z))
    for b in range(len(z)):
        if not scores[b] > -np.inf:
            continue
        if finished is not None and finished[b]:
            values[b, end_token] = scores[b]
            continue
        if np.any(np.isnan(z[b])) or np.any(z[b] == np.inf) or np.all(z[b] == -np.inf):
            continue
        m = z[b].max()
        with np.errstate(invalid="ignore"):
            d = z[b] - m
            e = np.exp(d)
            values[b] = scores[b] + (d - np.log(e.sum()))
            distance[b] = np.nansum(np.where(e > 0, -d * e, 0)) / e.sum()
    return values, distance


def beam_select(values, logits, n_select):
    """The n_select best (value, beam, token) of one group: by value, then beam, then token; a beam's own by logit."""
    beams, vocab = values.shape
    best = []
    for b in range(beams):
        order = np.lexsort((np.arange(vocab), -np.asarray(logits[b], np.float64), -values[b]))[:n_select]
        best += [(-values[b, t], b, i, int(t)) for i, t in enumerate(order) if values[b, t] > -np.inf]
    best.sort(key=lambda c: c[:3])
    out = [(-v, b, t) for v, b, _, t in best[:n_select]]
    return out + [(-np.inf, -1, -1)] * (n_select - len(out))


def cache_positions(k, v, slots, positions):
    """Logical rows [len, hkv, dh] of `positions` in the slots that hold them: k [n_slots, hkv, page, dh], v in tiles
    [n_slots, hkv, page / 32, dh, 32]."""
    return k[slots, :, positions], v[slots, :, positions // 32, :, positions % 32]


def prefix_attention(q, k, v, table, lens, offsets, prefix):
    """(o, a, weakest) for q [n, hq, dh], one layer's cache, host arrays.

    o [n, hq, dh]; a the same with |v| in place of v (what relative errors of weights are scaled by); slack [n, hq]: what
    an error of one step in the smallest numbers of fp16, of each weight below 2^-14, adds up to."""
    n, hq, dh = q.shape
    hkv, page = k.shape[1], k.shape[2]
    o, a, slack = np.zeros(q.shape), np.zeros(q.shape), np.zeros((n, hq))
    for i in range(n):
        groups = [g for g in range(len(prefix)) if offsets[g] <= i < offsets[g + 1]]
        p = int(prefix[groups[0]]) if groups else 0
        owner = offsets[groups[0]] if groups else i
        at = np.arange(int(lens[i]))
        if len(at) == 0:
            continue
        slots = np.where(at < p, table[owner][np.minimum(at // page, len(table[owner]) - 1)], table[i][at // page])
        keys, values = (x.astype(np.float64) for x in cache_positions(k, v, slots, at % page))
        for h in range(hq):
            g = h // (hq // hkv)
            s = keys[:, g] @ q[i, h].astype(np.float64) / np.sqrt(dh)
            w = np.exp(s - s.max())
            o[i, h] = w @ values[:, g] / w.sum()
            a[i, h] = w @ np.abs(values[:, g]) / w.sum()
            slack[i, h] = len(at) * 2.0 ** -25 * np.abs(values[:, g]).max() / w.sum()
    return o, a, slack
