"""Oracle of the distillation loss from a teacher's top logits and of its gradient: NumPy long double.

Readings: an id of -1, or a target id without a draft id, is none; rows without ids add nothing; an id outside the vocabulary, a NaN or +inf
among a row's kept log-probabilities or its logits makes loss and gradient NaN; a row that the student masks whole adds nothing; ids at -inf
get no gradient; temperatures as in oracle/logprobs.py; where a student's other ids have no probability in 64 bits, a remainder of up to 2^-20 is
the rounding of the log-probabilities and counts as 0.
"""
from __future__ import annotations

import numpy as np

DROP, RENORMALISE, BUCKET = 0, 1, 2
F = np.longdouble


def top_distill(Z, top_ids, top_logprobs, T=None, rest=DROP, grad_loss=None, tmap=None):
    """(loss [M], kept [M], gradient [M, V], and per row the largest size of the gradient's parts, [M, V]) in long double."""
    Z = np.asarray(Z, F)
    M, V = Z.shape
    loss, kept, grad, size = np.zeros(M, F), np.zeros(M, F), np.zeros((M, V), F), np.zeros((M, V), F)
    for m in range(M):
        t = 1.0 if T is None or not T[m] > 0 else min(max(F(T[m]), F(2) ** -126), F(np.finfo(np.float32).max))
        g = F(1) if grad_loss is None else F(grad_loss[m])
        pairs, broken = [], False
        for v, lp in zip(top_ids[m], top_logprobs[m]):
            v, lp = int(v), F(lp)
            if v < -1 or v >= (V if tmap is None else len(tmap)):
                broken = True
            elif v >= 0 and (tmap is None or tmap[v] >= 0):
                pairs.append((v if tmap is None else int(tmap[v]), lp))
        broken = broken or any(np.isnan(lp) or lp == np.inf for _, lp in pairs)
        z = Z[m]
        if not broken and not pairs:
            continue
        if broken or np.isnan(z).any() or (z == np.inf).any():
            loss[m] = grad[m] = np.nan
            kept[m] = np.nan if broken else sum(np.exp(lp) for _, lp in pairs)
            continue
        P = sum(np.exp(lp) for _, lp in pairs)
        kept[m] = P
        if z.max() == -np.inf:
            continue
        with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
            e = np.exp((z - z.max()) / t)
            lnS = np.log(e.sum())
            lq = (z - z.max()) / t - lnS
            q = np.exp(lq)
            shift = max(lp for _, lp in pairs) if rest == RENORMALISE else F(0)      # (p / P is that of any common factor)
            shift = shift if shift > -np.inf else F(0)
            norm = sum(np.exp(lp - shift) for _, lp in pairs) if rest == RENORMALISE else F(1)
            own = np.zeros(V, F)
            ids = np.zeros(V, bool)
            for v, lp in pairs:
                ids[v] = True
                if np.exp(lp - shift) > 0 and norm > 0:
                    loss[m] += np.exp(lp - shift) / norm * (lp - shift - np.log(norm) - lq[v])
                    own[v] += np.exp(lp - shift) / norm
            if rest == BUCKET:
                left = max(F(0), 1 - P)
                others = np.where(ids, -np.inf, (z - z.max()) / t)
                top = others.max()
                if left <= F(2) ** -20 and np.exp(np.float64(top)) == 0:
                    left = F(0)
                inside = np.where(others > -np.inf, np.exp(others - (top if top > -np.inf else 0)), 0)
                if left > 0:
                    loss[m] += left * (np.log(left) - (top + np.log(inside.sum()) - lnS if top > -np.inf else -np.inf))
                back = left * inside / (inside.sum() if top > -np.inf else 1)
                mass = F(1) if left > 0 else P
                d, parts = mass * q - own - back, mass * q + own + back
            else:
                mass = P if rest == DROP else F(norm > 0)
                d, parts = mass * q - own, mass * q + own
            d[z == -np.inf] = 0
            grad[m], size[m] = d * g / t, np.abs(parts * g / t)
    return loss, kept, grad, size
