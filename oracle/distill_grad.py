"""Oracle of the hybrid distillation loss's gradient with respect to the drafter's logits: token by token from the derivative of every
term (oracle/distill.py has the terms themselves), in NumPy's long double: with a drafter that is sure of its token, q(d_1) - pi and 1 - q
are differences of numbers next to 1, of which 64 bits leave little.
"""
from __future__ import annotations

import numpy as np

from .verify import inverse_map, map_merge, widen


def _log_softmax(z, T):
    z = np.asarray(z, dtype=np.longdouble) / T
    z = z - z.max()
    return z - np.log(np.exp(z).sum())


def hybrid_loss_grad(*, row_off, draft_ids, draft_logits, direct_map, V_t, cache, max_ngram_len, temperature, target_logits,
                     draft_temperature=None, dtype="f32", lam=0.2, lambda_mode="fixed", ngram_term="nll", n_accept=None, grad_loss=1.0):
    """(gradient [K, V_d], scale [K, V_d], soft [K, V_d]), the last two for tolerances.  `scale` bounds the terms that an element is the sum
    of.  `soft` is what an error of 2^-23 in each ln q does to an element through ln(q(d_1) - pi): the difference is then off by up to
    L 2^-23 q(d_1), which next to a tiny difference (a drafter sure of every sub-token) is a large change of its logarithm, or takes the
    difference to 0 and its term away."""
    Zq, Z = widen(draft_logits, dtype), np.asarray(target_logits, dtype=np.float64)
    dmap = np.asarray(direct_map)
    tmap = inverse_map(dmap, V_t)
    mapped = np.flatnonzero(dmap >= 0)
    grad, scale, soft, n = np.zeros(Zq.shape), np.zeros(Zq.shape), np.zeros(Zq.shape), 0
    for b in range(len(row_off) - 1):
        r0, q0 = int(row_off[b]), int(row_off[b]) - b
        k = int(row_off[b + 1]) - r0 - 1
        T = float(temperature[b])
        Td = T if draft_temperature is None else float(draft_temperature[b])
        if T <= 0 or Td <= 0:
            continue
        d = [int(x) for x in draft_ids[q0:q0 + k]]
        if any(not 0 <= x < Zq.shape[1] for x in d):
            continue
        tokens, spans, _, _ = map_merge(d, dmap, cache, max_ngram_len)
        for j, (t, (s, L)) in enumerate(zip(tokens, spans)):
            if L > 1 and n_accept is not None and j >= int(n_accept[b]):
                continue
            n += L
            lp = _log_softmax(Z[r0 + j], T)
            lq = [_log_softmax(Zq[q0 + s + i], Td) for i in range(L)]
            w = 1.0 if L == 1 else (np.float64(np.float32(lam)) if lambda_mode == "fixed" else np.exp(lp[t]))
            with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
                a = np.zeros(Zq.shape[1], np.longdouble)   # dTerm / dq(i) of the first row through q'
                a[mapped] = np.where(lq[0][mapped] > -np.inf, lq[0][mapped] - lp[dmap[mapped]] + 1.0, 0.0)
                push, loose = 0.0, 0.0                   # dTerm / dlog pi; uncertainty of ln(q(d_1) - pi)
                if L > 1 and ngram_term == "nll":
                    a[:] = 0.0
                    push = -1.0
                elif L > 1:
                    ln_pi = sum(lq[i][d[s + i]] for i in range(L))
                    pi = np.exp(ln_pi)
                    rest = -np.exp(lq[0][d[s]]) * np.expm1(ln_pi - lq[0][d[s]])
                    if tmap[t] >= 0:
                        a[tmap[t]] = 0.0
                    by_pi = ln_pi - lp[t] + 1.0 if pi > 0 else 0.0
                    pre = int(dmap[d[s]])
                    if pre >= 0 and pre != t:
                        a[d[s]] = np.log(rest) - lp[pre] + 1.0 if rest > 0 else 0.0
                        by_pi -= a[d[s]]
                        x = L * 2.0 ** -23 * np.exp(lq[0][d[s]]) / rest if rest > 0 else 1.0
                        loose = float(max(np.log1p(x), np.abs(a[d[s]]) if x > 0.5 else 2 * x))
                    push = pi * by_pi
                q = np.exp(lq[0])
                A = np.where(q > 0, q * a, 0.0).sum()
                grad[q0 + s] += w / Td * np.where(q > 0, q * (a - A), 0.0)
                scale[q0 + s] += w / Td * q * (1.0 + np.abs(a) + abs(A))
                if loose:
                    soft[q0 + s] += w / Td * q * q[d[s]] * loose
                    soft[q0 + s, d[s]] += w / Td * q[d[s]] * loose
                for i in range(L if L > 1 else 0):
                    one = np.zeros(Zq.shape[1])
                    one[d[s + i]] = 1.0
                    off = -np.exp(lq[i])
                    off[d[s + i]] = -np.expm1(lq[i][d[s + i]])
                    grad[q0 + s + i] += w / Td * push * off
                    scale[q0 + s + i] += w / Td * (abs(push) + (0.0 if ngram_term == "nll" else pi * (1 + abs(ln_pi)))) * (one + np.exp(lq[i]))
                    soft[q0 + s + i] += w / Td * (pi * loose if loose else 0.0) * (one + np.exp(lq[i]))
    up = grad_loss / max(1, n)
    return grad * up, scale * abs(up), soft * abs(up)


def hybrid_loss_grad_case(case, **kw):
    """The same on a workloads.VerifyCase (target logits of a case with hidden states: the oracle's product)."""
    from .verify import build_cache, lm_head_logits
    Z = case.target_logits
    if Z is None:
        Z = lm_head_logits(case.hidden, case.W, case.dtype)
    cache = build_cache(case.ngram_key_off, case.ngram_key_ids, case.ngram_target_ids)
    return hybrid_loss_grad(row_off=case.row_off, draft_ids=case.draft_ids, draft_logits=case.draft_logits, direct_map=case.direct_map,
                            V_t=case.V_t, cache=cache, max_ngram_len=case.max_ngram_len, temperature=case.temperature,
                            draft_temperature=case.draft_temperature, dtype=case.dtype, target_logits=Z, **kw)
