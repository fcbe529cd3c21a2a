"""Oracle of token log-probabilities, entropy and alternatives of rows of logits, and of their gradient: NumPy float64.

Readings: ids at -inf have probability 0 and are no alternatives; a row without any other id has no distribution (logprob -inf, entropy
0); one with a NaN or +inf gives NaN; temperatures that are not above 0 count as 1, those below 2^-126 as that, +inf as the largest
float32; a token of -1 is none (logprob 0), one outside [-1, V) gives NaN; of equal logits the lowest id comes first.
"""
from __future__ import annotations

import numpy as np

LARGEST = float(np.finfo(np.float32).max)


def token_logprobs(Z, tokens, T, n_top: int = 0, given_rows_only: bool = False) -> dict:
    Z = np.asarray(Z, dtype=np.float64)
    M, V = Z.shape
    tokens = np.zeros((M, 0), np.int64) if tokens is None else np.asarray(tokens).reshape(M, -1)
    out = {"logprob": np.zeros(tokens.shape), "entropy": np.zeros(M), "row_max": np.full(M, -np.inf), "row_sumexp": np.zeros(M),
           "top_ids": np.full((M, n_top), -1, np.int64), "top_logprobs": np.full((M, n_top), -np.inf), "lp": np.full((M, V), -np.inf)}
    for m in range(M):
        z, t = Z[m], min(max(float(T[m]), 2.0 ** -126), LARGEST) if T[m] > 0 else 1.0
        given = [(i, int(v)) for i, v in enumerate(tokens[m]) if v != -1]
        for i, v in given:
            if not 0 <= v < V:
                out["logprob"][m, i] = np.nan
        if given_rows_only and not given:
            continue
        given = [(i, v) for i, v in given if 0 <= v < V]
        if np.isnan(z).any() or (z == np.inf).any():
            for i, _ in given:
                out["logprob"][m, i] = np.nan
            out["entropy"][m] = out["row_sumexp"][m] = np.nan
            out["row_max"][m] = np.where(np.isnan(z), -np.inf, z).max()
            out["lp"][m] = np.nan
            continue
        mx = z.max()
        out["row_max"][m] = mx
        if mx == -np.inf:
            for i, _ in given:
                out["logprob"][m, i] = -np.inf
            continue
        with np.errstate(over="ignore", invalid="ignore"):
            lp = (z - mx) / t
        S = np.exp(lp).sum()
        out["row_sumexp"][m] = S
        lp = lp - np.log(S)
        p = np.exp(lp)
        out["lp"][m] = lp
        out["entropy"][m] = -(p[p > 0] * lp[p > 0]).sum()
        for i, v in given:
            out["logprob"][m, i] = lp[v]
        order = [v for v in np.argsort(-z, kind="stable")[:n_top] if z[v] > -np.inf]
        out["top_ids"][m, :len(order)] = order
        out["top_logprobs"][m, :len(order)] = lp[order]
    return out


def token_logprobs_grad(Z, tokens, T, grad_logprob=None, grad_entropy=None, given_rows_only: bool = False) -> np.ndarray:
    Z = np.asarray(Z, dtype=np.float64)
    M, V = Z.shape
    tokens = np.zeros((M, 0), np.int64) if tokens is None else np.asarray(tokens).reshape(M, -1)
    fwd = token_logprobs(Z, tokens, T, given_rows_only=given_rows_only)
    grad = np.zeros((M, V))
    for m in range(M):
        if fwd["row_sumexp"][m] == 0:
            continue
        if np.isnan(fwd["row_sumexp"][m]):
            grad[m] = np.nan
            continue
        t = min(max(float(T[m]), 2.0 ** -126), LARGEST) if T[m] > 0 else 1.0
        lp = fwd["lp"][m]
        p = np.exp(lp)
        G = 0.0
        for i, v in enumerate(tokens[m]):
            if grad_logprob is not None and 0 <= v < V:
                g = float(np.asarray(grad_logprob, dtype=np.float64).reshape(M, -1)[m, i])
                G += g
                grad[m, v] += g
        gH = 0.0 if grad_entropy is None else float(grad_entropy[m])
        some = p > 0
        grad[m, some] -= p[some] * (G + gH * (lp[some] + fwd["entropy"][m]))
        grad[m, Z[m] == -np.inf] = 0.0
        grad[m] /= t
    return grad
