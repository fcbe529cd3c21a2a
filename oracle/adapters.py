"""Oracle of low-rank adapters beside a head: NumPy float64, row by row.

Readings: a row's adapter of -1 is none; one outside [-1, n) makes the row NaN; both matrices are [outputs, inputs].
"""
from __future__ import annotations

import numpy as np


def adapter_logits(hidden, down, up, scale, adapter, logits=None) -> np.ndarray:
    hidden, down, up = (np.asarray(x, np.float64) for x in (hidden, down, up))
    n, V = up.shape[0], up.shape[1]
    out = np.zeros((hidden.shape[0], V)) if logits is None else np.array(logits, np.float64)
    for m, a in enumerate(adapter):
        if a == -1:
            continue
        if not 0 <= a < n:
            out[m] = np.nan
            continue
        out[m] += (1.0 if scale is None else float(scale[a])) * (up[a] @ (down[a] @ hidden[m]))
    return out
