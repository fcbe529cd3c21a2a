"""Oracle of penalties, biases and masks on rows of logits: NumPy float64, id by id.

Readings: repetition looks at prompt, output and the window's tokens in front of the row, the other two at output and window; of equal bias ids
the last entry counts; an id at -inf stays there; ids outside the vocabulary are none; a mask index outside [-1, n) makes the row NaN.
"""
from __future__ import annotations

from collections import Counter

import numpy as np


def adjust_logits(z, row_off=None, history=None, n_history=None, n_prompt=None, window=None, repetition=None, frequency=None, presence=None,
                  bias_ids=None, bias=None, masks=None, mask_of_row=None) -> np.ndarray:
    z = np.array(z, np.float64)
    M, V = z.shape
    off = np.arange(M + 1) if row_off is None else np.asarray(row_off)
    for b in range(len(off) - 1):
        ids = [] if history is None else [int(i) for i in history[b][:max(0, len(history[b]) if n_history is None else int(n_history[b]))]]
        first = max(0, 0 if n_prompt is None else int(n_prompt[b]))
        biases = {} if bias_ids is None else {int(i): float(x) for i, x in zip(bias_ids[b], bias[b])}
        rho, f, g = (d if x is None else float(x[b]) for x, d in ((repetition, 1.0), (frequency, 0.0), (presence, 0.0)))
        for row in range(max(0, off[b]), min(M, off[b + 1])):
            before = [] if window is None else [int(i) for i in window[off[b]:row]]
            seen, said = set(ids + before), Counter(ids[first:] + before)
            for v in seen | set(biases):
                if not 0 <= v < V or z[row, v] == -np.inf:
                    continue
                x = z[row, v]
                if v in seen:
                    x = x / rho if x > 0 else x * rho
                if said[v]:
                    x = x - f * said[v] - g
                z[row, v] = x + biases.get(v, 0.0)
            m = -1 if masks is None else row if mask_of_row is None else int(mask_of_row[row])
            if m < -1 or (m >= 0 and m >= len(masks)):
                z[row] = np.nan
            elif m >= 0:
                words = np.asarray(masks[m]).astype(np.int64) & 0xFFFFFFFF
                bits = (words[:, None] >> np.arange(32)) & 1
                z[row][bits.ravel()[:V] == 0] = -np.inf
    return z
