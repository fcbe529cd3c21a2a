"""Oracle of a target head of 4-bit weights with group scales: NumPy float64, straight from the definition

    W[k, v] = scale[k // group, v] * (code[k, v] - zero[k // group, v]),   z = h . W.
"""
from __future__ import annotations

import numpy as np


def unpack(codes) -> np.ndarray:
    """uint8 [d / 2, V] -> int64 [d, V]: the low four bits of byte row i belong to hidden index 2 i, the high ones to 2 i + 1."""
    codes = np.asarray(codes, dtype=np.uint8).astype(np.int64)
    out = np.empty((2 * codes.shape[0], codes.shape[1]), np.int64)
    out[0::2], out[1::2] = codes & 15, codes >> 4
    return out


def dequantize(codes, scales, zeros, group: int) -> np.ndarray:
    c = unpack(codes)
    g = np.arange(c.shape[0]) // group
    zero = np.full(np.asarray(scales).shape, 8) if zeros is None else np.asarray(zeros).astype(np.int64) & 15
    return np.asarray(scales, dtype=np.float64)[g] * (c - zero[g])


def logits(hidden, codes, scales, zeros, group: int) -> np.ndarray:
    return np.asarray(hidden, dtype=np.float64) @ dequantize(codes, scales, zeros, group)
