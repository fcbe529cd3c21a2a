"""Windows of thousands of rows, of which a workgroup has several and reads the tokens in front of them."""
import numpy as np
import pytest
import torch

from test_gpu_adjust import _check, _logits, v  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("rows", [[2047], [2049], [4100], [1, 6200, 3], [4097, 4097]])
def test_rows_of_long_windows(v, rows, dtype):  # noqa: F811
    rng = np.random.default_rng(sum(rows))
    V, B, off = 70, len(rows), np.concatenate(([0], np.cumsum(rows))).astype(np.int32)
    M = int(off[-1])
    z = _logits(rng, M, V, dtype)
    window = rng.integers(-1, V + 1, M).astype(np.int32)
    window[rng.random(M) < 0.9] = -1                       # (an id that is said now and then, so that rows differ)
    _check(v, z, row_off=off, window=window, repetition=(1.0 + rng.random(B)).astype(np.float32), frequency=(0.01 * rng.random(B)).astype(np.float32),
           presence=rng.random(B).astype(np.float32), history=rng.integers(-1, V, (B, 5)).astype(np.int32))
