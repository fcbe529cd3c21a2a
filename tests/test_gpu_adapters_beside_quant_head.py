"""Adapters beside a head of 4-bit weights: lm_head with them is lm_head, then what the adapters add."""
import numpy as np
import pytest
import torch

from test_gpu_adapters import DEV, _near, _set

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("M,d,V_t", [(1, 128, 700), (20, 256, 1003), (70, 128, 333)])
def test_lm_head(M, d, V_t):
    from paper_2507_02659_amd.runner import QuantWeights, Verifier
    rng = np.random.default_rng(M)
    codes = torch.from_numpy(rng.integers(0, 256, (d // 2, V_t)).astype(np.uint8)).to(DEV)
    scales = torch.from_numpy((0.01 + 0.02 * rng.random((d // 64, V_t))).astype(np.float32)).bfloat16().to(DEV)
    zeros = torch.from_numpy(rng.integers(0, 16, (d // 64, V_t)).astype(np.uint8)).to(DEV)
    v = Verifier.quantized(QuantWeights(codes, scales, zeros, 64), V_d=1, direct_map=np.zeros(1, np.int32), max_batch=max(M, 1), max_k=0)
    a = _set(rng, 3, 16, d, V_t)
    hidden = torch.from_numpy(rng.standard_normal((M, d)).astype(np.float32)).bfloat16().to(DEV)
    adapter = rng.integers(-1, 3, M).astype(np.int32)
    got = v.lm_head(hidden, adapters=a, adapter_of_row=torch.from_numpy(adapter).to(DEV))
    _near(got, hidden, a, adapter, v.lm_head(hidden))
    v.close()
