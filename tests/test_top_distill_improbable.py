"""Renormalised distillation where all kept probabilities are too small for 64 bits, as at a teacher's low temperature behind an id without a draft id."""
import numpy as np
import pytest
import torch

from oracle.top_distill import BUCKET, DROP, RENORMALISE, top_distill
from test_gpu_top_distill import DEV, _case, _check, _put, _verifier


def test_oracle():
    rng = np.random.default_rng(0)
    z, ids = rng.standard_normal((3, 9)), np.array([[1, 2, 5], [1, 1, 3], [0, 4, -1]])
    lps = -3.0 * rng.random((3, 3))
    loss, _, grad, _ = top_distill(z, ids, lps, None, RENORMALISE)
    for shift in (700.0, 2.0 ** 14, 2.0 ** 30):
        far = top_distill(z, ids, lps - shift, None, RENORMALISE)
        assert (far[1] < 1e-300).all()
        np.testing.assert_allclose(far[0].astype(float), loss.astype(float), atol=2.0 ** -50 * shift)
        np.testing.assert_allclose(far[2].astype(float), grad.astype(float), atol=2.0 ** -50 * shift)


@pytest.fixture(scope="module")
def v():
    ver = _verifier()
    yield ver
    ver.close()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,n", [(50, 1), (300, 5), (900, 65), (9000, 256), (40003, 130), (70001, 20)])
def test_sums_below_64_bits(v, V, n, dtype):
    rng = np.random.default_rng(V)
    z, ids, lps = _case(rng, 12, V, n, dtype)
    lps = np.maximum(lps, -20.0)
    for m, shift in enumerate((590.0, 610.0, 700.0, 740.0, 760.0, 5000.0, 2.0 ** 17)):
        lps[m] -= np.float32(shift)
    lps[7] = -np.inf
    ids[8] = -1
    lps[9] = np.finfo(np.float32).min
    lps[10] -= 3000.0
    lps[10, n // 2] = np.nan
    lps[11] -= 900.0
    lps[11, n - 1] = -1000.0 - 2000.0 * rng.random()
    ids[5, n // 2:] = ids[5, 0]                            # named many times
    T, g = 0.3 + rng.random(12), rng.standard_normal(12).astype(np.float32)
    got = _check(v, z, ids, lps, T, RENORMALISE, g)
    for m in (1, 2, 3, 4, 5, 6, 9, 11):                    # the gradient of a distribution: it says something, and adds up to 0
        assert float(got["kept"][m]) == 0 and float(got["grad"][m].abs().max()) > 0
    assert float(got["loss"][7]) == 0 and (got["grad"][7] == 0).all()
    for rest in (DROP, BUCKET):
        _check(v, z, ids, lps, T, rest, g)


@pytest.mark.gpu
def test_a_shift_of_the_log_probabilities(v):
    """Log-probabilities that float32 holds exactly with and without the shift: the same loss and gradient."""
    rng = np.random.default_rng(3)
    z, ids, lps = _case(rng, 6, 2000, 100)
    lps = np.float32(np.round(np.maximum(lps, -15.0) * 256) / 256)
    near = v.top_distill_loss_grad(z, _put(ids), _put(lps), rest=RENORMALISE)
    far = v.top_distill_loss_grad(z, _put(ids), _put(lps - np.float32(4096.0)), rest=RENORMALISE)
    # formed in 64 bits from sums that differ by a few of their roundings, then rounded once
    assert float((near["loss"] - far["loss"]).abs().max()) <= 2.0 ** -22 * (1 + float(near["loss"].abs().max()))
    assert float((near["grad"] - far["grad"]).abs().max()) <= 2.0 ** -23
