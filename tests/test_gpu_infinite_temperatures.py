"""A temperature of +inf: a uniform distribution over the ids that are not masked."""
import numpy as np
import pytest
import torch

from oracle.logprobs import token_logprobs
from oracle.top_distill import BUCKET, DROP, RENORMALISE
from test_gpu_top_distill import DEV, _case, _check, _put, _verifier

pytestmark = pytest.mark.gpu
INF = float("inf")


@pytest.fixture(scope="module")
def v():
    ver = _verifier()
    yield ver
    ver.close()


@pytest.mark.parametrize("rest", [DROP, RENORMALISE, BUCKET])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [50, 9000, 70001])
def test_distillation(v, V, dtype, rest):
    rng = np.random.default_rng(V)
    z, ids, lps = _case(rng, 6, V, 20, dtype)
    z[1, torch.from_numpy(rng.random(V) < 0.5).to(DEV)] = -INF
    z[2, ids[2, 0]] = -INF
    z[3] = -INF
    lps[2, 0] = -np.inf
    got = _check(v, z, ids, lps, np.float32([INF, INF, INF, INF, np.finfo(np.float32).max, 1.0]), rest, rng.standard_normal(6).astype(np.float32))
    assert not got["loss"].isnan().any() and not got["grad"].isnan().any()
    p = np.exp(lps[0].astype(np.float64))
    p = p / p.sum() if rest == RENORMALISE else p
    want = (p * (np.log(p) + np.log(V))).sum()
    if rest == BUCKET and p.sum() < 1:
        want += (1 - p.sum()) * (np.log(1 - p.sum()) - np.log(1 - 20 / V))
    assert float(got["loss"][0]) == pytest.approx(want, rel=1e-5, abs=1e-5)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [50, 9000, 70001])
def test_log_probabilities(v, V, dtype):
    rng = np.random.default_rng(V)
    z, _, _ = _case(rng, 4, V, 1, dtype)
    z[1, torch.from_numpy(rng.random(V) < 0.5).to(DEV)] = -INF
    z[2, 1:] = -INF
    z[3] = -INF
    z[:3, 0] = 0.5
    T, tokens = np.full(4, INF, np.float32), np.array([[0, V - 1]] * 4, np.int32)
    want = token_logprobs(z.double().cpu().numpy(), tokens, T, 3)
    got = v.token_logprobs(z, tokens=_put(tokens), temperature=_put(T), n_top=3)
    n = (z > -INF).sum(1).double().cpu().numpy()
    for name in ("logprob", "entropy", "top_logprobs"):
        # every exponential is 1: ln n, formed in 64 bits, rounded to float32
        np.testing.assert_allclose(got[name].double().cpu().numpy(), want[name], rtol=2.0 ** -22, atol=2.0 ** -22)
    np.testing.assert_allclose(got["entropy"].double().cpu().numpy(), np.log(np.maximum(n, 1)), rtol=2.0 ** -22, atol=2.0 ** -22)
    assert np.array_equal(got["top_ids"].cpu().numpy(), want["top_ids"])
    ones = torch.ones(4, device=DEV)
    grad = v.token_logprobs_grad(z, _put(tokens), got, grad_logprob=torch.ones(4, 2, device=DEV), grad_entropy=ones, temperature=_put(T))
    assert float(grad.abs().max()) <= 100 * 2.0 ** -128     # (a NaN is not)
