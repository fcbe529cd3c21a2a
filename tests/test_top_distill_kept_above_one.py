"""Distillation from top logits where the kept probabilities add up to more than 1: ids that are named twice, log-probabilities stored in few bits."""
import numpy as np
import pytest
import torch

from oracle.top_distill import BUCKET, DROP, RENORMALISE, top_distill
from test_gpu_top_distill import DEV, _check, _put, _verifier

RESTS = [DROP, RENORMALISE, BUCKET]


def _rows(rng, M, V, n):
    """Probabilities that add up to 1 to 2 (of the first row to a little above 1), in every second row of an id that is named twice."""
    ids = np.stack([rng.permutation(V)[:n] for _ in range(M)]).astype(np.int32)
    ids[::2, 1] = ids[::2, 0]
    total = 1.0 + rng.random(M)
    total[0] = 1.0 + 2.0 ** -9
    lps = np.log(rng.dirichlet(np.ones(n), M) * total[:, None]).astype(np.float32)
    return 2.0 * rng.standard_normal((M, V)).astype(np.float32), ids, lps


@pytest.mark.parametrize("rest", RESTS)
def test_oracle_against_differences(rest):
    rng = np.random.default_rng(rest)
    z, ids, lps = _rows(rng, 4, 9, 4)
    z = z.astype(np.longdouble)
    T, g = np.array([1.0, 0.3, 2.0, 0.7]), rng.standard_normal(4)
    _, kept, grad, _ = top_distill(z, ids, lps, T, rest, g)
    assert (kept > 1).all()
    np.testing.assert_allclose(grad.sum(1).astype(float), 0.0, atol=1e-14)
    h = np.longdouble(1e-6)
    for m in range(4):
        for v in range(9):
            up, down = z.copy(), z.copy()
            up[m, v] += h
            down[m, v] -= h
            d = g[m] * (top_distill(up, ids, lps, T, rest)[0][m] - top_distill(down, ids, lps, T, rest)[0][m]) / (2 * h)
            assert float(grad[m, v]) == pytest.approx(float(d), abs=1e-9), (m, v)


@pytest.fixture(scope="module")
def v():
    ver = _verifier()
    yield ver
    ver.close()


@pytest.mark.gpu
@pytest.mark.parametrize("rest", RESTS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [8, 700, 9000, 40003, 70001])
def test_loss_and_gradient(v, V, dtype, rest):
    rng = np.random.default_rng(V)
    z, ids, lps = _rows(rng, 5, V, min(V, 20))
    _check(v, torch.from_numpy(z).to(dtype).to(DEV), ids, lps, 0.3 + rng.random(5), rest, rng.standard_normal(5).astype(np.float32))


@pytest.mark.gpu
@pytest.mark.parametrize("rest", RESTS)
def test_against_differences(v, rest):
    """The difference of two float32 losses, and the sum of a row's gradient, which a shift of all of its logits makes 0: an entry is off by
    at most (78 + 158 + 5) 2^-24 of its parts (distances up to 24 in base 2), and these add up to twice the probabilities'."""
    rng = np.random.default_rng(5)
    z, ids, lps = _rows(rng, 2, 30, 5)
    z, h = torch.from_numpy(z).to(DEV), 2.0 ** -6
    for m in range(2):
        got = v.top_distill_loss_grad(z[m:m + 1], _put(ids[m:m + 1]), _put(lps[m:m + 1]), rest=rest)
        P = float(got["kept"][0])
        assert P > 1
        many = z[m:m + 1].repeat(60, 1)
        many[:30] += h * torch.eye(30, device=DEV)
        many[30:] -= h * torch.eye(30, device=DEV)
        loss = v.top_distill_loss(many, _put(ids[m:m + 1].repeat(60, 0)), _put(lps[m:m + 1].repeat(60, 0)), rest=rest)["loss"].double()
        d = (loss[:30] - loss[30:]) / (2 * h)
        # a third derivative (at most P, of the logarithm of the sum) times h^2 / 6, and the losses' roundings over 2 h
        tol = P * h * h / 6 + 2 * (2.0 ** -23 * float(loss.abs().max()) + P * 2.0 ** -20) / (2 * h)
        assert float((got["grad"][0].double() - d).abs().max()) <= tol
        assert abs(float(got["grad"].double().sum())) <= 2 * P * 2.0 ** -16
