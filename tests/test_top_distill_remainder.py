"""Distillation with the rest as one token more, where the student has no other ids than those that are kept: what a sum of rounded probabilities lacks of 1
is no remainder."""
import numpy as np
import pytest
import torch

from oracle.top_distill import BUCKET, top_distill
from test_gpu_top_distill import DEV, _check, _put, _verifier

LOWEST = float(np.finfo(np.float32).min)


def test_oracle():
    z = np.array([[1.0, 0.5, -np.inf, -np.inf], [1.0, 0.5, LOWEST, -np.inf], [1.0, 0.5, -1.0, -np.inf], [1.0, 0.5, -np.inf, -np.inf], [1.0, 0.5, LOWEST, LOWEST]])
    ids = np.array([[0, 1]] * 5)
    p = np.array([[0.6, 0.4 - 2.0 ** -21]] * 3 + [[0.6, 0.4 - 2.0 ** -19]] * 2)
    loss, _, grad, _ = top_distill(z, ids, np.log(p), None, BUCKET)
    q = np.exp(z[0, :2]) / np.exp(z[0, :2]).sum()
    want = (p[0] * np.log(p[0] / q)).sum()
    np.testing.assert_allclose(loss[:2].astype(float), want, rtol=1e-13)
    np.testing.assert_allclose(grad[:2, :2].astype(float), [p[0].sum() * q - p[0]] * 2, rtol=1e-9)
    assert (grad[:2, 2:] == 0).all() and np.isfinite(loss[2]) and loss[3] == np.inf and loss[4] > 1e30


@pytest.fixture(scope="module")
def v():
    ver = _verifier()
    yield ver
    ver.close()


def _masked(rng, M, V, left, dtype):
    """Rows of a teacher and a student under one mask that leaves so many ids of a row."""
    keep = torch.zeros(M, V, dtype=torch.bool, device=DEV)
    keep.scatter_(1, _put(np.stack([rng.permutation(V)[:left] for _ in range(M)])).long(), True)
    put = lambda scale: torch.from_numpy((scale * rng.standard_normal((M, V))).astype(np.float32)).to(DEV)  # noqa: E731
    return keep, put(3.0), put(2.0).to(dtype)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V,left", [(15, 15), (15, 14), (3000, 12), (9000, 19), (70001, 5)])
def test_teacher_and_student_under_one_mask(v, V, left, dtype):
    rng = np.random.default_rng(V + left)
    M = 200
    keep, teacher, z = _masked(rng, M, V, left, dtype)
    known = v.token_logprobs(torch.where(keep, teacher, -float("inf")), n_top=20)
    ids, lps = known["top_ids"].cpu().numpy(), known["top_logprobs"].cpu().numpy()
    total = np.exp(lps.astype(np.float64)).sum(1)
    assert (total < 1).any() and np.abs(total - 1).max() < 2.0 ** -20
    low = torch.finfo(dtype).min
    for nothing in (-float("inf"), low):
        got = _check(v, torch.where(keep, z, nothing), ids, lps, None, BUCKET)
        assert got["loss"].isfinite().all() and float(got["loss"].max()) < 100
        assert (got["grad"][~keep] == 0).all()
    # half of the ids that the teacher has, and no others: what is not kept has no place
    lps[:, ::2] = -np.inf
    ids[:, ::2] = -1
    at = _put(np.where(ids[:, 1::2] < 0, V, ids[:, 1::2])).long()      # (free places: a column behind the last)
    few = torch.zeros(M, V + 1, dtype=torch.bool, device=DEV).scatter_(1, at, True)[:, :V]
    got = _check(v, torch.where(few, z, -float("inf")), ids, lps, None, BUCKET)
    assert (got["loss"] == float("inf")).all()
