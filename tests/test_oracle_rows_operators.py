"""Pins of the oracles of adapters, adjusted logits and the distillation from top logits: worked examples, and gradients against differences."""
import numpy as np
import pytest

from oracle.adapters import adapter_logits
from oracle.adjust import adjust_logits
from oracle.top_distill import BUCKET, DROP, RENORMALISE, top_distill


def test_adapters():
    hidden = np.array([[1.0, 2.0], [3.0, -1.0], [1.0, 1.0], [0.0, 1.0]])
    down, up = np.array([[[1.0, 1.0]], [[2.0, 0.0]]]), np.array([[[1.0], [0.0], [-1.0]], [[0.0], [3.0], [1.0]]])
    z = np.ones((4, 3))
    got = adapter_logits(hidden, down, up, [0.5, 2.0], [0, 1, -1, 2], z)
    np.testing.assert_array_equal(got[:3], [[2.5, 1.0, -0.5], [1.0, 37.0, 13.0], [1.0, 1.0, 1.0]])
    assert np.isnan(got[3]).all()
    np.testing.assert_array_equal(adapter_logits(hidden[:1], down, up, None, [0]), [[3.0, 0.0, -3.0]])


def test_adjusted_logits():
    z = np.array([[2.0, -2.0, 1.0, -np.inf, 3.0]] * 3)
    got = adjust_logits(z, row_off=[0, 2, 3], history=[[0, 1, 1, 9], [2, 2, 3, -1]], n_history=[3, 4], n_prompt=[1, 0], window=[4, 0, 1], repetition=[2.0, 4.0],
                        frequency=[0.25, 0.5], presence=[1.0, 0.0], bias_ids=[[4, 4, -1], [3, 7, 0]], bias=[[9.0, 0.5, 9.0], [5.0, 5.0, -np.inf]],
                        masks=[[0b10111, 0], [0b01111, 0]], mask_of_row=[-1, 0, 1])
    np.testing.assert_array_equal(got[0], [1.0, -4.0 - 0.5 - 1.0, 1.0, -np.inf, 3.5])            # 4 is not said yet
    np.testing.assert_array_equal(got[1], [1.0, -5.5, 1.0, -np.inf, 1.5 - 0.25 - 1.0 + 0.5])     # and now it is
    np.testing.assert_array_equal(got[2], [-np.inf, -2.0, 0.25 - 1.0, -np.inf, -np.inf])
    assert np.isnan(adjust_logits(z, masks=[[31]], mask_of_row=[0, 1, -2])[1:]).all()


@pytest.mark.parametrize("rest", [DROP, RENORMALISE, BUCKET])
def test_distillation(rest):
    z = np.log(np.array([[0.5, 0.25, 0.125, 0.125]]))
    ids, lp = [[1, 0, -1]], np.log([[0.5, 0.25, 1.0]])
    loss, kept, grad, _ = top_distill(z, ids, lp, rest=rest)
    p = np.array([0.25, 0.5]) / (0.75 if rest == RENORMALISE else 1.0)
    want = (p * np.log(p / [0.5, 0.25])).sum() + (0.25 * np.log(0.25 / 0.25) if rest == BUCKET else 0.0)
    assert float(loss[0]) == pytest.approx(want) and float(kept[0]) == pytest.approx(0.75)
    mass = 0.75 if rest == DROP else 1.0
    own = np.array([*p, 0.0, 0.0])
    want = mass * np.array([0.5, 0.25, 0.125, 0.125]) - own - (np.array([0, 0, 0.125, 0.125]) if rest == BUCKET else 0)
    np.testing.assert_allclose(grad[0].astype(float), want, atol=1e-15)


@pytest.mark.parametrize("rest", [DROP, RENORMALISE, BUCKET])
def test_distillation_against_differences(rest):
    rng = np.random.default_rng(rest)
    V, n = 12, 5
    z = rng.standard_normal((4, V)).astype(np.longdouble)
    z[1, 3] = -np.inf
    tmap = np.array([3, -1, 0, 7, 11, 2, 5, 5, 9, 1])       # (two target ids of one draft id: an id that is named twice)
    ids = np.array([[0, 2, 6, 7, 3], [2, 6, -1, 1, 4], [5, 8, 9, 3, 4], [2, 2, 2, 2, 0]])
    lp = np.log(rng.dirichlet(np.ones(n + 1), 4)[:, :n])
    T, g = np.array([1.0, 0.3, 2.0, 0.7]), rng.standard_normal(4)
    _, _, grad, _ = top_distill(z, ids, lp, T, rest, g, tmap)
    h = np.longdouble(1e-6)
    for m in range(4):
        for v in range(V):
            if z[m, v] == -np.inf:
                assert grad[m, v] == 0
                continue
            up, down = z.copy(), z.copy()
            up[m, v] += h
            down[m, v] -= h
            d = g[m] * (top_distill(up, ids, lp, T, rest, None, tmap)[0][m] - top_distill(down, ids, lp, T, rest, None, tmap)[0][m]) / (2 * h)
            assert float(grad[m, v]) == pytest.approx(float(d), abs=1e-9), (m, v)


def test_distillation_of_rows_that_say_nothing():
    z = np.zeros((7, 3))
    z[1] = -np.inf
    z[2, 1] = np.nan
    z[3, 0] = -np.inf
    ids = [[-1, -1], [0, 1], [0, 1], [0, 1], [0, 3], [0, 1], [2, 1]]
    lp = np.log([[0.5, 0.5]] * 5 + [[0.5, 0.5], [0.5, 0.5]])
    lp[5, 0] = np.nan
    lp[6] = -np.inf
    for rest in (DROP, RENORMALISE, BUCKET):
        loss, kept, grad, _ = top_distill(z, ids, lp, None, rest)
        assert loss[0] == loss[1] == 0 and (grad[:2] == 0).all() and kept[0] == 0
        assert np.isnan(loss[[2, 4, 5]]).all() and np.isnan(grad[[2, 4, 5]]).all()
        assert loss[3] == np.inf and grad[3, 0] == 0 and np.isfinite(grad[3]).all()
        assert float(loss[6]) == pytest.approx(np.log(3.0) if rest == BUCKET else 0.0) and kept[6] == 0
