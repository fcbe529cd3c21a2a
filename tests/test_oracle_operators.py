"""Pins of the oracles of the 4-bit head, of token log-probabilities and of the loss's gradient; the new structs' layout; refusals that need
no GPU."""
import ctypes as C
import os
import re

import numpy as np
import pytest
import scipy.special
import scipy.stats

from oracle import distill as od
from oracle import distill_grad as og
from oracle import logprobs as ol
from oracle import quant_head as oq

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_quantized_product_by_hand():
    # hidden index 0: code 3, 1: code 9; 2: 15, 3: 0; groups of two
    codes = np.array([[3 | 9 << 4], [15 | 0 << 4]], np.uint8)
    W = oq.dequantize(codes, np.array([[0.5], [2.0]]), np.array([[4], [8]]), 2)
    assert W[:, 0].tolist() == [-0.5, 2.5, 14.0, -16.0]
    assert oq.dequantize(codes, np.array([[0.5], [2.0]]), None, 2)[:, 0].tolist() == [-2.5, 0.5, 14.0, -16.0]
    assert oq.logits([[1.0, 2.0, 3.0, 4.0]], codes, np.array([[0.5], [2.0]]), np.array([[4], [8]]), 2) == [[-0.5 + 5.0 + 42.0 - 64.0]]


def _rows(seed=3, M=5, V=23):
    rng = np.random.default_rng(seed)
    Z = 2.0 * rng.standard_normal((M, V))
    Z[1, rng.permutation(V)[:15]] = -np.inf
    return rng, Z, rng.integers(0, V, (M, 2)), np.array([1.0, 0.7, 0.0, 2.0, 0.3])


def test_logprobs_are_the_library_softmax():
    _, Z, tokens, T = _rows()
    got = ol.token_logprobs(Z, tokens, T, 4)
    for m in range(5):
        lp = scipy.special.log_softmax(Z[m] / (T[m] or 1.0))
        np.testing.assert_allclose(got["logprob"][m], lp[tokens[m]], rtol=1e-12)
        assert got["entropy"][m] == pytest.approx(scipy.stats.entropy(np.exp(lp)), rel=1e-12)
        assert got["top_ids"][m].tolist() == sorted(range(23), key=lambda v: (-Z[m, v], v))[:4]


def test_logprobs_readings():
    Z = np.array([[-np.inf] * 3, [0.0, np.nan, 1.0], [1.0, 1.0, -np.inf]])
    got = ol.token_logprobs(Z, [[0], [2], [1]], np.ones(3), 3)
    assert got["logprob"][0, 0] == -np.inf and got["entropy"][0] == 0 and got["top_ids"][0].tolist() == [-1] * 3
    assert np.isnan(got["logprob"][1, 0]) and np.isnan(got["entropy"][1]) and got["top_ids"][1].tolist() == [-1] * 3
    assert got["top_ids"][2].tolist() == [0, 1, -1] and got["logprob"][2, 0] == pytest.approx(-np.log(2))
    got = ol.token_logprobs(Z, [[-1], [-1], [5]], np.ones(3), 1, True)
    assert got["logprob"][0, 0] == 0 and got["entropy"][1] == 0 and np.isnan(got["logprob"][2, 0])


def test_logprob_gradient_against_differences():
    rng, Z, tokens, T = _rows()
    tokens[2, 0], tokens[3] = -1, 7                       # a token that is none; the same token twice
    g, gH = rng.standard_normal((5, 2)), rng.standard_normal(5)

    def value(Z):
        f = ol.token_logprobs(Z, tokens, T)
        with np.errstate(invalid="ignore"):
            return float(np.where(np.isfinite(f["logprob"]), g * f["logprob"], 0.0).sum() + (gH * f["entropy"]).sum())

    grad = ol.token_logprobs_grad(Z, tokens, T, g, gH)
    keep = [m for m in range(5) if np.isfinite(Z[m, tokens[m]]).all()]
    for m in keep:
        for v in range(Z.shape[1]):
            if Z[m, v] == -np.inf:
                assert grad[m, v] == 0
                continue
            up, down = Z.copy(), Z.copy()
            up[m, v] += 1e-5
            down[m, v] -= 1e-5
            assert grad[m, v] == pytest.approx((value(up) - value(down)) / 2e-5, abs=1e-7)


@pytest.mark.parametrize("lambda_mode,ngram_term", [("fixed", "nll"), ("target_prob", "approx_kl"), ("fixed", "approx_kl")])
def test_loss_gradient_against_differences(lambda_mode, ngram_term, monkeypatch):
    for oracle in (od, og):                               # draft logits in 64 bits, so that their differences are
        monkeypatch.setattr(oracle, "widen", lambda x, dtype: np.asarray(x, np.float64))
    rng = np.random.default_rng(8)
    V_d, V_t, ks, T = 9, 11, [4, 0, 3], [1.0, 1.0, 0.7]
    row_off = np.concatenate([[0], np.cumsum([k + 1 for k in ks])])
    dmap = np.array([4, -1, 0, 7, 2, 10, -1, 5, 1])
    # a target without a pre-image; one whose pre-image is another draft id; the image of the first sub-token itself; an unmapped first one
    cache = {(3, 1): 3, (0, 2, 4): 5, (2, 2): 0, (1, 7): 9}
    ids = np.array([3, 1, 5, 8] + [0, 2, 4])
    for ids in (ids, np.array([2, 2, 1, 7] + [4, 3, 1]), np.array([8, 0, 2, 4] + [1, 7, 5])):
        args = dict(row_off=row_off, draft_ids=ids, direct_map=dmap, V_t=V_t, cache=cache, max_ngram_len=3, temperature=T,
                    target_logits=rng.standard_normal((10, V_t)).astype(np.float32), dtype="f64", lam=0.3, lambda_mode=lambda_mode, ngram_term=ngram_term)
        Zq = rng.standard_normal((7, V_d))
        grad, scale, _ = og.hybrid_loss_grad(draft_logits=Zq, grad_loss=2.5, **args)
        assert np.all(np.abs(grad) <= scale * (1 + 1e-12))
        for i in np.ndindex(Zq.shape):
            up, down = Zq.copy(), Zq.copy()
            up[i] += 1e-5
            down[i] -= 1e-5
            want = 2.5 * (od.hybrid_loss(draft_logits=up, **args)["loss"] - od.hybrid_loss(draft_logits=down, **args)["loss"]) / 2e-5
            assert grad[i] == pytest.approx(want, abs=2e-8)


def test_struct_layouts_match_the_header():
    from paper_2507_02659_amd import binding as ot
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", "otverify.h")).read(), flags=re.S)
    for cls, size in ((ot.ot_quant_weights, 8 + 3 * 8), (ot.ot_logprob_in, 8 * 4 + 8 + 4 * 8), (ot.ot_logprob_out, 6 * 8)):
        body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (cls.__name__, cls.__name__), text, flags=re.S).group(1)
        names = []
        for decl in filter(None, (d.strip() for d in body.split(";"))):
            names += [n.strip().lstrip("*") for n in re.sub(r"^(const\s+)?\w+\s*\**", "", decl).split(",")]
        assert [f[0] for f in cls._fields_] == names, cls.__name__
        assert C.sizeof(cls) == size


def test_refusals_without_a_gpu():
    from paper_2507_02659_amd import binding as ot
    good = dict(d=64, V_t=100, V_d=50, max_batch=2, max_k=4, max_ngram_len=3, codes=0x1000, scales=0x1000, zeros=None, group=64,
                scale_dtype=ot.OT_F16, direct_map=np.full(50, -1, np.int32))

    def code(**kw):
        with pytest.raises(ot.OtError) as e:
            ot.ot_verify_init_quantized(**dict(good, **kw))
        assert "ot_verify_init" in e.value.message
        return e.value.code

    assert code(codes=None) == ot.OT_ERR_NULL and code(scales=None) == ot.OT_ERR_NULL and code(direct_map=None) == ot.OT_ERR_NULL
    assert code(group=16) == ot.OT_ERR_SHAPE and code(group=0) == ot.OT_ERR_SHAPE and code(group=256) == ot.OT_ERR_SHAPE
    assert code(scale_dtype=ot.OT_F32) == ot.OT_ERR_DTYPE and code(dtype=ot.OT_F32) == ot.OT_ERR_DTYPE and code(dtype=ot.OT_F16) == ot.OT_ERR_DTYPE
    assert code(d=60) == ot.OT_ERR_SHAPE and code(V_t=0) == ot.OT_ERR_SHAPE and code(max_k=64) == ot.OT_ERR_SHAPE
    lib = ot.load_library()
    assert lib.ot_verify_init_quantized(None, None, None) == ot.OT_ERR_NULL
    assert lib.ot_lm_head(None, 1, None, None, 1) == ot.OT_ERR_NULL
    assert lib.ot_token_logprobs(None, None, None) == ot.OT_ERR_NULL
    assert lib.ot_token_logprobs_grad(None, None, None, None, None, None, 1) == ot.OT_ERR_NULL
    assert lib.ot_distill_loss_grad(None, None, None, None, None, None, None, None) == ot.OT_ERR_NULL


def test_weights_are_checked_before_the_library_is_called():
    torch = pytest.importorskip("torch")
    from paper_2507_02659_amd.runner import QuantWeights
    codes, scales = torch.zeros(32, 10, dtype=torch.uint8), torch.zeros(1, 10, dtype=torch.float16)
    QuantWeights(codes, scales, None, 64).check()
    QuantWeights(codes, scales, codes[:1], 128).check()
    for bad in (QuantWeights(codes.int(), scales, None, 64), QuantWeights(codes, scales.float(), None, 64), QuantWeights(codes, scales, scales, 64)):
        with pytest.raises(TypeError):
            bad.check()
    for bad in (QuantWeights(codes, scales, None, 32), QuantWeights(codes, scales, codes[:2], 64)):
        with pytest.raises(ValueError):
            bad.check()
