"""The distillation loss's gradient with respect to the drafter's logits, against oracle/distill_grad.py."""
import numpy as np
import pytest
import torch

from oracle import distill_grad as og
from oracle import verify as ov
from test_gpu_distill import MODES
from workloads import CaseSpec, make_case

pytestmark = pytest.mark.gpu


def _compare(case, modes=MODES, grad_loss=None, rel=8e-6, with_qprime=False):
    """rel: an element's terms carry the fast exponential and the drafter's row sum (2e-7 each), a (two logits' 2^-24 of values up to 30 times
    the terms' own size) and A (the loss's KL value: 2e-6 relative plus 1e-6 as its own test has it, times 1 + |A|).
    The row sums are sums of float32 exponentials, so every ln q is known to 2^-23 at best: `soft` is what that does to ln(q(d_1) - pi)."""
    from paper_2507_02659_amd import binding as ot
    from paper_2507_02659_amd.runner import Verifier
    from_logits = case.hidden is None
    ref = ov.verify_case(case)
    v = Verifier.for_case(case)
    try:
        inp = v.upload(case)
        v.step(inp, from_logits=from_logits)
        step = v.results(inp)
        for lambda_mode, ngram_term, accepted_only in modes:
            if accepted_only and not np.array_equal(step["n_accept"], ref["n_accept"]):
                continue
            print(f"loss gradient {case.name} B={case.B} K={case.K} V_t={case.V_t} V_d={case.V_d} {case.dtype} {lambda_mode}/{ngram_term}/{accepted_only}", flush=True)
            want, scale, soft = og.hybrid_loss_grad_case(case, lambda_mode=lambda_mode, ngram_term=ngram_term, n_accept=ref["n_accept"] if accepted_only else None,
                                                   grad_loss=1.0 if grad_loss is None else grad_loss)
            how = dict(from_logits=from_logits, lam=0.2, lambda_mode=ot.OT_LAMBDA_TARGET_PROB if lambda_mode == "target_prob" else ot.OT_LAMBDA_FIXED,
                       ngram_term=ot.OT_NGRAM_TERM_APPROX_KL if ngram_term == "approx_kl" else ot.OT_NGRAM_TERM_NLL, accepted_only=accepted_only)
            plain = v.distill_loss(inp, **how)
            up = None if grad_loss is None else torch.tensor([grad_loss], dtype=torch.float32, device="cuda:0")
            got = v.distill_loss_grad(inp, grad_loss=up, with_qprime=with_qprime, **how)
            assert got["grad"].dtype == inp["draft_logits"].dtype and tuple(got["grad"].shape) == (case.K, case.V_d)
            # the values are ot_distill_loss's: the KL terms from float32 q and float32 differences of two logits (2^-22 of exponents up to
            # 40 or so), which the mean over q brings to the tolerance that the loss's own test has; the others alike
            for n in ("kind", "nll", "weight"):
                np.testing.assert_allclose(got[n].cpu().numpy()[:case.M], plain[n], rtol=1e-12)
            np.testing.assert_allclose(got["kl"].cpu().numpy()[:case.M], plain["kl"], rtol=2e-6, atol=1e-6)
            totals = got["totals"].cpu().numpy()
            np.testing.assert_allclose(totals, [plain[n] for n in ("loss_dm", "loss_ngram", "n_dm", "n_ngram_tokens", "loss")], rtol=1e-5, atol=1e-5)
            grad = got["grad"].double().cpu().numpy()
            half = 2.0 ** -8 if case.dtype == "bf16" else 2.0 ** -24
            tol = rel * scale + soft
            tol = tol + half * (np.abs(want) + tol) + 1e-37
            off = np.abs(grad - want) - tol
            assert off.size == 0 or off.max() <= 0, (off.max(), np.unravel_index(off.argmax(), off.shape))
            assert not grad[scale == 0].any()
    finally:
        v.close()


def _spec(name, ks, seed, **kw):
    base = dict(name=name, dtype="f32", d=8, V_t=600, V_d=301, k=ks, temperature=[[1.0, 0.7, 0.0, 1.0][i % 4] if len(ks) > 1 else 1.0 for i in range(len(ks))], n_direct=240,
                n_ngram=80, ngram_len=(2, 4), plant_cover=0.5, align=0.5, data_seed=seed, philox_seed=5, logits_only=True)
    return CaseSpec(**dict(base, **kw))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("ks", [[0], [1], [4], [0, 0, 3], [3, 0, 5, 1, 0, 4, 4, 2, 5], [2] * 40, [63, 0, 1]])
def test_windows(ks, dtype):
    _compare(make_case(_spec("windows", ks, len(ks) + sum(ks), dtype=dtype)))


@pytest.mark.parametrize("V_t,V_d,n_direct", [(40, 17, 0), (40, 17, 17), (1000, 999, 600), (300, 1001, 150), (9000, 8192, 7000), (5003, 4099, 4000), (3000, 40001, 2500)])
def test_vocabularies(V_t, V_d, n_direct):
    for dtype in ("f32", "bf16"):
        _compare(make_case(_spec("vocabularies", [5, 3, 6], V_d, dtype=dtype, V_t=V_t, V_d=V_d, n_direct=n_direct, n_ngram=min(60, V_t - n_direct))))


@pytest.mark.parametrize("V_d", [4095, 8185, 8192, 16377, 20000, 32768, 38377, 38378, 38400])
def test_many_rows_of_every_width(V_d):
    """64 rows and more, which one workgroup each takes where a row fits LDS: every number of vectors per thread, the last widths that fit, and
    the first that do not."""
    for dtype in ("f32", "bf16"):
        case = make_case(_spec("widths", [6, 7] * 5 + [0, 3], V_d, dtype=dtype, V_t=4000, V_d=V_d, n_direct=min(3000, V_d), n_ngram=60))
        assert case.K >= 64
        _compare(case, modes=[("target_prob", "approx_kl", False), ("fixed", "nll", True)])


@pytest.mark.parametrize("V_d", [301, 20000])
def test_targets_masked_with_the_lowest_number(V_d):
    """The target masks ids that the drafter proposes with a finite lowest number: the loss and the gradients are huge, and finite."""
    from paper_2507_02659_amd.runner import Verifier
    case = make_case(_spec("lowest", [3, 3], 5, n_ngram=0, temperature=[1.0, 1.0], n_direct=300, V_d=V_d))
    case.target_logits[0, case.direct_map[case.direct_map >= 0][:5]] = -3.0e38
    want, scale, _ = og.hybrid_loss_grad_case(case)
    v = Verifier.for_case(case)
    inp = v.upload(case)
    v.step(inp, from_logits=True)
    got = v.distill_loss_grad(inp, from_logits=True)
    loss = v.distill_loss(inp, from_logits=True)
    grad = got["grad"].double().cpu().numpy()
    np.testing.assert_allclose(got["kl"].cpu().numpy()[:case.M], loss["kl"], rtol=1e-5, atol=1e-6)
    assert np.isfinite(grad).all() and (np.abs(grad - want) <= 2e-5 * scale + 2.0 ** -23 * np.abs(want)).all()
    v.close()


def test_one_vocabulary_on_both_sides():
    for V in (1000, 40000):
        _compare(make_case(_spec("identity", [5, 0, 6], V, V_t=V, V_d=V, n_direct=0, identity_map=True, permute_frac=0.02, n_ngram=0)))


def test_targets_of_ngrams_that_are_images():
    """N-gram targets anywhere: images of other draft ids, of their own first sub-token, or none; first sub-tokens without an image."""
    case = make_case(_spec("targets", [6] * 30, 77, V_t=60, V_d=50, n_direct=35, n_ngram=25))
    rng = np.random.default_rng(1)
    case.ngram_target_ids = rng.integers(0, 60, case.ngram_target_ids.size).astype(np.int32)
    first = case.ngram_key_ids[case.ngram_key_off[:-1]]
    own = case.direct_map[first]
    use = (own >= 0) & (rng.random(own.size) < 0.4)
    case.ngram_target_ids[use] = own[use]
    assert use.any()
    _compare(case)


@pytest.mark.parametrize("V_d", [301, 1001, 16379])
def test_what_shared_memory_held_before_does_not_matter(V_d):
    """A 4-bit head that has just taken hidden rows of NaN leaves them in the shared memory of every compute unit; the draft rows end inside a
    vector of 8."""
    from paper_2507_02659_amd import binding as ot
    from paper_2507_02659_amd.runner import QuantWeights, Verifier
    d, V = 4096, 8192
    codes = torch.zeros(d // 2, V, dtype=torch.uint8, device="cuda:0")
    head = Verifier.quantized(QuantWeights(codes, torch.ones(d // 128, V, device="cuda:0").bfloat16(), None, 128), V_d=1, direct_map=np.zeros(1, np.int32),
                              max_batch=16, max_k=0)
    hidden = torch.full((16, d), float("nan"), device="cuda:0").bfloat16()
    case = make_case(_spec("after_nan", [4] * 40, 7, dtype="bf16", V_t=max(600, V_d), V_d=V_d))
    v = Verifier.for_case(case)
    try:
        inp = v.upload(case)
        v.step(inp, from_logits=True)
        how = dict(from_logits=True, lam=0.2, ngram_term=ot.OT_NGRAM_TERM_APPROX_KL)
        plain = v.distill_loss(inp, **how)
        for _ in range(3):
            assert torch.isnan(head.lm_head(hidden)).all()
            torch.cuda.synchronize()
            got = v.distill_loss_grad(inp, **how)
            np.testing.assert_allclose(got["kl"].cpu().numpy()[:case.M], plain["kl"], rtol=2e-6, atol=1e-6)
            assert torch.isfinite(got["grad"].float()).all()
    finally:
        v.close()
        head.close()


def test_draft_temperatures_and_upstream_gradient():
    case = make_case(_spec("temperatures", [4, 3, 5, 2, 6], 21, temperature=[1.0, 0.5, 1.0, 0.7, 0.0], draft_temperature=[0.6, 1.0, 0.0, 1.5, 1.0]))
    _compare(case, grad_loss=-2.5)
    _compare(case, grad_loss=0.0)
    _compare(case, grad_loss=1e-3, with_qprime=True)


def test_peaked_and_masked_draft_rows():
    """Drafted tokens of probability near 1, masked draft ids, masked target ids that no draft id maps to."""
    case = make_case(_spec("peaked", [5, 4, 6], 31, V_t=500, V_d=200, n_direct=150))
    rng = np.random.default_rng(2)
    z = case.draft_logits
    z[np.arange(case.K), case.draft_ids] += 30.0
    out = rng.random(z.shape) < 0.3
    out[np.arange(case.K), case.draft_ids] = False
    z[out] = -np.inf
    free = np.setdiff1d(np.arange(500), case.direct_map)
    free = np.setdiff1d(free, case.ngram_target_ids)
    case.target_logits[:, free[::2]] = -np.inf
    _compare(case)


def test_an_infinite_term_spoils_its_rows_alone():
    """The target masks an id that the drafter proposes with q' > 0: the loss is infinite, its rows' gradients are not finite."""
    from paper_2507_02659_amd.runner import Verifier
    case = make_case(_spec("infinite", [3, 3], 5, n_ngram=0, temperature=[1.0, 1.0], n_direct=300))
    case.target_logits[0, case.direct_map[case.direct_map >= 0][0]] = -np.inf
    v = Verifier.for_case(case)
    inp = v.upload(case)
    v.step(inp, from_logits=True)
    got = v.distill_loss_grad(inp, from_logits=True)
    grad, kind = got["grad"].cpu().numpy(), got["kind"].cpu().numpy()
    assert kind[0] == 1 and not np.isfinite(grad[0]).all() and np.isfinite(grad[1:]).all()
    v.close()


def test_after_a_step_on_hidden_states():
    """Statistics and logits as the LM-head launch left them, in every launch structure's form; a ragged vocabulary, bf16."""
    from paper_2507_02659_amd import binding as ot
    from paper_2507_02659_amd.runner import Verifier
    case = make_case(CaseSpec(name="hidden", dtype="bf16", d=512, V_t=5003, V_d=2001, k=[5, 8, 0, 3], temperature=[1.0, 0.7, 1.0, 0.0], n_direct=1500, n_ngram=300,
                              ngram_len=(2, 4), zipf_a=1.1, plant_cover=0.4, align=0.6, data_seed=3, philox_seed=4))
    _compare(case, rel=6e-5)                              # logits to 1e-5, and the KL value to 1e-4 + 1e-5 times 1 + |A| on a share of it
    grads = []
    for side in (ot.OT_DRAFT_SIDE_IN_LM_HEAD, ot.OT_DRAFT_SIDE_SEPARATE):
        v = Verifier.for_case(case, draft_side=side)
        inp = v.upload(case)
        v.step(inp)
        grads.append(v.distill_loss_grad(inp)["grad"].float().cpu())
        v.close()
    assert float((grads[0] - grads[1]).norm() / grads[1].norm()) < 2.0 ** -8


def test_replayed_from_a_graph():
    from paper_2507_02659_amd.runner import Verifier
    stream = torch.cuda.Stream()
    case = make_case(_spec("graph", [5, 3, 6], 12, V_t=3000, V_d=2000, n_direct=1500))
    v = Verifier.for_case(case, stream=stream)
    with torch.cuda.stream(stream):
        inp = v.upload(case)
        v.step(inp, from_logits=True)
        ups = [torch.tensor([x], dtype=torch.float32, device="cuda:0") for x in (1.0, -3.0, 0.5)]
        eager = [v.distill_loss_grad(inp, from_logits=True, grad_loss=u)["grad"].clone() for u in ups]
        up = ups[0].clone()
        stream.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            out = v.distill_loss_grad(inp, from_logits=True, grad_loss=up)["grad"]
        for turn in range(2):
            for u, want in zip(ups, eager):
                up.copy_(u)
                graph.replay()
                stream.synchronize()
                assert torch.equal(out, want)
                assert torch.equal(v.distill_loss_grad(inp, from_logits=True, grad_loss=u)["grad"], want)
    v.close()


def test_refusals_and_an_empty_batch():
    from paper_2507_02659_amd import binding as ot
    from paper_2507_02659_amd.runner import Verifier
    case = make_case(_spec("refusals", [2, 1], 2))
    v = Verifier.for_case(case)
    inp = v.upload(case)
    v.step(inp, from_logits=True)
    v.distill_loss(inp, from_logits=True)
    buf = v._loss_buffers(inp, False)
    grad = torch.empty(case.K, case.V_d, device="cuda:0")
    names = ("B", "step", "row_off", "row_off_host", "hidden", "draft_logits", "draft_ids", "temperature", "draft_temperature", "seq_id", "seed")
    good = dict(lam=0.2, lambda_mode=0, ngram_term=0, accepted_only=False, buffers=buf, grad_loss=None, grad=grad)

    def code(B=inp["B"], **kw):
        sin = ot.make_step_in(**dict({n: inp[n] for n in names}, B=B))
        with pytest.raises(ot.OtError) as e:
            ot.ot_distill_loss_grad(v.ctx, sin, ot.make_step_out(inp["out"]), inp["target_logits"], **dict(good, **kw))
        return e.value.code

    assert code(grad=None) == ot.OT_ERR_NULL and code(grad=grad.data_ptr() + 2) == ot.OT_ERR_SHAPE and code(lambda_mode=5) == ot.OT_ERR_SHAPE
    assert code(ngram_term=2) == ot.OT_ERR_SHAPE and code(B=-1) == ot.OT_ERR_SHAPE and code(B=99) == ot.OT_ERR_SHAPE
    assert code(buffers=dict(buf, kl=None)) == ot.OT_ERR_NULL
    assert code(B=99, grad=None) == ot.OT_ERR_SHAPE      # sizes first: the offsets of 99 sequences are not there
    assert code(grad=inp["draft_logits"]) == ot.OT_ERR_SHAPE
    with pytest.raises(ValueError):
        v.distill_loss_grad(inp, from_logits=True, grad_loss=torch.ones(1, dtype=torch.float64, device="cuda:0"))
    empty = dict({n: None for n in names}, B=0, step=0, seed=0)
    ot.ot_distill_loss_grad(v.ctx, ot.make_step_in(**empty), ot.make_step_out({}), None, **dict(good, grad=None))
    assert buf["totals"].cpu().numpy().tolist() == [0.0] * 5
    v.close()
