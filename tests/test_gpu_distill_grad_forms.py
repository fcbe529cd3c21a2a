"""The two forms of the loss's gradient (a draft row in one workgroup; behind the loss's launch, which q' rows ask for) where float32 has no
room for what the row's temperatures and masks make of its logits: both against the oracle and against ot_distill_loss."""
import numpy as np
import pytest

from test_gpu_distill_grad import MODES, _compare, _spec
from workloads import make_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("with_qprime", [False, True])
@pytest.mark.parametrize("V_d", [301, 9001])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tiny_draft_temperatures(dtype, V_d, with_qprime):
    """Above and below the temperature from which a row is done in 64 bits; masked draft ids, whose exponent is the largest."""
    temps = [1.0, 3e-8, 2e-8, 5e-9, 4e-9, 1e-12, 1e-30, 1e-36]
    case = make_case(_spec("tiny_draft", [5, 3, 6, 4, 4, 7, 2, 5], 41, dtype=dtype, V_t=max(600, V_d), V_d=V_d, temperature=[1.0] * 8, draft_temperature=temps))
    low = np.float32(-np.inf) if dtype == "f32" else np.uint16(0xFF80)
    out = np.random.default_rng(2).random(case.draft_logits.shape) < 0.3
    out[np.arange(case.K), case.draft_ids] = False
    case.draft_logits[out] = low
    _compare(case, modes=MODES, with_qprime=with_qprime)


@pytest.mark.parametrize("with_qprime", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_tiny_target_temperatures(dtype, with_qprime):
    """ln p down to -1e31, which the gradient follows."""
    temps = [1.0, 3e-8, 2e-8, 1e-9, 1e-20, 1e-30]
    case = make_case(_spec("tiny_target", [5, 3, 6, 4, 4, 7], 43, dtype=dtype, temperature=temps, draft_temperature=[1.0, 0.7, 1.0, 1.0, 0.5, 1.0]))
    _compare(case, modes=MODES, with_qprime=with_qprime)


def _two_forms(case, **how):
    """ot_distill_loss, and the gradient's outputs of both forms, as numpy arrays."""
    from paper_2507_02659_amd.runner import Verifier
    v = Verifier.for_case(case)
    inp = v.upload(case)
    v.step(inp, from_logits=True)
    loss = v.distill_loss(inp, from_logits=True, **how)
    got = [{n: t.double().cpu().numpy() for n, t in v.distill_loss_grad(inp, from_logits=True, with_qprime=q, **how).items()} for q in (False, True)]
    v.close()
    return loss, got


def _tail_ids(case, b, td):
    """Mapped draft ids of sequence b's first row whose q is there in 64 bits and below 2^-126 at the draft temperature."""
    row = np.asarray(case.draft_logits[int(case.row_off[b]) - b], np.float64) / td
    lq = row - row.max() - np.log(np.exp(row - row.max()).sum())
    return np.flatnonzero((lq < -90) & (lq > -600) & (case.direct_map >= 0))


@pytest.mark.parametrize("V_t,V_d,n_direct", [(600, 301, 300), (9500, 9001, 9000)])
def test_a_masked_target_under_a_tiny_probability(V_t, V_d, n_direct):
    """The target gives 0 to an id that the drafter proposes with q' of 1e-40 and less: the term is infinite in every form."""
    case = make_case(_spec("far", [4, 3, 5], 9, n_ngram=0, temperature=[1.0] * 3, draft_temperature=[0.05, 0.05, 1.0], n_direct=n_direct, V_t=V_t, V_d=V_d))
    ids = _tail_ids(case, 0, 0.05)
    assert ids.size > 3
    case.target_logits[0, case.direct_map[ids[0]]] = -np.inf
    loss, got = _two_forms(case)
    assert loss["kind"][0] == 1 and loss["kl"][0] == np.inf and np.isfinite(loss["kl"][1:]).all() and loss["loss"] == np.inf
    for g in got:
        np.testing.assert_allclose(g["kl"][:case.M], loss["kl"], rtol=2e-6, atol=1e-6)
        assert g["totals"][4] == np.inf
        assert not np.isfinite(g["grad"][0]).all() and np.isfinite(g["grad"][1:]).all()
    np.testing.assert_array_equal(np.isnan(got[0]["grad"]), np.isnan(got[1]["grad"]))


@pytest.mark.parametrize("with_qprime", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_targets_masked_with_low_numbers(dtype, with_qprime):
    """A third of the target's ids masked with -1e37, n-gram targets and first sub-tokens' images among them: huge terms, and finite."""
    case = make_case(_spec("low", [5, 3, 6, 4, 4, 7], 47, dtype=dtype, temperature=[1.0, 0.7, 1.0, 1.0, 0.8, 1.0], draft_temperature=[1.0, 0.05, 1.0, 0.3, 1.0, 0.1]))
    case.target_logits[np.random.default_rng(3).random(case.target_logits.shape) < 0.3] = -1e37
    _compare(case, modes=MODES, with_qprime=with_qprime)


@pytest.mark.parametrize("approx_kl", [False, True])
@pytest.mark.parametrize("tiny", [False, True])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_rows_without_a_distribution(dtype, tiny, approx_kl):
    """Draft rows that the mask leaves empty (no mass: nothing is added, gradients 0), that hold a NaN at a mapped or an unmapped id or +inf
    (NaN), target rows without a logit above -inf and with a NaN; the rows next to them stay as they are."""
    from paper_2507_02659_amd import binding as ot
    bits = {"f32": (np.float32(-np.inf), np.float32(np.nan), np.float32(np.inf)), "bf16": (np.uint16(0xFF80), np.uint16(0x7FC0), np.uint16(0x7F80))}[dtype]
    case = make_case(_spec("empty", [2] * 8, 51, dtype=dtype, n_ngram=0, n_direct=300, V_t=600, temperature=[1.0] * 8, draft_temperature=[1e-9 if tiny else 0.7] * 8))
    mapped, unmapped = np.flatnonzero(case.direct_map >= 0), np.flatnonzero(case.direct_map < 0)
    assert (case.direct_map[case.draft_ids] >= 0).all()
    case.draft_logits[0] = bits[0]
    case.draft_logits[2, mapped[7]] = bits[1]
    case.draft_logits[4, unmapped[0]] = bits[1]
    case.draft_logits[6, mapped[9]] = bits[2]
    case.target_logits[12] = -np.inf                      # of draft row 8
    case.target_logits[15, case.direct_map[mapped[0]]] = np.nan   # of draft row 10
    how = dict(ngram_term=ot.OT_NGRAM_TERM_APPROX_KL if approx_kl else ot.OT_NGRAM_TERM_NLL)
    loss, (one, gather) = _two_forms(case, **how)
    assert (loss["kind"].reshape(8, 3)[:, :2] == 1).all()
    for g in (one, gather):
        kl, grad = g["kl"][:case.M], g["grad"]
        assert kl[0] == 0 and not grad[0].any()
        assert np.isnan(kl[[3, 6, 9, 12, 15]]).all() and np.isnan(g["totals"][4])
        assert np.isnan(grad[[2, 4, 6]]).all() and np.isnan(grad[[8, 10]]).any(1).all()
        others = np.setdiff1d(np.arange(case.K), [0, 2, 4, 6, 8, 10])
        rows = others + others // 2
        assert np.isfinite(grad[others]).all() and (tiny or grad[others].any())
        np.testing.assert_allclose(kl[rows], loss["kl"][rows], rtol=2e-6, atol=1e-6)
    np.testing.assert_array_equal(np.isnan(one["grad"]), np.isnan(gather["grad"]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_a_gradient_over_the_logits_is_refused(dtype):
    """At the logits, and anywhere that shares a byte with them: one id before or behind, a row further, the last id; next to them it is taken."""
    import torch

    from paper_2507_02659_amd import binding as ot
    from paper_2507_02659_amd.runner import Verifier
    case = make_case(_spec("overlap", [3, 2], 3, dtype=dtype))
    v = Verifier.for_case(case)
    inp = v.upload(case)
    K, V_d, size = case.K, case.V_d, 2 if dtype == "bf16" else 4
    memory = torch.zeros(3 * K, V_d, dtype=inp["draft_logits"].dtype, device="cuda:0")
    memory[K:2 * K] = inp["draft_logits"]
    inp["draft_logits"] = memory[K:2 * K]
    v.step(inp, from_logits=True)
    want = v.distill_loss_grad(inp, from_logits=True)["grad"]
    names = ("B", "step", "row_off", "row_off_host", "hidden", "draft_logits", "draft_ids", "temperature", "draft_temperature", "seq_id", "seed")
    sin, sout = ot.make_step_in(**{n: inp[n] for n in names}), ot.make_step_out(inp["out"])

    def call(at):
        ot.ot_distill_loss_grad(v.ctx, sin, sout, inp["target_logits"], lam=0.2, lambda_mode=0, ngram_term=0, accepted_only=False,
                                buffers=v._loss_buffers(inp, False), grad_loss=None, grad=memory.data_ptr() + size * at)

    for at in (K * V_d, K * V_d + 1, K * V_d - 1, (K + 1) * V_d, 2 * K * V_d - 1, 1):
        with pytest.raises(ot.OtError) as e:
            call(at)
        assert e.value.code == ot.OT_ERR_SHAPE and "overlaps" in e.value.message
    for first in (0, 2 * K):
        call(first * V_d)
        v.synchronize()
        assert torch.equal(memory[first:first + K], want)
    v.close()


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("V_t,V_d,n_direct", [(600, 301, 240), (9000, 8000, 7000), (20000, 33001, 15000)])
@pytest.mark.parametrize("up", [6, 14, 22])
def test_a_sure_drafter(up, V_t, V_d, n_direct, dtype):
    """Rows whose likeliest id has all of q but 1e-1 to 1e-8: its gradient is made of what the others have, and is right relative to that.  (The
    tolerance of every other id is that of the other tests; of the likeliest one, q (a - A) = q (a rest - sum of the others' q a), D (1 - q) =
    D rest: the terms' own bounds times rest, and the others'.  rest, a float32 sum of V_d / 1024 values in a thread, is off by 2^-24 each at most.)"""
    from oracle import distill_grad as og
    case = make_case(_spec("sure", [6, 7, 5, 6] * 4, 31 + up, dtype=dtype, V_t=V_t, V_d=V_d, n_direct=n_direct, temperature=[1.0] * 16))
    rng = np.random.default_rng(up)
    rows, ids = np.arange(case.K), np.where(rng.random(case.K) < 0.8, case.draft_ids, rng.integers(0, V_d, case.K))
    z = (case.draft_logits.astype(np.uint32) << 16).view(np.float32) if dtype == "bf16" else case.draft_logits
    z[rows, ids] = np.round(z.max(1) + up)                # whole numbers: bfloat16 holds them
    case.draft_logits = (z.view(np.uint32) >> 16).astype(np.uint16) if dtype == "bf16" else z
    assert case.K >= 64
    want, scale, _ = og.hybrid_loss_grad_case(case)
    wide = z.astype(np.longdouble)
    e = np.exp(wide - wide.max(1, keepdims=True))
    e[rows, ids] = 0.0
    rest = (e.sum(1) / (1.0 + e.sum(1))).astype(np.float64)
    others = scale.copy()
    others[rows, ids] = 0.0
    scale[rows, ids] = scale[rows, ids] * rest + others.sum(1)
    _, forms = _two_forms(case)
    tol = 8e-6 * scale
    tol += (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * (np.abs(want) + tol) + 1e-37
    for got in forms:
        off = np.abs(got["grad"] - want) / tol
        assert off.max() <= 1.0, (off.max(), np.unravel_index(off.argmax(), off.shape))
