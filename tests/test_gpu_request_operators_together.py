"""A serving iteration with what its requests bring: hidden rows through the head and each request's adapter, penalties, biases and grammars on the rows
of the windows, the verification step from these logits, the emitted tokens' log-probabilities, and the drafter's gradient from the target's top logits."""
import numpy as np
import pytest
import torch

from oracle import logprobs as ol
from oracle import verify as ov
from oracle.adapters import adapter_logits
from oracle.adjust import adjust_logits
from oracle.top_distill import BUCKET, top_distill
from workloads import CaseSpec, make_case

import parity

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _put(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_an_iteration(dtype):
    from paper_2507_02659_amd.runner import Adapters, Verifier
    rng = np.random.default_rng(8)
    case = make_case(CaseSpec(name="requests", dtype=dtype, d=256, V_t=5003, V_d=2001, k=[5, 0, 8, 3, 6], temperature=[1.0, 1.0, 0.7, 0.0, 1.0], n_direct=1500,
                              n_ngram=300, ngram_len=(2, 4), plant_cover=0.4, data_seed=3, philox_seed=4))
    kind = torch.bfloat16 if dtype == "bf16" else torch.float32
    v = Verifier.for_case(case)
    inp = v.upload(case)
    a = Adapters(torch.randn(3, 16, 256, device=DEV).div(16).to(kind), torch.randn(3, 5003, 16, device=DEV).div(4).to(kind), torch.tensor([0.5, 1.0, 2.0], device=DEV))
    of_row = np.repeat([0, -1, 2, 1, 0], case.k + 1).astype(np.int32)
    z = v.lm_head(inp["hidden"], adapters=a, adapter_of_row=_put(of_row))
    head = v.lm_head(inp["hidden"]).double().cpu().numpy()
    host = lambda t: t.double().cpu().numpy()  # noqa: E731
    want = adapter_logits(host(inp["hidden"]), host(a.down), host(a.up), host(a.scale), of_row, head)
    np.testing.assert_allclose(host(z), want, atol=1e-5 * np.abs(want).max())

    # the proposals of the windows: what a step on the plain logits translates them to (it needs no target logits)
    v.step(inp)
    window = v.results(inp)["mapped_ids"]
    keep = rng.random((4, 5003)) < 0.5
    keep[:, window[window >= 0]] = True
    words = np.zeros((4, 157 * 32), bool)
    words[:, :5003] = keep
    words = (words.reshape(4, 157, 32).astype(np.uint64) << np.arange(32, dtype=np.uint64)).sum(2).astype(np.uint32).view(np.int32)
    asked = dict(row_off=case.row_off.astype(np.int32), history=rng.integers(0, 5003, (5, 60)).astype(np.int32), n_history=np.array([60, 0, 31, 8, 44], np.int32),
                 n_prompt=np.array([20, 0, 31, 0, 10], np.int32), window=window.astype(np.int32), repetition=np.float32([1.2, 1.0, 1.5, 1.1, 0.9]),
                 frequency=np.float32([0.1, 0.2, 0.0, 0.3, 0.4]), presence=np.float32([0.3, 0.0, 0.1, 0.2, 0.5]), bias_ids=rng.integers(-1, 5003, (5, 4)).astype(np.int32),
                 bias=rng.standard_normal((5, 4)).astype(np.float32), masks=words, mask_of_row=rng.integers(-1, 4, case.M).astype(np.int32))
    before = host(z)
    adjusted = v.adjust_logits(z, out=z, **{n: _put(x) for n, x in asked.items()})
    want = adjust_logits(before, **asked)
    got = host(adjusted)
    np.testing.assert_array_equal(np.isinf(got), np.isinf(want))
    fine = np.isfinite(want)
    np.testing.assert_allclose(got[fine], want[fine], rtol=2.0 ** -23, atol=1e-9)

    # the step from these logits, and what it emitted
    inp["target_logits"] = adjusted
    v.step(inp, from_logits=True)
    res = v.results(inp)
    case.target_logits, case.hidden = adjusted.cpu().numpy(), None
    rep = parity.compare(case, res, ov.verify_case(case), logits_from_gpu=True)
    assert not rep.failures and rep.divergent <= 1, rep.failures[:5]
    emitted = v.step_logprobs(inp, from_logits=True, n_top=20)
    T = np.repeat(case.temperature, case.k + 1)
    lps = ol.token_logprobs(got, res["out_tokens"], T, 20, True)
    assert np.array_equal(emitted["top_ids"].cpu().numpy(), lps["top_ids"])
    for row in range(case.M):                             # what a mask leaves out is never emitted
        if res["out_tokens"][row] >= 0:
            assert np.isfinite(got[row, res["out_tokens"][row]])

    # the target's top logits of the drafted rows teach the drafter
    rows = np.concatenate([np.arange(o, o + k) for o, k in zip(case.row_off[:-1], case.k)]).astype(np.int64)
    teacher = v.token_logprobs(adjusted[_put(rows)], n_top=20)
    g = np.full(case.K, 1.0 / case.K, np.float32)
    learn = v.top_distill_loss_grad(inp["draft_logits"], teacher["top_ids"], teacher["top_logprobs"], rest=BUCKET, grad_loss=_put(g), through_map=True)
    tmap = np.full(5003, -1)
    mapped = np.flatnonzero(case.direct_map >= 0)
    tmap[case.direct_map[mapped]] = mapped
    loss, kept, grad, size = top_distill(host(inp["draft_logits"]), teacher["top_ids"].cpu().numpy(), teacher["top_logprobs"].cpu().numpy(), None, BUCKET, g, tmap)
    np.testing.assert_allclose(host(learn["loss"]), loss.astype(float), rtol=2e-6, atol=2e-6)
    np.testing.assert_allclose(host(learn["kept"]), kept.astype(float), rtol=1e-6)
    off = np.abs(host(learn["grad"]) - grad.astype(float)) - 8e-6 * size.astype(float) - (2.0 ** -8 if dtype == "bf16" else 2.0 ** -24) * np.abs(grad.astype(float))
    assert off.max() <= 1e-37
    v.close()


def test_calls_without_rows():
    from paper_2507_02659_amd.runner import Adapters, Verifier
    v = Verifier(d=8, V_t=16, V_d=1, dtype="bf16", W=torch.zeros(8, 16, dtype=torch.bfloat16, device=DEV), direct_map=np.zeros(1, np.int32), max_batch=1, max_k=0)
    a = Adapters(torch.zeros(1, 8, 8, device=DEV), torch.zeros(1, 16, 8, device=DEV))
    none = torch.zeros(0, dtype=torch.int32, device=DEV)
    assert v.adapter_logits(torch.zeros(0, 8, device=DEV), a, none, torch.zeros(0, 16, device=DEV)).shape == (0, 16)
    assert v.adjust_logits(torch.zeros(0, 16, device=DEV), presence=torch.zeros(0, device=DEV)).shape == (0, 16)
    assert v.adjust_logits(torch.zeros(0, 16, device=DEV), row_off=torch.zeros(3, dtype=torch.int32, device=DEV)).shape == (0, 16)
    z, ids = torch.zeros(0, 16, device=DEV), torch.zeros(0, 4, dtype=torch.int32, device=DEV)
    got = v.top_distill_loss_grad(z, ids, torch.zeros(0, 4, device=DEV))
    assert got["loss"].shape == (0,) and got["grad"].shape == (0, 16)
    v.close()


def test_inputs_dropped_before_the_work_is_done():
    """Calls on a busy stream of the verifier's own whose inputs the caller drops at once: what is allocated and written next does not land in them."""
    from paper_2507_02659_amd.runner import Adapters, Verifier
    stream = torch.cuda.Stream()
    v = Verifier(d=8, V_t=16, V_d=1, dtype="bf16", W=torch.zeros(8, 16, dtype=torch.bfloat16, device=DEV), direct_map=np.zeros(1, np.int32), max_batch=1, max_k=0,
                 stream=stream)
    rng = np.random.default_rng(1)
    put = lambda x: torch.from_numpy(x).to(DEV)  # noqa: E731
    h, down, up = (rng.standard_normal(s).astype(np.float32) for s in ((20, 32), (2, 8, 32), (2, 700, 8)))
    z, ids = rng.standard_normal((20, 700)).astype(np.float32), rng.integers(0, 700, (20, 9)).astype(np.int32)
    one = np.ones(20, np.float32)
    calls = (lambda: v.adapter_logits(put(h), Adapters(put(down), put(up), put(one[:2])), put(ids[:, 0] % 2), put(z)),
             lambda: v.adjust_logits(put(z), history=put(ids), presence=put(one), bias_ids=put(ids), bias=put(z[:, :9].copy())),
             lambda: v.top_distill_loss_grad(put(z), put(ids), put(np.log(0.1 * np.ones((20, 9), np.float32))), grad_loss=put(one))["grad"])
    for call in calls:
        torch.cuda.synchronize()
        want = call().clone()
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            busy = torch.randn(8192, 8192, device=DEV)
            for _ in range(4):
                busy = (busy @ busy) * 1e-3
        torch.cuda.current_stream().synchronize()
        got = call()
        junk = [torch.full((n,), float("nan"), device=DEV) for n in (14000, 640, 512, 11200, 180, 20) for _ in range(8)]
        torch.cuda.synchronize()
        assert torch.equal(got, want)
        del junk
    v.close()
