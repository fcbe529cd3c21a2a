"""Rows of logits that a call of the log-probabilities does not read, and rows whose largest logits are shared by as many lanes as a list of
alternatives holds, or one more."""
import numpy as np
import pytest
import torch

from oracle import logprobs as ol
from test_gpu_logprobs import DEV, v  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V", [5, 1003, 40003])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_that_are_not_given_may_hold_anything(v, V, dtype):  # noqa: F811
    """With given_rows_only the rows without a token are unwritten memory of the caller's: here NaN and infinities.  Their gradients are zeros, those
    of the others are what they are without the option; also over the logits themselves, and with tokens of which one in a row is -1."""
    rng = np.random.default_rng(V)
    M = 9
    z = torch.from_numpy(rng.standard_normal((M, V)).astype(np.float32)).to(dtype).to(DEV)
    tokens = rng.integers(0, V, (M, 2)).astype(np.int32)
    tokens[[1, 2, 5, 8]] = -1
    tokens[3, 0] = -1
    absent = [1, 2, 5, 8]
    for i, bad in zip(absent, (float("nan"), float("inf"), -float("inf"), 3.0)):
        z[i] = bad
    tok = torch.from_numpy(tokens).to(DEV)
    g, gH = torch.randn(M, 2, device=DEV), torch.randn(M, device=DEV)
    keep = [m for m in range(M) if m not in absent]
    print(f"given rows V={V} {dtype}", flush=True)
    full = z.clone()                                      # the same batch (rows start at the same places) with nothing unwritten
    full[absent] = 1.0
    want = v.token_logprobs_grad(full, tok, v.token_logprobs(full, tok), grad_logprob=g, grad_entropy=gH)
    fwd = v.token_logprobs(z, tok, given_rows_only=True)
    got = v.token_logprobs_grad(z, tok, fwd, grad_logprob=g, grad_entropy=gH, given_rows_only=True)
    assert not got[absent].any() and torch.equal(got[keep], want[keep])
    from paper_2507_02659_amd import binding as ot
    given = v._logprob_in(z, tok, None, None, 0, True)
    ot.ot_token_logprobs_grad(v.ctx, given, ot.make_logprob_out(fwd), g, gH, z, V)
    assert torch.equal(z, got)


@pytest.mark.parametrize("n_top", [1, 63, 64])
@pytest.mark.parametrize("n_best", [62, 63, 64, 65, 256])
def test_best_logits_in_as_many_lanes(v, n_best, n_top):  # noqa: F811
    """n_best lanes of a workgroup hold one largest logit each, equal ones or not; the lanes next to them hold second best ones."""
    z = torch.full((3, 256 * 16), -1.0, device=DEV)
    lanes = torch.arange(n_best, device=DEV) * 4              # the first vector of lane i
    z[:, lanes] = 5.0
    z[1, lanes] += torch.randperm(n_best, device=DEV) * 0.01
    z[2, lanes + 1] = torch.linspace(1, 4, n_best, device=DEV)
    got = v.token_logprobs(z, n_top=n_top)
    want = ol.token_logprobs(z.double().cpu().numpy(), None, np.ones(3), n_top)
    print(f"lanes {n_best} alternatives {n_top}", flush=True)
    np.testing.assert_array_equal(got["top_ids"].cpu().numpy(), want["top_ids"])
    # exponents up to 6 * log2(e): three roundings of 2^-24 |t| and six half-steps on each exponential, as many on ln S; and the result's
    np.testing.assert_allclose(got["top_logprobs"].cpu().numpy(), want["top_logprobs"], rtol=2.0 ** -24, atol=(3 * 10 + 6) * 2.0 ** -24)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_gradients_that_share_memory_with_the_logits(v, dtype):  # noqa: F811
    """Rows next to the logits' rows, in front of them, behind all of them are taken; rows that end or start inside of them are refused, whatever
    the distance of the rows."""
    from paper_2507_02659_amd import binding as ot
    M, V, ld = 5, 100, 250
    gen = torch.Generator(device=DEV).manual_seed(1)
    memory = torch.zeros(4 * M * ld, dtype=dtype, device=DEV)
    start = M * ld + 70                                   # of the logits, whose rows lie ld apart
    rows = lambda at, step: memory[at:at + M * step].view(M, step)[:, :V]  # noqa: E731
    rows(start, ld).copy_(torch.randn(M, V, generator=gen, device=DEV))
    z = rows(start, ld).contiguous()
    tok, g = torch.zeros(M, dtype=torch.int32, device=DEV), torch.randn(M, generator=gen, device=DEV)
    fwd = v.token_logprobs(rows(start, ld), tok)
    want = v.token_logprobs_grad(z, tok, fwd, grad_logprob=g)
    size = memory.element_size()

    def call(at, step, M=M):
        given = ot.make_logprob_in(M=M, V=V, dtype=ot.OT_BF16 if dtype == torch.bfloat16 else ot.OT_F32, logits=memory.data_ptr() + start * size, ld=ld,
                                   tokens=tok, n_tok=1)
        ot.ot_token_logprobs_grad(v.ctx, given, ot.make_logprob_out(fwd), g, None, memory.data_ptr() + at * size, step)

    for at, step in ((start + 1, ld), (start - 1, ld), (start + V - 1, ld), (start - V + 1, ld), (start + ld, ld), (start + 2 * ld - 1, ld), (start - 3 * ld + 99, ld),
                     (start + V, ld + 1), (start + V, 101), (start - V, 120), (start - 3 * V, V)):
        with pytest.raises(ot.OtError) as e:
            call(at, step)
        assert e.value.code == ot.OT_ERR_SHAPE and "overlap" in e.value.message, (at - start, step)
    with pytest.raises(ot.OtError):
        call(start + 50, ld, M=1)
    # bit for bit only where rows start alike: the others' exponentials are the same, their places in a vector are not
    for at, step in ((start + V, ld), (start - V, ld), (start + V + 50, ld), (start - V - 50 - 2 * ld, ld), (start + M * ld, ld), (start + M * ld, V), (start - M * V, V), (0, V)):
        before = memory.clone()
        call(at, step)
        torch.cuda.synchronize()
        np.testing.assert_allclose(rows(at, step).float().cpu().numpy(), want.float().cpu().numpy(), rtol=2.0 ** -7 if dtype == torch.bfloat16 else 2.0 ** -22, atol=1e-30)
        assert torch.equal(rows(start, ld), z)
        rows(at, step).copy_(before[at:at + M * step].view(M, step)[:, :V])
        assert torch.equal(memory, before)                # nothing else was written
    call(start, ld)
    np.testing.assert_allclose(rows(start, ld).float().cpu().numpy(), want.float().cpu().numpy(), rtol=2.0 ** -7 if dtype == torch.bfloat16 else 2.0 ** -22, atol=1e-30)
