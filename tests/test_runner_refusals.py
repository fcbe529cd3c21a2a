"""What the Python entry points refuse on the host, before an address reaches the library: tensors that are not on the verifier's device,
statistics and logits of another shape or type.  No GPU and no context: a call that is not refused ends in Reached."""
import pytest
import torch

from paper_2507_02659_amd import binding as ot
from paper_2507_02659_amd.runner import QuantWeights, Verifier


class Reached(Exception):
    pass


@pytest.fixture
def v(monkeypatch):
    def reached(*args, **kw):
        raise Reached

    for name in ("ot_lm_head", "ot_token_logprobs", "ot_token_logprobs_grad", "ot_distill_loss_grad", "ot_verify_init_quantized"):
        monkeypatch.setattr(ot, name, reached)
    v = Verifier.__new__(Verifier)
    v.device, v.stream, v.ctx, v.cache, v._number = torch.device("cpu"), None, None, None, -1   # (stands for the GPU)
    v.dtype, v.d, v.V_t, v.V_d = "bf16", 16, 40, 30
    return v


def _elsewhere(v):
    v.device = torch.device("cuda:0")


def _case():
    z = torch.zeros(4, 40)
    return dict(logits=z, tokens=torch.zeros(4, dtype=torch.int32)), {n: torch.zeros(4) for n in ("row_max", "row_sumexp", "entropy")}


def test_hidden_rows_elsewhere(v):
    hidden = torch.zeros(2, 16, dtype=torch.bfloat16)
    with pytest.raises(Reached):
        v.lm_head(hidden)
    _elsewhere(v)
    with pytest.raises(ValueError, match="hidden is on cpu"):
        v.lm_head(hidden)


def test_rows_of_logits_elsewhere(v, monkeypatch):
    given, _ = _case()
    more = dict(temperature=torch.ones(2), row_off=torch.tensor([0, 2, 4], dtype=torch.int32))
    with pytest.raises(Reached):
        v.token_logprobs(**given, **more)
    here = Verifier._here
    for name in ("logits", "tokens", "temperature", "row_off"):

        def one_elsewhere(self, **tensors):
            here(self, **{n: t for n, t in tensors.items() if n != name})
            self.device = torch.device("cuda:0")
            here(self, **{n: t for n, t in tensors.items() if n == name})

        monkeypatch.setattr(Verifier, "_here", one_elsewhere)
        v.device = torch.device("cpu")
        with pytest.raises(ValueError, match=name + " is on cpu"):
            v.token_logprobs(**given, **more)


def test_statistics_of_another_call(v):
    given, forward = _case()
    grads = dict(grad_logprob=torch.zeros(4), grad_entropy=torch.zeros(4))
    with pytest.raises(Reached):
        v.token_logprobs_grad(**given, forward=forward, **grads)
    for name in forward:
        for bad in (torch.zeros(3), torch.zeros(4, 1), torch.zeros(4, dtype=torch.float64), None):
            with pytest.raises(ValueError, match=name):
                v.token_logprobs_grad(**given, forward=dict(forward, **{name: bad}), **grads)
        with pytest.raises(ValueError, match=name):
            v.token_logprobs_grad(**given, forward={n: t for n, t in forward.items() if n != name}, **grads)
    with pytest.raises(Reached):                          # without a gradient of the entropy it is not read
        v.token_logprobs_grad(**given, forward=dict(forward, entropy=None), grad_logprob=grads["grad_logprob"])
    for name in ("row_max", "row_sumexp", "entropy", "grad_logprob", "grad_entropy"):
        away = torch.zeros(4, device="meta")
        with pytest.raises(ValueError, match=name + " is on meta"):
            v.token_logprobs_grad(**given, forward=dict(forward, **({name: away} if name in forward else {})), **dict(grads, **({name: away} if name in grads else {})))


def test_draft_logits_of_another_type(v):
    none = {n: None for n in ("row_off", "row_off_host", "hidden", "draft_ids", "temperature", "draft_temperature", "seq_id", "target_logits")}
    out = {n: None for n in ("n_mapped", "n_accept", "mapped_ids", "span_start", "span_len", "p_tok")}
    inp = dict(none, B=1, M=3, K=2, step=0, seed=0, out=out, draft_logits=torch.zeros(2, 30, dtype=torch.bfloat16))
    with pytest.raises(Reached):
        v.distill_loss_grad(inp)
    for bad in (torch.zeros(2, 30), torch.zeros(2, 29, dtype=torch.bfloat16), torch.zeros(1, 30, dtype=torch.bfloat16),
                torch.zeros(2, 30, dtype=torch.bfloat16, device="meta")):
        with pytest.raises(ValueError, match="draft"):
            v.distill_loss_grad(dict(inp, draft_logits=bad))
    with pytest.raises(ValueError, match="grad_loss is on meta"):
        v.distill_loss_grad(inp, grad_loss=torch.ones(1, device="meta"))


@pytest.mark.parametrize("away", ["codes", "scales", "zeros"])
def test_weights_elsewhere(v, monkeypatch, away):
    for name in ("is_available", "set_device", "current_device", "synchronize"):
        monkeypatch.setattr(torch.cuda, name, {"is_available": lambda: True, "current_device": lambda: 0}.get(name, lambda *a: None))
    w = dict(codes=torch.zeros(8, 40, dtype=torch.uint8), scales=torch.zeros(1, 40, dtype=torch.bfloat16), zeros=torch.zeros(1, 40, dtype=torch.uint8))
    args = dict(V_d=1, direct_map=None, max_batch=1, max_k=0, device="cpu")
    with pytest.raises(Reached):
        Verifier.quantized(QuantWeights(**w), **args)
    with pytest.raises(ValueError, match=away + " is on meta"):
        Verifier.quantized(QuantWeights(**dict(w, **{away: w[away].to("meta")})), **args)


def test_the_binding_takes_no_host_memory(monkeypatch):
    """The entry points' mirrors: a tensor or an array in host memory is refused wherever the device reads or writes, before the library is called."""
    import numpy as np

    class Library:
        def __getattr__(self, name):
            return lambda *args: pytest.fail("reached the library")

    monkeypatch.setattr(ot, "load_library", Library)
    for host in (torch.zeros(4), np.zeros(4, np.float32)):
        for args in ((None, 1, host, 0x1000, 4), (None, 1, 0x1000, host, 4)):
            with pytest.raises(ValueError, match="host memory"):
                ot.ot_lm_head(*args)
        given = dict(M=1, V=4, dtype=ot.OT_F32, logits=0x1000, ld=4, tokens=0x1000, n_tok=1, temperature=0x1000, row_off=0x1000, B=1)
        for name in ("logits", "tokens", "temperature", "row_off"):
            with pytest.raises(ValueError, match="host memory"):
                ot.make_logprob_in(**dict(given, **{name: host}))
        for name in ot.LOGPROB_OUT:
            with pytest.raises(ValueError, match="host memory"):
                ot.make_logprob_out({name: host})
        for at in (3, 4, 5):
            args = [None, ot.make_logprob_in(**given), ot.make_logprob_out({}), 0x1000, 0x1000, 0x1000, 4]
            args[at] = host
            with pytest.raises(ValueError, match="host memory"):
                ot.ot_token_logprobs_grad(*args)
        weights = dict(codes=0x1000, scales=0x1000, zeros=None)
        for name in weights:
            with pytest.raises(ValueError, match="host memory"):
                ot.ot_verify_init_quantized(d=8, V_t=4, V_d=1, max_batch=1, max_k=0, max_ngram_len=2, group=32, scale_dtype=ot.OT_BF16, direct_map=None,
                                            **dict(weights, **{name: host}))
        for name in ("grad_loss", "grad"):
            sin = ot.make_step_in(B=0, step=0, seed=0, **{n: None for n in ("row_off", "row_off_host", "hidden", "draft_logits", "draft_ids", "temperature",
                                                                            "draft_temperature", "seq_id")})
            with pytest.raises(ValueError, match="host memory"):
                ot.ot_distill_loss_grad(None, sin, ot.make_step_out({}), None, lam=0.2, lambda_mode=0, ngram_term=0, accepted_only=False, buffers={},
                                        **dict(dict(grad_loss=None, grad=0x1000), **{name: host}))
