"""An error names the entry point that was called, also where that shares its checks with another one."""
import numpy as np
import pytest

from paper_2507_02659_amd import binding as ot

GOOD = dict(d=64, V_t=100, V_d=50, max_batch=2, max_k=4, max_ngram_len=3, direct_map=np.full(50, -1, np.int32))
BAD = [dict(d=0), dict(d=60), dict(max_k=64), dict(max_ngram_len=1), dict(direct_map=None), dict(draft_side=9), dict(max_batch=1 << 20),
       dict(direct_map=np.full(50, 100, np.int32)), dict(direct_map=np.zeros(50, np.int32))]


def _message(call, *args, **kw):
    with pytest.raises(ot.OtError) as e:
        call(*args, **kw)
    return e.value.message


@pytest.mark.parametrize("bad", BAD)
def test_init(bad):
    """Nothing here reaches a HIP call."""
    for name, more in (("ot_verify_init", dict(W=0x1000, dtype=ot.OT_BF16)),
                       ("ot_verify_init_quantized", dict(codes=0x1000, scales=0x1000, zeros=None, group=32, scale_dtype=ot.OT_BF16))):
        assert _message(getattr(ot, name), **{**GOOD, **more, **bad}).startswith(name + ": ")


def _loss(ctx, grad, **kw):
    empty = dict({n: None for n in ("row_off", "row_off_host", "hidden", "draft_logits", "draft_ids", "temperature", "draft_temperature", "seq_id")},
                 B=1, step=0, seed=0)
    args = dict(dict(lam=0.2, lambda_mode=0, ngram_term=0, accepted_only=False, buffers={n: 0x1000 for n in ot.LOSS_OUT}), **kw)
    more = dict(grad_loss=None, grad=0x1000) if grad else {}
    call = ot.ot_distill_loss_grad if grad else ot.ot_distill_loss
    return _message(call, ctx, ot.make_step_in(**empty), ot.make_step_out({}), None, **args, **more)


def test_loss_without_a_context():
    assert _loss(None, False).startswith("ot_distill_loss: ")
    assert _loss(None, True).startswith("ot_distill_loss_grad: ")


@pytest.mark.gpu
def test_loss():
    import torch
    v = ot.ot_verify_init(**GOOD, dtype=ot.OT_F32, W=torch.zeros(64, 100, device="cuda:0"))
    for bad in (dict(lambda_mode=7), dict(ngram_term=7), dict(buffers={}), {}):
        assert _loss(v, False, **bad).startswith("ot_distill_loss: "), bad
        assert _loss(v, True, **bad).startswith("ot_distill_loss_grad: "), bad
    ot.ot_verify_destroy(v)
