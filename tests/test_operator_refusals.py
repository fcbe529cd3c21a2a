"""What adapters, adjusted logits and the distillation from top logits refuse, all on the host and before a device is asked for: the context is a
block of zeros (V_d = 0) and no address is followed.  What is not refused ends in the question for the current device, or on a GPU there."""
import ctypes as C

import pytest
import torch

from paper_2507_02659_amd import binding as ot
from paper_2507_02659_amd.runner import Adapters, Verifier

CTX = C.create_string_buffer(1 << 14)
AT = 0x10000


def _code(call, *args):
    with pytest.raises(ot.OtError) as e:
        call(C.addressof(CTX), *args)
    name = call.__name__ if hasattr(call, "__name__") else ""
    assert e.value.message.startswith(name + ": "), e.value.message
    return e.value.code


# Sizes that a launch cannot count pass every check but the last one.
def _adapter(out=AT + (1 << 40), ld_out=100, **kw):
    base = dict(M=4, d=16, V=100, rank=8, n_adapters=2, dtype=ot.OT_BF16, hidden=AT, down=AT, up=AT, adapter=AT, logits=AT, ld=100)
    return _code(ot.ot_adapter_logits, ot.make_adapter_in(**dict(base, **kw)), out, ld_out)


def test_adapters():
    S, N, D = ot.OT_ERR_SHAPE, ot.OT_ERR_NULL, ot.OT_ERR_DTYPE
    for kw in (dict(M=-1), dict(d=0), dict(d=2 ** 24 + 8), dict(V=0), dict(V=2 ** 30 + 1, ld=2 ** 31, ld_out=2 ** 31), dict(n_adapters=0), dict(ld=99), dict(ld_out=99), dict(rank=0),
               dict(rank=264), dict(rank=4), dict(rank=12), dict(d=12), dict(rank=6, dtype=ot.OT_F32), dict(reserved=1), dict(hidden=AT + 8), dict(down=AT + 4),
               dict(up=AT + 2), dict(logits=AT + 2), dict(out=AT + 1), dict(out=AT + 4), dict(out=AT, ld_out=101), dict(out=AT + 4 * 99), dict(out=AT - 4 * 350),
               dict(V=2 ** 30, ld=2 ** 30, ld_out=2 ** 30, M=2048, out=1 << 50)):
        assert _adapter(**kw) == S, kw
    for name in ("hidden", "down", "up", "adapter"):
        assert _adapter(**{name: None}) == N, name
    assert _adapter(out=None) == N
    for kw in (dict(dtype=ot.OT_F16), dict(dtype=7), dict(logits_dtype=ot.OT_F16), dict(logits_dtype=-1)):
        assert _adapter(**kw) == D, kw
    lib = ot.load_library()
    assert lib.ot_adapter_logits(None, None, None, 0) == N
    ot.ot_adapter_logits(C.addressof(CTX), ot.make_adapter_in(M=0, d=16, V=100, rank=8, n_adapters=2, dtype=ot.OT_BF16, hidden=None, down=None, up=None, adapter=None),
                         None, 100)


def _adjust(out=AT + (1 << 40), ld_out=100, **kw):
    base = dict(M=4, V=100, B=4, dtype=ot.OT_F32, ld=100, logits=AT)
    return _code(ot.ot_adjust_logits, ot.make_adjust_in(**dict(base, **kw)), out, ld_out)


def test_adjusted_logits():
    S, N, D = ot.OT_ERR_SHAPE, ot.OT_ERR_NULL, ot.OT_ERR_DTYPE
    for kw in (dict(M=-1), dict(V=0), dict(V=2 ** 30 + 1, ld=2 ** 31, ld_out=2 ** 31), dict(ld=99), dict(ld_out=99), dict(B=3), dict(B=5), dict(B=-1, row_off=AT),
               dict(reserved=(1, 0)), dict(reserved=(0, 1)), dict(n_bias=-1), dict(n_bias=4097, bias=AT, bias_ids=AT), dict(history=AT, ld_history=2 ** 29 + 1), dict(n_masks=-1), dict(ld_history=-1), dict(masks=AT, n_masks=4, ld_mask=3),
               dict(window=AT), dict(masks=AT, n_masks=3, ld_mask=4), dict(logits=AT + 2), dict(out=AT + 2), dict(out=AT, ld_out=101),
               dict(out=AT + 4 * 99), dict(V=2 ** 30, ld=2 ** 30, ld_out=2 ** 30, M=100, B=100, out=1 << 50)):
        assert _adjust(**kw) == S, kw
    for kw in (dict(logits=None), dict(out=None), dict(n_bias=2, bias=AT), dict(n_bias=2, bias_ids=AT), dict(ld_history=3), dict(n_masks=4, ld_mask=4)):
        assert _adjust(**kw) == N, kw
    assert _adjust(dtype=ot.OT_F16) == D and _adjust(dtype=5) == D
    lib = ot.load_library()
    assert lib.ot_adjust_logits(None, None, None, 0) == N
    for kw in (dict(M=0, B=0), dict(M=0, B=3, row_off=AT), dict(M=4, B=0, row_off=AT)):
        ot.ot_adjust_logits(C.addressof(CTX), ot.make_adjust_in(**dict(dict(V=100, dtype=ot.OT_F32, ld=100), **kw)), None, 100)


def _distill(grad=False, loss=AT, out=AT + (1 << 40), ld_grad=100, **kw):
    base = dict(M=4, V=100, dtype=ot.OT_F32, n_top=5, logits=AT, ld=100, top_ids=AT, top_logprobs=AT)
    given = ot.make_top_distill_in(**dict(base, **kw))
    if grad:
        return _code(ot.ot_top_distill_loss_grad, given, loss, None, None, out, ld_grad)
    return _code(ot.ot_top_distill_loss, given, loss, None)


@pytest.mark.parametrize("grad", [False, True])
def test_distillation_from_top_logits(grad):
    S, N, D = ot.OT_ERR_SHAPE, ot.OT_ERR_NULL, ot.OT_ERR_DTYPE
    wide = dict(ld_grad=2 ** 22) if grad else {}
    for kw in (dict(M=-1), dict(V=0), dict(V=2 ** 20 + 1, ld=2 ** 22, **wide), dict(ld=99), dict(n_top=0), dict(n_top=257), dict(rest=-1), dict(rest=3), dict(reserved=1),
               dict(through_map=True), dict(row_off=AT, temperature=AT), dict(row_off=AT, B=2), dict(logits=AT + 2), dict(M=2 ** 23, **(dict(out=1 << 50) if grad else {}))):
        assert _distill(grad, **kw) == S, kw
    for kw in (dict(logits=None), dict(top_ids=None), dict(top_logprobs=None), dict(loss=None)):
        assert _distill(grad, **kw) == N, kw
    assert _distill(grad, dtype=ot.OT_F16) == D and _distill(grad, dtype=5) == D
    if grad:
        for kw in (dict(ld_grad=99), dict(out=AT + 2), dict(out=AT, ld_grad=101), dict(out=AT + 4 * 99)):
            assert _distill(True, **kw) == S, kw
        assert _distill(True, out=None) == N
    lib = ot.load_library()
    assert lib.ot_top_distill_loss(None, None, None, None) == N and lib.ot_top_distill_loss_grad(None, None, None, None, None, None, 0) == N


# ------------------------------------------------------------------------------------------------ the Python methods
class Reached(Exception):
    pass


@pytest.fixture
def v(monkeypatch):
    def reached(*args, **kw):
        raise Reached

    for name in ("ot_lm_head", "ot_adapter_logits", "ot_adjust_logits", "ot_top_distill_loss", "ot_top_distill_loss_grad"):
        monkeypatch.setattr(ot, name, reached)
    v = Verifier.__new__(Verifier)
    v.device, v.stream, v.ctx, v.cache, v._number = torch.device("cpu"), None, None, None, -1   # (stands for the GPU)
    v.dtype, v.d, v.V_t, v.V_d = "bf16", 16, 40, 30
    return v


def _try(call, good, bad):
    with pytest.raises(Reached):
        call(**good)
    for change in bad:
        with pytest.raises((ValueError, TypeError)):
            call(**dict(good, **change))
    for name, t in good.items():
        if isinstance(t, torch.Tensor):
            with pytest.raises(ValueError, match=name + " is "):
                call(**dict(good, **{name: t.to("meta")}))


def test_adapter_method(v):
    bf16 = torch.bfloat16
    down, up, scale = torch.zeros(2, 8, 16, dtype=bf16), torch.zeros(2, 40, 8, dtype=bf16), torch.ones(2)
    hidden, of_row, z = torch.zeros(3, 16, dtype=bf16), torch.zeros(3, dtype=torch.int32), torch.zeros(3, 40)
    good = dict(hidden=hidden, adapters=Adapters(down, up, scale), adapter_of_row=of_row, logits=z, out=torch.zeros(3, 44)[:, :40])
    bad = [dict(adapters=Adapters(*a)) for a in ((down.float(), up), (down.half(), up.half()), (down[0], up[0]), (down, up[:1]), (down[:, :4], up), (down.transpose(1, 2), up),
                                                 (down, up, scale.double()), (down, up, scale[:1]), (down, up.transpose(1, 2)))]
    bad += [dict(hidden=h) for h in (hidden.float(), hidden[:, :8], hidden[0], torch.zeros(16, 3, dtype=bf16).t())]
    bad += [dict(adapter_of_row=a) for a in (of_row.long(), of_row[:2], of_row[:, None])]
    bad += [dict(logits=x) for x in (z[:2], z[:, :39], z.half(), torch.zeros(40, 3).t())]
    bad += [dict(out=x) for x in (z.bfloat16(), z[:2], torch.zeros(40, 3).t(), z[:1].expand(3, 40))]
    _try(v.adapter_logits, good, bad)
    for name, a in (("down", Adapters(down.to("meta"), up)), ("up", Adapters(down, up.to("meta"))), ("scale", Adapters(down, up, scale.to("meta")))):
        with pytest.raises(ValueError, match=name + " is on meta"):
            v.adapter_logits(**dict(good, adapters=a))
    with pytest.raises(ValueError, match="head's adapters"):
        v.lm_head(hidden, adapters=Adapters(down, up[:, :39]), adapter_of_row=of_row)
    with pytest.raises(ValueError, match="together"):
        v.lm_head(hidden, adapters=Adapters(down, up))
    with pytest.raises(ValueError, match="together"):
        v.lm_head(hidden, adapter_of_row=of_row)


def test_adjust_method(v):
    i32 = torch.int32
    good = dict(logits=torch.zeros(5, 40), row_off=torch.tensor([0, 2, 5], dtype=i32), history=torch.zeros(2, 7, dtype=i32), n_history=torch.zeros(2, dtype=i32),
                n_prompt=torch.zeros(2, dtype=i32), window=torch.zeros(5, dtype=i32), repetition=torch.ones(2), frequency=torch.ones(2), presence=torch.ones(2),
                bias_ids=torch.zeros(2, 3, dtype=i32), bias=torch.zeros(2, 3), masks=torch.zeros(4, 2, dtype=i32), mask_of_row=torch.zeros(5, dtype=i32))
    bad = [{n: t[:1]} for n, t in good.items() if n not in ("logits", "masks")] + [{n: t.double()} for n, t in good.items()]
    bad += [dict(bias=None), dict(bias_ids=None), dict(bias_ids=good["bias_ids"][0]), dict(history=good["history"][0]), dict(masks=good["masks"][:, :1]),
            dict(masks=good["masks"][0]), dict(mask_of_row=None), dict(out=torch.zeros(5, 39)), dict(out=torch.zeros(5, 40).bfloat16()), dict(logits=torch.zeros(40, 5).t())]
    _try(v.adjust_logits, good, bad)


def test_distill_methods(v):
    good = dict(logits=torch.zeros(4, 30), top_ids=torch.zeros(4, 3, dtype=torch.int32), top_logprobs=torch.zeros(4, 3), temperature=torch.ones(2),
                row_off=torch.tensor([0, 2, 4], dtype=torch.int32))
    bad = [dict(top_ids=good["top_ids"][:3]), dict(top_ids=good["top_ids"][:, :2]), dict(top_ids=good["top_ids"].long()), dict(top_logprobs=torch.zeros(4, 2)),
           dict(top_logprobs=torch.zeros(4, 3).double()), dict(top_ids=good["top_ids"][0]), dict(temperature=torch.ones(4)), dict(row_off=good["row_off"].long()),
           dict(logits=torch.zeros(4, 30).half()), dict(logits=torch.zeros(30, 4).t()), dict(logits=torch.zeros(4, 40), through_map=True)]
    _try(v.top_distill_loss, good, bad)
    _try(v.top_distill_loss_grad, dict(good, grad_loss=torch.ones(4), through_map=True),
         bad + [dict(grad_loss=torch.ones(3)), dict(grad_loss=torch.ones(4).double()), dict(out=torch.zeros(4, 29)), dict(out=torch.zeros(4, 30).bfloat16())])


def test_the_binding_takes_no_host_memory(monkeypatch):
    class Library:
        def __getattr__(self, name):
            return lambda *args: pytest.fail("reached the library")

    monkeypatch.setattr(ot, "load_library", Library)
    host = torch.zeros(4)
    adapter = dict(M=1, d=8, V=4, rank=8, n_adapters=1, dtype=0, hidden=AT, down=AT, up=AT, adapter=AT, scale=AT, logits=AT, ld=4)
    distill = dict(M=1, V=4, dtype=1, n_top=1, logits=AT, ld=4, top_ids=AT, top_logprobs=AT, temperature=AT, row_off=AT, B=1)
    adjust = dict({n: AT for n in ot.ADJUST_ARRAYS}, M=1, V=4, B=1, dtype=1, ld=4)
    for make, given in ((ot.make_adapter_in, adapter), (ot.make_top_distill_in, distill), (ot.make_adjust_in, adjust)):
        make(**given)
        for name, x in given.items():
            if x == AT:
                with pytest.raises(ValueError, match="host memory"):
                    make(**dict(given, **{name: host}))
    for call, args in ((ot.ot_adapter_logits, (None, ot.make_adapter_in(**adapter), host, 4)), (ot.ot_adjust_logits, (None, ot.make_adjust_in(**adjust), host, 4)),
                       (ot.ot_top_distill_loss, (None, ot.make_top_distill_in(**distill), host, None)),
                       (ot.ot_top_distill_loss, (None, ot.make_top_distill_in(**distill), AT, host)),
                       (ot.ot_top_distill_loss_grad, (None, ot.make_top_distill_in(**distill), AT, None, host, AT, 4)),
                       (ot.ot_top_distill_loss_grad, (None, ot.make_top_distill_in(**distill), AT, None, None, host, 4))):
        with pytest.raises(ValueError, match="host memory"):
            call(*args)


def test_struct_layouts_match_the_header():
    import os
    import re
    text = re.sub(r"/\*.*?\*/", "", open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include", "otverify.h")).read(), flags=re.S)
    for cls, size in ((ot.ot_adapter_in, 8 * 4 + 8 + 6 * 8), (ot.ot_adjust_in, 8 * 4 + 3 * 8 + 13 * 8), (ot.ot_top_distill_in, 8 * 4 + 8 + 5 * 8)):
        body = re.search(r"typedef struct %s \{(.*?)\} %s;" % (cls.__name__, cls.__name__), text, flags=re.S).group(1)
        names = []
        for decl in filter(None, (d.strip() for d in body.split(";"))):
            names += [re.sub(r"\[.*\]", "", n).strip().lstrip("*") for n in re.sub(r"^(const\s+)?\w+\s*\**", "", decl).split(",")]
        assert [f[0] for f in cls._fields_] == names and C.sizeof(cls) == size, cls.__name__
