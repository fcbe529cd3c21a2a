"""Distances between rows past the address space: whether outputs overlap inputs is found out without leaving 64 bits or dividing by 0."""
import ctypes as C

import pytest

from paper_2507_02659_amd import binding as ot

AT = 0x10000
MEMORY = C.create_string_buffer(b"\xff" * (1 << 14))      # a context of device -1, which is never the current one: no address is followed
CTX = C.addressof(MEMORY)
REFUSED, REACHED = (ot.OT_ERR_SHAPE,), (ot.OT_ERR_HIP, ot.OT_ERR_CTX_MISMATCH)      # reached: the question for the current device


def _adjust(M, ld, out):
    ot.ot_adjust_logits(CTX, ot.make_adjust_in(M=M, V=100, B=M, dtype=ot.OT_F32, ld=ld, logits=AT), out, ld)


def _adapter(M, ld, out):
    given = ot.make_adapter_in(M=M, d=16, V=100, rank=8, n_adapters=1, dtype=ot.OT_BF16, hidden=AT, down=AT, up=AT, adapter=AT, logits=AT, ld=ld)
    ot.ot_adapter_logits(CTX, given, out, ld)


def _distill(M, ld, out):
    given = ot.make_top_distill_in(M=M, V=100, dtype=ot.OT_F32, n_top=5, logits=AT, ld=ld, top_ids=AT, top_logprobs=AT)
    ot.ot_top_distill_loss_grad(CTX, given, AT, None, None, out, ld)


@pytest.mark.parametrize("call", [_adjust, _adapter, _distill])
@pytest.mark.parametrize("M", [1, 2, 3])
@pytest.mark.parametrize("ld", [2 ** 62, 2 ** 61 + 2 ** 30, 2 ** 63 - 1])
def test_rows_that_share_memory_are_refused(call, M, ld):
    for out, codes in ((AT + 4 * 99, REFUSED), (AT - 4 * 99, REFUSED), (AT + 4 * 100, REACHED), (AT - 4 * 100, REACHED)):
        with pytest.raises(ot.OtError) as e:
            call(M, ld, out)
        assert e.value.code in codes, (out - AT, e.value.message)
