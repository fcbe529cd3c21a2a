"""A window that could be counted into the flags beside a count is refused, on the host."""
import ctypes as C

import pytest

from paper_2507_02659_amd import binding as ot

AT = 0x10000
MEMORY = C.create_string_buffer(b"\xff" * (1 << 14))      # a context of device -1, which is never the current one: no address is followed


def test_windows_longer_than_a_count_holds():
    """2^29 ids of history and 2^29 - 1 tokens of a window in front of its last row: together below 2^30, where the flags begin."""
    def code(M, **kw):
        given = ot.make_adjust_in(M=M, V=1, B=1, dtype=ot.OT_F32, ld=1, logits=AT, row_off=AT, **kw)
        with pytest.raises(ot.OtError) as e:
            ot.ot_adjust_logits(C.addressof(MEMORY), given, AT + (1 << 40), 1)
        assert e.value.message.startswith("ot_adjust_logits: ")
        return e.value.code

    assert code(2 ** 29 + 1, window=AT) == ot.OT_ERR_SHAPE
    assert code(2 ** 31 - 1, window=AT, history=AT, ld_history=2 ** 29) == ot.OT_ERR_SHAPE
    for M, kw in ((2 ** 29, dict(window=AT)), (2 ** 29 + 1, {})):     # these get as far as the device
        assert code(M, **kw) in (ot.OT_ERR_HIP, ot.OT_ERR_CTX_MISMATCH)
