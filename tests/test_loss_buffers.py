"""The buffers that the loss's calls share: allocated and filled on the verifier's stream, and by each verifier for itself (host only)."""
import contextlib

import torch

from paper_2507_02659_amd.runner import Verifier


def _verifier(V_t, stream):
    v = Verifier.__new__(Verifier)
    v.device, v.V_t, v.stream, v.ctx, v.cache = torch.device("cpu"), V_t, stream, None, None
    v._number = next(Verifier._numbers)
    return v


def _watch(monkeypatch):
    """Every torch.full with the stream that is current then."""
    current, filled, full = [None], [], torch.full

    @contextlib.contextmanager
    def stream(s):
        before, current[0] = current[0], s
        yield
        current[0] = before

    def watched(*args, **kw):
        filled.append(current[0])
        return full(*args, **kw)

    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch, "full", watched)
    return filled


def test_filled_on_the_verifiers_stream(monkeypatch):
    """The launches on that stream write and read them: a fill on any other one may come between."""
    filled = _watch(monkeypatch)
    own = object()
    for with_qprime in (False, True):
        v, inp = _verifier(7, own), {"M": 3}
        buf = v._loss_buffers(inp, with_qprime)
        assert len(filled) >= 5 and all(s is own for s in filled)
        assert v._loss_buffers(inp, with_qprime) is buf
        filled.clear()


def test_two_verifiers_of_one_batch_have_their_own(monkeypatch):
    _watch(monkeypatch)
    inp = {"M": 3}
    a, b = _verifier(7, object()), _verifier(9, object())
    first, second = a._loss_buffers(inp, True), b._loss_buffers(inp, True)
    assert first is not second and tuple(first["qprime"].shape) == (3, 7) and tuple(second["qprime"].shape) == (3, 9)
    assert not {t.data_ptr() for t in first.values()} & {t.data_ptr() for t in second.values()}
    assert a._loss_buffers(inp, True) is first and b._loss_buffers(inp, True) is second
