"""Calls made while another stream than the verifier's is current, and busy."""
import pytest
import torch

from test_gpu_distill_grad import _spec
from workloads import make_case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("with_qprime", [False, True])
@pytest.mark.parametrize("V_d", [301, 20000])
def test_the_loss_gradient_of_a_first_call(V_d, with_qprime):
    """The call's buffers are new.  Both forms of the gradient: rows in one workgroup, and (q' rows wanted, or few wide rows) the gather."""
    from paper_2507_02659_amd.runner import Verifier
    case = make_case(_spec("streams", [5, 3, 6], 12, V_t=3000, V_d=V_d, n_direct=250))
    v = Verifier.for_case(case, stream=torch.cuda.Stream())
    inp = v.upload(case)
    torch.cuda.synchronize()                              # inputs are ready on every stream
    v.step(inp, from_logits=True)
    v.synchronize()
    busy = torch.randn(8192, 8192, device="cuda:0")
    print(f"first call V_d={V_d} q'={with_qprime}", flush=True)
    for _ in range(4):
        busy = (busy @ busy) * 1e-3                       # tens of milliseconds on the default stream
    first = v.distill_loss_grad(inp, from_logits=True, with_qprime=with_qprime)
    v.synchronize()
    torch.cuda.synchronize()
    first = {n: t.clone() for n, t in first.items()}
    again = v.distill_loss_grad(inp, from_logits=True, with_qprime=with_qprime)
    torch.cuda.synchronize()
    for n in first:
        assert torch.equal(first[n], again[n]), n
    v.close()


def test_inputs_dropped_before_the_work_is_done():
    """Tensors of the default stream that the caller drops right after the call, while the verifier's stream is still busy: what the default
    stream allocates and writes next does not land in them."""
    import numpy as np

    from paper_2507_02659_amd.runner import Verifier
    d, V, M = 512, 4099, 40
    gen = torch.Generator(device="cuda:0").manual_seed(5)
    W = torch.randn(d, V, generator=gen, device="cuda:0").bfloat16()
    v = Verifier(d=d, V_t=V, V_d=1, dtype="bf16", W=W, direct_map=np.zeros(1, np.int32), max_batch=M, max_k=0, stream=torch.cuda.Stream())
    hidden = torch.randn(M, d, generator=gen, device="cuda:0").bfloat16()
    z = torch.randn(M, V, generator=gen, device="cuda:0")
    tok = torch.randint(0, V, (M,), generator=gen, device="cuda:0", dtype=torch.int32)
    T, g, gH = torch.rand(M, generator=gen, device="cuda:0") + 0.5, torch.randn(M, generator=gen, device="cuda:0"), torch.randn(M, generator=gen, device="cuda:0")
    torch.cuda.synchronize()
    want = v.lm_head(hidden)
    fwd = v.token_logprobs(z, tok, temperature=T, n_top=5)
    grad = v.token_logprobs_grad(z, tok, fwd, grad_logprob=g, grad_entropy=gH, temperature=T)
    busy = torch.randn(8192, 8192, device="cuda:0")
    torch.cuda.synchronize()
    with torch.cuda.stream(v.stream):
        for _ in range(4):
            busy = (busy @ busy) * 1e-3                   # tens of milliseconds on the verifier's stream
    copies = [t.clone() for t in (hidden, z, tok, T, g, gH)]
    torch.cuda.current_stream().synchronize()             # ready
    got = v.lm_head(copies[0])
    lp = v.token_logprobs(copies[1], copies[2], temperature=copies[3], n_top=5)
    dz = v.token_logprobs_grad(copies[1], copies[2], fwd, grad_logprob=copies[4], grad_entropy=copies[5], temperature=copies[3])
    shapes = [(t.shape, t.dtype) for t in copies]
    del copies
    held = [torch.zeros(shape, dtype=dtype, device="cuda:0") for _ in range(3) for shape, dtype in shapes]
    torch.cuda.synchronize()
    assert torch.equal(got, want) and torch.equal(dz, grad) and all(torch.equal(lp[n], fwd[n]) for n in fwd) and len(held) == 18
    v.close()
