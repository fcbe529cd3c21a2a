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
