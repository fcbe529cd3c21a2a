"""Long rows in other workgroups where there are few of them: the same values, with the loss alone the same bits."""
import numpy as np
import pytest
import torch

from oracle.top_distill import BUCKET
from test_gpu_top_distill import _case, _check, _verifier

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("V,dtype", [(33003, torch.float32), (81920, torch.float32), (196608, torch.bfloat16), (196609, torch.bfloat16), (300003, torch.bfloat16)])
def test_on_both_sides_of_the_compute_units(V, dtype):
    cu = torch.cuda.get_device_properties(0).multi_processor_count
    rng = np.random.default_rng(V)
    v = _verifier()
    z, ids, lps = _case(rng, 2, V, 20, dtype)
    pairs = _check(v, z, ids, lps, None, BUCKET)
    many = {}
    for M in (cu // 2, cu // 2 + 1, cu, cu + 1):      # (the oracle's two rows, again and again)
        at = torch.arange(M, device=z.device) % 2
        put = lambda x: torch.from_numpy(x).to(z.device)[at]  # noqa: E731
        own = z[at]
        loss = v.top_distill_loss(own, put(ids), put(lps), rest=BUCKET)
        many[M] = v.top_distill_loss_grad(own, put(ids), put(lps), rest=BUCKET, out=own)
        for n in loss:
            assert torch.equal(loss[n], many[M][n])
        # sums in another order: each addition in 64 bits, of exponentials whose tree sums of eight are the same; rounded once
        assert float((many[M]["loss"] - pairs["loss"][at]).abs().max()) <= 2.0 ** -22 * (1 + float(pairs["loss"].abs().max()))
        assert torch.equal(many[M]["grad"][:2], many[M]["grad"][cu // 2 - 2:cu // 2])
    v.close()
