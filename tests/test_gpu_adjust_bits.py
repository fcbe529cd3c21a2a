"""Adjusted logits: an id that nothing names keeps its bits, also next to one that something does; there a NaN of bfloat16 stays one."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.mark.parametrize("L", [3, 8200])
def test_every_bfloat16_next_to_a_marked_id(L):
    """All 65536 patterns, NaNs of every kind among them, with one id of each vector of eight named in turn."""
    from paper_2507_02659_amd.runner import Verifier
    v = Verifier(d=8, V_t=16, V_d=1, dtype="bf16", W=torch.zeros(8, 16, dtype=torch.bfloat16, device=DEV), direct_map=np.zeros(1, np.int32), max_batch=1, max_k=0)
    bits = torch.from_numpy(np.random.default_rng(0).permutation(65536).astype(np.uint16).view(np.int16)).to(DEV).view(torch.bfloat16)
    z = bits.repeat(8, 1)
    n = 4096
    ids = torch.stack([torch.arange(n, device=DEV) * 8 + m for m in range(8)]).int()
    keep = torch.ones(8, 65536, dtype=torch.bool, device=DEV).scatter_(1, ids.long(), False)
    masks = torch.full((8, 2048), -1, dtype=torch.int32, device=DEV)
    masks[1::2, 1::2] = 0x7FFFFFFF                        # ids of 31 mod 64 left out
    keep[1::2, 63::64] = False
    history = torch.full((8, L), -1, dtype=torch.int32, device=DEV)
    history[:, 0] = ids[:, 0]
    given = dict(history=history, presence=torch.ones(8, device=DEV), bias_ids=ids, bias=torch.ones(8, n, device=DEV), masks=masks)
    own = z.clone()
    for got in (v.adjust_logits(z, **given), v.adjust_logits(own, out=own, **given)):
        numbers = keep & ~z.isnan()
        assert torch.equal(got.view(torch.int16)[numbers], z.view(torch.int16)[numbers])
        assert got[keep & z.isnan()].isnan().all()
    v.close()
