"""Inner sums of adapters that are not finite, and those next to the largest float: the row is NaN, or whole, whatever the type and the rank."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def v():
    from paper_2507_02659_amd.runner import Verifier
    ver = Verifier(d=8, V_t=16, V_d=1, dtype="bf16", W=torch.zeros(8, 16, dtype=torch.bfloat16, device=DEV), direct_map=np.zeros(1, np.int32),
                   max_batch=1, max_k=0)
    yield ver
    ver.close()


@pytest.mark.parametrize("dtype,R", [(torch.bfloat16, R) for R in (8, 16, 24, 32, 64, 72, 256)] + [(torch.float32, R) for R in (4, 16, 20, 32, 64, 68, 80, 256)])
@pytest.mark.parametrize("logits_type", [torch.float32, torch.bfloat16])
def test_rows_of_infinite_inner_sums_are_nan(v, dtype, R, logits_type):
    from paper_2507_02659_amd.runner import Adapters
    gen = torch.Generator(device=DEV).manual_seed(R)
    randn = lambda *s: torch.randn(*s, generator=gen, device=DEV)  # noqa: E731
    d, V = 32, 300
    down, up = (randn(2, R, d) / 6).to(dtype), (randn(2, V, R) / 4).to(dtype)
    hidden, z = randn(9, d).to(dtype), randn(9, V).to(logits_type)
    at = torch.tensor([0, 0, 0, 1, -1, 0, 1, 0, 0], dtype=torch.int32, device=DEV)
    scale = torch.tensor([1.0, 2.0], device=DEV)
    down[0, 0, :4] = 1.0
    up[:, :7, :R // 2] = 0.0
    hidden[7:, :4] = 2.0
    clean = v.adapter_logits(hidden, Adapters(down, up, scale), at, z)
    hidden[1, 3] = float("inf")
    hidden[2, 3] = -float("inf")
    hidden[3, :] = torch.where(down[1, 0] < 0, -3e38, 3e38)   # finite, but not their sum
    hidden[4, 0] = float("inf")                               # a row without an adapter
    hidden[5, :4] = 3e38                                      # one of the sums, of 4 products
    hidden[5, 4:] = 0
    for given in (z, None):
        got = v.adapter_logits(hidden, Adapters(down, up, scale), at, given)
        for m in (1, 2, 3, 5):
            assert got[m].isnan().all(), (m, given is None)
        if given is not None:
            assert torch.equal(got[[0, 4, 6, 7, 8]], clean[[0, 4, 6, 7, 8]])
    # through the scale
    got = v.adapter_logits(hidden[6:], Adapters(down, up, torch.tensor([3e38, 1.0], device=DEV)), at[6:], z[6:])
    big = (hidden[7:].double() @ down[0].double().t()).abs().amax(1) * 3e38 > 3.5e38
    assert big.all() and got[1:].isnan().all() and not got[0].isnan().any()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_the_largest_inner_sums(v, dtype):
    """24 significant bits below 2^128, from three bytes each: float32 holds them, the nearest bfloat16 may be infinite."""
    from paper_2507_02659_amd.runner import Adapters
    rng = np.random.default_rng(5)
    whole = np.concatenate(([2 ** 24 - 1, 0xFF8000, 0xFF7FFF, 0xFF0001], rng.integers(0xFF0000, 2 ** 24, 20))).astype(np.int64)
    M, d = whole.size, 32
    hidden = np.zeros((M, d))
    for k in range(3):
        hidden[:, k] = ((whole >> (8 * k)) & 255) * 256.0 ** k * 2.0 ** 104
    hidden[1::2] *= -1
    down, up = torch.zeros(1, 16, d), torch.zeros(1, 50, 16)
    down[0, 2, :3] = 1.0
    up[0, 13, 2], up[0, 14, 2] = 1.0, 0.5
    a = Adapters(down.to(dtype).to(DEV), up.to(dtype).to(DEV))
    got = v.adapter_logits(torch.from_numpy(hidden).to(dtype).to(DEV), a, torch.zeros(M, dtype=torch.int32, device=DEV)).cpu().numpy()
    want = (hidden.sum(1)).astype(np.float32)
    assert np.isfinite(want).all() and np.array_equal(got[:, 13], want) and np.array_equal(got[:, 14], want * np.float32(0.5))
    assert (got[:, :13] == 0).all() and (got[:, 15:] == 0).all()
