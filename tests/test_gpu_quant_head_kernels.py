"""Every kernel of the 4-bit head that a size can reach: row tiles, column tiles and wavefronts per workgroup, 32-deep steps per scale, parts of
the hidden dimension; vocabularies up to several rounds of the chip and ragged ones, hidden dimensions that leave a remainder of blocks."""
import numpy as np
import pytest
import torch

from test_gpu_quant_head import DEV, _verifier

pytestmark = pytest.mark.gpu


def _ceil(a, b):
    return -(-a // b)


def _choice(M, d, V, group, n_cu):
    """The launch that a call takes: ("up to 16", column tiles, ...) or ("above 16", row tiles, column tiles, wavefronts, steps per scale)."""
    tiles, blocks, steps = _ceil(V, 16), _ceil(d, 128), group // 32
    if M <= 16:
        rounds = _ceil(tiles, 64 * n_cu)
        per_cu = _ceil(tiles, rounds * n_cu)
        S = _ceil(per_cu, 16)
        return "up to 16", S, max(1, min(16 // _ceil(per_cu, S), blocks)) > 1, steps
    m_blocks = _ceil(M, 144)
    RT = _ceil(M, 16 * m_blocks)
    best = None
    for s in (1, 2, 4)[:3 if steps == 4 and RT <= 5 else 2]:
        for waves in (8, 7, 6):
            cost = _ceil(_ceil(tiles, s * waves) * m_blocks, n_cu) * s * waves * {4: 6, 2: 7, 1: 8}[s]
            if best is None or (cost, -s) < best[0]:
                best = (cost, -s), s, waves
    return "above 16", RT, best[1], best[2], steps


def _whole_numbers(gen, d, V, group):
    """Random codes, zero points, scales that are powers of two; the weights in 64 bits."""
    from paper_2507_02659_amd.runner import QuantWeights
    G = _ceil(d, group)
    codes = torch.randint(0, 256, (d // 2, V), generator=gen, device=DEV, dtype=torch.uint8)
    zeros = torch.randint(0, 16, (G, V), generator=gen, device=DEV, dtype=torch.uint8)
    scales = torch.exp2(torch.randint(-2, 3, (G, V), generator=gen, device=DEV).float()).bfloat16()
    W = torch.stack((codes & 15, codes >> 4), 1).reshape(d, V).double()
    each = torch.arange(d, device=DEV) // group
    return QuantWeights(codes, scales, zeros, group), (W - zeros.double()[each]) * scales.double()[each]


WIDTHS = [(1003, 392), (26003, 136), (30003, 264), (40003, 640), (50003, 264), (60003, 136), (66003, 520), (100003, 264), (128001, 136)]
REACHED = set()


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("V,d", WIDTHS)
def test_above_16_rows(V, d, group):
    gen = torch.Generator(device=DEV).manual_seed(V + d + group)
    w, W = _whole_numbers(gen, d, V, group)
    v = _verifier(w, 161)
    n_cu = torch.cuda.get_device_properties(0).multi_processor_count
    for M in [16 * rt - 3 for rt in range(2, 10)] + ([145, 161] if V < 70000 else []):
        h = torch.randint(-1, 2, (M, d), generator=gen, device=DEV).bfloat16()
        kernel = _choice(M, d, V, group, n_cu)
        print(f"{M}x{d}x{V} groups of {group}: {kernel}", flush=True)
        got = v.lm_head(h)
        assert torch.equal(got.double(), h.double() @ W), kernel
        REACHED.add(kernel)
    v.close()


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("V,d", [(4099, 640), (20003, 1032), (60003, 264), (70003, 392), (140003, 136), (200003, 264), (280003, 136)])
def test_up_to_16_rows(V, d, group):
    gen = torch.Generator(device=DEV).manual_seed(V + d + group)
    w, W = _whole_numbers(gen, d, V, group)
    v = _verifier(w, 16)
    n_cu = torch.cuda.get_device_properties(0).multi_processor_count
    for M in (1, 2, 7, 16):
        h = torch.randint(-1, 2, (M, d), generator=gen, device=DEV).bfloat16()
        kernel = _choice(M, d, V, group, n_cu)
        print(f"{M}x{d}x{V} groups of {group}: {kernel}", flush=True)
        assert torch.equal(v.lm_head(h).double(), h.double() @ W), kernel
        REACHED.add(kernel)
    v.close()


def test_every_kernel_was_reached():
    """Of the tests above, where all of them ran on a whole MI355X."""
    if torch.cuda.get_device_properties(0).multi_processor_count != 256 or len(REACHED) < 20:
        pytest.skip("the sizes are chosen for 256 compute units and all tests of this file")
    tall = {k[1:3] + k[4:] for k in REACHED if k[0] == "above 16"}
    want = {(rt, s, steps) for rt in range(2, 10) for s in (1, 2, 4) for steps in (1, 2, 4) if s < 4 or (steps == 4 and rt <= 5)}
    assert tall == want, want - tall
    assert {k[3] for k in REACHED if k[0] == "above 16"} == {6, 7, 8}
    assert {k[1::2] for k in REACHED if k[0] == "up to 16"} == {(s, steps) for s in (1, 2, 3, 4) for steps in (1, 2, 4)}
    assert {k[2] for k in REACHED if k[0] == "up to 16"} == {True, False}
