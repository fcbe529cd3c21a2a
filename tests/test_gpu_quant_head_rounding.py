"""How far the 4-bit head's logits are from the product of the weights in 64 bits: hidden rows with a mean, with an outlier channel, columns whose
codes equal their zero point, rows with an infinity."""
import numpy as np
import pytest
import torch

from test_gpu_quant_head import DEV, _verifier

pytestmark = pytest.mark.gpu


def _inputs(M, d, V, group, rows, columns):
    from paper_2507_02659_amd.runner import QuantWeights
    gen = torch.Generator(device=DEV).manual_seed(M + group)
    G = -(-d // group)
    each = torch.arange(d, device=DEV) // group
    zeros = torch.randint(4, 12, (G, V), generator=gen, device=DEV, dtype=torch.uint8)
    codes = (8.0 + 2.6 * torch.randn(d, V, generator=gen, device=DEV)).round().clamp(0, 15).to(torch.uint8)
    if columns == "equal":
        zeros = 7 + zeros % 2
        codes = zeros[each]
    scales = (0.01 * (0.5 + torch.rand(G, V, generator=gen, device=DEV))).bfloat16()
    h = torch.randn(M, d, generator=gen, device=DEV)
    h = h + 2.0 if rows == "mean" else h
    if rows == "outlier":
        h[:, 5] = 300.0
    return h.bfloat16(), QuantWeights((codes[0::2] | codes[1::2] << 4).contiguous(), scales, zeros, group), codes.double(), zeros.double()[each], scales.double(), each


@pytest.mark.parametrize("columns", ["normal", "equal"])
@pytest.mark.parametrize("rows", ["normal", "mean", "outlier"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("M", [6, 16, 40, 144])
def test_roundings(M, group, rows, columns):
    """Root mean square over all logits.  A rounding is off by at most 2^-24 of a partial sum, uniformly: 2^-24 / sqrt(3) rms.  Of a group's `group`
    additions every partial sum is within B / sqrt(2) rms, B the larger of the terms' 2-norm (a random walk's end) and of the sum itself; the
    sum of hidden states times |zp - 7.5| is another such sum, and its product and difference are two roundings more.  The total is rounded
    once a group (and, above 16 rows, once more an offset) at T / sqrt(2), T its end's 2-norm, and up to four groups' offsets."""
    d, V = 1024, 1003
    h, w, c, zp, s, each = _inputs(M, d, V, group, rows, columns)
    v = _verifier(w, M)
    print(f"roundings M={M} group={group} {rows} {columns}", flush=True)
    got = v.lm_head(h).double()
    v.close()
    H, k, G = h.double(), c - 7.5, s.shape[0]
    square, true, offset = 0.0, 0.0, 0.0
    for g in range(G):
        hg, kg, zg = H[:, each == g], k[each == g], (zp[each == g][0] - 7.5).abs()
        B = torch.maximum(((hg ** 2) @ (kg ** 2)).sqrt(), (hg @ kg).abs())
        U = zg * torch.maximum((hg ** 2).sum(1).sqrt(), hg.sum(1).abs())[:, None]
        square = square + s[g] ** 2 * (group / 2 * (B ** 2 + U ** 2) + 2 * torch.maximum(B, U) ** 2)
        true = true + (s[g] * (hg @ (c - zp)[each == g])) ** 2
        offset = torch.maximum(torch.as_tensor(offset, device=DEV), s[g] * zg * hg.sum(1).abs()[:, None])
    total = 2 * G * ((true / 2).sqrt() + (4 * offset if M > 16 else 0.0)) ** 2
    bound = 2.0 ** -24 / 3 ** 0.5 * (square + total).mean().sqrt()
    rms = (got - H @ ((c - zp) * s[each])).square().mean().sqrt()
    assert rms <= bound, (float(rms), float(bound))


@pytest.mark.parametrize("M", [1, 16, 40, 144])
def test_codes_that_equal_the_zero_point_of_8(M):
    """Up to 16 rows every group's product is exactly half the sum of its hidden states, and the logits are 0."""
    h, w, *_ = _inputs(M, 1024, 515, 128, "mean", "normal")
    w.codes.fill_(0x88)
    w.zeros = None
    v = _verifier(w, M)
    got = v.lm_head(h)
    v.close()
    # above 16 rows the scaled products of up to four groups stand in the total before their offsets are taken off: eight roundings per four groups
    # of sums of at most four times 0.5 * 0.015 sum |h|
    most = 0.0 if M <= 16 else 2 * 8 * 2.0 ** -24 * 4 * 0.5 * 0.015 * float(h.double().abs().view(M, 8, 128).sum(2).max())
    assert float(got.abs().max()) <= most


@pytest.mark.parametrize("M", [3, 16, 30, 100])
@pytest.mark.parametrize("value", [float("inf"), -float("inf"), float("nan")])
def test_rows_with_an_infinity_are_nan(M, value):
    """Whatever the codes: all above 7.5, all below, the zero point itself; a scale of 0."""
    h, w, *_ = _inputs(M, 264, 203, 64, "normal", "normal")
    h[1, 263] = value
    w.codes[:, :50], w.codes[:, 50:100], w.codes[:, 100:120] = 0xFF, 0x00, 0x77
    w.zeros[:, 100:120] = 7
    w.scales[:, 110:130] = 0.0
    v = _verifier(w, M)
    got = v.lm_head(h)
    v.close()
    assert torch.isnan(got[1]).all() and torch.isfinite(got[torch.arange(M, device=DEV) != 1]).all()
