"""The 4-bit head against oracle/quant_head.py: exact where the arithmetic is (small whole numbers), else within its rounding; every
kernel of it, ragged sizes, both scale types, every group; logits of other heads through ot_lm_head; steps; refusals."""
import numpy as np
import pytest
import torch

from oracle import quant_head as oq
from oracle import verify as ov

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def _weights(rng, d, V, group, scales, zeros, exact=False):
    from paper_2507_02659_amd.runner import QuantWeights
    G = -(-d // group)
    codes = rng.integers(0, 256, (d // 2, V)).astype(np.uint8)
    s = 2.0 ** rng.integers(-2, 3, (G, V)) if exact else rng.uniform(0.002, 0.02, (G, V)) * rng.choice([1.0, 1.0, 1.0, 0.01, -1.0, 0.0], (G, V))
    s = torch.from_numpy(s).to(torch.bfloat16 if scales == "bf16" else torch.float16)
    z = rng.integers(0, 16, (G, V)).astype(np.uint8) if zeros else None
    put = lambda a: None if a is None else torch.from_numpy(a).to(DEV)  # noqa: E731
    return QuantWeights(put(codes), s.to(DEV), put(z), group), (codes, s.double().numpy(), z, group)


def _verifier(w, rows):
    from paper_2507_02659_amd.runner import Verifier
    return Verifier.quantized(w, V_d=1, direct_map=np.zeros(1, np.int32), max_batch=rows, max_k=0)


def _tolerance(hidden, codes, scales, zeros, group):
    """Per element.  A group's sum holds products h (16 + c): its partial sums are at most about 3 B_g, with B_g the larger of the terms'
    2-norm (a random walk's) and of the sum itself, and up to 128 roundings of 2^-24 of those add up as a random walk, sqrt(128) 2^-24 3 B_g
    at the most; the offset's product and difference add two more.  Seven standard deviations of that are under 7 * 3 * 12 * 2^-24 B_g =
    252 * 2^-24 B_g; partial sums grow from nothing (their mean square is a third) and 128 roundings happen only if the matrix instruction
    rounds every addition: 100 * 2^-24.  Groups add as a random walk; the total is rounded once per group, at 3 times its own norm."""
    c, g = oq.unpack(codes), np.arange(hidden.shape[1]) // group
    G = scales.shape[0]
    zero = np.full(scales.shape, 8) if zeros is None else zeros & 15
    square, total = 0.0, 0.0
    for i in range(G):
        h, k = hidden[:, g == i], 16.0 + c[g == i]
        B = np.maximum(np.sqrt(h ** 2 @ k ** 2), np.maximum(np.abs(h @ k), np.abs(h.sum(1))[:, None] * (16.0 + zero[i])))
        square = square + (scales[i] * B) ** 2
        total = total + (scales[i] * (h @ (c[g == i] - zero[i]))) ** 2
    return 2.0 ** -24 * (100 * np.sqrt(square) + 7 * 3 * np.sqrt(G * total)) + 1e-30


def _bf16(x):
    t = torch.from_numpy(np.ascontiguousarray(x)).float().bfloat16()
    return t.to(DEV), t.double().numpy()


SHAPES = [(1, 128, 16), (1, 8, 1), (2, 40, 17), (3, 264, 100), (5, 1024, 515), (6, 136, 4099), (15, 392, 70), (16, 256, 257), (16, 4096, 1000), (17, 520, 64), (24, 2056, 333),
          (31, 128, 1000), (33, 1000, 515), (47, 640, 300), (64, 256, 2049), (65, 384, 70), (81, 904, 600), (96, 256, 500), (112, 264, 129), (128, 512, 300),
          (144, 1032, 1000), (145, 256, 515), (161, 384, 300), (300, 264, 700), (1000, 136, 333), (8, 8200, 130), (16, 12288, 60), (40, 12296, 33)]


@pytest.mark.parametrize("M,d,V", SHAPES)
def test_whole_numbers_come_out_exactly(M, d, V):
    """Small whole hidden states and scales that are powers of two: every sum is a whole number of quarters below 2^24 of them."""
    for i, (group, scales, zeros) in enumerate([(32, "bf16", True), (64, "f16", False), (128, "bf16", True), (128, "f16", False)]):
        rng = np.random.default_rng([M, d, V, i])
        w, given = _weights(rng, d, V, group, scales, zeros, exact=True)
        dev, h = _bf16(rng.integers(-1, 2, (M, d)).astype(np.float64))
        v = _verifier(w, M)
        print(f"exact {M}x{d}x{V} group {group} {scales} zeros {zeros}", flush=True)
        got = v.lm_head(dev).cpu().numpy()
        v.close()
        want = oq.logits(h, *given)
        assert np.abs(want).max() < 2 ** 22
        np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("M,d,V", [s for s in SHAPES if s[0] * s[1] * s[2] < 2e8])
def test_logits_within_their_rounding(M, d, V):
    for i, (group, scales, zeros) in enumerate([(128, "f16", True), (64, "bf16", True), (32, "f16", False)]):
        rng = np.random.default_rng([d, V, M, i])
        w, given = _weights(rng, d, V, group, scales, zeros)
        spread = rng.choice([0.01, 1.0, 1.0, 30.0], (M, 1)) * np.exp(rng.normal(0, 1, (1, d)))
        dev, h = _bf16((rng.standard_normal((M, d)) + rng.choice([0.0, 0.0, 2.0], (M, 1))) * spread)
        v = _verifier(w, M)
        print(f"logits {M}x{d}x{V} group {group} {scales}", flush=True)
        got = v.lm_head(dev).cpu().numpy()
        v.close()
        off = np.abs(got - oq.logits(h, *given)) / _tolerance(h, *given)
        assert off.max() <= 1.0, (off.max(), np.unravel_index(off.argmax(), off.shape))


def test_rows_are_their_own():
    """A NaN or an infinity stays in its row; rows past M and columns past V_t of the caller's memory stay as they were."""
    rng = np.random.default_rng(4)
    for M in (3, 16, 30, 100):
        w, given = _weights(rng, 264, 203, 64, "bf16", True)
        dev, h = _bf16(rng.standard_normal((M, 264)))
        dev[1, 5], dev[2, 263] = float("nan"), float("inf")
        from paper_2507_02659_amd import binding as ot
        v = _verifier(w, M)
        out = torch.full((M + 2, 256), -7.0, device=DEV)
        print("rows of their own", M, flush=True)
        ot.ot_lm_head(v.ctx, M, dev, out, 256)
        got = out.cpu().numpy()
        v.close()
        assert (got[M:] == -7).all() and (got[:, 203:] == -7).all()
        assert not np.isfinite(got[1:3, :203]).any()
        keep = [m for m in range(M) if m not in (1, 2)]
        want, tol = oq.logits(h[keep], *given), _tolerance(h[keep], *given)
        assert (np.abs(got[keep][:, :203] - want) <= tol).all()


def test_same_results_every_time_and_from_a_graph():
    from paper_2507_02659_amd.runner import Verifier
    rng = np.random.default_rng(6)
    stream = torch.cuda.Stream()
    for M in (2, 40):
        w, _ = _weights(rng, 512, 3001, 128, "f16", True)
        hidden = [_bf16(rng.standard_normal((M, 512)))[0] for _ in range(3)]
        v = Verifier.quantized(w, V_d=1, direct_map=np.zeros(1, np.int32), max_batch=M, max_k=0, stream=stream)
        with torch.cuda.stream(stream):
            eager = [v.lm_head(h).clone() for h in hidden]
            static = hidden[0].clone()
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                out = v.lm_head(static)
            for turn in range(2):
                for h, want in zip(hidden, eager):
                    static.copy_(h)
                    graph.replay()
                    stream.synchronize()
                    assert torch.equal(out, want)
                    assert torch.equal(v.lm_head(h), want)
        v.close()


@pytest.mark.parametrize("dtype,M", [("bf16", 1), ("bf16", 30), ("bf16", 200), ("f32", 5), ("f32", 40)])
def test_other_heads_give_their_steps_logits(dtype, M):
    """ot_lm_head of a bf16 or fp32 context: bit for bit what a step of as many rows leaves in the workspace in its separate structure."""
    from paper_2507_02659_amd import binding as ot
    from paper_2507_02659_amd.runner import Verifier
    from workloads import CaseSpec, make_case
    case = make_case(CaseSpec(name="lm_head", dtype=dtype, d=520, V_t=3001, V_d=400, k=[0] * M, temperature=[1.0] * M, n_direct=300, data_seed=M))
    v = Verifier.for_case(case, draft_side=ot.OT_DRAFT_SIDE_SEPARATE)
    inp = v.upload(case)
    v.step(inp)
    want = v.workspace(M, 0, with_logits=True)["logits"]
    got = v.lm_head(inp["hidden"]).cpu().numpy()
    v.close()
    np.testing.assert_array_equal(got, want)


@pytest.mark.parametrize("head,M", [("bf16", 1), ("bf16", 30), ("bf16", 200), ("f32", 5), ("f32", 40), ("4 bit", 3), ("4 bit", 40)])
def test_rows_of_logits_anywhere(head, M):
    """Rows an odd number of elements apart, from any element on: the same logits, and nothing between the rows is written."""
    from paper_2507_02659_amd import binding as ot
    from paper_2507_02659_amd.runner import Verifier
    d, V, ld = 520, 1003, 1009
    dtype = torch.float32 if head == "f32" else torch.bfloat16
    if head == "4 bit":
        v = _verifier(_weights(np.random.default_rng(M), d, V, 64, "bf16", True)[0], M)
    else:
        v = Verifier(d=d, V_t=V, V_d=1, dtype=head, W=torch.randn(d, V, device=DEV).to(dtype), direct_map=np.zeros(1, np.int32), max_batch=M, max_k=0)
    h = torch.randn(M, d, device=DEV).to(dtype)
    want = v.lm_head(h)
    for start in (0, 1, 2, 3):
        memory = torch.full((M * ld + 8,), -7.0, device=DEV)
        ot.ot_lm_head(v.ctx, M, h, memory.data_ptr() + 4 * start, ld)
        rows = memory[start: start + M * ld].view(M, ld)
        assert torch.equal(rows[:, :V], want)
        assert (rows[:, V:] == -7).all() and (memory[:start] == -7).all() and (memory[start + M * ld:] == -7).all()
    v.close()


@pytest.mark.parametrize("draft_side", ["AUTO", "IN_LM_HEAD"])
def test_a_step_through_a_quantized_head(draft_side):
    """Against the step of the oracle on the head's own logits: integers equal, probabilities to 1e-3."""
    import parity
    from paper_2507_02659_amd import binding as ot
    from paper_2507_02659_amd.runner import Verifier
    from workloads import CaseSpec, make_case
    rng = np.random.default_rng(12)
    for k in ([5], [3, 0, 4, 2], [8, 1, 0, 5, 8, 6, 2, 7]):
        case = make_case(CaseSpec(name="quant_step", dtype="bf16", d=264, V_t=2003, V_d=700, k=k, temperature=[[1.0, 0.7, 0.0][i % 3] for i in range(len(k))],
                                  n_direct=500, n_ngram=60, ngram_len=(2, 3), plant_cover=0.3, data_seed=len(k), philox_seed=9))
        w, given = _weights(rng, 264, 2003, 64, "bf16", True)
        v = Verifier.quantized(w, V_d=700, direct_map=case.direct_map, max_batch=case.B, max_k=8, max_ngram_len=case.max_ngram_len,
                               draft_side=getattr(ot, "OT_DRAFT_SIDE_" + draft_side))
        v.set_cache(case.ngram_key_off, case.ngram_key_ids, case.ngram_target_ids)
        assert ot.ot_verify_structure(v.ctx, case.B, case.M) == (ot.OT_STRUCTURE_SEPARATE, 3)
        inp = v.upload(case)
        v.step(inp)
        res = v.results(inp)
        ws = v.workspace(case.M, case.K, with_logits=True)
        v.close()
        h = ov.widen(case.hidden, "bf16")
        assert (np.abs(ws["logits"] - oq.logits(h, *given)) <= _tolerance(h, *given)).all()
        case.W, case.hidden, case.target_logits = None, None, ws["logits"]
        rep = parity.compare(case, res, ov.verify_case(case), logits_from_gpu=True)
        assert not rep.failures, rep.failures[:5]


def test_refusals():
    from paper_2507_02659_amd import binding as ot
    w, _ = _weights(np.random.default_rng(1), 64, 50, 32, "f16", False)
    v = _verifier(w, 4)
    h, out = torch.zeros(5, 64, dtype=torch.bfloat16, device=DEV), torch.empty(5, 50, device=DEV)

    def code(*args):
        with pytest.raises(ot.OtError) as e:
            ot.ot_lm_head(v.ctx, *args)
        return e.value.code

    assert code(5, h, out, 50) == ot.OT_ERR_SHAPE and code(-1, h, out, 50) == ot.OT_ERR_SHAPE
    assert code(4, h, out, 49) == ot.OT_ERR_SHAPE
    assert code(4, None, out, 50) == ot.OT_ERR_NULL and code(4, h, None, 50) == ot.OT_ERR_NULL
    assert code(4, h.data_ptr() + 2, out, 50) == ot.OT_ERR_SHAPE
    ot.ot_lm_head(v.ctx, 0, None, None, 50)
    for bad in (h.float(), h[:, :32], h[0]):
        with pytest.raises(ValueError):
            v.lm_head(bad)
    v.close()
