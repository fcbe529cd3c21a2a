"""The distillation loss from a teacher's top logits and its gradient against oracle/top_distill.py."""
import numpy as np
import pytest
import torch

from oracle.top_distill import BUCKET, DROP, RENORMALISE, top_distill

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
RESTS = [DROP, RENORMALISE, BUCKET]


def _verifier(V_t=16, V_d=1, dmap=None, **kw):
    from paper_2507_02659_amd.runner import Verifier
    return Verifier(d=8, V_t=V_t, V_d=V_d, dtype="bf16", W=torch.zeros(8, V_t, dtype=torch.bfloat16, device=DEV),
                    direct_map=np.zeros(V_d, np.int32) if dmap is None else dmap, max_batch=1, max_k=0, **kw)


@pytest.fixture(scope="module")
def v():
    ver = _verifier()
    yield ver
    ver.close()


def _put(x):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x)).to(DEV)


def _check(v, z, ids, lps, T=None, rest=DROP, g=None, tmap=None, row_off=None, temps=None, out=None, in_place=True):
    """Loss and gradient.  An exponential outside the kept ids takes a base-2 argument t with three roundings of 2^-24 |t|, the instruction and
    the sums in front of 64 bits six more half-steps: it is off by at most (3 |t| + 6) 2^-24 of itself, and the sum of the others by the mean of
    that under their distribution.  What the kept ids give is formed in 64 bits.  Results are rounded once (a gradient outside the kept ids: the
    factor, the product, then the type)."""
    M, V = z.shape
    print(f"top distill M={M} V={V} {z.dtype} stride={z.stride()} at {z.data_ptr() % 16} n={np.asarray(ids).shape[1]} rest={rest} map={tmap is not None}", flush=True)
    ids, lps = np.asarray(ids, np.int32), np.asarray(lps, np.float32)
    T_rows = None if T is None else np.asarray(T, np.float32)
    if temps is None:
        temps = T_rows
    Z = z.double().cpu().numpy()
    want, kept, grad, size = (x.astype(np.float64) for x in top_distill(Z, ids, lps, T_rows, rest, g, tmap))
    kw = dict(rest=rest, temperature=_put(temps), row_off=_put(row_off), through_map=tmap is not None)
    alone = v.top_distill_loss(z, _put(ids), _put(lps), **kw)
    got = v.top_distill_loss_grad(z, _put(ids), _put(lps), grad_loss=_put(g), out=out, **kw)
    assert got["grad"].dtype == z.dtype and got["grad"].shape == z.shape
    for n in alone:
        assert torch.equal(alone[n].nan_to_num(nan=-9.5), got[n].nan_to_num(nan=-9.5)), n
    t_rows = np.ones(M) if T_rows is None else np.where(T_rows > 0, np.maximum(T_rows.astype(np.float64), 2.0 ** -126), 1.0)
    with np.errstate(invalid="ignore", over="ignore", divide="ignore"):
        others = Z.copy()
        for m in range(M):
            for i in ids[m]:
                s = i if tmap is None or not 0 <= i < len(tmap) else tmap[i]
                if 0 <= s < V:
                    others[m, s] = -np.inf
        t = (others - others.max(1, keepdims=True)) / t_rows[:, None] / np.log(2)
        t = np.where(others > -np.inf, np.abs(t), 0.0)
        share = np.where(others > -np.inf, np.exp2(-t), 0.0)
        whole = share.sum(1, keepdims=True)
        share = share / np.where(whole > 0, whole, 1.0)
        each = (3 * t + 6) * 2.0 ** -24
        tol_S = (share * each).sum(1) + 2.0 ** -24
    P = np.where(np.isnan(kept), 0, kept)
    weight = np.maximum(P, 1.0)                           # in front of ln S, and of the others' logarithm
    host = {n: x.double().cpu().numpy() for n, x in got.items()}

    def near(a, b, tol):
        np.testing.assert_array_equal(np.isnan(a), np.isnan(b))
        big = np.isinf(b) | (np.abs(b) > 3e38)
        np.testing.assert_array_equal(np.where(big, a, 0), np.where(big, np.float32(b), 0))
        off = np.where(np.isnan(b) | big, 0, np.abs(a - b) - tol)
        assert off.max(initial=0) <= 0, (off.max(), np.unravel_index(off.argmax(), off.shape))

    magnitude = np.where(np.isfinite(want), np.abs(want), 0)
    near(host["loss"], want, 2.0 ** -24 * magnitude + 2 * weight * tol_S + 1e-12 * (1 + magnitude))
    near(host["kept"], kept, 2.0 ** -24 * P + 1e-15)
    size = np.where(np.isfinite(size), size, 0)
    tol = size * (np.where(others > -np.inf, each, 0) + 2 * tol_S[:, None] + 4 * 2.0 ** -24) + 2.0 ** -24 * np.abs(np.where(np.isfinite(grad), grad, 0)) + 1e-37
    factor = 4 * (np.ones(M) if g is None else np.abs(g)) * weight / t_rows      # the instruction flushes exponentials below 2^-126
    tol = tol + 2.0 ** -126 * factor[:, None]
    if z.dtype == torch.bfloat16:
        tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(np.where(np.isfinite(grad), grad, 0))
    with np.errstate(over="ignore"):
        near(host["grad"], grad, tol)
    if in_place and z.is_contiguous():
        own = z.clone()
        again = v.top_distill_loss_grad(own, _put(ids), _put(lps), grad_loss=_put(g), out=own, **kw)
        for n in got:
            assert torch.equal(again[n].nan_to_num(nan=-9.5), got[n].nan_to_num(nan=-9.5)), n
    return got


def _case(rng, M, V, n, dtype=torch.float32, V_teacher=None):
    """Distinct ids with probabilities that leave a little; a student near them."""
    V_teacher = V_teacher or V
    ids = np.stack([rng.permutation(V_teacher)[:n] for _ in range(M)]) if V_teacher < 5000 else np.stack([rng.choice(V_teacher, n, replace=False) for _ in range(M)])
    if ids.shape[1] < n:
        ids = np.concatenate((ids, np.full((M, n - ids.shape[1]), -1)), 1)
    lps = np.log(rng.dirichlet(np.full(n + 1, 0.3), M)[:, :n] + 1e-9).astype(np.float32)
    z = (2.0 * rng.standard_normal((M, V))).astype(np.float32)
    return torch.from_numpy(z).to(dtype).to(DEV), ids.astype(np.int32), lps


@pytest.mark.parametrize("rest", RESTS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 3, 5, 31, 64, 65, 127, 1000, 1023, 4096, 4097, 8192, 8201, 32003, 65543, 98311, 131073, 152064])
def test_lengths(v, V, dtype, rest):
    rng = np.random.default_rng(V)
    z, ids, lps = _case(rng, 3, V, 20, dtype)
    _check(v, z, ids, lps, 0.3 + rng.random(3), rest, rng.standard_normal(3).astype(np.float32))


@pytest.mark.parametrize("rest", RESTS)
@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 128, 129, 255, 256])
def test_numbers_of_ids(v, n, rest):
    rng = np.random.default_rng(n)
    for V, dtype in ((40, torch.float32), (256, torch.bfloat16), (5000, torch.float32)):
        z, ids, lps = _case(rng, 4, V, n, dtype)
        _check(v, z, ids, lps, None, rest)


@pytest.mark.parametrize("M,V", [(1, 32000), (2, 300), (257, 700), (600, 513), (3000, 100)])
def test_numbers_of_rows(v, M, V):
    rng = np.random.default_rng(M)
    z, ids, lps = _case(rng, M, V, 7, torch.bfloat16 if M % 2 else torch.float32)
    _check(v, z, ids, lps, 0.5 + rng.random(M), BUCKET, (rng.standard_normal(M) / M).astype(np.float32))


@pytest.mark.parametrize("rest", RESTS)
@pytest.mark.parametrize("V,dtype", [(16385, torch.float32), (32767, torch.float32), (32769, torch.bfloat16), (50257, torch.bfloat16)])
def test_more_long_rows_than_compute_units(v, V, dtype, rest):
    """Other workgroups than for a few such rows."""
    rng = np.random.default_rng(V)
    z, ids, lps = _case(rng, 300, V, 12, dtype)
    _check(v, z, ids, lps, 0.5 + rng.random(300), rest, rng.standard_normal(300).astype(np.float32))


@pytest.mark.parametrize("rest", RESTS)
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [50, 9000, 70001])
def test_masks_and_special_values(v, V, dtype, rest):
    rng = np.random.default_rng(V)
    M = 18
    z, ids, lps = _case(rng, M, V, 20, dtype)
    low, inf, nan = torch.finfo(dtype).min, float("inf"), float("nan")
    keep = torch.zeros(M, V, dtype=torch.bool, device=DEV)
    keep.scatter_(1, _put(ids).long(), True)
    z[0] = -inf                                           # masked whole
    z[1] = torch.where(keep[1], z[1], -inf)               # nothing outside the kept ids
    z[2] = torch.where(keep[2], -inf, z[2])               # nothing within them
    z[3, torch.from_numpy(rng.random(V) < 0.9).to(DEV)] = -inf
    z[4] = low
    z[5, torch.from_numpy(rng.random(V) < 0.9).to(DEV)] = low
    z[6, ids[6, 0]] = nan
    z[7, int((~keep[7]).nonzero()[0])] = nan
    z[8, ids[8, 3]] = inf
    z[9, int((~keep[9]).nonzero()[1])] = inf
    z[10] = nan
    ids[11] = -1                                          # no ids
    z[11] = nan
    ids[12, ::2] = -1
    lps[13] = -np.inf                                     # ids of probability 0
    lps[14, 2:] = -np.inf
    z[14, ids[14, 5]] = -inf                              # masked, and not asked for
    lps[15, 3] = np.nan
    lps[16, 3] = np.inf
    ids[17, 4] = V
    for T in (None, np.full(M, 0.01), np.full(M, 30.0), np.float32([0.0, -1.0, 1.0] * 6)):
        _check(v, z, ids, lps, T, rest, rng.standard_normal(M).astype(np.float32))
    ids[17, 4] = -2
    got = v.top_distill_loss_grad(z[17:], _put(ids[17:]), _put(lps[17:]), rest=rest)
    assert got["loss"].isnan().all() and got["grad"].isnan().all()


@pytest.mark.parametrize("rest", RESTS)
def test_rows_that_hold_a_nan_and_no_probability(v, rest):
    """The row is NaN whether its ids ask for it or not."""
    rng = np.random.default_rng(2)
    z, ids, lps = _case(rng, 4, 70, 5)
    lps[:] = -np.inf
    z[0, ids[0, 1]] = float("nan")
    z[1, int((torch.arange(70, device=DEV)[:, None] != _put(ids[1])[None]).all(1).nonzero()[0])] = float("nan")
    z[2, ids[2, 0]] = float("inf")
    got = _check(v, z, ids, lps, None, rest)
    assert got["loss"][:3].isnan().all() and not got["loss"][3].isnan()


@pytest.mark.parametrize("rest", RESTS)
def test_tiny_temperatures(v, rest):
    """Gradients past float32 and exponentials of 0 beside them: what is masked or too far to be reached stays 0."""
    rng = np.random.default_rng(1)
    z, ids, lps = _case(rng, 3, 300, 5)
    z[:, 200:] = -float("inf")
    got = v.top_distill_loss_grad(z, _put(ids), _put(lps), rest=rest, temperature=torch.full((3,), 1e-42, device=DEV), grad_loss=torch.full((3,), 1e3, device=DEV))
    assert not got["grad"].isnan().any() and (got["grad"][:, 200:] == 0).all()
    _check(v, z, ids, lps, np.full(3, 1e-6), rest)


@pytest.mark.parametrize("rest", RESTS)
@pytest.mark.parametrize("gap", [3.0, 12.0, 40.0, 300.0])
def test_a_sure_student(v, gap, rest):
    """The student all but agrees with a sure teacher, or is sure of another id: gradients and losses keep their digits."""
    rng = np.random.default_rng(int(gap))
    V = 3000
    z, ids, lps = _case(rng, 4, V, 6)
    z[0, ids[0, 0]] = gap                                 # the teacher's likeliest
    z[1, ids[1, :2]] = gap
    z[2, 2999] = gap                                      # one that it does not keep
    ids[2] = np.where(ids[2] == 2999, 0, ids[2])
    q = torch.log_softmax(z.double(), 1).cpu().numpy()
    for m in (0, 1, 3):                                   # of the student's own probabilities, nearly
        lps[m] = q[m, ids[m]] + 1e-3
    _check(v, z, ids, lps, None, rest)


@pytest.mark.parametrize("rest", RESTS)
def test_an_id_that_is_named_twice(v, rest):
    rng = np.random.default_rng(3)
    for n in (2, 70, 256):
        z, ids, lps = _case(rng, 3, 900, n)
        ids[0] = 5
        ids[1, 1::2] = ids[1, ::2][:ids[1, 1::2].size]
        ids[2, n // 2:] = ids[2, 0]
        _check(v, z, ids, lps, None, rest)


@pytest.mark.parametrize("rest", RESTS)
def test_through_the_direct_map(rest):
    rng = np.random.default_rng(4)
    V_t, V_d = 4000, 1501
    dmap = np.full(V_d, -1, np.int32)
    dmap[rng.permutation(V_d)[:1200]] = rng.permutation(V_t)[:1200]
    tmap = np.full(V_t, -1, np.int32)
    tmap[dmap[dmap >= 0]] = np.flatnonzero(dmap >= 0)
    ver = _verifier(V_t, V_d, dmap)
    z, ids, lps = _case(rng, 9, V_d, 40, torch.bfloat16, V_t)
    ids[0, :] = np.flatnonzero(tmap < 0)[:40]             # none of them has a draft id
    ids[1, ::3] = -1
    ids[2, 0] = V_t                                       # no target id
    ids[3, 0] = V_t - 1
    ids[4] = np.flatnonzero(tmap >= 0)[:40]
    got = _check(ver, z, ids, lps, 0.5 + rng.random(9), rest, None, tmap)
    assert got["loss"][0] == 0 and (got["grad"][0] == 0).all() and got["loss"][2].isnan()
    ver.close()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_and_alignment(v, dtype):
    rng = np.random.default_rng(9)
    for V, ld, at, ld_out, at_out in ((1003, 1003, 1, 1003, 1), (1003, 1003, 3, 1003, 0), (1000, 1024, 5, 1000, 2), (8192, 8200, 7, 8193, 3), (70001, 70001, 1, 70003, 0), (17, 40, 2, 17, 0)):
        z0, ids, lps = _case(rng, 5, V, 9, dtype)
        flat, to = torch.full((at + 5 * ld + 16,), float("nan"), device=DEV, dtype=dtype), torch.full((at_out + 5 * ld_out + 16,), -7.0, device=DEV, dtype=dtype)
        z, out = flat[at:at + 5 * ld].view(5, ld)[:, :V], to[at_out:at_out + 5 * ld_out].view(5, ld_out)[:, :V]
        z.copy_(z0)
        got = _check(v, z, ids, lps, None, BUCKET, out=out, in_place=False)   # (rows elsewhere: sums in another order)
        want = got["grad"].clone()
        out.fill_(-7.0)
        assert (to == -7).all()
        v.top_distill_loss_grad(z, _put(ids), _put(lps), rest=BUCKET, out=z)
        assert torch.equal(z, want)
        z.fill_(float("nan"))
        assert flat.isnan().all()


def test_temperatures_by_sequence(v):
    rng = np.random.default_rng(5)
    row_off, T = np.array([0, 3, 4, 9, 10], np.int32), np.array([1.0, 0.0, 0.4, 2.0], np.float32)
    z, ids, lps = _case(rng, 10, 900, 6)
    _check(v, z, ids, lps, np.repeat(T, np.diff(row_off)), BUCKET, row_off=row_off, temps=T)


def test_offsets_past_32_bits(v):
    M, V, ld = 5, 1500, 600_000_000
    z = torch.zeros((M - 1) * ld + V, dtype=torch.bfloat16, device=DEV).as_strided((M, V), (ld, 1))
    rng = np.random.default_rng(0)
    z0, ids, lps = _case(rng, M, V, 5, torch.bfloat16)
    z.copy_(z0)
    got = _check(v, z, ids, lps, None, BUCKET)
    own = v.top_distill_loss_grad(z, _put(ids), _put(lps), rest=BUCKET, out=z)
    assert torch.equal(own["grad"], got["grad"])


@pytest.mark.parametrize("V", [499_000, 1 << 20])
def test_the_widest_rows(v, V):
    """Rows whose bitmap takes most of a workgroup's shared memory."""
    rng = np.random.default_rng(1)
    z, ids, lps = _case(rng, 2, V, 9, torch.bfloat16)
    _check(v, z, ids, lps, None, BUCKET)


def test_rows_behind_the_last_stay_as_they_were(v):
    from paper_2507_02659_amd import binding as ot
    rng = np.random.default_rng(1)
    z, ids, lps = _case(rng, 3, 100, 4)
    ids, lps = _put(ids), _put(lps)
    given = ot.make_top_distill_in(M=3, V=100, dtype=ot.OT_F32, n_top=4, logits=z, ld=100, top_ids=ids, top_logprobs=lps, rest=BUCKET)
    loss, kept, grad = torch.full((5,), -7.0, device=DEV), torch.full((5,), -7.0, device=DEV), torch.full((5, 100), -7.0, device=DEV)
    ot.ot_top_distill_loss_grad(v.ctx, given, loss, kept, None, grad, 100)
    for x in (loss, kept, grad):
        assert (x[3:] == -7).all() and (x[:3] != -7).all()
    again = torch.full((5,), -7.0, device=DEV)
    ot.ot_top_distill_loss(v.ctx, given, again, None)
    assert torch.equal(again, loss)


def test_against_differences(v):
    """float32 logits moved by a quarter; the loss's differences in float32 are good to 2^-23 of the loss over the step."""
    rng = np.random.default_rng(2)
    z, ids, lps = _case(rng, 1, 30, 5)
    for rest in RESTS:
        got = v.top_distill_loss_grad(z, _put(ids), _put(lps), rest=rest)
        h = 2.0 ** -6
        many = z.repeat(60, 1)
        many[:30] += h * torch.eye(30, device=DEV)
        many[30:] -= h * torch.eye(30, device=DEV)
        loss = v.top_distill_loss(many, _put(ids.repeat(60, 0)), _put(lps.repeat(60, 0)), rest=rest)["loss"].double()
        d = (loss[:30] - loss[30:]) / (2 * h)
        # central differences: a third derivative (at most 1, of each of the two logarithms) times h^2 / 6, and the losses' roundings over 2 h
        tol = 2 * h * h / 6 + 2 * (2.0 ** -23 * float(loss.abs().max()) + 2.0 ** -20) / (2 * h)
        assert float((got["grad"][0].double() - d).abs().max()) <= tol


def test_what_token_logprobs_leaves(v):
    """The teacher's rows through token_logprobs: its alternatives are the ids, places that remain free are none."""
    rng = np.random.default_rng(7)
    teacher = torch.from_numpy((3 * rng.standard_normal((6, 2000))).astype(np.float32)).to(DEV)
    teacher[2, 10:] = -float("inf")                       # ten ids for twenty places
    teacher[3] = -float("inf")                            # none
    left = v.token_logprobs(teacher, n_top=20)
    z = torch.from_numpy((2 * rng.standard_normal((6, 2000))).astype(np.float32)).to(DEV)
    for rest in RESTS:
        got = _check(v, z, left["top_ids"].cpu().numpy(), left["top_logprobs"].cpu().numpy(), None, rest)
        assert got["loss"][3] == 0 and (got["grad"][3] == 0).all()
        assert float(got["kept"][2]) == pytest.approx(1.0, abs=1e-6)


def test_from_graphs_and_on_another_stream():
    rng = np.random.default_rng(6)
    stream = torch.cuda.Stream()
    ver = _verifier(stream=stream)
    with torch.cuda.stream(stream):
        made = []
        for M, V, n in ((1, 50001, 20), (40, 9000, 256), (2, 600_000, 9)):
            sets = []
            for _ in range(3):
                z, ids, lps = _case(rng, M, V, n)
                sets.append((z, _put(ids), _put(lps), torch.randn(M, device=DEV)))
            call = lambda z, i, p, g: ver.top_distill_loss_grad(z, i, p, rest=BUCKET, grad_loss=g)  # noqa: E731
            eager = [{k: x.clone() for k, x in call(*s).items()} for s in sets]
            own = [x.clone() for x in sets[0]]
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                out = call(*own)
            made.append((sets, eager, own, graph, out, call))
        for turn in (0, 1, 2, 1):
            for sets, eager, own, graph, out, call in made:
                for x, y in zip(own, sets[turn]):
                    x.copy_(y)
                graph.replay()
                again = call(*sets[turn])
                stream.synchronize()
                for k, want in eager[turn].items():
                    assert torch.equal(out[k], want) and torch.equal(again[k], want), k
    ver.close()
