"""Penalties, biases and masks against oracle/adjust.py."""
import numpy as np
import pytest
import torch

from oracle.adjust import adjust_logits

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def v():
    from paper_2507_02659_amd.runner import Verifier
    ver = Verifier(d=8, V_t=16, V_d=1, dtype="bf16", W=torch.zeros(8, 16, dtype=torch.bfloat16, device=DEV), direct_map=np.zeros(1, np.int32),
                   max_batch=1, max_k=0)
    yield ver
    ver.close()


def _put(x):
    if x is None or isinstance(x, torch.Tensor):
        return x
    x = np.asarray(x)
    return torch.from_numpy(np.ascontiguousarray(x, np.int32 if x.dtype.kind in "iu" else np.float32)).to(DEV)


def _words(bits):
    """bool [n, V] as int32 words."""
    n, V = bits.shape
    b = np.zeros((n, -(-V // 32) * 32), bool)
    b[:, :V] = bits
    return (b.reshape(n, -1, 32).astype(np.uint64) << np.arange(32, dtype=np.uint64)).sum(2).astype(np.uint32).view(np.int32)


def _check(v, z, out=None, in_place=True, **kw):
    """Every id against the oracle.  The value is formed in 64 bits from a few operands and rounded once to float32 and, of bfloat16 logits, once
    more: half a step of the type, plus 2^-24 for bfloat16's first rounding, plus 2^-50 of the operands."""
    print(f"adjust {tuple(z.shape)} {z.dtype} stride={z.stride()} at {z.data_ptr() % 16} " + " ".join(f"{n}={np.asarray(x).shape}" for n, x in kw.items()), flush=True)
    Z = z.double().cpu().numpy()
    want = adjust_logits(Z, **kw)
    as_type = torch.from_numpy(want).float().to(z.dtype).double().numpy()
    want = np.where(np.isinf(as_type), as_type, want)     # past the type's range
    given = {n: _put(x) for n, x in kw.items()}
    got = v.adjust_logits(z, out=out, **given)
    assert torch.equal(z.double().cpu().nan_to_num(), torch.from_numpy(Z).nan_to_num()), "the input"
    f = {n: np.abs(np.asarray(kw.get(n, 0.0), np.float64)).max(initial=0) for n in ("repetition", "frequency", "presence")}
    bias = np.asarray(kw.get("bias", np.zeros(1)), np.float64)
    many = f["frequency"] * 1e5 + f["presence"] + np.abs(np.where(np.isfinite(bias), bias, 0)).max(initial=0)
    rho = np.asarray(kw.get("repetition", np.ones(1)), np.float64)
    operands = np.where(np.isfinite(Z), np.abs(Z), 0) * max(rho.max(initial=1), (1 / rho).max(initial=1)) + many
    bf16 = z.dtype == torch.bfloat16
    with np.errstate(invalid="ignore", over="ignore"):
        tol = np.abs(want) * (2.0 ** -8 + 2.0 ** -24 if bf16 else 2.0 ** -24) + 2.0 ** -50 * operands + (2.0 ** -133 if bf16 else 2.0 ** -149)
        for x in (got, v.adjust_logits(z.clone(), **given) if z.is_contiguous() else None):
            if x is None:
                continue
            host = x.double().cpu().numpy()
            np.testing.assert_array_equal(np.isnan(host), np.isnan(want))
            np.testing.assert_array_equal(np.isinf(host) * np.sign(host), np.isinf(want) * np.sign(want))
            off = np.where(np.isfinite(want), np.abs(host - want) - tol, 0)
            assert off.max(initial=0) <= 0, (off.max(), np.unravel_index(off.argmax(), off.shape))
            same = (want == Z) | (np.isnan(want) & np.isnan(Z))
            assert (host[same & ~np.isnan(Z)] == Z[same & ~np.isnan(Z)]).all(), "what nothing names"
    if in_place:
        own = z.clone() if z.is_contiguous() else z
        back = v.adjust_logits(own, out=own, **given)
        assert back.data_ptr() == own.data_ptr() and torch.equal(back.view(torch.int32 if z.element_size() == 4 else torch.int16),
                                                                 got.view(torch.int32 if z.element_size() == 4 else torch.int16))
    return got


def _logits(rng, M, V, dtype=torch.float32):
    return torch.from_numpy((2.0 * rng.standard_normal((M, V))).astype(np.float32)).to(dtype).to(DEV)


def _all(rng, B, rows, V, L=40, n_bias=5, n_masks=None, masked=0.7):
    """Every argument, for sequences of the given numbers of rows."""
    off = np.concatenate(([0], np.cumsum(rows))).astype(np.int32)
    M = int(off[-1])
    n_masks = max(1, M // 2) if n_masks is None else n_masks
    ids = lambda *shape: np.where(rng.random(shape) < 0.5, rng.integers(-1, V + 2, shape), rng.integers(0, max(1, V // 20), shape)).astype(np.int32)  # noqa: E731
    kw = dict(row_off=off, history=ids(B, L), n_history=rng.integers(0, L + 1, B).astype(np.int32), window=ids(M), repetition=(0.5 + rng.random(B)).astype(np.float32),
              frequency=rng.standard_normal(B).astype(np.float32), presence=rng.standard_normal(B).astype(np.float32),
              bias_ids=ids(B, n_bias), bias=(3 * rng.standard_normal((B, n_bias))).astype(np.float32),
              masks=_words(rng.random((n_masks, V)) < masked), mask_of_row=rng.integers(-1, n_masks, M).astype(np.int32))
    kw["n_prompt"] = (kw["n_history"] * rng.random(B)).astype(np.int32)
    return M, kw


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("V", [1, 2, 7, 31, 32, 33, 64, 255, 1000, 1023, 1024, 1025, 2047, 2049, 4095, 4096, 4097, 8191, 12289, 32003, 130001])
def test_lengths(v, V, dtype):
    rng = np.random.default_rng(V)
    rows = [3, 1, 4] if V < 9000 else [2, 1]
    M, kw = _all(rng, len(rows), rows, V)
    _check(v, _logits(rng, M, V, dtype), **kw)


@pytest.mark.parametrize("V", [1, 33, 4095, 16383, 16385, 40003])
def test_long_histories(v, V):
    """The larger workgroups: slices of 16384 ids, of ragged windows."""
    rng = np.random.default_rng(V)
    M, kw = _all(rng, 3, [2, 70, 1], V, L=8500, n_bias=9)
    _check(v, _logits(rng, M, V), **kw)
    _check(v, _logits(rng, M, V, torch.bfloat16), **kw)


@pytest.mark.parametrize("rows", [[1], [64], [1] * 70, [5, 0, 9, 1, 64, 2], [200], [3] * 300])
@pytest.mark.parametrize("V", [300, 5000])
def test_numbers_of_rows(v, rows, V):
    rng = np.random.default_rng(len(rows) + V)
    M, kw = _all(rng, len(rows), rows, V)
    _check(v, _logits(rng, M, V, torch.bfloat16 if len(rows) % 2 else torch.float32), **kw)


def test_each_alone(v):
    """One argument at a time, none at all, single tokens without row_off."""
    rng = np.random.default_rng(0)
    for dtype in (torch.float32, torch.bfloat16):
        z = _logits(rng, 6, 5003, dtype)
        M, kw = _all(rng, 6, [1] * 6, 5003)
        assert torch.equal(v.adjust_logits(z), z)
        got = v.adjust_logits(z, history=_put(kw["history"]))              # without penalties a history changes nothing
        assert torch.equal(got, z)
        del kw["row_off"], kw["window"]
        for names in (("history", "repetition"), ("history", "frequency"), ("history", "presence"), ("history", "n_history", "frequency", "presence"),
                      ("history", "n_prompt", "presence"), ("bias_ids", "bias"), ("masks", "mask_of_row")):
            _check(v, z, **{n: kw[n] for n in names})
        _check(v, z, masks=_words(rng.random((8, 5003)) < 0.3))            # more masks than rows: a row's own
        # arrays without entries
        _check(v, z, history=np.zeros((6, 0), np.int32), n_history=np.zeros(6, np.int32), presence=kw["presence"], bias_ids=np.zeros((6, 0), np.int32),
               bias=np.zeros((6, 0), np.float32), masks=np.zeros((0, 157), np.int32), mask_of_row=np.array([-1, -1, 0, -1, 5, -2], np.int32))
        _check(v, z, row_off=np.array([0, 2, 6], np.int32), window=kw["history"][:6, 0].copy(), frequency=np.float32([0.5, 2.0]))


@pytest.mark.parametrize("L", [0, 1, 2, 255, 257, 5000, 40000])
def test_histories(v, L):
    """One id thousands of times, many ids, lengths past the array and below 0, a prompt past the length."""
    rng = np.random.default_rng(L)
    V = 9001
    history = rng.integers(-2, V + 5, (5, L)).astype(np.int32)
    history[0, :] = 77
    history[1, L // 2:] = V - 1
    kw = dict(history=history, n_history=np.array([L, L, L + 9, -3, L // 2], np.int32), n_prompt=np.array([L // 3, L + 4, -1, 2, 0], np.int32),
              repetition=np.float32([1.5, 0.8, 1.2, 3.0, 1.0]), frequency=np.float32([0.01, 0.3, -0.2, 1.0, 0.5]), presence=np.float32([0.5, -0.5, 0, 1, 2]))
    _check(v, _logits(rng, 5, V), **kw)
    _check(v, _logits(rng, 5, V, torch.bfloat16), **kw)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masks_and_special_values(v, dtype):
    rng = np.random.default_rng(4)
    V = 4500
    z = _logits(rng, 12, V, dtype)
    low, high = torch.finfo(dtype).min, torch.finfo(dtype).max
    z[0, ::3] = -float("inf")
    z[1] = -float("inf")
    z[2, ::5] = float("nan")
    z[3, ::7] = float("inf")
    z[4, ::2] = low
    z[5, ::2] = high
    z[6] = 0.0
    z[7] = -0.0
    z[8] = torch.finfo(dtype).tiny
    bits = rng.random((6, V)) < 0.5
    bits[0] = False                                       # nothing is left
    bits[1] = True
    bits[2] = False
    bits[2, V - 1] = True
    bits[3, :V // 2] = False
    M, kw = _all(rng, 12, [1] * 12, V, L=3000, n_bias=200)
    kw["masks"] = _words(bits)
    kw["bias"][:, ::4] = -np.inf
    for index in (rng.integers(-1, 6, 12), np.full(12, 2), np.arange(12) - 3):     # (the last: some below -1, some past the last)
        kw["mask_of_row"] = index.astype(np.int32)
        _check(v, z, **kw)
    del kw["mask_of_row"]
    kw["masks"] = _words(rng.random((12, V)) < 0.1)
    _check(v, z, **kw)
    kw["repetition"] = np.full(12, 2.0, np.float32)       # products past the type's range
    _check(v, z, **kw)


@pytest.mark.parametrize("n_bias", [1, 2, 3, 64, 300, 4096])
@pytest.mark.parametrize("L", [3, 8200])
def test_bias_lists(v, n_bias, L):
    """Lists up to the longest, of ids in one place and all over, with both sizes of workgroups."""
    rng = np.random.default_rng(n_bias)
    V = 20011
    M, kw = _all(rng, 3, [2, 1, 2], V, L=L, n_bias=n_bias)
    kw["bias_ids"][0] = 5000 + rng.permutation(n_bias)
    kw["bias_ids"][1] = rng.permutation(V)[:n_bias]
    _check(v, _logits(rng, M, V), **kw)
    _check(v, _logits(rng, M, V, torch.bfloat16), **kw)


def test_an_id_that_the_bias_list_names_twice(v):
    z = torch.zeros(2, 5000, device=DEV)
    ids = np.full((2, 300), 4097, np.int32)
    ids[1, 1::2] = 3
    bias = np.arange(600, dtype=np.float32).reshape(2, 300)
    got = _check(v, z, bias_ids=ids, bias=bias)
    assert got[0, 4097] == 299 and got[1, 4097] == 598 and got[1, 3] == 599


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_strides_and_alignment(v, dtype):
    rng = np.random.default_rng(9)
    for V, ld, at, ld_out, at_out in ((1003, 1003, 1, 1003, 1), (1003, 1003, 3, 1003, 0), (1000, 1024, 5, 1000, 2), (8192, 8200, 7, 8193, 3), (8200, 8201, 0, 8201, 0), (17, 40, 2, 17, 0)):
        M, kw = _all(rng, 2, [3, 2], V)
        flat, to = _logits(rng, 1, at + 5 * ld + 16, dtype)[0], torch.full((at_out + 5 * ld_out + 16,), -7.0, device=DEV, dtype=dtype)
        z, out = flat[at:at + 5 * ld].view(5, ld)[:, :V], to[at_out:at_out + 5 * ld_out].view(5, ld_out)[:, :V]
        before = flat.clone()
        got = _check(v, z, out=out, in_place=False, **kw)
        around = to.clone()
        around[at_out:at_out + 5 * ld_out].view(5, ld_out)[:, :V] = -7.0
        assert (around == -7).all()
        v.adjust_logits(z, out=z, **{n: _put(x) for n, x in kw.items()})
        assert torch.equal(z, got)
        z.copy_(before[at:at + 5 * ld].view(5, ld)[:, :V])
        assert torch.equal(flat, before)                  # what lies around the rows is as it was


def test_rows_of_no_sequence_stay_as_they_were(v):
    rng = np.random.default_rng(1)
    z = _logits(rng, 7, 900)
    out = torch.full((7, 900), -7.0, device=DEV)
    kw = dict(row_off=np.array([1, 3, 5], np.int32), window=rng.integers(0, 900, 7).astype(np.int32), presence=np.float32([1.0, 2.0]))
    v.adjust_logits(z, out=out, **{n: _put(x) for n, x in kw.items()})
    want = adjust_logits(z.double().cpu().numpy(), **kw)
    assert (out[[0, 5, 6]] == -7).all()
    np.testing.assert_allclose(out[1:5].cpu().numpy(), want[1:5], rtol=2.0 ** -24)
    # offsets that leave the rows: only those that are there
    kw["row_off"] = np.array([-4, 2, 90], np.int32)
    out.fill_(-7.0)
    v.adjust_logits(z, out=out, **{n: _put(x) for n, x in dict(row_off=kw["row_off"], presence=kw["presence"]).items()})
    assert torch.equal(out, z)


def test_offsets_past_32_bits(v):
    """Rows of logits, histories and masks past 2^31 elements of the first."""
    M, V, ld = 5, 1500, 600_000_000
    flat = torch.zeros((M - 1) * ld + V, dtype=torch.bfloat16, device=DEV)
    z = flat.as_strided((M, V), (ld, 1))
    rng = np.random.default_rng(0)
    z.copy_(_logits(rng, M, V, torch.bfloat16))
    history = torch.full((M, 500_000_000), -1, dtype=torch.int32, device=DEV)
    ids = rng.integers(0, V, (M, 900)).astype(np.int32)
    history[:, :900] = _put(ids)
    masks = torch.zeros(M, 500_000_000, dtype=torch.int32, device=DEV)
    words = _words(rng.random((M, V)) < 0.5)
    masks[:, :words.shape[1]] = _put(words)
    kw = dict(frequency=np.float32([0.1, 0.2, 0.3, 0.4, 0.5]), n_history=np.full(M, 900, np.int32))
    want = adjust_logits(z.double().cpu().numpy(), history=ids, masks=words, **kw)
    got = v.adjust_logits(z, history=history, masks=masks, **{n: _put(x) for n, x in kw.items()}).double().cpu().numpy()
    np.testing.assert_array_equal(np.isinf(got), np.isinf(want))
    fine = np.isfinite(want)
    assert (np.abs(got - want)[fine] <= 2.0 ** -8 * np.abs(want[fine]) * (1 + 2.0 ** -15) + 1e-12).all()


def test_from_graphs_and_on_another_stream():
    """Two captured graphs on a verifier's own stream, replayed in turn with eager calls between them; every call gives the same bits."""
    from paper_2507_02659_amd.runner import Verifier
    rng = np.random.default_rng(6)
    stream = torch.cuda.Stream()
    ver = Verifier(d=8, V_t=16, V_d=1, dtype="bf16", W=torch.zeros(8, 16, dtype=torch.bfloat16, device=DEV), direct_map=np.zeros(1, np.int32),
                   max_batch=1, max_k=0, stream=stream)
    with torch.cuda.stream(stream):
        made = []
        for rows, V, L in (([9] * 4, 32003, 40), ([1], 9000, 40), ([2, 3], 20011, 9000)):   # (the last: the larger workgroups)
            sets = []
            for _ in range(3):
                M, kw = _all(rng, len(rows), rows, V, L=L, n_masks=3)
                sets.append((_logits(rng, M, V), {n: _put(x) for n, x in kw.items()}))
            eager = [ver.adjust_logits(z, **kw).clone() for z, kw in sets]
            z, kw = sets[0][0].clone(), {n: x.clone() for n, x in sets[0][1].items()}
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                out = ver.adjust_logits(z, **kw)
            made.append((sets, eager, z, kw, graph, out))
        for turn in (0, 1, 2, 1):
            for sets, eager, z, kw, graph, out in made:
                z.copy_(sets[turn][0])
                for n, x in kw.items():
                    x.copy_(sets[turn][1][n])
                graph.replay()
                again = ver.adjust_logits(sets[turn][0], **sets[turn][1])
                stream.synchronize()
                assert torch.equal(out, eager[turn]) and torch.equal(again, eager[turn])
    ver.close()
