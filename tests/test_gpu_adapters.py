"""Low-rank adapters beside the head against oracle/adapters.py."""
import numpy as np
import pytest
import torch

from oracle.adapters import adapter_logits

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


@pytest.fixture(scope="module")
def v():
    from paper_2507_02659_amd.runner import Verifier
    ver = Verifier(d=8, V_t=16, V_d=1, dtype="bf16", W=torch.zeros(8, 16, dtype=torch.bfloat16, device=DEV), direct_map=np.zeros(1, np.int32),
                   max_batch=1, max_k=0)
    yield ver
    ver.close()


def _set(rng, n, R, d, V, dtype=torch.bfloat16, scale=True):
    from paper_2507_02659_amd.runner import Adapters
    put = lambda a: torch.from_numpy(a.astype(np.float32)).to(dtype).to(DEV)  # noqa: E731
    s = torch.from_numpy((0.5 + rng.random(n)).astype(np.float32)).to(DEV) if scale else None
    return Adapters(put(rng.standard_normal((n, R, d)) / np.sqrt(d)), put(rng.standard_normal((n, V, R)) / np.sqrt(R)), s)


def _near(got, hidden, a, adapter, logits):
    """A sum of n products in float32, rounded at every addition by at most a step of the partial sums: n 2^-23 of the sum of their sizes.  The
    inner one (d products, one rounding of scale), kept to 2^-24 by its three parts, then the outer one (three parts of rank products), then the
    logit's addition and the output's rounding."""
    h, s = hidden.double().cpu().numpy(), None if a.scale is None else a.scale.double().cpu().numpy()
    down, up = a.down.double().cpu().numpy(), a.up.double().cpu().numpy()
    z = None if logits is None else logits.double().cpu().numpy()
    want = adapter_logits(h, down, up, s, adapter, z)
    R, d = down.shape[1:]
    sizes = adapter_logits(np.abs(h), np.abs(down), np.abs(up), s, adapter)      # the inner sum's sizes through the outer one's
    tol = np.where(np.isnan(sizes), 0, sizes) * ((d + 4) * 2.0 ** -23 + (3 * R + 4) * 2.0 ** -23) + 2.0 ** -24 * (0 if z is None else np.abs(z)) + 2.0 ** -24 * np.abs(want) + 1e-36
    if got.dtype == torch.bfloat16:
        tol = tol * (1 + 2.0 ** -8) + 2.0 ** -8 * np.abs(want)
    host = got.double().cpu().numpy()
    np.testing.assert_array_equal(np.isnan(host), np.isnan(want))
    off = np.where(np.isnan(want), 0, np.abs(host - want) - tol)
    assert off.max(initial=0) <= 0, (off.max(), np.unravel_index(off.argmax(), off.shape))
    none = np.asarray(adapter) == -1
    if z is not None and none.any():
        assert torch.equal(got[torch.from_numpy(none).to(DEV)], logits[torch.from_numpy(none).to(DEV)])


def _check(v, rng, M, n, R, d, V, dtype=torch.bfloat16, logits_type=torch.float32, adapter=None, scale=True, base=True):
    a = _set(rng, n, R, d, V, dtype, scale)
    hidden = torch.from_numpy(rng.standard_normal((M, d)).astype(np.float32)).to(dtype).to(DEV)
    adapter = rng.integers(-1, n, M).astype(np.int32) if adapter is None else np.asarray(adapter, np.int32)
    at = torch.from_numpy(adapter).to(DEV)
    z = torch.from_numpy((2 * rng.standard_normal((M, V))).astype(np.float32)).to(logits_type).to(DEV) if base else None
    print(f"adapters M={M} n={n} R={R} d={d} V={V} {dtype} {logits_type} base={base} rows={adapter[:12].tolist()}", flush=True)
    got = v.adapter_logits(hidden, a, at, z)
    _near(got, hidden, a, adapter, z)
    if z is not None:
        own = z.clone()
        assert torch.equal(v.adapter_logits(hidden, a, at, own, out=own).nan_to_num(), got.nan_to_num()) and torch.equal(own.nan_to_num(), got.nan_to_num())
    return got


@pytest.mark.parametrize("dtype,R", [(torch.bfloat16, R) for R in (8, 16, 24, 32, 40, 64, 72, 96, 128, 136, 200, 256)] + [(torch.float32, R) for R in (4, 12, 16, 20, 36, 64, 68, 100, 132, 192, 256)])
def test_ranks(v, dtype, R):
    rng = np.random.default_rng(R)
    _check(v, rng, 11, 3, R, 72, 333, dtype)
    _check(v, rng, 70, 2, R, 264, 130, dtype, torch.bfloat16)


@pytest.mark.parametrize("V", [1, 2, 3, 4, 5, 15, 16, 17, 63, 64, 65, 255, 256, 257, 1000, 4099])
def test_lengths(v, V):
    rng = np.random.default_rng(V)
    for dtype in (torch.bfloat16, torch.float32):
        for logits_type in (torch.float32, torch.bfloat16):
            _check(v, rng, 5, 2, 16, 40, V, dtype, logits_type)


@pytest.mark.parametrize("d", [1, 3, 8, 16, 31, 40, 63, 128, 500, 520, 1024, 2056, 4096, 8200])
def test_hidden_sizes(v, d):
    rng = np.random.default_rng(d)
    _check(v, rng, 7, 3, 8, d, 100, torch.float32)
    if d % 8 == 0:
        _check(v, rng, 7, 3, 24, d, 100)


@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 63, 64, 65, 129, 700, 2047, 2048, 2049, 4200])
def test_numbers_of_rows(v, M):
    rng = np.random.default_rng(M)
    _check(v, rng, M, 5, 16, 32, 70)
    _check(v, rng, M, 1, 16, 32, 70, adapter=np.zeros(M))
    _check(v, rng, M, 4, 8, 16, 70, torch.float32, adapter=np.repeat(np.arange(-1, 5), -(-M // 6))[:M] % 5 - 1)


def test_few_strips_and_many_tiles(v):
    """Blocks whose tiles are shared out over workgroups: few ids, many adapters, rows in any order."""
    rng = np.random.default_rng(11)
    for M, n, R, V in ((56, 5, 64, 2251), (64, 64, 16, 1100), (130, 20, 136, 700), (64, 1, 16, 513), (33, 7, 8, 9)):
        for logits_type in (torch.float32, torch.bfloat16):
            _check(v, rng, M, n, R, 48, V, torch.bfloat16, logits_type)
            _check(v, rng, M, n, R, 48, V, torch.float32, logits_type)


def test_many_adapters(v):
    """A row each, all in one block and in many; an adapter that no row has."""
    rng = np.random.default_rng(3)
    _check(v, rng, 64, 64, 8, 32, 130, adapter=rng.permutation(64))
    _check(v, rng, 64, 300, 8, 32, 130, adapter=rng.permutation(300)[:64])
    _check(v, rng, 200, 1000, 8, 16, 66, adapter=rng.permutation(1000)[:200])
    _check(v, rng, 300, 100, 8, 16, 66, torch.float32)


def test_rows_without_an_adapter_and_without_logits(v):
    rng = np.random.default_rng(4)
    for dtype in (torch.bfloat16, torch.float32):
        _check(v, rng, 9, 2, 16, 32, 500, dtype, adapter=np.full(9, -1))
        _check(v, rng, 9, 2, 16, 32, 500, dtype, adapter=[0, -1, 1, 2, -2, 0, 2 ** 31 - 1, -2 ** 31, 1])
        got = _check(v, rng, 9, 2, 16, 32, 500, dtype, adapter=[0, -1, 1, 2, -2, 0, 1, 1, -1], base=False, scale=False)
        assert (got[1] == 0).all() and (got[8] == 0).all()
    # an infinity among the hidden states or the matrices stays in its rows
    a = _set(rng, 2, 16, 32, 100)
    hidden = torch.randn(6, 32, device=DEV).bfloat16()
    at = torch.tensor([0, 1, 0, -1, 1, 0], dtype=torch.int32, device=DEV)
    z = torch.randn(6, 100, device=DEV)
    clean = v.adapter_logits(hidden, a, at, z)
    hidden[2, 5] = float("inf")
    hidden[3] = float("nan")
    a.up[1, 7, 3] = float("nan")
    got = v.adapter_logits(hidden, a, at, z)
    assert got[2].isnan().all() and got[1, 7].isnan() and got[4, 7].isnan()
    keep = torch.ones(6, 100, dtype=torch.bool, device=DEV)
    keep[2], keep[1, 7], keep[4, 7] = False, False, False
    assert torch.equal(got[keep], clean[keep])


def test_an_inner_sum_keeps_its_digits(v):
    """Inner sums that float32 holds exactly, with 24 significant bits, through a column of the identity: the output is their float32 value."""
    from paper_2507_02659_amd.runner import Adapters
    rng = np.random.default_rng(5)
    d = 32
    hidden = torch.zeros(40, d)
    whole = rng.integers(2 ** 23, 2 ** 24, 40)
    for k in range(3):                                     # bytes as bfloat16, exactly
        hidden[:, k] = torch.from_numpy(((whole >> (8 * k)) & 255) * 256.0 ** k)
    down, up = torch.zeros(1, 8, d), torch.zeros(1, 50, 8)
    down[0, 2, :3] = 1.0
    up[0, 13, 2] = 1.0
    a = Adapters(down.bfloat16().to(DEV), up.bfloat16().to(DEV))
    got = v.adapter_logits(hidden.bfloat16().to(DEV), a, torch.zeros(40, dtype=torch.int32, device=DEV))
    assert np.array_equal(got[:, 13].cpu().numpy(), whole.astype(np.float32)) and (got[:, :13] == 0).all()


@pytest.mark.parametrize("logits_type", [torch.float32, torch.bfloat16])
def test_strides_and_alignment(v, logits_type):
    rng = np.random.default_rng(8)
    M, n, R, d = 19, 3, 16, 48
    for V, ld, at, ld_out, at_out in ((1003, 1003, 1, 1003, 3), (130, 150, 5, 131, 2), (257, 257, 0, 300, 1)):
        a = _set(rng, n, R, d, V)
        hidden = torch.from_numpy(rng.standard_normal((M, d)).astype(np.float32)).bfloat16().to(DEV)
        adapter = rng.integers(-1, n, M).astype(np.int32)
        flat = torch.randn(at + M * ld + 8, device=DEV).to(logits_type)
        to = torch.full((at_out + M * ld_out + 8,), -7.0, device=DEV, dtype=logits_type)
        z, out = flat[at:at + M * ld].view(M, ld)[:, :V], to[at_out:at_out + M * ld_out].view(M, ld_out)[:, :V]
        of_row = torch.from_numpy(adapter).to(DEV)
        before = flat.clone()
        got = v.adapter_logits(hidden, a, of_row, z, out=out)
        _near(got, hidden, a, adapter, z)
        assert torch.equal(flat, before)
        want = got.clone()
        out.fill_(-7.0)
        assert (to == -7).all()                           # nothing beside the rows was written
        v.adapter_logits(hidden, a, of_row, z, out=z)
        assert torch.equal(z, want)
        z.copy_(before[at:at + M * ld].view(M, ld)[:, :V])
        assert torch.equal(flat, before)


def test_offsets_past_32_bits(v):
    """Logits past 2^31 elements of the first, and an adapter whose matrices lie as far behind the first one's."""
    from paper_2507_02659_amd.runner import Adapters
    rng = np.random.default_rng(0)
    M, V, ld = 5, 1500, 600_000_000
    z = torch.zeros((M - 1) * ld + V, dtype=torch.bfloat16, device=DEV).as_strided((M, V), (ld, 1))
    a = _set(rng, 2, 16, 32, V)
    hidden = torch.randn(M, 32, device=DEV).bfloat16()
    adapter = np.array([0, 1, -1, 1, 0], np.int32)
    got = v.adapter_logits(hidden, a, torch.from_numpy(adapter).to(DEV), z)
    _near(got, hidden, a, adapter, z)
    own = v.adapter_logits(hidden, a, torch.from_numpy(adapter).to(DEV), z, out=z)
    assert torch.equal(own, got)
    n, R, d, V = 300, 256, 32768, 32768                   # 2.5e9 elements each
    down, up = torch.zeros(n, R, d, dtype=torch.bfloat16, device=DEV), torch.zeros(n, V, R, dtype=torch.bfloat16, device=DEV)
    last = _set(rng, 1, R, d, V, scale=False)
    down[-1], up[-1] = last.down[0], last.up[0]
    hidden = torch.randn(3, d, device=DEV).bfloat16()
    far = v.adapter_logits(hidden, Adapters(down, up), torch.full((3,), n - 1, dtype=torch.int32, device=DEV))
    assert torch.equal(far, v.adapter_logits(hidden, last, torch.zeros(3, dtype=torch.int32, device=DEV)))
    assert far.abs().max() > 0


def test_beside_the_head():
    """The verifier's own head, bf16 and fp32, with adapters."""
    from paper_2507_02659_amd.runner import Verifier
    rng = np.random.default_rng(2)
    for name, dtype in (("bf16", torch.bfloat16), ("f32", torch.float32)):
        W = (torch.randn(128, 700, device=DEV) * 0.1).to(dtype)
        ver = Verifier(d=128, V_t=700, V_d=1, dtype=name, W=W, direct_map=np.zeros(1, np.int32), max_batch=20, max_k=0)
        a = _set(rng, 3, 16, 128, 700, dtype)
        hidden = torch.randn(20, 128, device=DEV).to(dtype)
        adapter = rng.integers(-1, 3, 20).astype(np.int32)
        got = ver.lm_head(hidden, adapters=a, adapter_of_row=torch.from_numpy(adapter).to(DEV))
        _near(got, hidden, a, adapter, ver.lm_head(hidden))
        ver.close()


def test_from_graphs_that_share_the_workspace():
    from paper_2507_02659_amd.runner import Verifier
    rng = np.random.default_rng(6)
    stream = torch.cuda.Stream()
    ver = Verifier(d=8, V_t=16, V_d=1, dtype="bf16", W=torch.zeros(8, 16, dtype=torch.bfloat16, device=DEV), direct_map=np.zeros(1, np.int32),
                   max_batch=1, max_k=0, stream=stream)
    with torch.cuda.stream(stream):
        made = []
        for M, R, d, V in ((1, 16, 512, 9000), (100, 64, 256, 3001)):
            a = _set(rng, 4, R, d, V)
            sets = [(torch.randn(M, d, device=DEV).bfloat16(), torch.randint(-1, 4, (M,), device=DEV, dtype=torch.int32), torch.randn(M, V, device=DEV)) for _ in range(3)]
            eager = [ver.adapter_logits(h, a, t, z).clone() for h, t, z in sets]
            own = [x.clone() for x in sets[0]]
            stream.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=stream):
                out = ver.adapter_logits(own[0], a, own[1], own[2])
            made.append((a, sets, eager, own, graph, out))
        for turn in (0, 1, 2, 1):
            for a, sets, eager, own, graph, out in made:
                for x, y in zip(own, sets[turn]):
                    x.copy_(y)
                graph.replay()
                again = ver.adapter_logits(sets[turn][0], a, sets[turn][1], sets[turn][2])
                stream.synchronize()
                assert torch.equal(out, eager[turn]) and torch.equal(again, eager[turn])
    ver.close()
