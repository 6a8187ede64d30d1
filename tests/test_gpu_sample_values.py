"""ml2_sample on long rows of 16-bit scores with one draw, which are counted
by score: against the definition in 64 bits, and against the same call with
more draws, which takes the way that float32 rows take.  Weights are whole
numbers in both, so indices and log-probabilities have to be the same bits."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2411_10764_amd import ml2  # noqa: E402
from tests import test_gpu_sample as base  # noqa: E402

DEV = "cuda:0"
TYPES = [torch.bfloat16, torch.float16]
MORE = 9  # draws of a row that take the other way, four of them one by one too


def _both(scores, valid=None, seed=0, **lim):
    """Draws one by one and the same among more, equal bit by bit."""
    rows, n = scores.shape
    rng = np.random.default_rng(seed)
    u = torch.from_numpy(base._u(rng, rows, MORE)).to(DEV)
    par = {}
    for a, t in (("temperature", torch.float32), ("top_k", torch.int32),
                 ("top_p", torch.float32), ("min_p", torch.float32)):
        v = lim.get(a)
        if v is not None:
            par[a] = torch.as_tensor(np.broadcast_to(np.asarray(v), (rows,)).copy()).to(t).to(DEV)
    many = ml2.Sampler(rows, n, MORE)
    idx, logp = (v[:, :4].cpu().numpy() for v in many.run(scores, u, valid, **par))
    one = ml2.Sampler(rows, n, 1)
    for j in range(4):
        one.idx.fill_(-77)
        one.ws.fill_(255)
        i, p = one.run(scores, u[:, j: j + 1].contiguous(), valid, **par)
        assert np.array_equal(i[:, 0].cpu().numpy(), idx[:, j])
        assert np.array_equal(p[:, 0].cpu().numpy().view(np.int32), logp[:, j].view(np.int32))
    return idx, logp


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [14337, 16384, 16389, 57344, 57345, 70001])
def test_lengths_and_limits(dtype, n):
    print(f"[sample values] {dtype} n={n}", flush=True)
    rng = np.random.default_rng(n)
    for j, lim in enumerate(base.LIMITS):
        rows = 2
        x = torch.from_numpy(rng.standard_normal((rows, n)).astype(np.float32) * 2.5)
        valid = None if j % 2 else (rng.random((rows, n)) < 0.7).astype(np.uint8)
        par = {a: np.full(rows, b) for a, b in lim.items()}
        for u in (0.0, 0.37, 0.81, 0.99):
            idx, logp, (want, want_logp, sure) = base._run(
                x.to(dtype).to(DEV), np.full((rows, 1), u, np.float32), valid, **par)
            assert np.array_equal(idx[sure], want[sure])
            assert np.all(np.abs(logp[sure] - want_logp[sure]) <= base.TOL)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [14337, 50021, 65536, 65537, 131072, 262144, 262145])
def test_same_as_with_more_draws(dtype, n):
    print(f"[sample values] {dtype} n={n}", flush=True)
    g = torch.Generator(device=DEV)
    g.manual_seed(n)
    x = (torch.randn(3, n, generator=g, device=DEV) * 2).to(dtype)
    valid = (torch.rand(n, generator=g, device=DEV) < 0.6).to(torch.uint8)
    for seed, lim in enumerate((dict(), dict(top_k=50), dict(top_k=n - 1), dict(top_p=0.9),
                                dict(top_k=n // 3, top_p=0.95), dict(top_k=1000, top_p=0.3),
                                dict(min_p=0.05), dict(top_p=0.99, min_p=0.9),
                                dict(temperature=0.2, top_p=0.9), dict(temperature=0.0),
                                dict(temperature=50.0, top_k=n // 2, top_p=0.5, min_p=0.9))):
        _both(x, None, seed, **lim)
        _both(x, valid, seed, **lim)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("levels", [1, 2, 5, 40])
def test_ties_across_parts(dtype, levels):
    """Entries of the cut's score are kept by index, wherever parts end."""
    rng = np.random.default_rng(levels)
    rows, n = 3, 120001
    x = rng.integers(0, levels, (rows, n)).astype(np.float32) / 4
    x[x == 0] = rng.choice([0.0, -0.0], (x == 0).sum())
    x = torch.from_numpy(x).to(dtype).to(DEV)
    valid = torch.from_numpy((rng.random((rows, n)) < 0.5).astype(np.uint8)).to(DEV)
    for v in (None, valid):
        for seed, lim in enumerate((dict(top_k=1), dict(top_k=3), dict(top_k=n // 5),
                                    dict(top_k=n // 2 + 1), dict(top_k=n - 1), dict(top_p=0.0),
                                    dict(top_p=0.4), dict(top_p=0.9), dict(top_k=n // 3, top_p=0.5),
                                    dict(top_k=n // 3, min_p=0.99), dict())):
            idx, _ = _both(x, v, seed, **lim)
            if levels == 1 and v is None and "top_k" in lim and "top_p" not in lim:
                k = min(lim["top_k"], n)
                assert (idx[:, 0] == 0).all() and (idx[:, 1] == k - 1).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_specials_in_long_rows(dtype):
    """Rows without an entry, with one, and infinities, NaN and the type's
    lowest value in and out of the mask."""
    n = 60013
    inf, nan, low = np.inf, np.nan, torch.finfo(dtype).min
    rng = np.random.default_rng(3)
    fills = ([nan], [-inf], [low], [-inf, nan, 1.5], [inf, 1.0, -inf], [low, low, 3.0],
             [-low, low, 0.0], [0.0, -0.0, nan], [1e-7, 0.0, -1e-7], [inf, -low, 2.0, nan])
    x = np.array([np.resize(np.array(f, np.float64), n) for f in fills]).astype(np.float32)
    one = np.full((1, n), -inf, np.float32)
    one[0, 59999] = -3.0
    x = torch.from_numpy(np.concatenate([x, one])).to(dtype).to(DEV)
    none = torch.zeros(x.shape, dtype=torch.uint8, device=DEV)
    half = torch.from_numpy((rng.random(x.shape) < 0.5).astype(np.uint8)).to(DEV)
    for valid in (None, none, half):
        for seed, lim in enumerate((dict(), dict(top_k=3), dict(top_p=0.6), dict(min_p=0.5),
                                    dict(temperature=0.0), dict(temperature=1e-38),
                                    dict(temperature=np.inf), dict(temperature=1e-45, top_k=2),
                                    dict(top_k=n // 2, top_p=0.7, min_p=0.2))):
            idx, logp = _both(x, valid, seed, **lim)
            assert (idx[:2] == -1).all() and (logp[:2] == -np.inf).all()
            if valid is none:
                assert (idx == -1).all()
            elif valid is None:
                assert (idx[-1] == 59999).all() and (logp[-1] == 0).all()


@pytest.mark.parametrize("dtype", TYPES)
def test_every_bit_pattern(dtype):
    """All 65,536 patterns, both signs of every NaN among them, in every place."""
    rng = np.random.default_rng(11)
    rows = 4
    bits = np.stack([rng.permutation(65536) for _ in range(rows)])
    bits[1, bits[1] % 3 > 0] = 0x7FFF      # two thirds NaN, positive
    bits[2, bits[2] % 3 > 0] = 0xFFFF      # negative
    bits[3, rng.random(65536) < 0.5] = torch.tensor(torch.inf, dtype=dtype).view(torch.int16) + 1
    x = torch.from_numpy(bits.astype(np.uint16).view(np.int16)).to(DEV).view(dtype)
    finite = x.float().where(x.float().abs() < 1000, torch.nan).to(dtype)
    for scores in (x, finite):
        for seed, lim in enumerate((dict(), dict(top_k=3), dict(top_k=1000), dict(top_k=20000),
                                    dict(top_k=60000), dict(top_p=0.9),
                                    dict(top_k=500, top_p=0.5), dict(temperature=0.0))):
            _both(scores, None, seed, **lim)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("offset,pad", [(1, 0), (3, 5), (1, 1), (0, 64)])
def test_strides_alignment_and_shared_mask(dtype, offset, pad):
    rng = np.random.default_rng(offset * 7 + pad)
    rows, n = 3, 30011
    flat = torch.full((offset + rows * (n + pad),), 99.0, dtype=dtype, device=DEV)
    x = flat[offset:].view(rows, n + pad)[:, :n]
    x.copy_(torch.from_numpy(rng.standard_normal((rows, n)).astype(np.float32) * 2))
    mask = torch.from_numpy((rng.random(offset + rows * (n + pad)) < 0.8).astype(np.uint8)).to(DEV)
    for valid in (mask[offset:].view(rows, n + pad)[:, :n], mask[offset: offset + n]):
        idx, _ = _both(x, valid, 1, top_k=700, top_p=0.95)
        at = np.broadcast_to(valid.cpu().numpy(), (rows, n))
        assert np.take_along_axis(at, idx.astype(np.int64), 1).all()


def test_rows_with_their_own_settings_and_many_rows():
    rng = np.random.default_rng(5)
    rows, n = 700, 50021  # more than one set of launches
    g = torch.Generator(device=DEV)
    g.manual_seed(1)
    x = torch.randn(rows, n, generator=g, device=DEV, dtype=torch.float32).mul_(2.5)
    _both(x.to(torch.float16), None, 2, temperature=rng.choice([0.0, -1.0, np.nan, 0.3, 1.0], rows),
          top_k=rng.choice([-3, 0, 1, 2, 50, n, n + 9], rows),
          top_p=rng.choice([np.nan, 2.0, 1.0, 0.9, 0.2, 0.0, -1.0], rows),
          min_p=rng.choice([np.nan, -1.0, 0.0, 0.01, 0.5, 1.0, 7.0], rows))


def test_captured_and_replayed():
    n, rows = 50021, 4
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    x = (torch.randn(rows, n, generator=g, device=DEV) * 2).to(torch.bfloat16)
    u = torch.rand(rows, 1, generator=g, device=DEV)
    p = torch.full((rows,), 0.9, device=DEV)
    s, eager = ml2.Sampler(rows, n), ml2.Sampler(rows, n)
    s.run(x, u, top_p=p)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        s.run(x, u, top_p=p)
    for _ in range(3):
        u.copy_(torch.rand(rows, 1, generator=g, device=DEV))
        x.copy_(torch.randn(rows, n, generator=g, device=DEV).to(torch.bfloat16))
        graph.replay()
        idx, logp = eager.run(x, u, top_p=p)
        torch.cuda.synchronize()
        assert torch.equal(s.idx, idx) and torch.equal(s.logprob, logp)
