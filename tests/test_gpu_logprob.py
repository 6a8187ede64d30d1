"""ml2_logprob and ml2_logprob_grad against the formula in 64 bits and against
differences.

Tolerances.  An exponent z is two float32 roundings from its value and the
exponential adds one: relative error (|z| + 2) 2^-23 of a weight, at most 30 *
2^-23 where the weight matters.  A sum adds 2^-24 for each of the up to about
300 terms a lane and the joins add in a row.  So l is within 330 * 2^-23 =
4e-5 of its value, a log-probability within 4e-5 + 2^-22 |z| of its own, a
gradient within 8e-5 of its two terms, plus the rounding to its type."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2411_10764_amd import ml2  # noqa: E402
from tests import drawutil  # noqa: E402

DEV = "cuda:0"
TYPES = [torch.float32, torch.bfloat16, torch.float16]
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.float32: 1e-37, torch.bfloat16: 1e-37, torch.float16: 2.0 ** -24}


def _reference(x, valid, T, targets, weight):
    lp, g = [], []
    for r in range(x.shape[0]):
        v = None if valid is None else valid if valid.ndim == 1 else valid[r]
        a, b = drawutil.logprob_row(x[r], v, T[r], targets[r], weight[r])
        lp.append(a)
        g.append(b)
    return np.stack(lp), np.stack(g)


def _check_logprob(got, want):
    fin = np.isfinite(want)
    assert np.array_equal(np.isneginf(got), np.isneginf(want))
    assert np.all(np.abs(got[fin] - want[fin]) <= 4e-5 + 2.0 ** -22 * np.abs(want[fin]))


def _check_grad(got, want, x, valid, T, targets, weight, dtype):
    """Relative to the size of the two terms each entry's gradient is made of."""
    for r in range(x.shape[0]):
        v = None if valid is None else valid if valid.ndim == 1 else valid[r]
        _, size = drawutil.logprob_row(x[r], v, T[r], targets[r], np.zeros(targets.shape[1]))
        t = float(T[r]) if T[r] > 0 else 1.0
        ok = drawutil.included(x[r], v)
        w = np.abs(weight[r]) * [bool(0 <= j < x.shape[1] and ok[j]) for j in targets[r]]
        z = np.full(x.shape[1], -np.inf)
        if ok.any():
            y = x[r][ok].astype(np.float64)
            with np.errstate(all="ignore"):
                z[ok] = np.where(y == y.max(), 0, (y - y.max()) / t)
            z -= np.log(np.exp(z).sum())
        size = np.exp(z) * w.sum() / t
        for j, q in zip(targets[r], w):
            if 0 <= j < x.shape[1]:
                size[j] += q / t
        tol = 8e-5 * size + ROUND[dtype] * np.abs(want[r]) + TINY[dtype]
        bad = np.abs(got[r] - want[r]) > tol
        assert not bad.any(), (r, np.nonzero(bad)[0][:5], got[r][bad][:5], want[r][bad][:5])


def _case(rng, rows, n, d, dtype, masked, spread=2.0):
    x = torch.from_numpy(rng.standard_normal((rows, n)).astype(np.float32) * spread).to(dtype)
    valid = (rng.random((rows, n)) < 0.6).astype(np.uint8) if masked else None
    targets = rng.integers(-1, n + 1, (rows, d)).astype(np.int32)
    if d > 3:
        targets[:, d // 2:] = targets[:, : d - d // 2]  # repeated targets
    weight = rng.standard_normal((rows, d)).astype(np.float32)
    T = rng.choice([0.5, 1.0, 2.0, 0.0], rows).astype(np.float32)
    return x, valid, targets, weight, T


def _run(x, valid, targets, weight, T):
    rows, n = x.shape
    d = targets.shape[1]
    f = ml2.LogProb(rows, n, d, grad_dtype=x.dtype)
    dev = [torch.from_numpy(a).to(DEV) if a is not None else None
           for a in (targets, valid, T, weight)]
    f.logprob.fill_(7.0)
    a = f.run(x.to(DEV), dev[0], dev[1], dev[2]).clone()
    f.logprob.fill_(7.0)
    f.grad.fill_(7.0)
    b, g = f.run_grad(x.to(DEV), dev[0], dev[3], dev[1], dev[2])
    torch.cuda.synchronize()
    return a.cpu().numpy(), b.cpu().numpy(), drawutil.as_float(g)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n,d", [(1, 1, 1), (2, 2, 3), (3, 63, 5), (2, 65, 1), (5, 1000, 33),
                                      (2, 4097, 64), (300, 517, 2), (1, 50021, 17),
                                      (7, 20011, 1), (1, 300007, 1500), (600, 2048, 1),
                                   (2, 100, 16384), (1, 50021, 16384), (1, 1000003, 5000),
                                      (2, 131072, 1), (40, 70001, 2)])
def test_formula(dtype, rows, n, d):
    print(f"[logprob] {dtype} {rows} x {n}, {d}", flush=True)
    for masked in (False, True):
        rng = np.random.default_rng(rows + n + d)
        x, valid, targets, weight, T = _case(rng, rows, n, d, dtype, masked)
        a, b, g = _run(x, valid, targets, weight, T)
        xf = drawutil.as_float(x)
        lp, grad = _reference(xf, valid, T, targets, weight)
        _check_logprob(a, lp)
        _check_logprob(b, lp)
        _check_grad(g, grad, xf, valid, T, targets, weight, dtype)


def test_specials():
    """Rows without an entry, infinities and NaN in and out of the mask."""
    inf, nan, low = np.inf, np.nan, np.finfo(np.float32).min
    x = np.array([[nan] * 6, [-inf] * 6, [low] * 6, [inf, 1, inf, -inf, 0, 2],
                  [low, 3, low, low, nan, 1], [-low, low, -low, 0, 1, 2],
                  [0.0, -0.0, nan, -inf, inf, 5]], np.float32)
    rng = np.random.default_rng(2)
    targets = rng.integers(-1, 7, (len(x), 9)).astype(np.int32)
    weight = rng.standard_normal(targets.shape).astype(np.float32)
    T = np.array([1, 1, 2, 1, 0.5, 1, np.nan], np.float32)
    for valid in (None, np.zeros(x.shape, np.uint8), (rng.random(x.shape) < 0.5).astype(np.uint8)):
        a, b, g = _run(torch.from_numpy(x), valid, targets, weight, T)
        lp, grad = _reference(x, valid, np.nan_to_num(T), targets, weight)
        _check_logprob(a, lp)
        _check_logprob(b, lp)
        _check_grad(g, grad, x, valid, np.nan_to_num(T), targets, weight, torch.float32)


@pytest.mark.parametrize("T", [1e-38, 1e-45, np.inf])
def test_extreme_temperatures(T):
    x = torch.tensor([[1.0, 2.0, 2.0, -3.0, 0.5]], device=DEV)
    f = ml2.LogProb(1, 5, 5, grad_dtype=torch.float32)
    t = torch.arange(5, dtype=torch.int32, device=DEV)[None]
    lp = f.run(x, t, temperature=torch.tensor([T], device=DEV)).cpu().numpy()[0]
    if np.isinf(T):
        assert np.allclose(lp, -np.log(5), atol=4e-5)
    else:
        assert np.allclose(lp[[1, 2]], -np.log(2), atol=4e-5) and np.all(lp[[0, 3, 4]] < -1e30)


@pytest.mark.parametrize("offset,pad,gpad", [(0, 0, 3), (1, 5, 0), (3, 0, 1)])
@pytest.mark.parametrize("dtype", TYPES)
def test_strides_and_alignment(dtype, offset, pad, gpad):
    rng = np.random.default_rng(offset + pad)
    rows, n, d = 5, 3001, 4
    x, valid, targets, weight, T = _case(rng, rows, n, d, dtype, True)
    flat = torch.full((offset + rows * (n + pad),), 50.0, dtype=dtype, device=DEV)
    xs = flat[offset:].view(rows, n + pad)[:, :n]
    xs.copy_(x)
    gflat = torch.full((offset + rows * (n + gpad),), 3.0, dtype=dtype, device=DEV)
    grad = gflat[offset:].view(rows, n + gpad)
    dev = [torch.from_numpy(a).to(DEV) for a in (targets, weight, valid[0], T)]
    ws = ml2.LogProb(rows, n, d).ws
    ml2.ml2_logprob_grad(xs, dev[0], dev[1], grad[:, :n], ws, None, dev[2], dev[3])
    torch.cuda.synchronize()
    assert torch.all(grad[:, n:] == 3.0) and torch.all(gflat[:offset] == 3.0)
    xf = drawutil.as_float(x)
    _, want = _reference(xf, valid[0], T, targets, weight)
    _check_grad(drawutil.as_float(grad[:, :n]), want, xf, valid[0], T, targets, weight, dtype)


def test_differences():
    """Central differences of ml2_logprob's own weighted sum: with steps of
    2^-6 the difference's own error is step^2 / 6 * 2 = 8e-5 of a weight and
    the sum's rounding 4e-5 / 2^-6 * its weights' size is far above what two
    sums that share their rounding leave: 5e-3 in all."""
    rng = np.random.default_rng(4)
    n, d, h = 40, 6, 2.0 ** -6
    x = torch.from_numpy(rng.standard_normal((1, n)).astype(np.float32)).to(DEV)
    valid = torch.from_numpy((rng.random(n) < 0.8).astype(np.uint8)).to(DEV)
    t = torch.from_numpy(rng.integers(0, n, (1, d)).astype(np.int32)).to(DEV)
    t[0, 3] = t[0, 1]
    valid[t[0].long()] = 1
    w = torch.from_numpy(rng.standard_normal((1, d)).astype(np.float32)).to(DEV)
    T = torch.tensor([0.8], device=DEV)
    _, g = ml2.LogProb(1, n, d, grad_dtype=torch.float32).run_grad(x, t, w, valid, T)
    many = x.repeat(2 * n, 1)
    at = torch.arange(n, device=DEV)
    many[at, at] += h
    many[n + at, at] -= h
    lp = ml2.LogProb(2 * n, n, d).run(many, t.repeat(2 * n, 1), valid, T.repeat(2 * n))
    f = (lp.double() * w.double()).sum(1)
    diff = ((f[:n] - f[n:]) / (2 * h)).cpu().numpy()
    assert np.all(np.abs(diff - g[0].double().cpu().numpy()) <= 5e-3)


def test_same_bits_every_run_and_in_a_graph():
    rng = np.random.default_rng(6)
    for rows, n, d in ((1, 400000, 700), (64, 5000, 3)):
        x, valid, targets, weight, T = _case(rng, rows, n, d, torch.float32, True)
        dev = [torch.from_numpy(a).to(DEV) for a in (targets, weight, valid, T)]
        xd = x.to(DEV)
        f = ml2.LogProb(rows, n, d, grad_dtype=torch.float32)
        want = [t.clone() for t in f.run_grad(xd, *dev)]
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        f.run_grad(xd, *dev, stream=side)
        torch.cuda.synchronize()
        assert torch.equal(want[0], f.logprob) and torch.equal(want[1], f.grad)
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            f.run_grad(xd, *dev)
        for _ in range(4):
            f.grad.fill_(9.0)
            f.ws.fill_(255)
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(want[0], f.logprob) and torch.equal(want[1], f.grad)
            xd.mul_(0.95)
            want = [t.clone() for t in f.run_grad(xd, *dev)]


def test_large_gradient():
    """A gradient beyond what the caches hold (written past them): sampled rows."""
    rows, n = 1400, 65536
    g = torch.Generator(device=DEV)
    g.manual_seed(3)
    x = (torch.randn(rows, n, generator=g, device=DEV) * 2).to(torch.bfloat16)
    targets = torch.randint(n, (rows, 2), generator=g, device=DEV, dtype=torch.int32)
    weight = torch.randn(rows, 2, generator=g, device=DEV)
    lp, grad = ml2.LogProb(rows, n, 2, grad_dtype=torch.bfloat16).run_grad(x, targets, weight)
    torch.cuda.synchronize()
    some = [0, 1, 255, 700, rows - 1]
    xf, t, w = drawutil.as_float(x[some]), targets[some].cpu().numpy(), weight[some].cpu().numpy()
    T = np.ones(len(some), np.float32)
    want_lp, want = _reference(xf, None, T, t, w)
    _check_logprob(lp[some].cpu().numpy(), want_lp)
    _check_grad(drawutil.as_float(grad[some]), want, xf, None, T, t, w, torch.bfloat16)


@pytest.mark.parametrize("n,d", [(4096, 100), (4096, 500), (100, 16384), (300000, 128),
                                 (300000, 5000)])
def test_targets_that_mostly_repeat(n, d):
    """Nine of ten targets are one entry, as where a sure policy draws one again and again."""
    rng = np.random.default_rng(n + d)
    x, valid, targets, weight, T = _case(rng, 2, n, d, torch.float32, False)
    targets[:, : d - d // 10] = n // 2
    a, b, g = _run(x, valid, targets, weight, T)
    xf = drawutil.as_float(x)
    lp, grad = _reference(xf, valid, T, targets, weight)
    _check_logprob(a, lp)
    _check_logprob(b, lp)
    _check_grad(g, grad, xf, valid, T, targets, weight, torch.float32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [60, 3001, 50021, 300007])
def test_signaling_nan_is_like_any_nan(dtype, n):
    """Scores of a bit pattern that operations quieten: draws, log-probabilities
    and gradients are those of the same row with quiet ones."""
    rng = np.random.default_rng(n)
    x = torch.from_numpy(rng.standard_normal((2, n)).astype(np.float32) * 2).to(dtype)
    bits = torch.int32 if dtype == torch.float32 else torch.int16
    signaling = torch.tensor(torch.inf, dtype=dtype).view(bits) + 1
    at = torch.from_numpy(rng.random((2, n)) < 0.4)
    at[:, n // 2:n // 2 + 3] = torch.tensor([True, False, True])
    x[:, n // 2 + 1] = 9.0  # the best, between two of them
    loud = x.view(bits).where(~at, signaling.expand_as(at)).view(dtype).to(DEV)
    quiet = x.masked_fill(at, float("nan")).to(DEV)
    t = torch.from_numpy(rng.integers(0, n, (2, 7)).astype(np.int32)).to(DEV)
    w = torch.from_numpy(rng.standard_normal((2, 7)).astype(np.float32)).to(DEV)
    p = torch.full((2,), 0.8, device=DEV)
    for d in (1, 40):
        u = torch.from_numpy(rng.random((2, d), dtype=np.float32)).to(DEV)
        got = [[v.clone() for v in ml2.Sampler(2, n, d).run(s, u, top_p=p)] for s in (loud, quiet)]
        assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
    f = [ml2.LogProb(2, n, 7, grad_dtype=dtype) for _ in range(2)]
    got = [a.run_grad(s, t, w) for a, s in zip(f, (loud, quiet))]
    assert torch.equal(got[0][0], got[1][0]) and torch.equal(got[0][1], got[1][1])
