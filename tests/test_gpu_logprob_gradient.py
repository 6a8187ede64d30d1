"""ml2_logprob_grad at every entry: a gradient that is NaN, or not 0 where an
entry is not included, fails (the tolerances: drawutil.gradient_tolerance)."""
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


def _run(x, valid, targets, weight, T):
    """(ml2_logprob, ml2_logprob_grad's logprob, gradient), buffers filled before."""
    rows, n = x.shape
    f = ml2.LogProb(rows, n, targets.shape[1], grad_dtype=x.dtype)
    t, v, w, at = [torch.from_numpy(a).to(DEV) if a is not None else None
                   for a in (targets, valid, weight, T)]
    f.logprob.fill_(7.0)
    forward = f.run(x.to(DEV), t, v, at).clone()
    f.logprob.fill_(7.0)
    f.grad.fill_(7.0)
    lp, g = f.run_grad(x.to(DEV), t, w, v, at)
    torch.cuda.synchronize()
    return forward.cpu().numpy(), lp.cpu().numpy(), drawutil.as_float(g)


def _check(x, valid, targets, weight, T):
    """The case against the 64-bit form: a log-probability within the tolerance of
    its sum (4e-5) and of its own two roundings, the gradient as check_gradient."""
    forward, lp, g = _run(x, valid, targets, weight, T)
    xf = drawutil.as_float(x)
    for r in range(x.shape[0]):
        v = None if valid is None else valid if valid.ndim == 1 else valid[r]
        want, _ = drawutil.logprob_row(xf[r], v, T[r], targets[r])
        fin = np.isfinite(want)
        for got in (forward[r], lp[r]):
            assert np.array_equal(got[~fin], want[~fin]), (r, got, want)
            off = np.abs(got[fin] - want[fin])
            assert np.all(off <= 4e-5 + 2.0 ** -22 * np.abs(want[fin])), (r, got, want)
    drawutil.check_gradient(g, xf, valid, T, targets, weight, ROUND[x.dtype], TINY[x.dtype],
                            float(torch.finfo(x.dtype).max))


def _case(rng, rows, n, d, dtype, masked):
    x = torch.from_numpy(rng.standard_normal((rows, n)).astype(np.float32) * 2).to(dtype)
    valid = (rng.random((rows, n)) < 0.6).astype(np.uint8) if masked else None
    targets = rng.integers(-1, n + 1, (rows, d)).astype(np.int32)
    if d > 3:
        targets[:, d // 2:] = targets[:, : d - d // 2]  # repeated targets
    weight = rng.standard_normal((rows, d)).astype(np.float32)
    T = rng.choice([0.5, 1.0, 2.0, 0.0], rows).astype(np.float32)
    return x, valid, targets, weight, T


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,n,d", [(1, 1, 1), (3, 63, 5), (5, 1000, 33), (300, 517, 2),
                                      (70, 20011, 3), (1, 50021, 17), (2, 100, 2000),
                                      (3, 131072, 200), (40, 70001, 2)])
@pytest.mark.parametrize("masked", [False, True])
def test_formula(dtype, rows, n, d, masked):
    rng = np.random.default_rng(7 * rows + n + d)
    x, valid, targets, weight, T = _case(rng, rows, n, d, dtype, masked)
    _check(x, valid, targets, weight, T)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [9, 3001, 70001])
def test_specials(dtype, n):
    """Rows of infinities, NaN and the type's lowest value, in and out of the mask."""
    inf, nan, low = np.inf, np.nan, float(torch.finfo(dtype).min)
    head = np.array([[nan] * 6, [-inf] * 6, [low] * 6, [inf, 1, inf, -inf, 0, 2],
                     [low, 3, low, low, nan, 1], [-low, low, -low, 0, 1, 2],
                     [0.0, -0.0, nan, -inf, inf, 5]])
    rng = np.random.default_rng(n)
    x = np.ascontiguousarray(head[:, rng.integers(0, 6, n)])
    x[:, :6] = head
    x = torch.from_numpy(x).to(dtype)
    targets = rng.integers(-1, 12, (len(x), 9)).astype(np.int32)
    weight = rng.standard_normal(targets.shape).astype(np.float32)
    T = np.array([1, 1, 2, 1, 0.5, 1, 0], np.float32)
    for valid in (None, np.zeros(n, np.uint8), (rng.random(x.shape) < 0.5).astype(np.uint8)):
        _check(x, valid, targets, weight, T)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("n", [6, 3001, 70001])
def test_not_included_is_zero_whatever_the_weights(dtype, n):
    """Weights whose sum or share over a small temperature passes float32's range:
    entries that are not included get 0 all the same, and so do those without
    probability and a target that holds all of it."""
    rng = np.random.default_rng(n)
    rows = 8
    x = torch.from_numpy(rng.uniform(-9, -1, (rows, n)).astype(np.float32)).to(dtype)
    x[:, 0] = 0.0
    x[4:, 1] = 0.0  # two that share the probability
    x[:, 2] = -np.inf
    x[1::2, 3] = np.nan
    valid = np.ones((rows, n), np.uint8)
    valid[:, 4] = 0
    targets = np.array([[0, -1, 4, n]] * rows, np.int32)
    weight = np.array([[10.0, 3.0, 5.0, 2.0]] * rows, np.float32)
    T = np.full(rows, 1e-38, np.float32)
    T[2:4] = 3e-39
    T[6:] = 1e-45  # 1 / T itself is infinite
    _check(x, valid, targets, weight, T)
    weight[:] = 3e38
    T[:] = 1.0
    _check(x, valid, targets, weight, T)


@pytest.mark.parametrize("rows,n", [(5, 3001), (2, 70001)])
def test_scores_and_gradient_in_one_buffer(rows, n):
    """Columns of one buffer are taken; the scores' own memory is refused."""
    rng = np.random.default_rng(n)
    x, valid, targets, weight, T = _case(rng, rows, n, 6, torch.float32, True)
    both = torch.full((rows, 2 * n), 3.0, device=DEV)
    both[:, :n] = x.to(DEV)
    t, v, w, at = [torch.from_numpy(a).to(DEV) for a in (targets, valid, weight, T)]
    ws = ml2.LogProb(rows, n, 6).ws
    ml2.ml2_logprob_grad(both[:, :n], t, w, both[:, n:], ws, None, v, at)
    torch.cuda.synchronize()
    assert torch.equal(both[:, :n].cpu(), x)
    drawutil.check_gradient(both[:, n:].cpu().numpy(), x.numpy(), valid, T, targets, weight,
                            ROUND[torch.float32], TINY[torch.float32],
                            float(np.finfo(np.float32).max))
    for grad in (both[:, :n], both[:, 1:n + 1]):
        with pytest.raises(ml2.Ml2Error, match="overlaps"):
            ml2.ml2_logprob_grad(both[:, :n], t, w, grad, ws, None, v, at)
    torch.cuda.synchronize()
    assert torch.equal(both[:, :n].cpu(), x)
