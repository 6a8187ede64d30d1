"""ml2_logprob and ml2_logprob_grad at small temperatures, in the one-workgroup
kernel and in the chunked one.

A weight is exp2 of s * c - m * c with c = log2(e) / T.  Where m / T passes
2^24, the rounding of m * c is worth whole powers of two of every weight; the
maxima here are chosen by it."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from tests.test_gpu_logprob_gradient import TYPES, _check  # noqa: E402

LOG2E = np.float32(1.44269504088896340736)


def _maxima(T, dtype, low, high, count, rng):
    """Scores of 1 .. 32 whose product with log2(e) / T rounds by `low` .. `high`
    powers of two (fewer than `count` where the type has fewer)."""
    m = torch.from_numpy(rng.uniform(1, 32, 400000).astype(np.float32)).to(dtype)
    m = np.unique(m.float().numpy())
    c = np.float32(1) / np.float32(T) * LOG2E
    off = m.astype(np.float64) * np.float64(c) - (m * c).astype(np.float64)  # exact
    m = m[(off >= low) & (off < high)]
    return rng.permutation(m)[:count]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T", [1e-6, 3e-8, 1e-8, 2e-9, 1e-10])
@pytest.mark.parametrize("n", [40, 3001, 20011, 70001])
def test_small_temperatures(dtype, T, n):
    rng = np.random.default_rng(n)
    m = [_maxima(T, dtype, a, b, 8, rng)
         for a, b in ((126, 128), (60, 126), (28, 60), (1, 28), (-1, 1), (-28, -1), (-150, -28),
                      (128, 300))]
    m.append(np.array([1.0, 30.0], np.float32))
    if dtype == torch.float32:
        m.append(np.array([22.596845626831055], np.float32))
    m = np.concatenate(m)
    rows = len(m)
    if n == 20011:  # as many rows as take them whole
        m = np.resize(m, max(rows, 64))
        rows = len(m)
    x = torch.from_numpy(rng.uniform(-3, 0.9, (rows, n)).astype(np.float32)).to(dtype)
    at = rng.integers(0, n, rows)
    x[np.arange(rows), at] = torch.from_numpy(m).to(dtype)
    x[np.arange(rows)[::3], (at[::3] + 1) % n] = torch.from_numpy(m[::3]).to(dtype)  # ties
    targets = np.stack([at, (at + 1) % n, (at + 2) % n, at], 1).astype(np.int32)
    weight = (rng.standard_normal((rows, 4)) * T).astype(np.float32)
    valid = np.ones((rows, n), np.uint8)
    valid[:, 5::7] = 0
    valid[np.arange(rows), at] = 1
    for v in (None, valid):
        _check(x, v, targets, weight, np.full(rows, T, np.float32))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n", [40, 3001, 70001])
@pytest.mark.parametrize("T", [1e-38, 4e-39, 3.2e-39])
def test_temperatures_as_small_as_the_scores(dtype, n, T):
    """Scores of about T where 1 / T is finite, log2(e) / T not: the exponents are
    ordinary numbers.  Scores are whole numbers of 2^-133, bfloat16's smallest."""
    rng = np.random.default_rng(n)
    x = torch.from_numpy(rng.integers(-250, 20, (3, n)).astype(np.float32) * 2.0 ** -133).to(dtype)
    x[:, 0] = 40 * 2.0 ** -133
    valid = (rng.random((3, n)) < 0.6).astype(np.uint8)
    valid[:, 0] = 1
    targets = rng.integers(-1, n + 1, (3, 5)).astype(np.int32)
    targets[:, 0] = 0
    weight = (rng.standard_normal((3, 5)) * 0.01).astype(np.float32)
    _check(x, valid, targets, weight, np.full(3, T, np.float32))
