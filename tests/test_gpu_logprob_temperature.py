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
