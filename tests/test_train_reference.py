"""The reference of the 8-bit states, and what rounding at random is for, on the CPU."""
import numpy as np
import torch

from tests import trainutil as t


def test_codes_are_torch_float8_e4m3fn():
    codes = np.arange(256).astype(np.uint8)
    ours, theirs = t.values(codes), torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn)
    theirs = theirs.double().numpy()
    ok = ~np.isnan(theirs)
    assert ok.sum() == 254 and np.array_equal(ours[ok], theirs[ok])


def test_numbers_of_the_format_stay():
    for bits in (0, 1, 32768, 65535):
        size = t.values(np.arange(127).astype(np.uint8))
        assert np.array_equal(t.rounded(size, np.full(127, bits), 0), np.arange(127))


def test_rounding_is_unbiased_and_hashes_are_spread():
    """Mean of 20,000 roundings of one value, its standard error being at most half a step over
    their root; upper and lower halves of the hash are uncorrelated."""
    n = 20000
    h = t.hashed(5, 3, 0, np.arange(n))
    for bits in (h >> 16, h & 0xFFFF):
        for size in (1.03, 300.0, 0.011, 0.0011):
            codes = t.rounded(np.full(n, size), bits, 0).astype(np.uint8)
            step = max(2.0 ** (np.floor(np.log2(size)) - 3), 2.0 ** -9)
            assert abs(t.values(codes).mean() - size) < 5 * step / 2 / n ** 0.5
        other = t.hashed(5, 4, 0, np.arange(n)) >> 16
        assert abs(np.corrcoef(bits, other)[0, 1]) < 5 / n ** 0.5
    assert abs(np.corrcoef(h >> 16, h & 0xFFFF)[0, 1]) < 5 / n ** 0.5


def test_layer_norm_gradient_is_the_derivative():
    """The 64-bit gradients against differences of the 64-bit forward pass."""
    rng = np.random.default_rng(3)
    x, w, b, d = (rng.standard_normal(s) for s in ((4, 9), 9, 9, (4, 9)))
    eps, h = 1e-3, 1e-5
    _, _, rstd, _ = t.layer_norm(x, w, b, eps)
    dx, dw, db, _ = t.layer_norm_grad(x, d, w, rstd)

    def loss(x, w, b):
        return (t.layer_norm(x, w, b, eps)[0] * d).sum()

    for grad, at in ((dx, 0), (dw, 1), (db, 2)):
        args = [x, w, b]
        v = rng.standard_normal(args[at].shape)
        up, down = list(args), list(args)
        up[at], down[at] = args[at] + h * v, args[at] - h * v
        slope = (loss(*up) - loss(*down)) / (2 * h)
        assert abs(slope - (grad * v).sum()) < 1e-7 * (1 + abs(slope))
