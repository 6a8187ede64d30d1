"""The check that gradients go through refuses what is not the gradient: the
mistakes are planted in the 64-bit form's own answer, on the CPU."""
import numpy as np
import pytest

from tests import drawutil

F32 = (2.0 ** -24, 1e-37, float(np.finfo(np.float32).max))
F16 = (2.0 ** -11, 2.0 ** -24, 65504.0)


def _case():
    rng = np.random.default_rng(1)
    x = rng.standard_normal((3, 40)).astype(np.float32)
    valid = (rng.random((3, 40)) < 0.6).astype(np.uint8)
    x[1, 3], x[2, 5] = np.nan, -np.inf
    T = np.array([1.0, 0.5, 0.0], np.float32)
    targets = rng.integers(-1, 41, (3, 6)).astype(np.int32)
    weight = rng.standard_normal((3, 6)).astype(np.float32)
    got = np.stack([drawutil.logprob_row(x[r], valid[r], T[r], targets[r], weight[r])[1]
                    for r in range(3)]).astype(np.float32)
    return got, (x, valid, T, targets, weight)


def test_the_formula_passes():
    got, case = _case()
    drawutil.check_gradient(got, *case, *F32)
    drawutil.check_gradient(-0.0 + got.astype(np.float16).astype(np.float32), *case, *F16)


@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf, 1e-3])
@pytest.mark.parametrize("included", [True, False])
def test_a_planted_mistake_is_refused(value, included):
    got, case = _case()
    ok = drawutil.included(case[0][1], case[1][1])
    at = np.nonzero(ok == included)[0][2]
    got[1, at] = value
    with pytest.raises(AssertionError):
        drawutil.check_gradient(got, *case, *F32)


def test_a_row_of_nan_is_refused():
    got, case = _case()
    got[0] = np.nan
    with pytest.raises(AssertionError):
        drawutil.check_gradient(got, *case, *F32)


def test_overflow_is_infinite_of_the_same_sign():
    x, T = np.zeros((1, 2), np.float32), np.array([1e-5], np.float32)
    targets, weight = np.array([[0]], np.int32), np.array([[4.0]], np.float32)
    case = (x, None, T, targets, weight)
    drawutil.check_gradient(np.array([[np.inf, -np.inf]]), *case, *F16)
    for wrong in ([np.inf, np.inf], [65504.0, -65504.0], [np.nan, -np.inf]):
        with pytest.raises(AssertionError):
            drawutil.check_gradient(np.array([wrong]), *case, *F16)
