"""Which memory ml2_logprob_grad's outputs may share with its inputs: none, and
nothing else is refused.  Without a GPU: the calls that pass this check end at
the next one, a workspace that is missing."""
import random

import pytest

from paper_2411_10764_amd import ml2

A = 0x1000000  # an aligned address that nothing here reads


def _overlaps(dtype, rows, n, scores, ld, grad, grad_ld, per_row=1, targets=1 << 40,
              weight=1 << 41, logprob=1 << 42):
    """Whether the call is refused for its memory."""
    status = ml2.lib().ml2_logprob_grad(dtype, scores, n, ld, rows, None, 0, None, targets, weight,
                                        per_row, logprob, grad, grad_ld, None, 0, None)
    assert status == ml2.ML2_ERR_INVALID_ARG
    said = ml2.lib().ml2_last_error().decode()
    assert said.startswith("ml2_logprob_grad:") and ("overlaps" in said) != ("workspace" in said)
    return "overlaps" in said


def test_gradient_over_the_scores():
    for dtype, size in ((ml2.ML2_F32, 4), (ml2.ML2_BF16, 2), (ml2.ML2_F16, 2)):
        assert _overlaps(dtype, 4, 100, A, 100, A, 100)
        assert _overlaps(dtype, 4, 100, A, 128, A, 128)
        assert _overlaps(dtype, 4, 100, A, 100, A + 399 * size, 100)
        assert not _overlaps(dtype, 4, 100, A, 100, A + 400 * size, 100)
        assert not _overlaps(dtype, 4, 100, A + 400 * size, 100, A, 100)
        assert not _overlaps(dtype, 4, 100, A, 200, A + 100 * size, 200)  # one buffer's halves
        assert not _overlaps(dtype, 4, 100, A + 100 * size, 200, A, 200)
        assert _overlaps(dtype, 4, 100, A, 199, A + 100 * size, 199)
        assert not _overlaps(dtype, 2097152, 1, A, 1 << 40, A + size, 1 << 40)


def test_against_the_elements_themselves():
    rng = random.Random(3)
    seen = set()
    for _ in range(4000):
        rows, n = rng.randint(1, 5), rng.randint(1, 7)
        ld, grad_ld = n + rng.randint(0, 9), n + rng.randint(0, 9)
        if rng.random() < 0.5:
            grad_ld = ld
        off = rng.randint(-60, 60)
        scores = {r * ld + i for r in range(rows) for i in range(n)}
        want = any(off + r * grad_ld + i in scores for r in range(rows) for i in range(n))
        got = _overlaps(ml2.ML2_BF16, rows, n, A, ld, A + 2 * off, grad_ld)
        assert got == want, (rows, n, ld, grad_ld, off)
        seen.add((got, ld == grad_ld))
    assert len(seen) == 4


@pytest.mark.parametrize("rows,per_row", [(1, 1), (3, 5)])
def test_logprob_over_targets_or_weight(rows, per_row):
    size = 4 * rows * per_row
    for name in ("targets", "weight"):
        for off, want in ((0, True), (size - 4, True), (4 - size, True), (size, False),
                          (-size, False)):
            got = _overlaps(ml2.ML2_F32, rows, 10, A, 10, 2 * A, 10, per_row,
                            **{name: (1 << 42) + off})
            assert got == want, (name, off)
