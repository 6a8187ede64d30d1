"""Cuts among a few scores that the bins cannot tell apart: each of the ways that
settle such a list, by its length and by which limits cut it."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")
from paper_2411_10764_amd import ml2  # noqa: E402
from tests import drawutil  # noqa: E402

DEV = "cuda:0"


@pytest.mark.parametrize("n", [4096, 14336, 100000])
@pytest.mark.parametrize("entries", [10, 64, 65, 96, 128, 129, 400])
def test_lists_of_distinct_scores(n, entries):
    """`entries` scores in one bin under the best one, the rest without weight:
    top-k cuts them by count, top-p by weight, both by the nearer of the two."""
    rng = np.random.default_rng(n + entries)
    rows, draws = 2, 40
    x = np.full((rows, n), -40.0, np.float32)
    for r in range(rows):
        at = rng.permutation(np.arange(1, n))[:entries]
        x[r, at] = np.float32(-1.01) - np.float32(0.015) * rng.random(entries, dtype=np.float32)
    x[:, 0] = 0.0
    u = rng.random((rows, draws), dtype=np.float32)
    scores, given = torch.from_numpy(x).to(DEV), torch.from_numpy(u).to(DEV)
    sampler = ml2.Sampler(rows, n, draws)
    for k, p in ((entries // 2, 1.0), (0, 0.6), (entries - 3, 0.6), (entries // 3, 0.97)):
        idx, logp = sampler.run(scores, given, top_k=torch.full((rows,), k, dtype=torch.int32, device=DEV),
                                top_p=torch.full((rows,), p, device=DEV))
        torch.cuda.synchronize()
        want = drawutil.sample(x, None, np.ones(rows, np.float32), np.full(rows, k),
                               np.full(rows, p, np.float32), np.zeros(rows, np.float32), u)
        sure = want[2]
        assert sure.mean() > 0.9, (k, p, sure.mean())
        assert np.array_equal(idx.cpu().numpy()[sure], want[0][sure]), (k, p)
        # log M: weights of one rounding and 1 ulp of exp each
        assert np.all(np.abs(logp.cpu().numpy() - want[1])[sure] <= 4e-6), (k, p)
